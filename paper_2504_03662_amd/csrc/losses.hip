// Losses of logits with the logits' gradient: log probabilities of tokens and cross entropy, the clipped policy loss, the
// preference loss of pairs of sequences, distillation from a teacher's top logits.
//
// With a = scale z (a row of logits), p = exp(a - lse) and lse = log sum exp a, every one of them is a function of a row's lse and
// of a few of its logits, and its gradient is dz = -c p with a constant c of the row, but for those few logits.  So there is one
// row kernel: it reads a row, keeps maximum and sum of exponentials of what a thread has met, joins them over the workgroup, forms
// the loss and c from them, and writes the gradient.  It is bound by memory: 8 bytes an element (fp32) or 4 (bf16) against
// about 20 instructions.
// Sums over a thread's elements are fp32; from there on (sums over threads, log sums, losses) they are fp64, which is free: losses
// are small differences of log sums, and a sequence's reward adds up over thousands of tokens.
#include "../../include/gx.h"
#include "gx_kernels.h"
#include <type_traits>

namespace {

using namespace gx;

constexpr int MAX_ROWS = 1 << 21, MAX_VOCAB = 1 << 19, MAX_TOP = 1024, MAX_PAIRS = 1 << 20;
// So few rows that read their teachers in one launch with the rest; more of them in a launch before, where no registers wait for it
constexpr int READ_HERE = 256;
// So few rows and pairs that a launch of its own for the pairs takes longer than adding them up for every row
constexpr int FEW_ROWS = 1024, FEW_PAIRS = 256;
constexpr long MAX_GRID = (1 << 24) - 1;                       // workgroups of 256: a launch has less than 2^32 threads
constexpr float NO_LOGIT = -INFINITY, MIN_SCALE = 1.f / (1 << 20);

template <int N> using Int = std::integral_constant<int, N>;
template <bool B> using Flag = std::bool_constant<B>;

template <typename T> struct Lanes;                            // elements of 16 bytes
template <> struct Lanes<float> { static constexpr int N = 4; typedef f32x4 type; };
template <> struct Lanes<bf16> { static constexpr int N = 8; typedef bf16x8 type; };

// A row cut at the borders of 16 bytes: `head` elements before the first, `body` chunks, the rest behind the last.  The elements at the
// ends (fewer than two chunks) go one to a thread.  `lead`: chunks from the last border of 128 bytes to the first chunk: threads
// count from there, so that a wavefront's 64 chunks are whole lines.
template <typename T>
struct Cut {
  static constexpr int N = Lanes<T>::N;
  int head, body, ends, lead, vocab;
  GX_DEVINL Cut(const void* row, int v) : vocab(v) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = min(v, (N - off) % N);
    body = (v - head) / N;
    ends = v - body * N;                                       // before and behind together
    lead = (int)((reinterpret_cast<uintptr_t>(row) + (uintptr_t)head * sizeof(T)) >> 4 & 7);
  }
  GX_DEVINL bool has(int c) const { return (unsigned)c < (unsigned)body; }
  GX_DEVINL int end_at(int i) const { return i < head ? i : vocab - ends + i; }
};

template <typename T> GX_DEVINL typename Lanes<T>::type splat(float x) {
  typename Lanes<T>::type v;
#pragma unroll
  for (int e = 0; e < Lanes<T>::N; e++) v[e] = from_f32<T>(x);
  return v;
}

// An id: its column here, or what it is instead
constexpr int IGNORED = -1, ELSEWHERE = -2, INVALID = -3;
struct Ids {
  const void* p;
  int bytes;
  long first, whole, ignore;
  GX_DEVINL int column(int row, int vocab) const {
    const long id = bytes == 8 ? static_cast<const long*>(p)[row] : static_cast<const int*>(p)[row];
    if (id == ignore) return IGNORED;
    if (id < 0 || id >= whole) return INVALID;
    const long c = id - first;
    return c >= 0 && c < vocab ? (int)c : ELSEWHERE;
  }
};

// Exponential and logarithm in fp64, to about 2^-50: a power of two, and a series in what is left of it (of exp up to the 12th power for
// |r| <= log(2) / 2, of log m = 2 atanh((m - 1) / (m + 1)) up to the 19th for m between sqrt(1/2) and sqrt(2)).  Every
// wavefront of a row computes a few of them: a quarter of the instructions of a library's.
GX_DEVINL double exp_f64(double x) {
  const double c = fmin(fmax(x, -1100.0), 1100.0), n = rint(c * 1.4426950408889634074), r = fma(n, -0.69314718055994530942, c);
  double p = 1.0 / 479001600.0;
  const double coef[12] = {1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0,
                           1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
  for (int i = 0; i < 12; i++) p = fma(p, r, coef[i]);
  return x == x ? ldexp(p, (int)n) : x;
}
GX_DEVINL double log_f64(double x) {                           // of 0, of positive normal numbers or of NaN
  int n = __builtin_amdgcn_frexp_exp(x);
  double m = __builtin_amdgcn_frexp_mant(x);                   // 0.5 .. 1
  if (m < 0.70710678118654752440) {
    m *= 2.0;
    n--;
  }
  const double t = (m - 1.0) / (m + 1.0), t2 = t * t;
  double p = 2.0 / 19.0;
#pragma unroll
  for (int k = 17; k > 0; k -= 2) p = fma(p, t2, 2.0 / k);
  return x == 0.0 ? -(double)INFINITY : fma((double)n, 0.69314718055994530942, p * t);
}

// Maximum and sum of exponentials (relative to the maximum) of a set of logits; the empty set has -inf and 0
struct Sums {
  float m;
  double s;
};

// What a row's teacher says, as top_kernel leaves it: the sum of q; of q (log q - scale (z - m)); 1 - sum of q, or 0; and m and
// the sum over the student's logits that have an entry.  An entry: its column, or -1, the student's logit there, q.
struct TopRow {
  double q_sum, terms, rest;
  Sums own;
};
struct TopEntry {
  int col;
  float z, q, pad;
};

struct None {};

enum Kind { SCORE, TOKEN, POLICY, DISTILL };
struct RowArgs {
  const void* z;
  void* dz;                                                    // null: losses only
  long stride, grad_stride;
  int rows, vocab, kind;
  float scale, c_hi, c_lo;                                     // c_hi + c_lo = scale log2(e)
  Ids ids;
  const float* weights;
  float *loss, *logp, *lse;
  // policy
  const float *old_logp, *ref_logp, *adv;
  float low, high, kl;
  // for a later pass over the same logits: log probability, (maximum, 1 / sum of exponentials), the weight that counts
  double* logp64;
  f32x2* stats;
  float* counted;
  // distillation
  const TopRow* top_rows;                                      // null: the row's workgroup reads its teacher itself
  const TopEntry* entries;
  int top, rest, lds_bytes;                                    // lds_bytes: of a row's columns that are taken out
};

// exp(scale d) for d = z - maximum.  c_lo: the rounding of the constant would shift every term of a sum the same way.  It is
// positive, so that d = -inf gives 0.
GX_DEVINL float exp_scaled(float d, float c_hi, float c_lo) { return __builtin_amdgcn_exp2f(fmaf(d, c_lo, d * c_hi)); }

// the same for a gradient of type T: of bf16 the constant's low part would be lost
template <typename T>
GX_DEVINL float exp_gradient(float d, float c_hi, float c_lo) {
  return sizeof(T) == 2 ? __builtin_amdgcn_exp2f(d * c_hi) : exp_scaled(d, c_hi, c_lo);
}

GX_DEVINL double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

GX_DEVINL float reference(float m) { return m == NO_LOGIT ? 0.f : m; }
GX_DEVINL double rescaled(Sums x, float m, const RowArgs& a) {
  return x.s == 0.0 ? 0.0 : x.s * (double)exp_scaled(x.m - m, a.c_hi, a.c_lo);
}
GX_DEVINL Sums joined(Sums x, Sums y, const RowArgs& a) {
  const float m = fmaxf(x.m, y.m);
  return {m, rescaled(x, m, a) + rescaled(y, m, a)};
}
GX_DEVINL double log_sum(Sums x, const RowArgs& a) { return (double)a.scale * (double)x.m + log_f64(x.s); }

template <typename T>
GX_DEVINL void clear_row(T* row, int vocab, int tid, int threads) {
  typedef typename Lanes<T>::type Raw;
  const Cut<T> k(row, vocab);
  for (int c = tid; c < k.body; c += threads) reinterpret_cast<Raw*>(row + k.head)[c] = Raw{};
  if (tid < k.ends) row[k.end_at(tid)] = from_f32<T>(0.f);
}

// Past the caches: whoever reads the gradient next reads it as fast (1024 to 4096 rows of 32000, bf16: a sum over it 35 to 93 us, after stores
// into the caches 35 to 101), and the row kernel takes 28 rather than 31 us at 1024 rows, 205 rather than 206 at 8192 of 32768, 190 rather
// than 206 at 4096 of 64013.
template <typename T>
GX_DEVINL void store_chunk(T* p, const float (&x)[Lanes<T>::N], bool aligned) {
  typedef typename Lanes<T>::type Raw;
  Raw v;
#pragma unroll
  for (int e = 0; e < Lanes<T>::N; e++) v[e] = from_f32<T>(x[e]);
  if (aligned) {
    __builtin_nontemporal_store(v, reinterpret_cast<Raw*>(p));
  } else {                                                     // a gradient whose rows lie otherwise than the logits'
#pragma unroll
    for (int e = 0; e < Lanes<T>::N; e++) p[e] = v[e];
  }
}

// The policy loss of a token and its derivative by logp, without the weight.  A ratio beyond a border counts with the border,
// and has no gradient, where that makes the gain smaller; no advantage, no gain, whatever the ratio.
GX_DEVINL float policy_slope(const RowArgs& a, double logp, float old, float ref, float adv) {
  const float r = expf((float)(logp - (double)old)), gain = r * adv;
  const float cut = fminf(fmaxf(r, 1.f - a.low), 1.f + a.high) * adv;
  float g = adv != 0.f && !(gain > cut) ? -gain : 0.f;
  if (a.kl != 0.f) g -= a.kl * expm1f((float)((double)ref - logp));
  return g;
}
GX_DEVINL double policy_loss(const RowArgs& a, double logp, float old, float ref, float adv) {
  const double r = exp_f64(logp - (double)old);
  double l = 0.0;
  if (adv != 0.f) {
    const double cut = fmin(fmax(r, 1.0 - (double)a.low), 1.0 + (double)a.high), gain = r * (double)adv;
    l = gain <= cut * (double)adv ? -gain : -cut * (double)adv;
    if (r != r) l = r;
  }
  if (a.kl != 0.f) {
    const double d = (double)ref - logp;
    l += (double)a.kl * (exp_f64(d) - d - 1.0);
  }
  return l;
}

// Reads a row's teacher with THREADS threads, in fp64 but for the entry's q.
// An index that comes twice is one column with two entries; the first of them stands for the column, with the sum of their q.
// Whether there is such an index is asked of a table of at least twice as many places as entries (so that a search ends), and only
// then entries are compared with all others.
struct TopArgs {
  const void* z;
  long stride;
  int rows, vocab, top, places, id_bytes, top_bf16;
  float scale;
  const void *ids, *logits;
  const float *lse, *weights;
  TopRow* out;
  TopEntry* entries;
};
__host__ __device__ inline int top_words(const TopArgs& a) { return a.places + 2 * a.top; }       // of LDS for a row

template <typename T, int THREADS>
GX_DEVINL TopRow read_top(const TopArgs& a, int row, int tid, int* table, double (*part)[3]) {
  constexpr int WAVES = THREADS / 64;
  const int wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  auto all_here = [] {
    if (WAVES > 1) __syncthreads();
    else __threadfence_block();
  };
  int* const cols = table + a.places;
  float* const qs = reinterpret_cast<float*>(cols + a.top);
  const T* zr = static_cast<const T*>(a.z) + (size_t)row * a.stride;
  TopEntry* const entries = a.entries + (size_t)row * a.top;
  const size_t first_entry = (size_t)row * a.top;
  auto column = [&](int i) {
    const long id = a.id_bytes == 8 ? static_cast<const long*>(a.ids)[first_entry + i] : static_cast<const int*>(a.ids)[first_entry + i];
    return id >= 0 && id < a.vocab ? (int)id : -1;
  };
  auto teacher = [&](int i) {
    return a.top_bf16 ? (float)static_cast<const bf16*>(a.logits)[first_entry + i] : static_cast<const float*>(a.logits)[first_entry + i];
  };
  // a thread's first entry stays in registers; more than THREADS entries are read again
  const bool one = tid < a.top;
  const int col0 = one ? column(tid) : -1;
  const float t0 = one ? teacher(tid) : 0.f, z0 = col0 >= 0 ? to_f32(zr[col0]) : 0.f;
  auto col_of = [&](int i) { return i == tid ? col0 : column(i); };
  auto t_of = [&](int i) { return i == tid ? t0 : teacher(i); };
  auto z_of = [&](int i, int col) { return i == tid ? z0 : to_f32(zr[col]); };
  for (int i = tid; i < a.places; i += THREADS) table[i] = -1;
  all_here();
  float mz = NO_LOGIT, mt = NO_LOGIT;
  int again = 0;
  for (int i = tid; i < a.top; i += THREADS) {
    const int col = col_of(i);
    cols[i] = col;
    if (col < 0) continue;
    mz = fmaxf(mz, z_of(i, col));
    mt = fmaxf(mt, t_of(i));
    for (unsigned at = (unsigned)col * 2654435761u;; at++) {
      const int there = atomicCAS(&table[at & (a.places - 1)], -1, col);
      if (there == col) again = 1;
      if (there == col || there == -1) break;
    }
  }
  again = __any(again);
  mz = wave_max(mz);
  if (!a.lse) mt = wave_max(mt);
  if (WAVES > 1) {
    if ((tid & 63) == 0) {
      part[wave][0] = (double)mz;
      part[wave][1] = (double)mt;
      part[wave][2] = (double)again;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < WAVES; k++) {
      mz = fmaxf(mz, (float)part[k][0]);
      mt = fmaxf(mt, (float)part[k][1]);
      again |= part[k][2] != 0.0;
    }
    __syncthreads();
  } else {
    __threadfence_block();
  }
  const double scale = (double)a.scale, ref = (double)reference(mz);
  double lse;
  if (a.lse) {
    lse = (double)a.lse[row];
  } else {
    double s = 0.0;
    for (int i = tid; i < a.top; i += THREADS)
      if (cols[i] >= 0) s += exp_f64(scale * ((double)t_of(i) - (double)mt));
    s = wave_sum_f64(s);
    if (WAVES > 1) {
      if ((tid & 63) == 0) part[wave][0] = s;
      __syncthreads();
      s = 0.0;
#pragma unroll
      for (int k = 0; k < WAVES; k++) s += part[k][0];
      __syncthreads();
    }
    lse = scale * (double)mt + log_f64(s);
  }
  double sums[3] = {0.0, 0.0, 0.0};
  for (int i = tid; i < a.top; i += THREADS) {
    TopEntry e = {cols[i], 0.f, 0.f, 0.f};
    if (e.col >= 0) {
      e.z = z_of(i, e.col);
      const double logq = scale * (double)t_of(i) - lse, q = exp_f64(logq), az = scale * ((double)e.z - ref);
      sums[0] += q;
      if (q != 0.0) sums[1] += q * (logq - az);
      e.q = (float)q;
      qs[i] = e.q;
      bool first = true;
      if (again)
        for (int j = 0; j < i; j++) first &= cols[j] != e.col;
      if (!first) e.col = -1;
      else if (a.lse) sums[2] += exp_f64(az);
    }
    entries[i] = e;
  }
  if (again) {
    all_here();
    for (int i = tid; i < a.top; i += THREADS) {
      if (entries[i].col < 0) continue;
      float q = qs[i];
      for (int j = i + 1; j < a.top; j++)
        if (cols[j] == cols[i]) q += qs[j];
      entries[i].q = q;
    }
  }
#pragma unroll
  for (int n = 0; n < 3; n++) {
    if (n == 2 && !a.lse) continue;
    sums[n] = wave_sum_f64(sums[n]);
    if (WAVES > 1 && (tid & 63) == 0) part[wave][n] = sums[n];
  }
  if (WAVES > 1) {
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 3; n++) {
      sums[n] = 0.0;
      if (n == 2 && !a.lse) continue;
#pragma unroll
      for (int k = 0; k < WAVES; k++) sums[n] += part[k][n];
    }
  }
  return {sums[0], sums[1], a.lse ? fmax(0.0, 1.0 - sums[0]) : 0.0, {mz, sums[2]}};
}

// A row to a wavefront, or for more than 64 entries to a workgroup
template <typename T, int THREADS>
__global__ void __launch_bounds__(256) top_kernel(TopArgs a) {
  constexpr int ROWS = 256 / THREADS;
  extern __shared__ int lds_top[];
  __shared__ double part[4][3];
  const int of_group = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x * ROWS + of_group, tid = ROWS == 1 ? threadIdx.x : threadIdx.x & 63;
  if (row >= a.rows) return;
  if (a.weights && a.weights[row] == 0.f) return;              // nobody reads its record
  const TopRow t = read_top<T, THREADS>(a, row, tid, lds_top + of_group * top_words(a), part);
  if (tid == 0) a.out[row] = t;
}

// A row to a workgroup of THREADS, or with 64 one to each of a workgroup's four wavefronts.  A thread has CH chunks in flight; with
// STREAM as many of those steps as the row needs, and reads them again for the gradient, without it one.
template <typename T, int THREADS, int CH, bool STREAM, bool TOP, bool AGAIN>
__global__ void __launch_bounds__(THREADS < 256 ? 256 : THREADS, 4) loss_row_kernel(RowArgs a, std::conditional_t<TOP, TopArgs, None> teacher) {
  constexpr int N = Lanes<T>::N, WAVES = THREADS / 64, ROWS = THREADS < 256 ? 256 / THREADS : 1;
  typedef typename Lanes<T>::type Raw;
  extern __shared__ unsigned lds[];
  __shared__ Sums part[WAVES];
  const int wave_of_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = ROWS == 1 ? blockIdx.x : blockIdx.x * ROWS + wave_of_group;
  if (ROWS > 1 && row >= a.rows) return;
  const int tid = ROWS == 1 ? threadIdx.x : lane, wave = ROWS == 1 ? wave_of_group : 0;
  const T* zr = static_cast<const T*>(a.z) + (size_t)row * a.stride;
  T* dr = a.dz ? static_cast<T*>(a.dz) + (size_t)row * a.grad_stride : nullptr;
  const float w = a.weights ? a.weights[row] : 1.f;
  const int y = TOP ? ELSEWHERE : a.ids.column(row, a.vocab);
  const bool counts = w != 0.f && y != IGNORED;
  if (!counts) {
    if (tid == 0) {
      if (a.loss) a.loss[row] = 0.f;
      if (a.logp) a.logp[row] = 0.f;
      if (a.lse) a.lse[row] = 0.f;
      if (a.logp64) {
        a.logp64[row] = 0.0;
        a.stats[row] = f32x2{0.f, 0.f};
        a.counted[row] = 0.f;
      }
    }
    if (dr) clear_row(dr, a.vocab, tid, THREADS);
    return;
  }
  __shared__ TopRow read_here[ROWS];
  if constexpr (TOP) {
    if (!a.top_rows) {
      __shared__ double sums[WAVES][3];
      const TopRow t = read_top<T, THREADS>(teacher, row, tid, reinterpret_cast<int*>(lds) + (ROWS > 1 ? wave_of_group * top_words(teacher) : 0), sums);
      if (tid == 0) read_here[ROWS > 1 ? wave_of_group : 0] = t;
      if (WAVES > 1) __syncthreads();
      else __threadfence_block();
    }
  }
  auto top_row = [&]() { return a.top_rows ? a.top_rows[row] : read_here[ROWS > 1 ? wave_of_group : 0]; };
  const Cut<T> k(zr, a.vocab);
  const Raw* body = reinterpret_cast<const Raw*>(zr + k.head);
  // chunk j of a step, and whether this wavefront has one
  auto chunk = [&](int base, int j) { return base + j * THREADS + tid - k.lead; };
  auto there = [&](int base, int j) { return base + j * THREADS + wave * 64 - k.lead < k.body; };
  const TopEntry* entries = TOP ? a.entries + (size_t)row * a.top : nullptr;
  int col = -1;
  if (TOP && a.rest && tid < a.top) col = entries[tid].col;
  Raw v[CH];
  auto load = [&](int base, auto past) {
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int c = chunk(base, j);
      v[j] = splat<T>(NO_LOGIT);
      if (k.has(c)) {
        if (decltype(past)::value) v[j] = __builtin_nontemporal_load(body + c);
        else v[j] = body[c];
      }
    }
  };
  const Flag<!AGAIN && !STREAM> only_time;                     // a row that is read twice is to stay near in between
  load(0, only_time);
  const bool has_end = tid < k.ends;
  const int end_col = k.end_at(tid);
  float end = has_end ? to_f32(zr[end_col]) : NO_LOGIT;
  float zy = 0.f;
  if (!TOP && y >= 0) zy = to_f32(zr[y]);

  // With a rest, columns that have an entry are taken out of the row: the others' sum can be far smaller than theirs
  const bool take = TOP && a.rest;
  // a byte for each chunk, that of chunk c at c + 8; c = -1 and c = body stand for the ends
  unsigned* const columns_out = lds + (ROWS > 1 ? wave_of_group * (a.lds_bytes / 4) : 0);
  const unsigned char* const out_bytes = reinterpret_cast<const unsigned char*>(columns_out) + 8;
  auto all_here = [] {                                         // the threads of a row; LDS keeps a wavefront's order
    if (WAVES > 1) __syncthreads();
    else __threadfence_block();
  };
  if (take) {
    for (int i = tid; i < a.lds_bytes / 4; i += THREADS) columns_out[i] = 0;
    all_here();
    for (int i = tid;;) {
      if (col >= 0) {
        const int at = col - k.head, c = at < 0 ? -1 : min(at / N, k.body), e = at < 0 ? col : at - c * N;
        atomicOr(&columns_out[(c + 8) >> 2], 1u << (((c + 8) & 3) * 8 + e));
      }
      i += THREADS;
      if (i >= a.top) break;
      col = entries[i].col;
    }
    all_here();
    if (has_end && (end_col < k.head ? out_bytes[-1] >> end_col : out_bytes[k.body] >> (end_col - k.head - k.body * N)) & 1) end = NO_LOGIT;
  }
  // (a thread without a chunk has a byte nevertheless, and nothing but -inf to lose)
  auto take_out = [&](int base) {
    if (!take) return;
    unsigned on[CH];
#pragma unroll
    for (int j = 0; j < CH; j++) on[j] = out_bytes[chunk(base, j)];
#pragma unroll
    for (int j = 0; j < CH; j++) {
      if (on[j]) {
#pragma unroll
        for (int e = 0; e < N; e++)
          if (on[j] >> e & 1) v[j][e] = from_f32<T>(NO_LOGIT);
      }
    }
  };

  // maximum and sum of this thread's elements
  float m = end, s = end == NO_LOGIT ? 0.f : 1.f;
  if (end != end) s = end;                                     // NaN stays one
  for (int base = 0;;) {
    take_out(base);
    float top_here = m;
#pragma unroll
    for (int j = 0; j < CH; j++) {
      if (!there(base, j)) break;
#pragma unroll
      for (int e = 0; e < N; e++) top_here = fmaxf(top_here, to_f32(v[j][e]));
    }
    const float ref = reference(top_here);
    if (s != 0.f) s *= exp_scaled(m - ref, a.c_hi, a.c_lo);
    m = top_here;
#pragma unroll
    for (int j = 0; j < CH; j++) {
      if (!there(base, j)) break;
#pragma unroll
      for (int e = 0; e < N; e++) s += exp_scaled(to_f32(v[j][e]) - ref, a.c_hi, a.c_lo);
    }
    if (!STREAM) break;
    base += THREADS * CH;
    if (base >= k.body + k.lead) break;
    load(base, only_time);
  }
  Sums all;
  all.m = wave_max(m);
  all.s = wave_sum_f64(rescaled({m, (double)s}, all.m, a));
  if (WAVES > 1) {
    if (lane == 0) part[wave] = all;
    __syncthreads();
    all.m = part[0].m;
#pragma unroll
    for (int i = 1; i < WAVES; i++) all.m = fmaxf(all.m, part[i].m);
    all.s = 0.0;
#pragma unroll
    for (int i = 0; i < WAVES; i++) all.s += rescaled(part[i], all.m, a);
  }

  // the gradient is slope * exp(scale (z - ref)) of every element that has no value of its own
  const double scale = (double)a.scale;
  const double weight = (double)w;
  float ref = all.m, slope = 0.f, own = 0.f;                   // own: the gradient by logp
  double logp = 0.0, log_s = 0.0;
  float p_top = 0.f, ref_top = 0.f, mass = 0.f;                // TOP: p of an entry's column is p_top exp(scale (z - ref_top))
  bool others = false;                                         // TOP: whether there are columns without an entry
  if (TOP) {
    const TopRow t = top_row();
    others = a.rest && (all.m != NO_LOGIT || all.s != 0.0);
    const double r = others ? t.rest : 0.0, total = t.q_sum + r;
    const Sums row_sums = a.rest ? joined(all, t.own, a) : all;
    // total p - r exp(a - lse of the others), and what that is relative to the others' own sum
    slope = (float)(weight * scale * (total * rescaled(all, row_sums.m, a) / row_sums.s - r) / all.s);
    if (a.rest && !others && row_sums.s != 0.0) slope = 0.f;   // there is nothing to write, or zeros
    ref = reference(all.m);
    ref_top = row_sums.m;
    p_top = (float)(1.0 / row_sums.s);
    mass = (float)total;
  } else {
    own = -w;
    if (a.kind == POLICY) {                                    // (the others' logarithms can wait until the registers are free)
      log_s = log_f64(all.s);
      logp = scale * ((double)zy - (double)all.m) - log_s;
      own = w * policy_slope(a, logp, a.old_logp[row], a.kl != 0.f ? a.ref_logp[row] : 0.f, a.adv[row]);
    }
    if (y == INVALID) own = __builtin_nanf("");
    slope = (float)(-(double)own * scale / all.s);
  }

  if (dr) {
    const bool aligned = ((reinterpret_cast<uintptr_t>(dr) ^ reinterpret_cast<uintptr_t>(zr)) & 15) == 0;
    for (int base = 0;;) {
      if (STREAM) {
        load(base, Flag<true>());
        take_out(base);
      }
#pragma unroll
      for (int j = 0; j < CH; j++) {
        const int c = chunk(base, j);
        if (!k.has(c)) continue;
        float x[N];
#pragma unroll
        for (int e = 0; e < N; e++) x[e] = slope * exp_gradient<T>(to_f32(v[j][e]) - ref, a.c_hi, a.c_lo);
        store_chunk(dr + k.head + (size_t)c * N, x, aligned);
      }
      if (!STREAM) break;
      base += THREADS * CH;
      if (base >= k.body + k.lead) break;
    }
    if (has_end && (TOP || end_col != y)) dr[end_col] = from_f32<T>(slope * exp_scaled(end - ref, a.c_hi, a.c_lo));
  }

  if (TOP) {
    const TopRow t = top_row();
    if (tid == 0) {
      const double r = others ? t.rest : 0.0, log_all = log_sum(a.rest ? joined(all, t.own, a) : all, a);
      double l = t.terms;
      if (t.q_sum != 0.0) l += t.q_sum * (log_all - scale * (double)reference(t.own.m));
      if (r > 0.0) l += r * (log_f64(r) - (log_sum(all, a) - log_all));
      a.loss[row] = (float)(weight * l);
    }
    if (!dr) return;
    all_here();                                                // (the chunks are stored)
    const float ws = w * a.scale;
    for (int i = tid; i < a.top; i += THREADS) {
      const TopEntry e = entries[i];
      if (e.col >= 0) dr[e.col] = from_f32<T>(ws * (mass * p_top * exp_scaled(e.z - ref_top, a.c_hi, a.c_lo) - e.q));
    }
    return;
  }
  // the thread that has stored the chunk around y, or could have: it overwrites y after that
  const int at = y - k.head, by_end = at < 0 ? y : at - k.body * N + k.head;
  const int y_tid = y < 0 ? -1 : at >= 0 && at < k.body * N ? (at / N + k.lead) % THREADS : by_end;
  if (tid != 0 && tid != y_tid) return;
  if (a.kind != POLICY) {
    log_s = log_f64(all.s);
    logp = scale * ((double)zy - (double)all.m) - log_s;
  }
  if (y == ELSEWHERE) logp = -(scale * (double)all.m + log_s);
  if (y == INVALID) logp = __builtin_nan("");
  if (dr && tid == y_tid) dr[y] = from_f32<T>(own * a.scale * -expm1f((float)logp));        // g scale (1 - p), without the difference
  if (tid > 0) return;
  if (a.logp) a.logp[row] = (float)logp;
  if (a.lse) a.lse[row] = (float)(scale * (double)all.m + log_s);
  if (a.logp64) {
    a.logp64[row] = logp;
    a.stats[row] = f32x2{all.m, (float)(1.0 / all.s)};
    a.counted[row] = w;
  }
  if (a.kind == TOKEN) a.loss[row] = (float)(-weight * logp);
  if (a.kind == POLICY) a.loss[row] = (float)(weight * policy_loss(a, logp, a.old_logp[row], a.kl != 0.f ? a.ref_logp[row] : 0.f, a.adv[row]));
}

// Pairs of sequences: sequence j's reward is beta times the sum of w (logp - ref) over its tokens, the pair's loss a function of the
// difference of two rewards, and a token's share of the gradient its weight times the pair's slope.
struct PairArgs {
  const void* logp;
  const float *ref, *weights, *pair_weights;
  const int* starts;
  float *loss, *rewards, *dlogp;
  int pairs, rows;
  float beta, margin, smoothing;
};
GX_DEVINL int start_of(const PairArgs& a, int i) { return min(max(a.starts[i], 0), a.rows); }

// A workgroup of 256 adds up a pair: two rewards, and the slope of its loss by the chosen sequence's log probability
struct Pair {
  int at[3];
  double reward[2], x, slope;
  float weight;
  template <typename L>
  GX_DEVINL void add_up(const PairArgs& a, int pair, double (*part)[4]) {
    const int tid = threadIdx.x;
#pragma unroll
    for (int h = 0; h < 3; h++) at[h] = start_of(a, 2 * pair + h);
#pragma unroll
    for (int h = 0; h < 2; h++) {
      double s = 0.0;
      for (int t = at[h] + tid; t < at[h + 1]; t += 256) {
        const float w = a.weights ? a.weights[t] : 1.f;
        if (w != 0.f) s += (double)w * ((double)static_cast<const L*>(a.logp)[t] - (a.ref ? (double)a.ref[t] : 0.0));
      }
      s = wave_sum_f64(s);
      if ((tid & 63) == 0) part[h][tid >> 6] = s;
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; h++) reward[h] = (double)a.beta * ((part[h][0] + part[h][1]) + (part[h][2] + part[h][3]));
    weight = a.pair_weights ? a.pair_weights[pair] : 1.f;
    x = reward[0] - reward[1] - (double)a.margin;
    // the derivative by x is smoothing - sigmoid(-x), formed without a difference of numbers near 1
    slope = (double)a.beta * (double)weight * ((double)a.smoothing - 1.0 / (1.0 + exp_f64(x)));
  }
  GX_DEVINL void write(const PairArgs& a, int pair) const {
    const double low = log1p(exp_f64(-fabs(x))), sm = (double)a.smoothing;       // low: -log sigmoid(|x|)
    const double l = (1.0 - sm) * (low + fmax(-x, 0.0)) + sm * (low + fmax(x, 0.0));
    a.loss[pair] = weight != 0.f ? (float)((double)weight * (x == x ? l : x)) : 0.f;
    if (a.rewards) {
      a.rewards[2 * pair] = (float)reward[0];
      a.rewards[2 * pair + 1] = (float)reward[1];
    }
  }
  GX_DEVINL float by_logp(const PairArgs& a, bool rejected, int t) const {
    const float w = a.weights ? a.weights[t] : 1.f;
    return w != 0.f && weight != 0.f ? (float)((rejected ? -slope : slope) * (double)w) : 0.f;
  }
};

// A workgroup to a pair, one more to the tokens of no sequence
template <typename L>
__global__ void __launch_bounds__(256) pairs_kernel(PairArgs a) {
  __shared__ double part[2][4];
  const int tid = threadIdx.x, pair = blockIdx.x;
  if (pair == a.pairs) {
    for (int t = tid; t < start_of(a, 0); t += 256) a.dlogp[t] = 0.f;
    for (int t = start_of(a, 2 * a.pairs) + tid; t < a.rows; t += 256) a.dlogp[t] = 0.f;
    return;
  }
  Pair p;
  p.add_up<L>(a, pair, part);
  if (tid == 0) p.write(a, pair);
  if (!a.dlogp) return;
#pragma unroll
  for (int h = 0; h < 2; h++)
    for (int t = p.at[h] + tid; t < p.at[h + 1]; t += 256) a.dlogp[t] = p.by_logp(a, h, t);
}

// dz = g scale (1_y - p) where p = f exp(c (u z - m)): m = lse of the whole vocabulary (u = scale, c = 1, f = 1), or what the row
// kernel has left (u = 1, c = scale, m the maximum, f = 1 / sum).  A workgroup takes 256 * CH chunks of a row.
// PAIRS: g comes from the row's pair, which each of its rows' workgroups adds up, and one more to a pair for the losses
struct GradArgs {
  const void* z;
  void* dz;
  long stride, grad_stride;
  int rows, vocab, parts;
  float scale, unit, c_hi, c_lo;
  Ids ids;
  const float *lse, *dlogp;
  const f32x2* stats;
};
template <typename T, int CH, bool PAIRS>
__global__ void __launch_bounds__(256) loss_grad_kernel(GradArgs a, std::conditional_t<PAIRS, PairArgs, None> pairs) {
  constexpr int N = Lanes<T>::N;
  typedef typename Lanes<T>::type Raw;
  // from the last row on: of logits that have just been read whole, the last ones may still be near
  const int tid = threadIdx.x, block = a.rows * a.parts - 1 - (int)blockIdx.x, row = block < 0 ? 0 : block / a.parts, part = block - row * a.parts;
  float dlogp = 0.f;
  if constexpr (PAIRS) {
    __shared__ double sums[2][4];
    __shared__ int found;
    Pair p;
    if (block < 0) {
      p.add_up<double>(pairs, -1 - block, sums);
      if (tid == 0) p.write(pairs, -1 - block);
      return;
    }
    if (tid == 0) found = -1;
    __syncthreads();
    for (int i = tid; i < 2 * pairs.pairs; i += 256)
      if (start_of(pairs, i) <= row && row < start_of(pairs, i + 1)) found = i;
    __syncthreads();
    const int of = found;
    if (of >= 0) {
      p.add_up<double>(pairs, of / 2, sums);
      dlogp = p.by_logp(pairs, of & 1, row);
    }
  } else {
    dlogp = a.dlogp[row];
  }
  const T* zr = static_cast<const T*>(a.z) + (size_t)row * a.stride;
  T* dr = static_cast<T*>(a.dz) + (size_t)row * a.grad_stride;
  const Cut<T> k(zr, a.vocab);
  const int y = a.ids.column(row, a.vocab), first = part * 256 * CH + tid - k.lead;
  float g = dlogp * a.scale;
  const bool aligned = ((reinterpret_cast<uintptr_t>(dr) ^ reinterpret_cast<uintptr_t>(zr)) & 15) == 0;
  const bool counts = y != IGNORED && g != 0.f;
  if (counts && y == INVALID) g = __builtin_nanf("");
  const f32x2 st = !counts ? f32x2{0.f, 0.f} : a.stats ? a.stats[row] : f32x2{a.lse[row], 1.f};
  const float slope = -g * st[1];
  auto at = [&](float z) { return slope * exp_gradient<T>(fmaf(z, a.unit, -st[0]), a.c_hi, a.c_lo); };
  Raw v[CH];
  if (counts) {
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int c = first + j * 256;
      if (k.has(c)) {
        const Raw* p = reinterpret_cast<const Raw*>(zr + k.head) + c;
        v[j] = __builtin_nontemporal_load(p);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < CH; j++) {
    const int c = first + j * 256;
    if (!k.has(c)) continue;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; e++) x[e] = 0.f;
    if (counts) {
#pragma unroll
      for (int e = 0; e < N; e++) {
        x[e] = at(to_f32(v[j][e]));
        if (k.head + c * N + e == y) x[e] += g;
      }
    }
    store_chunk(dr + k.head + (size_t)c * N, x, aligned);
  }
  if (part == 0 && tid < k.ends) {
    const int col = k.end_at(tid);
    dr[col] = from_f32<T>(counts ? at(to_f32(zr[col])) + (col == y ? g : 0.f) : 0.f);
  }
}

// ------------------------------------------------------------------------------- host
bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
gx_status launched() { return hipGetLastError() == hipSuccess ? GX_OK : GX_ERR_LAUNCH; }

bool finite(float x) { return x - x == 0.f; }

gx_status check(const gx_logits_cfg* c) {
  if (!c) return GX_ERR_NULL;
  if (c->dtype != GX_F32 && c->dtype != GX_BF16) return GX_ERR_DTYPE;
  if (c->id_bytes != 4 && c->id_bytes != 8) return GX_ERR_DTYPE;
  if (c->flags) return GX_ERR_FLAGS;
  const int64_t far = (int64_t)1 << 40;
  if (c->rows < 0 || c->rows > MAX_ROWS || c->vocab <= 0 || c->vocab > MAX_VOCAB || c->stride < c->vocab || c->stride > far ||
      c->grad_stride < c->vocab || c->grad_stride > far || !(c->scale >= MIN_SCALE && c->scale <= 1.f / MIN_SCALE) || c->first_id < 0 ||
      c->whole_vocab < 0 || c->whole_vocab > far || (c->whole_vocab && c->first_id + c->vocab > c->whole_vocab) ||
      (!c->whole_vocab && c->first_id))
    return GX_ERR_SHAPE;
  return GX_OK;
}
gx_status check_whole(const gx_logits_cfg* c) {
  const gx_status st = check(c);
  return st == GX_OK && (c->first_id || (c->whole_vocab && c->whole_vocab != c->vocab)) ? GX_ERR_SHAPE : st;
}
gx_status check(const gx_pairs_cfg* c) {
  if (!c) return GX_ERR_NULL;
  if (c->flags) return GX_ERR_FLAGS;
  if (c->pairs < 0 || c->pairs > MAX_PAIRS || c->rows < 0 || c->rows > MAX_ROWS || !finite(c->beta) || !finite(c->margin) ||
      !(c->smoothing >= 0.f && c->smoothing <= 1.f))
    return GX_ERR_SHAPE;
  return GX_OK;
}
gx_status check(const gx_distill_cfg* c) {
  if (!c) return GX_ERR_NULL;
  if (c->top_dtype != GX_F32 && c->top_dtype != GX_BF16) return GX_ERR_DTYPE;
  if (c->flags) return GX_ERR_FLAGS;
  return c->top <= 0 || c->top > MAX_TOP ? GX_ERR_SHAPE : GX_OK;
}
bool logits_misaligned(const gx_logits_cfg& c, const void* p) { return misaligned(p, c.dtype == GX_BF16 ? 2 : 4); }

Ids ids_of(const gx_logits_cfg& c, const void* ids) {
  return Ids{ids, c.id_bytes, (long)c.first_id, (long)(c.whole_vocab ? c.whole_vocab : c.vocab), (long)c.ignore_id};
}
// scale log2(e) as a sum of two positive numbers
void set_scale(float scale, float& hi, float& lo) {
  const double c = (double)scale * 1.4426950408889634074;
  hi = (float)c;
  if ((double)hi >= c) hi = nextafterf(hi, 0.f);
  lo = (float)(c - (double)hi);
}
// The most chunks of a row, with those between a border of 128 bytes and the first
int chunks_of(const gx_logits_cfg& c, const void* z, int64_t stride) {
  const bool whole_lines = !misaligned(z, 128) && stride * (c.dtype == GX_BF16 ? 2 : 4) % 128 == 0;
  return c.vocab / (c.dtype == GX_BF16 ? 8 : 4) + (whole_lines ? 0 : 7);
}
RowArgs row_args(const gx_logits_cfg& c, Kind kind, const void* logits, void* dlogits, const float* weights, float* loss) {
  RowArgs a = {};
  a.z = logits;
  a.dz = dlogits;
  a.stride = (long)c.stride;
  a.grad_stride = (long)c.grad_stride;
  a.rows = c.rows;
  a.vocab = c.vocab;
  a.kind = kind;
  a.scale = c.scale;
  set_scale(c.scale, a.c_hi, a.c_lo);
  a.weights = weights;
  a.loss = loss;
  return a;
}

// again: the logits are read once more right after this.
// Rows stay in registers while a workgroup has room for them: the fewest threads that hold one in 16 chunks each do best (8192
// rows of 8000 / 16384 / 32768, bf16 cross entropy with gradient: 256 threads 51 / 96 / 200 us, 512 threads 57 / 104 / 203; read twice 60 / 101 / 219), up to
// 512 columns or so a wavefront a row; 50001: 294, read twice 335; 131072: 1024 threads with nothing beside them on a compute unit
// 215, read twice 234.  With few rows, which do not fill the chip, more threads to a row (512 rows of 32000: 17 and 15 us).
// Log probabilities alone, and entries to look up, do better reading twice than with 1024 threads and their barriers: 118 and 99 us, 275 and
// 246.  The rule does not ask whether a gradient is wanted: a loss has the same bits with and without.
gx_status run_rows(const gx_logits_cfg& c, RowArgs a, bool again, hipStream_t s, const TopArgs& teacher = TopArgs{}) {
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  const bool bf = c.dtype == GX_BF16, top = a.kind == DISTILL;
  const int per_row = chunks_of(c, a.z, c.stride);
  bool refused = false;
  auto go = [&](auto kernel, int threads, int step, auto more) {
    const int rows = threads < 256 ? 256 / threads : 1;
    size_t lds = 0;
    if (top) {                                                 // one after the other in the same place
      a.lds_bytes = a.rest ? (per_row > 0 ? cdiv(per_row, step) : 1) * step + 16 : 0;
      lds = a.top_rows ? 0 : (size_t)rows * 4 * top_words(teacher);
      if (lds < (size_t)rows * a.lds_bytes) lds = (size_t)rows * a.lds_bytes;
    }
    if (lds > 65536 &&
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
      refused = true;
      return;
    }
    hipLaunchKernelGGL(kernel, dim3(cdiv(a.rows, rows)), dim3(threads < 256 ? 256 : threads), lds, s, a, more);
  };
  auto with = [&](auto threads, auto ch, auto stream) {
    constexpr int TH = decltype(threads)::value, CH = decltype(ch)::value;
    constexpr bool ST = decltype(stream)::value;
    auto run = [&](auto of_bf16, auto of_f32, auto more) { bf ? go(of_bf16, TH, TH * CH, more) : go(of_f32, TH, TH * CH, more); };
    if (top) run(loss_row_kernel<bf16, TH, CH, ST, true, false>, loss_row_kernel<float, TH, CH, ST, true, false>, teacher);
    else if (again) run(loss_row_kernel<bf16, TH, CH, ST, false, true>, loss_row_kernel<float, TH, CH, ST, false, true>, None());
    else run(loss_row_kernel<bf16, TH, CH, ST, false, false>, loss_row_kernel<float, TH, CH, ST, false, false>, None());
  };
  const Flag<false> held;
  const Flag<true> twice;
  if (per_row <= 256) with(Int<64>(), Int<4>(), held);
  else if (per_row <= 512) with(Int<64>(), Int<8>(), held);
  else if (per_row <= 1024) with(Int<256>(), Int<4>(), held);
  else if (per_row <= 2048) with(Int<256>(), Int<8>(), held);
  else if (per_row <= 4096 && a.rows >= 1024) with(Int<256>(), Int<16>(), held);
  else if (per_row <= 4096) with(Int<512>(), Int<8>(), held);
  else if (per_row <= 8192) with(Int<512>(), Int<16>(), held);
  else if (per_row <= 16384 && a.kind != SCORE) with(Int<1024>(), Int<16>(), held);
  else if (per_row <= 16384) with(Int<1024>(), Int<4>(), twice);
  else with(Int<512>(), Int<8>(), twice);
  return refused ? GX_ERR_LAUNCH : launched();
}

gx_status run_grad(const gx_logits_cfg& c, GradArgs a, const PairArgs* pairs, hipStream_t s) {
  constexpr int CH = 4;
  const bool bf = c.dtype == GX_BF16;
  a.stride = (long)c.stride;
  a.grad_stride = (long)c.grad_stride;
  a.rows = c.rows;
  a.vocab = c.vocab;
  a.scale = c.scale;
  const int chunks = chunks_of(c, a.z, c.stride);
  a.parts = chunks > 0 ? cdiv(chunks, 256 * CH) : 1;
  if ((long)c.rows * a.parts > MAX_GRID) return GX_ERR_SHAPE;
  const dim3 grid((unsigned)(c.rows * a.parts + (pairs ? pairs->pairs : 0)));
  auto go = [&](auto kernel, auto more) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, more); };
  if (pairs) bf ? go(loss_grad_kernel<bf16, CH, true>, *pairs) : go(loss_grad_kernel<float, CH, true>, *pairs);
  else bf ? go(loss_grad_kernel<bf16, CH, false>, None()) : go(loss_grad_kernel<float, CH, false>, None());
  return launched();
}

PairArgs pair_args(const gx_pairs_cfg& c, const gx_pairs_in& in, const float* weights, const void* logp, float* loss, float* rewards,
                   float* dlogp) {
  return PairArgs{logp, in.ref_logp, weights, in.pair_weights, in.starts, loss, rewards, dlogp, c.pairs, c.rows,
                  c.beta, c.margin, c.smoothing};
}
template <typename L>
gx_status run_pairs(const PairArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(pairs_kernel<L>, dim3(a.pairs + (a.dlogp ? 1 : 0)), dim3(256), 0, s, a);
  return launched();
}

gx_status check_pairs_in(const gx_pairs_cfg& c, const gx_pairs_in* in, const float* loss) {
  if (!in || !in->starts || (c.pairs > 0 && !loss)) return GX_ERR_NULL;
  if (misaligned(in->starts, 4) || misaligned(in->weights, 4) || misaligned(in->ref_logp, 4) || misaligned(in->pair_weights, 4) ||
      misaligned(loss, 4))
    return GX_ERR_ALIGN;
  return GX_OK;
}

// Scratch of the preference loss: per row the log probability, (maximum, 1 / sum), the weight and the gradient by logp
struct PreferenceScratch {
  size_t logp, stats, counted, dlogp, bytes;
};
PreferenceScratch preference_scratch(int rows) {
  const size_t n = ((size_t)rows + 15) & ~(size_t)15;
  return {0, 8 * n, 16 * n, 20 * n, 24 * n};
}

// Scratch of the distillation: what top_kernel leaves of every row's teacher
struct DistillScratch {
  size_t rows, entries, bytes;
};
DistillScratch distill_scratch(int rows, int top) {
  const size_t head = (size_t)rows * sizeof(TopRow);
  static_assert(sizeof(TopRow) % 8 == 0 && sizeof(TopEntry) == 16, "");
  const size_t entries = (head + 15) & ~(size_t)15;
  return {0, entries, entries + (size_t)rows * top * sizeof(TopEntry)};
}

}  // namespace

extern "C" {

gx_status gx_logp_fwd(const gx_logits_cfg* cfg, const void* logits, const void* ids, float* logp, float* lse, void* hip_stream) {
  const gx_status st = check(cfg);
  if (st != GX_OK) return st;
  if (cfg->rows == 0) return GX_OK;
  if (!logits || !ids || !logp) return GX_ERR_NULL;
  if (logits_misaligned(*cfg, logits) || misaligned(ids, cfg->id_bytes) || misaligned(logp, 4) || misaligned(lse, 4)) return GX_ERR_ALIGN;
  RowArgs a = row_args(*cfg, SCORE, logits, nullptr, nullptr, nullptr);
  a.ids = ids_of(*cfg, ids);
  a.logp = logp;
  a.lse = lse;
  return run_rows(*cfg, a, true, static_cast<hipStream_t>(hip_stream));
}

gx_status gx_logp_bwd(const gx_logits_cfg* cfg, const void* logits, const void* ids, const float* lse, const float* dlogp, void* dlogits,
                      void* hip_stream) {
  const gx_status st = check(cfg);
  if (st != GX_OK) return st;
  if (cfg->rows == 0) return GX_OK;
  if (!logits || !ids || !lse || !dlogp || !dlogits) return GX_ERR_NULL;
  if (logits_misaligned(*cfg, logits) || logits_misaligned(*cfg, dlogits) || misaligned(ids, cfg->id_bytes) || misaligned(lse, 4) ||
      misaligned(dlogp, 4))
    return GX_ERR_ALIGN;
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  GradArgs a = {};
  a.z = logits;
  a.dz = dlogits;
  a.unit = cfg->scale;
  set_scale(1.f, a.c_hi, a.c_lo);
  a.ids = ids_of(*cfg, ids);
  a.lse = lse;
  a.dlogp = dlogp;
  return run_grad(*cfg, a, nullptr, static_cast<hipStream_t>(hip_stream));
}

gx_status gx_token_loss(const gx_logits_cfg* cfg, const void* logits, const void* ids, const float* weights, float* loss, float* logp,
                        void* dlogits, void* hip_stream) {
  const gx_status st = check_whole(cfg);
  if (st != GX_OK) return st;
  if (cfg->rows == 0) return GX_OK;
  if (!logits || !ids || !loss) return GX_ERR_NULL;
  if (logits_misaligned(*cfg, logits) || logits_misaligned(*cfg, dlogits) || misaligned(ids, cfg->id_bytes) || misaligned(weights, 4) ||
      misaligned(loss, 4) || misaligned(logp, 4))
    return GX_ERR_ALIGN;
  RowArgs a = row_args(*cfg, TOKEN, logits, dlogits, weights, loss);
  a.ids = ids_of(*cfg, ids);
  a.logp = logp;
  return run_rows(*cfg, a, false, static_cast<hipStream_t>(hip_stream));
}

gx_status gx_policy_loss(const gx_logits_cfg* cfg, const gx_policy_cfg* policy, const gx_policy_in* in, const void* logits,
                         const void* ids, float* loss, float* logp, void* dlogits, void* hip_stream) {
  const gx_status st = check_whole(cfg);
  if (st != GX_OK) return st;
  if (!policy || !in) return GX_ERR_NULL;
  if (policy->flags) return GX_ERR_FLAGS;
  if (!(policy->clip_low >= 0.f && policy->clip_low <= 1.f) || !(policy->clip_high >= 0.f) || !finite(policy->clip_high) ||
      !(policy->kl >= 0.f) || !finite(policy->kl))
    return GX_ERR_SHAPE;
  if (cfg->rows == 0) return GX_OK;
  if (!logits || !ids || !loss || !in->old_logp || !in->advantages || (policy->kl > 0.f && !in->ref_logp)) return GX_ERR_NULL;
  if (logits_misaligned(*cfg, logits) || logits_misaligned(*cfg, dlogits) || misaligned(ids, cfg->id_bytes) ||
      misaligned(in->weights, 4) || misaligned(in->old_logp, 4) || misaligned(in->ref_logp, 4) || misaligned(in->advantages, 4) ||
      misaligned(loss, 4) || misaligned(logp, 4))
    return GX_ERR_ALIGN;
  RowArgs a = row_args(*cfg, POLICY, logits, dlogits, in->weights, loss);
  a.ids = ids_of(*cfg, ids);
  a.logp = logp;
  a.old_logp = in->old_logp;
  a.ref_logp = in->ref_logp;
  a.adv = in->advantages;
  a.low = policy->clip_low;
  a.high = policy->clip_high;
  a.kl = policy->kl;
  return run_rows(*cfg, a, false, static_cast<hipStream_t>(hip_stream));
}

gx_status gx_pairs_loss(const gx_pairs_cfg* pairs, const gx_pairs_in* in, const float* logp, float* loss, float* rewards, float* dlogp,
                        void* hip_stream) {
  gx_status st = check(pairs);
  if (st != GX_OK) return st;
  if (pairs->rows > 0 && !logp) return GX_ERR_NULL;
  st = check_pairs_in(*pairs, in, loss);
  if (st != GX_OK) return st;
  if (misaligned(logp, 4) || misaligned(rewards, 4) || misaligned(dlogp, 4)) return GX_ERR_ALIGN;
  if (pairs->pairs == 0 && (!dlogp || pairs->rows == 0)) return GX_OK;
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  return run_pairs<float>(pair_args(*pairs, *in, in->weights, logp, loss, rewards, dlogp), static_cast<hipStream_t>(hip_stream));
}

size_t gx_preference_workspace_bytes(const gx_logits_cfg* cfg) {
  return check_whole(cfg) == GX_OK ? preference_scratch(cfg->rows).bytes : 0;
}

gx_status gx_preference_loss(const gx_logits_cfg* cfg, const gx_pairs_cfg* pairs, const gx_pairs_in* in, const void* logits,
                             const void* ids, float* loss, float* rewards, void* dlogits, void* workspace, void* hip_stream) {
  gx_status st = check_whole(cfg);
  if (st == GX_OK) st = check(pairs);
  if (st != GX_OK) return st;
  if (pairs->rows != cfg->rows) return GX_ERR_SHAPE;
  st = check_pairs_in(*pairs, in, loss);
  if (st != GX_OK) return st;
  if (cfg->rows > 0 && (!logits || !ids || !workspace)) return GX_ERR_NULL;
  if (logits_misaligned(*cfg, logits) || logits_misaligned(*cfg, dlogits) || misaligned(ids, cfg->id_bytes) || misaligned(rewards, 4) ||
      misaligned(workspace, 16))
    return GX_ERR_ALIGN;
  if (pairs->pairs == 0 && (!dlogits || cfg->rows == 0)) return GX_OK;
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const PreferenceScratch l = preference_scratch(cfg->rows);
  char* ws = static_cast<char*>(workspace);
  RowArgs a = row_args(*cfg, SCORE, logits, nullptr, in->weights, nullptr);
  a.ids = ids_of(*cfg, ids);
  a.logp64 = reinterpret_cast<double*>(ws + l.logp);
  a.stats = reinterpret_cast<f32x2*>(ws + l.stats);
  a.counted = reinterpret_cast<float*>(ws + l.counted);
  float* dlogp = reinterpret_cast<float*>(ws + l.dlogp);
  if (cfg->rows > 0 && (st = run_rows(*cfg, a, dlogits != nullptr, s)) != GX_OK) return st;
  // few rows: the workgroups of their gradients add the pairs up themselves
  const bool few = dlogits && cfg->rows > 0 && cfg->rows <= FEW_ROWS && pairs->pairs <= FEW_PAIRS;
  const PairArgs p = pair_args(*pairs, *in, a.counted, a.logp64, loss, rewards, dlogits ? dlogp : nullptr);
  if (!few && (st = run_pairs<double>(p, s)) != GX_OK) return st;
  if (!dlogits || cfg->rows == 0) return GX_OK;
  GradArgs g = {};
  g.z = logits;
  g.dz = dlogits;
  g.unit = 1.f;
  set_scale(cfg->scale, g.c_hi, g.c_lo);
  g.ids = a.ids;
  g.stats = a.stats;
  g.dlogp = dlogp;
  return run_grad(*cfg, g, few ? &p : nullptr, s);
}

size_t gx_distill_workspace_bytes(const gx_logits_cfg* cfg, const gx_distill_cfg* distill) {
  return check_whole(cfg) == GX_OK && check(distill) == GX_OK ? distill_scratch(cfg->rows, distill->top).bytes : 0;
}

gx_status gx_distill_loss(const gx_logits_cfg* cfg, const gx_distill_cfg* distill, const gx_distill_in* in, const void* logits,
                          float* loss, void* dlogits, void* workspace, void* hip_stream) {
  gx_status st = check_whole(cfg);
  if (st == GX_OK) st = check(distill);
  if (st != GX_OK) return st;
  if (!in) return GX_ERR_NULL;
  if (cfg->rows == 0) return GX_OK;
  if (!logits || !loss || !in->top_ids || !in->top_logits || !workspace) return GX_ERR_NULL;
  if (logits_misaligned(*cfg, logits) || logits_misaligned(*cfg, dlogits) || misaligned(in->top_ids, cfg->id_bytes) ||
      misaligned(in->top_logits, distill->top_dtype == GX_BF16 ? 2 : 4) || misaligned(in->top_lse, 4) || misaligned(in->weights, 4) ||
      misaligned(loss, 4) || misaligned(workspace, 16))
    return GX_ERR_ALIGN;
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const DistillScratch l = distill_scratch(cfg->rows, distill->top);
  char* ws = static_cast<char*>(workspace);
  TopArgs t = {};
  t.z = logits;
  t.stride = (long)cfg->stride;
  t.rows = cfg->rows;
  t.vocab = cfg->vocab;
  t.top = distill->top;
  for (t.places = 64; t.places < 2 * t.top;) t.places *= 2;
  t.id_bytes = cfg->id_bytes;
  t.top_bf16 = distill->top_dtype == GX_BF16;
  t.scale = cfg->scale;
  t.ids = in->top_ids;
  t.logits = in->top_logits;
  t.lse = in->top_lse;
  t.weights = in->weights;
  t.out = reinterpret_cast<TopRow*>(ws + l.rows);
  t.entries = reinterpret_cast<TopEntry*>(ws + l.entries);
  RowArgs a = row_args(*cfg, DISTILL, logits, dlogits, in->weights, loss);
  a.top = distill->top;
  a.rest = in->top_lse != nullptr;
  a.entries = t.entries;
  if (t.rows > READ_HERE) {
    a.top_rows = t.out;
    const int rows = t.top <= 64 ? 4 : 1;                      // of a workgroup
    auto read = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(cdiv(t.rows, rows)), dim3(256), rows * 4 * (size_t)top_words(t), s, t); };
    if (rows == 4) cfg->dtype == GX_BF16 ? read(top_kernel<bf16, 64>) : read(top_kernel<float, 64>);
    else cfg->dtype == GX_BF16 ? read(top_kernel<bf16, 256>) : read(top_kernel<float, 256>);
    if ((st = launched()) != GX_OK) return st;
  }
  return run_rows(*cfg, a, false, s, t);
}

}  // extern "C"
