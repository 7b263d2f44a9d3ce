// Losses of logits with the logits' gradient: log probabilities of tokens and cross entropy, the clipped policy loss, the
// preference loss of pairs of sequences, distillation from a teacher's top logits.
//
// With a = scale z (a row of logits), p = exp(a - lse) and lse = log sum exp a, every one of them is a function of a row's lse and
// of a few of its logits, and its gradient is dz = -c p with a constant c of the row, but for those few logits.  So there is one
// row kernel: it reads a row, keeps maximum and sum of exponentials of what a thread has met, joins them over the workgroup, forms
// the loss and c from them, and writes the gradient.  It is bound by memory: 8 bytes an element (fp32) or 4 (bf16) against
// about 20 instructions.
// The exponentials of a chunk are added up in fp32 as a tree, and from there on (sums over chunks and threads, log sums, losses) all is
// fp64, which costs nothing that could be measured: losses are small differences of log sums, and a sequence's reward adds up
// over thousands of tokens.  A log sum of 32768 logits (bf16) is off by 2e-8, and by 1e-9 at the mean.
//
// Measured, us (and TB/s of logits read and gradients written; a large copy moves 5.7), all rows counting, inputs of 1.2 GB in turn: cross
// entropy with gradient, bf16, 8192 x 32768 198 (5.4), 8192 x 50001 282 (5.8), 2048 x 131072 206 (5.2), 1024 x 262144, read twice, 236 (4.6),
// fp32 4096 x 32003 182 (5.8); 64 entries of a teacher, 8192 x 32768 212 (5.1), 2048 x 131072, read twice, 253 (4.2); preference
// loss, which reads twice, 8192 x 32768 264 (6.1, the second time in part from caches).  Small rows are bound by the instructions that every
// row costs (16384 x 1000 19, 3.4; 64 entries 42), few rows by latency (64 x 32000 8.4).  Below, figures next to a choice are both sides
// of it in one run, of the code as it was then; runs differ by up to 4 %.
#include "../../include/gx.h"
#include "gx_kernels.h"
#include <algorithm>
#include <type_traits>

namespace {

using namespace gx;

// Limits of the interface.  Rows times 1024 threads, and workgroups of 256 threads, are launches of less than 2^32 threads
constexpr int MAX_ROWS = 1 << 21, MAX_VOCAB = 1 << 19, MAX_TOP = 1024, MAX_PAIRS = 1 << 20;
constexpr long MAX_GRID = (1 << 24) - 1;
// So few rows and pairs that a launch of its own for the pairs takes longer than adding them up for every row (131 rows of 1001 15.4 us,
// 19 with the launch; 1001 rows of 5003 16.0, and 1025, with the launch, 18.9).  The rule does not ask for the length of rows: each of the
// workgroups of a long one adds its pair up before it asks for logits (1024 rows of 262144 304, and 2048 of 131072, with the launch, 271)
constexpr int FEW_ROWS = 1024, FEW_PAIRS = 256;
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

// A constant in scalar registers: of vector registers the series' coefficients took so many that a compute unit had a workgroup less
GX_DEVINL double scalar(double x) {
  asm("" : "+s"(x));
  return x;
}
// Exponential and logarithm in fp64, to about 2^-50 (the exponential for |x| up to 25; log(2) is one number whose rounding counts n times, so
// that it is off by 3e-14 at 700): a power of two, and a series in what is left of it (of exp up to the 12th power for
// |r| <= log(2) / 2, of log m = 2 atanh((m - 1) / (m + 1)) up to the 19th for m between sqrt(1/2) and sqrt(2)).  Every
// wavefront of a row computes a few of them: a quarter of the instructions of a library's.
GX_DEVINL double exp_f64(double x) {
  const double c = fmin(fmax(x, -1100.0), 1100.0), n = rint(c * 1.4426950408889634074), r = fma(n, -0.69314718055994530942, c);
  double p = 1.0 / 479001600.0;
  const double coef[12] = {1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0,
                           1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
  for (int i = 0; i < 12; i++) p = fma(p, r, scalar(coef[i]));
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
  for (int k = 17; k > 0; k -= 2) p = fma(p, t2, scalar(2.0 / k));
  return x == 0.0 ? -(double)INFINITY : fma((double)n, 0.69314718055994530942, p * t);
}

// Maximum and sum of exponentials (relative to the maximum) of a set of logits; the empty set has -inf and 0
struct Sums {
  float m;
  double s;
};

// What a row's teacher says: the sum of q; of q log q; 1 - sum of q, or 0.  An entry: its column, or -1, and its q.
struct TopRow {
  double q_sum, terms, rest;
};
struct TopEntry {
  double q;
  int col, pad;
};

struct None {};
__device__ const f32x4 something = {0.f, 0.f, 0.f, 0.f};       // 16 bytes that can be read

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
  int top, rest, words, lds_bytes;                             // words of marks to a thread; LDS of a row
};

// exp(scale d) for d = z - maximum.  c_lo: the rounding of the constant would shift every term of a sum the same way; the two products
// are rounded as one sum, for the same reason.  c_lo is positive, so that d = -inf gives 0.
GX_DEVINL float exp_scaled(float d, float c_hi, float c_lo) { return __builtin_amdgcn_exp2f(fmaf(d, c_hi, d * c_lo)); }

// the same for a gradient of type T: of bf16 the constant's low part would be lost
template <typename T>
GX_DEVINL float exp_gradient(float d, float c_hi, float c_lo) {
  return sizeof(T) == 2 ? __builtin_amdgcn_exp2f(d * c_hi) : exp_scaled(d, c_hi, c_lo);
}

// What N lanes have together (up to 16: of the first N, in lane order of no account), and what all 64 have, the same in every lane.  Lanes
// exchange in registers (neighbours, pairs, mirrored halves and rows of 16), and the four rows of 16 through scalar registers: an exchange
// through LDS is a round trip of some 100 cycles, and a row has about 40 of them one after another.
template <int CTRL> GX_DEVINL int crossed(int x) { return __builtin_amdgcn_update_dpp(x, x, CTRL, 0xf, 0xf, false); }
template <int CTRL> GX_DEVINL float crossed(float x) { return __builtin_bit_cast(float, crossed<CTRL>(__builtin_bit_cast(int, x))); }
template <int CTRL> GX_DEVINL double crossed(double x) {
  const unsigned long u = __builtin_bit_cast(unsigned long, x);
  const unsigned lo = crossed<CTRL>((int)u), hi = crossed<CTRL>((int)(u >> 32));
  return __builtin_bit_cast(double, (unsigned long)hi << 32 | lo);
}
GX_DEVINL float of_lane(float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); }
GX_DEVINL double of_lane(double x, int lane) {
  const unsigned long u = __builtin_bit_cast(unsigned long, x);
  const unsigned lo = __builtin_amdgcn_readlane((int)u, lane), hi = __builtin_amdgcn_readlane((int)(u >> 32), lane);
  return __builtin_bit_cast(double, (unsigned long)hi << 32 | lo);
}
template <int N, typename V, typename F>
GX_DEVINL V of_lanes(V v, F f) {
  static_assert(N == 64 || N == 16 || N == 8 || N == 4);
  v = f(v, crossed<0xB1>(v));                                  // lane ^ 1
  v = f(v, crossed<0x4E>(v));                                  // lane ^ 2
  if (N > 4) v = f(v, crossed<0x141>(v));                      // 7 - lane of 8
  if (N > 8) v = f(v, crossed<0x140>(v));                      // 15 - lane of 16
  return N < 64 ? of_lane(v, 0) : f(f(of_lane(v, 0), of_lane(v, 16)), f(of_lane(v, 32), of_lane(v, 48)));
}
template <int N> GX_DEVINL float max_of_lanes(float v) {
  return of_lanes<N>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int N> GX_DEVINL double sum_of_lanes(double v) {
  return of_lanes<N>(v, [](double a, double b) { return a + b; });
}

GX_DEVINL float reference(float m) { return m == NO_LOGIT ? 0.f : m; }
// exp(scale d) to 2^-32: there are few different maxima in a row of bf16, so that errors of the factors between them would not
// average out as those of a sum's terms do.  The series as in exp_f64, up to the 8th power.
GX_DEVINL double exp_exact(float d, const RowArgs& a) {
  if (d == NO_LOGIT) return 0.0;
  const double x = fmax((double)a.scale * (double)d, -1100.0), n = rint(x * 1.4426950408889634074), r = fma(n, -0.69314718055994530942, x);
  double p = 1.0 / 40320.0;
  const double coef[8] = {1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
  for (int i = 0; i < 8; i++) p = fma(p, r, scalar(coef[i]));
  return d == d ? ldexp(p, (int)n) : (double)d;
}
GX_DEVINL double rescaled(Sums x, float m, const RowArgs& a) { return x.s == 0.0 ? 0.0 : x.s * exp_exact(x.m - m, a); }
template <int N>
GX_DEVINL Sums joined_lanes(Sums x, const RowArgs& a) {
  const float m = max_of_lanes<N>(x.m);
  return {m, sum_of_lanes<N>(rescaled(x, m, a))};
}
GX_DEVINL float of_first_lane(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }
GX_DEVINL double of_first_lane(double x) {
  const unsigned long u = __builtin_bit_cast(unsigned long, x);
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)u), hi = __builtin_amdgcn_readfirstlane((unsigned)(u >> 32));
  return __builtin_bit_cast(double, (unsigned long)hi << 32 | lo);
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
GX_DEVINL void store_chunk(T* p, typename Lanes<T>::type v, bool aligned) {
  typedef typename Lanes<T>::type Raw;
  if (aligned) {
    __builtin_nontemporal_store(v, reinterpret_cast<Raw*>(p));
  } else {                                                     // a gradient whose rows lie otherwise than the logits'
#pragma unroll
    for (int e = 0; e < Lanes<T>::N; e++) p[e] = v[e];
  }
}
template <typename T>
GX_DEVINL typename Lanes<T>::type rounded(const float (&x)[Lanes<T>::N]) {
  typename Lanes<T>::type v;
#pragma unroll
  for (int e = 0; e < Lanes<T>::N; e++) v[e] = from_f32<T>(x[e]);
  return v;
}
// Where the bits of `on` are set those of a, elsewhere those of b
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
template <typename Raw>
GX_DEVINL Raw chosen(u32x4 on, Raw a, Raw b) {
  const u32x4 x = __builtin_bit_cast(u32x4, a), y = __builtin_bit_cast(u32x4, b);
  return __builtin_bit_cast(Raw, (on & x) | (~on & y));
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
  if (logp != logp) return logp;                               // no such token, or no distribution: whatever the advantage
  const double r = exp_f64(logp - (double)old);
  double l = 0.0;
  if (adv != 0.f) {
    const double cut = fmin(fmax(r, 1.0 - (double)a.low), 1.0 + (double)a.high), gain = r * (double)adv;
    l = gain <= cut * (double)adv ? -gain : -cut * (double)adv;
    if (r != r) l = r;
  }
  if (a.kl != 0.f) {
    const double d = (double)ref - logp;
    const double e = exp_f64(d);
    l += (double)a.kl * (e == (double)INFINITY ? e : e - d - 1.0);
  }
  return l;
}

// Reads a row's teacher with THREADS threads, in fp64.
// An index that comes twice is one column with two entries; the first of them stands for the column, with the sum of their q.
// Whether there is such an index is asked of a table of at least twice as many places as entries (so that a search ends), and only
// then entries are compared with all others.
struct TopArgs {
  int rows, vocab, top, places, id_bytes, top_bf16;
  float scale;
  const void *ids, *logits;
  const float *lse, *weights;
  TopRow* out;
  TopEntry* entries;
};
__host__ __device__ inline int top_words(const TopArgs& a) { return a.places + 4 * a.top; }       // of LDS for a row

template <int THREADS>
GX_DEVINL TopRow read_top(const TopArgs& a, int row, int tid, double* lds, double (*part)[2]) {
  constexpr int WAVES = THREADS / 64;
  const int wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  auto all_here = [] {
    if (WAVES > 1) __syncthreads();
    else __threadfence_block();
  };
  double* const qs = lds;
  int* const cols = reinterpret_cast<int*>(qs + a.top);
  int* const table = cols + 2 * a.top;
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
  const int col0 = tid < a.top ? column(tid) : -1;
  const float t0 = tid < a.top ? teacher(tid) : 0.f;
  auto t_of = [&](int i) { return i == tid ? t0 : teacher(i); };
  for (int i = tid; i < a.places; i += THREADS) table[i] = -1;
  all_here();
  float mt = NO_LOGIT;
  int again = 0;
  for (int i = tid; i < a.top; i += THREADS) {
    const int col = i == tid ? col0 : column(i);
    cols[i] = col;
    if (col < 0) continue;
    mt = fmaxf(mt, t_of(i));
    for (unsigned at = (unsigned)col * 2654435761u;; at++) {
      const int there = atomicCAS(&table[at & (a.places - 1)], -1, col);
      if (there == col) again = 1;
      if (there == col || there == -1) break;
    }
  }
  again = __any(again);
  if (!a.lse) mt = max_of_lanes<64>(mt);
  if (WAVES > 1) {
    if ((tid & 63) == 0) {
      part[wave][0] = (double)mt;
      part[wave][1] = (double)again;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < WAVES; k++) {
      mt = fmaxf(mt, (float)part[k][0]);
      again |= part[k][1] != 0.0;
    }
    __syncthreads();
  } else {
    __threadfence_block();
  }
  // q = e / total: the entries' own exponentials, or those by the teacher's log sum
  const double scale = (double)a.scale, lse = a.lse ? (double)a.lse[row] : scale * (double)mt;
  double sums[2] = {0.0, 0.0};
  for (int i = tid; i < a.top; i += THREADS) {
    if (cols[i] < 0) continue;
    const double x = scale * (double)t_of(i) - lse, e = exp_f64(x);
    qs[i] = e;
    sums[0] += e;
    if (e != 0.0) sums[1] += e * x;
  }
#pragma unroll
  for (int n = 0; n < 2; n++) {
    sums[n] = sum_of_lanes<64>(sums[n]);
    if (WAVES > 1 && (tid & 63) == 0) part[wave][n] = sums[n];
  }
  all_here();
  if (WAVES > 1) {
#pragma unroll
    for (int n = 0; n < 2; n++) {
      sums[n] = 0.0;
#pragma unroll
      for (int k = 0; k < WAVES; k++) sums[n] += part[k][n];
    }
  }
  const double total = a.lse || sums[0] == 0.0 ? 1.0 : sums[0], by = 1.0 / total;
  for (int i = tid; i < a.top; i += THREADS) {
    int col = cols[i];
    double q = col < 0 ? 0.0 : qs[i];
    if (again && col >= 0) {
      for (int j = 0; j < i; j++)
        if (cols[j] == cols[i]) col = -1;
      for (int j = i + 1; j < a.top; j++)
        if (cols[j] == cols[i]) q += qs[j];
    }
    entries[i] = {q * by, col, 0};
  }
  // sum of q log q = sum of (e / total) (x - log total)
  return {sums[0] * by, sums[1] * by - (total == 1.0 ? 0.0 : sums[0] * by * log_f64(total)), a.lse ? fmax(0.0, 1.0 - sums[0]) : 0.0};
}

// A row to a wavefront, or for more than 64 entries to a workgroup
template <int THREADS>
__global__ void __launch_bounds__(256) top_kernel(TopArgs a) {
  constexpr int ROWS = 256 / THREADS;
  extern __shared__ double lds_top[];
  __shared__ double part[4][2];
  const int of_group = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x * ROWS + of_group, tid = ROWS == 1 ? threadIdx.x : threadIdx.x & 63;
  if (row >= a.rows) return;
  if (a.weights && a.weights[row] == 0.f) return;              // nobody reads its record
  const TopRow t = read_top<THREADS>(a, row, tid, lds_top + of_group * (top_words(a) / 2), part);
  if (tid == 0) a.out[row] = t;
}

// LDS of a row's entries: two chunks to a slot, the ends' numbers, marks and slots of the threads
__host__ __device__ inline int top_bytes(int top, int words, int threads) {
  return (32 * (top + 1) + 64 + 4 * (words * threads + 2 + threads) + 15) & ~15;
}

// A row to a workgroup of THREADS, or with 64 one to each of a workgroup's four wavefronts.  A thread has CH chunks in flight; with
// STREAM as many of those steps as the row needs, and reads them again for the gradient, without it one.  Entries have barriers to wait at,
// so a compute unit is to have three workgroups of 512 (8192 x 32768, 64 entries, 220 us; with two, 248).
template <typename T, int THREADS, int CH, bool STREAM, bool TOP, bool AGAIN>
__global__ void __launch_bounds__(THREADS < 256 ? 256 : THREADS, TOP && CH <= 8 ? 6 : 4) loss_row_kernel(RowArgs a, std::conditional_t<TOP, TopArgs, None> teacher) {
  constexpr int N = Lanes<T>::N, WAVES = THREADS / 64, ROWS = THREADS < 256 ? 256 / THREADS : 1;
  typedef typename Lanes<T>::type Raw;
  extern __shared__ __attribute__((aligned(16))) char group_lds[];
  __shared__ Sums part[WAVES];
  const int wave_of_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = ROWS == 1 ? blockIdx.x : blockIdx.x * ROWS + wave_of_group;
  if (ROWS > 1 && row >= a.rows) return;
  const int tid = ROWS == 1 ? threadIdx.x : lane, wave = ROWS == 1 ? wave_of_group : 0;
  char* const lds = group_lds + (ROWS > 1 ? wave_of_group * a.lds_bytes : 0);          // the row's own
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
      __shared__ double sums[WAVES][2];
      const TopRow t = read_top<THREADS>(teacher, row, tid, reinterpret_cast<double*>(lds), sums);
      if (tid == 0) read_here[ROWS > 1 ? wave_of_group : 0] = t;
      if (WAVES > 1) __syncthreads();
      else __threadfence_block();
    }
  }
  auto top_row = [&]() { return a.top_rows ? a.top_rows[row] : read_here[ROWS > 1 ? wave_of_group : 0]; };
  const Cut<T> k(zr, a.vocab);
  // Loads are without branches (a thread beyond the row's ends reads its first or last chunk, and of a row without a chunk something
  // else), so that it is known at each use how many are still under way.
  const Raw* body = k.body > 0 ? reinterpret_cast<const Raw*>(zr + k.head) : reinterpret_cast<const Raw*>(&something);
  const int last = max(k.body - 1, 0);
  Raw v[CH];
  // chunk j of a step, and whether this wavefront has one
  auto chunk = [&](int base, int j) { return base + j * THREADS + tid - k.lead; };
  auto blank = [&](int base) {                                 // what is beyond the ends
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int first = base + j * THREADS + wave * 64 - k.lead;
      if (first >= 0 && first + 64 <= k.body) continue;
      if (!k.has(chunk(base, j))) v[j] = splat<T>(NO_LOGIT);
    }
  };
  auto there = [&](int base, int j) { return base + j * THREADS + wave * 64 - k.lead < k.body; };
  const TopEntry* entries = TOP ? a.entries + (size_t)row * a.top : nullptr;
  int col = -1;
  if (TOP) {
    col = entries[min(tid, a.top - 1)].col;
    if (tid >= a.top) col = -1;
  }
  auto load = [&](int base, auto past) {
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int c = min(max(chunk(base, j), 0), last);
      if (decltype(past)::value) v[j] = __builtin_nontemporal_load(body + c);
      else v[j] = body[c];
    }
  };
  const Flag<!AGAIN && !STREAM> only_time;                     // a row that is read twice is to stay near in between
  load(0, only_time);
  const bool has_end = tid < k.ends;
  const int end_col = k.end_at(tid);
  float end = has_end ? to_f32(zr[end_col]) : NO_LOGIT;
  float zy = 0.f;
  if (!TOP && y >= 0) zy = to_f32(zr[y]);

  auto all_here = [] {                                         // the threads of a row; LDS keeps a wavefront's order
    if (WAVES > 1) __syncthreads();
    else __threadfence_block();
  };
  // TOP: chunks with an entry's column are marked, bit by bit for the thread that has them, and have a slot in LDS: the bits of those
  // columns, and a chunk in which their logits go to the entries' threads and their gradients come back, so that they are stored
  // with the rest of their chunks.  (One by one they are a sector of memory each, read and written: 16 / 64 / 256 of 32768 columns,
  // 8192 rows, 214 / 223 / 334 us, so 210 / 215 / 239.)  Which slot is whose depends on the order in which threads ask, and nothing
  // else does.  All of it but the logits is there before the row is.
  u32x4* const columns = reinterpret_cast<u32x4*>(lds);
  Raw* const staged = reinterpret_cast<Raw*>(columns + a.top + 1);            // the last slot is for chunks without a column
  float* const end_value = reinterpret_cast<float*>(staged + a.top + 1);
  unsigned* const marks = reinterpret_cast<unsigned*>(end_value + 16);
  static_assert(CH <= 32);
  const int words = STREAM ? a.words : 1;
  unsigned* const end_marks = marks + words * THREADS;
  int* const slots = reinterpret_cast<int*>(end_marks + 2), *const slots_taken = slots - 1;
  // an entry's place: an end, or an element of a slot
  auto is_end = [&](int col) { return (unsigned)(col - k.head) >= (unsigned)(k.body * N); };
  auto end_of = [&](int col) { return col < k.head ? col : col - (k.vocab - k.ends); };
  auto element = [&](int col) {
    const int c = (col - k.head) / N + k.lead, owner = c % THREADS, n = c / THREADS;
    int slot = slots[owner];
    const int word = STREAM ? n >> 5 : 0;                      // a row in registers has one step of CH chunks, of 32 at most
#pragma unroll 1
    for (int i = 0; i < word; i++) slot += __popc(marks[i * THREADS + owner]);
    slot += __popc(marks[word * THREADS + owner] & ((1u << (n & 31)) - 1));
    return slot * N + (col - k.head) % N;
  };
  auto each_entry = [&](auto f) {
    for (int i = tid; i < a.top; i += THREADS) {
      if (i != tid) col = entries[i].col;
      if (col >= 0) f(i, col);
    }
    if (a.top > THREADS && tid < a.top) col = entries[tid].col;
  };
  if (TOP) {
    for (int i = tid; i < words * THREADS + 2; i += THREADS) marks[i] = 0;
    if (tid == 0) columns[a.top] = u32x4{0, 0, 0, 0};
    all_here();
    each_entry([&](int, int at) {
      if (is_end(at)) {
        atomicOr(end_marks, 1u << end_of(at));
      } else {
        const int c = (at - k.head) / N + k.lead, n = c / THREADS;
        atomicOr(&marks[(n >> 5) * THREADS + c % THREADS], 1u << (n & 31));
      }
    });
    all_here();
    int mine = 0;
#pragma unroll 1
    for (int i = 0; i < words; i++) mine += __popc(marks[i * THREADS + tid]);
    const int first = mine ? atomicAdd(slots_taken, mine) : 0;
    slots[tid] = first;
    for (int i = 0; i < mine; i++) columns[first + i] = u32x4{0, 0, 0, 0};
    all_here();
    each_entry([&](int, int at) {
      if (is_end(at)) return;
      if (sizeof(T) == 2) reinterpret_cast<unsigned short*>(columns)[element(at)] = 0xffff;
      else reinterpret_cast<unsigned*>(columns)[element(at)] = 0xffffffffu;
    });
    all_here();
    // no entry: nothing to learn, whatever the logits hold
    if (__builtin_amdgcn_readfirstlane((int)*end_marks | *slots_taken) == 0) {
      if (dr) clear_row(dr, a.vocab, tid, THREADS);
      if (tid == 0) a.loss[row] = 0.f;
      return;
    }
    if (has_end) end_value[tid] = end;
  }
  int slot = TOP ? slots[tid] : 0;
  // f(slot) for the thread's chunk of a step where any of the wavefront's chunks is marked
  auto if_marked = [&](int base, int j, auto f) {
    const int n = STREAM ? base / THREADS + j : j;
    const unsigned on = marks[(n >> 5) * THREADS + tid] >> (n & 31) & 1;
    if (!__any(on)) return;
    f(on ? slot : a.top);
    slot += on;
  };
  float most = TOP ? end : NO_LOGIT;                           // of what is taken out, and perhaps of others
  auto take_out = [&](int base) {
#pragma unroll
    for (int j = 0; j < CH; j++) {
      if (!there(base, j)) break;
      if_marked(base, j, [&](int here) {
        if (here != a.top) staged[here] = v[j];
        if (a.rest) {
#pragma unroll
          for (int e = 0; e < N; e++) most = fmaxf(most, to_f32(v[j][e]));
          v[j] = chosen(columns[here], splat<T>(NO_LOGIT), v[j]);
        }
      });
    }
  };

  // With a rest the columns that have an entry are taken out of the row: the others' sum can be far smaller than theirs
  if (TOP && has_end && a.rest && *end_marks >> tid & 1) end = NO_LOGIT;

  // The wavefront's maximum, and the sums of its threads relative to that: threads with maxima of their own would need an exponential
  // in fp64 each to join them
  float m = NO_LOGIT;
  double s = 0.0;
  for (int base = 0;;) {
    blank(base);
    if (TOP) take_out(base);
    float top_here = end;                                      // (the last that was asked for)
#pragma unroll
    for (int j = 0; j < CH; j++) {
      if (!there(base, j)) break;
#pragma unroll
      for (int e = 0; e < N; e++) top_here = fmaxf(top_here, to_f32(v[j][e]));
    }
    top_here = max_of_lanes<64>(STREAM ? fmaxf(m, top_here) : top_here);
    const float ref = reference(top_here);
    if (STREAM && m != top_here) s *= exp_exact(m - ref, a);
    m = top_here;
    // A chunk's exponentials are added up as a tree and the chunks in fp64: a divergence is a small difference of log sums, and a
    // reward the sum of many
#pragma unroll
    for (int j = 0; j < CH; j++) {
      if (!there(base, j)) break;
      float x[N];
#pragma unroll
      for (int e = 0; e < N; e++) x[e] = exp_scaled(to_f32(v[j][e]) - ref, a.c_hi, a.c_lo);
#pragma unroll
      for (int n = N / 2; n > 0; n >>= 1) {
#pragma unroll
        for (int e = 0; e < n; e++) x[e] += x[e + n];
      }
      s += (double)x[0];
    }
    if (!STREAM) break;
    base += THREADS * CH;
    if (base >= k.body + k.lead) break;
    load(base, only_time);
  }
  if (has_end) s += exp_exact(end - reference(m), a);
  Sums all = {m, sum_of_lanes<64>(s)};
  if (TOP && a.rest) most = max_of_lanes<64>(most);
  if constexpr (WAVES > 1) {
    __shared__ float most_part[TOP ? WAVES : 1];
    if (lane == 0) {
      part[wave] = all;
      if (TOP) most_part[wave] = most;
    }
    __syncthreads();
    if (TOP) most = max_of_lanes<WAVES>(lane < WAVES ? most_part[lane] : NO_LOGIT);
    all = joined_lanes<WAVES>(lane < WAVES ? part[lane] : Sums{NO_LOGIT, 0.0}, a);
  }
  all = {of_first_lane(all.m), of_first_lane(all.s)};          // (one register for all lanes)
  if (TOP) most = of_first_lane(most);

  // the gradient is slope * exp(scale (z - ref)) of every element that has no value of its own
  const double scale = (double)a.scale;
  const double weight = (double)w;
  float ref = all.m, slope = 0.f, own = 0.f;                   // own: the gradient by logp
  double logp = 0.0, log_s = 0.0;
  Sums row_sums = all;                                         // TOP with a rest: with the entries' columns
  double q_z = 0.0;                                            // TOP: sum of q z over the entries
  bool others = false;                                         // TOP: whether there are columns without an entry
  if (TOP) {
    const TopRow t = top_row();
    // sums over the entries: of q z, and with a rest of their columns' exponentials
    Sums taken = {fmaxf(most, all.m), 0.0};
    const float from = reference(taken.m);
    if (WAVES == 1) all_here();
    const T* const staged_values = reinterpret_cast<const T*>(staged);
    each_entry([&](int i, int at) {
      const float z = is_end(at) ? end_value[end_of(at)] : to_f32(staged_values[element(at)]);
      const double q = entries[i].q;
      if (q != 0.0) q_z += q * (double)z;
      if (a.rest) taken.s += exp_exact(z - from, a);
    });
    q_z = sum_of_lanes<64>(q_z);
    if (a.rest) taken.s = sum_of_lanes<64>(taken.s);
    if (WAVES > 1) {
      __shared__ double entries_part[WAVES][2];
      if (lane == 0) {
        entries_part[wave][0] = q_z;
        entries_part[wave][1] = taken.s;
      }
      __syncthreads();
      q_z = taken.s = 0.0;
      for (int i = 0; i < WAVES && 64 * i < a.top; i++) {      // no entry from there on
        q_z += entries_part[i][0];
        taken.s += entries_part[i][1];
      }
    }
    q_z = of_first_lane(q_z);
    taken.s = of_first_lane(taken.s);
    others = a.rest && (all.m != NO_LOGIT || all.s != 0.0);
    const double r = others ? t.rest : 0.0, total = t.q_sum + r;
    double of_others = all.s;                                  // their sum, relative to the row's maximum
    if (a.rest) {
      of_others = rescaled(all, taken.m, a);
      row_sums = {taken.m, of_others + taken.s};
    }
    // total p - r exp(a - lse of the others), and what that is relative to the others' own sum
    slope = of_first_lane((float)(weight * scale * (total * of_others / row_sums.s - r) / all.s));
    row_sums = {of_first_lane(row_sums.m), of_first_lane(row_sums.s)};
    if (a.rest && !others && row_sums.s != 0.0) slope = 0.f;   // there is nothing to write, or zeros
    ref = reference(all.m);
    if (dr) {
      const float mass_p = (float)(total / row_sums.s);
      const double ws = weight * scale;
      each_entry([&](int i, int at) {
        auto gradient = [&](float z) {
          return (float)(ws * ((double)(mass_p * exp_scaled(z - row_sums.m, a.c_hi, a.c_lo)) - entries[i].q));
        };
        if (is_end(at)) {
          float& z = end_value[end_of(at)];
          z = gradient(z);
        } else {
          T& z = reinterpret_cast<T*>(staged)[element(at)];
          z = from_f32<T>(gradient(to_f32(z)));
        }
      });
      all_here();
    }
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
    if (TOP) slot = slots[tid];
    for (int base = 0;;) {
      if (STREAM) load(base, Flag<true>());
#pragma unroll
      for (int j = 0; j < CH; j++) {
        const int c = chunk(base, j);
        if (!k.has(c)) continue;
        float x[N];
#pragma unroll
        for (int e = 0; e < N; e++) x[e] = slope * exp_gradient<T>(to_f32(v[j][e]) - ref, a.c_hi, a.c_lo);
        Raw d = rounded<T>(x);
        if (TOP) {
          if_marked(base, j, [&](int here) { d = chosen(columns[here], staged[here], d); });
        }
        store_chunk(dr + k.head + (size_t)c * N, d, aligned);
      }
      if (!STREAM) break;
      base += THREADS * CH;
      if (base >= k.body + k.lead) break;
    }
    if (has_end && (TOP || end_col != y)) {
      float x = slope * exp_scaled(end - ref, a.c_hi, a.c_lo);
      if (TOP && *end_marks >> tid & 1) x = end_value[tid];
      dr[end_col] = from_f32<T>(x);
    }
  }

  if (TOP) {
    if (tid > 0) return;
    const TopRow t = top_row();
    const double r = others ? t.rest : 0.0, log_all = log_sum(row_sums, a);
    double l = t.terms;
    if (t.q_sum != 0.0) l += t.q_sum * log_all - scale * q_z;
    if (r > 0.0) l += r * (log_f64(r) - (log_sum(all, a) - log_all));
    a.loss[row] = (float)(weight * l);
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
  const float lse = (float)(scale * (double)all.m + log_s);
  if (y == ELSEWHERE) logp = -(scale * (double)all.m + log_s);
  // a shard of nothing but -inf has no log sum to take from the token's logit, or to take from nothing
  if (a.ids.whole != a.vocab && lse == -INFINITY) logp = y == ELSEWHERE ? 0.0 : scale * (double)zy;
  if (y == INVALID) logp = __builtin_nan("");
  if (dr && tid == y_tid) dr[y] = from_f32<T>(own * a.scale * -expm1f((float)logp));        // g scale (1 - p), without the difference
  if (tid > 0) return;
  if (a.logp) a.logp[row] = (float)logp;
  if (a.lse) a.lse[row] = lse;
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
#pragma unroll 4
      for (int t = at[h] + tid; t < at[h + 1]; t += 256) {     // (loads that wait for nothing)
        const double logp = (double)static_cast<const L*>(a.logp)[t], ref = a.ref ? (double)a.ref[t] : 0.0;
        const float w = a.weights ? a.weights[t] : 1.f;
        s += w != 0.f ? (double)w * (logp - ref) : 0.0;
      }
      s = sum_of_lanes<64>(s);
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
    // x is infinite where a token of one sequence has probability 0: a part of factor 0 is none then either
    const double l = (sm < 1.0 ? (1.0 - sm) * (low + fmax(-x, 0.0)) : 0.0) + (sm > 0.0 ? sm * (low + fmax(x, 0.0)) : 0.0);
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
// kernel has left (u = 1, c = scale, m the maximum, f = 1 / sum).  A workgroup of 256 takes THREADS * CH chunks of each of 256 / THREADS rows.
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
  const double* logp;                                          // with stats: the tokens' log probabilities
};
template <typename T, int THREADS, int CH, bool PAIRS>
__global__ void __launch_bounds__(256) loss_grad_kernel(GradArgs a, std::conditional_t<PAIRS, PairArgs, None> pairs) {
  constexpr int N = Lanes<T>::N;
  typedef typename Lanes<T>::type Raw;
  // from the last row on: of logits that have just been read whole, the last ones may still be near
  static_assert(THREADS == 256 || (THREADS == 64 && !PAIRS));
  const int tid = THREADS == 256 ? threadIdx.x : threadIdx.x & 63;
  const int block = a.rows * a.parts - 1 - (THREADS == 256 ? (int)blockIdx.x : (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
  if (!PAIRS && block < 0) return;
  const int row = block < 0 ? 0 : block / a.parts, part = block - row * a.parts;
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
  const int y = a.ids.column(row, a.vocab), first = part * THREADS * CH + tid - k.lead;
  float g = dlogp * a.scale;
  const bool aligned = ((reinterpret_cast<uintptr_t>(dr) ^ reinterpret_cast<uintptr_t>(zr)) & 15) == 0;
  const bool counts = y != IGNORED && g != 0.f;
  if (counts && y == INVALID) g = __builtin_nanf("");
  const f32x2 st = !counts ? f32x2{0.f, 0.f} : a.stats ? a.stats[row] : f32x2{a.lse[row], 1.f};
  const float slope = -g * st[1];
  auto at = [&](float z) { return slope * exp_gradient<T>(fmaf(z, a.unit, -st[0]), a.c_hi, a.c_lo); };
  // g (1 - p) at the token, without the difference, which a p near 1 would leave nothing of
  auto at_token = [&](float z) { return -g * expm1f(a.logp ? (float)a.logp[row] : fmaf(z, a.unit, -st[0])); };
  Raw v[CH];
  if (counts) {
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int c = first + j * THREADS;
      if (k.has(c)) {
        const Raw* p = reinterpret_cast<const Raw*>(zr + k.head) + c;
        v[j] = __builtin_nontemporal_load(p);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < CH; j++) {
    const int c = first + j * THREADS;
    if (!k.has(c)) continue;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; e++) x[e] = 0.f;
    if (counts) {
#pragma unroll
      for (int e = 0; e < N; e++) x[e] = at(to_f32(v[j][e]));
    }
    store_chunk(dr + k.head + (size_t)c * N, rounded<T>(x), aligned);
  }
  // the thread that has stored the chunk around y overwrites y after that
  const int at_y = y - k.head;
  if (counts && at_y >= 0 && at_y < k.body * N) {
    float zy = 0.f;
    bool mine = false;
#pragma unroll
    for (int j = 0; j < CH; j++) {
      if (first + j * THREADS != at_y / N) continue;
      mine = true;
#pragma unroll
      for (int e = 0; e < N; e++) zy = at_y % N == e ? to_f32(v[j][e]) : zy;
    }
    if (mine) dr[y] = from_f32<T>(at_token(zy));
  }
  if (part == 0 && tid < k.ends) {
    const int col = k.end_at(tid);
    float x = 0.f;
    if (counts) {
      const float z = to_f32(zr[col]);
      x = col == y ? at_token(z) : at(z);
    }
    dr[col] = from_f32<T>(x);
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
      c->whole_vocab < 0 || c->whole_vocab > far || (c->whole_vocab && c->first_id > c->whole_vocab - c->vocab) ||
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

// again: the logits are read once more right after this, perhaps.
// Rows stay in registers while a workgroup has room for them, and up to 512 chunks a wavefront has one.  Cross entropy with gradient,
// bf16, us: 16384 rows of 1000, a wavefront with 4 / 8 chunks to a thread 18.1 / 18.6, 256 threads 37.5; 8192 rows of 4096 26.3, 256
// threads 28.6; of 8000, 256 threads with 4 / 8 chunks 47.1 / 47.5; of 16384, 256 threads with 8 / 16 90.6 / 93.4, read twice 99; of
// 32768, 512 threads with 8 196, 256 with 16 202, read twice 212; of 50001, 512 with 16 279, read twice 319; 2048 rows of
// 131072, 1024 threads with 16 210, read twice 231.
// Only the last shape has a compute unit for one row alone.  With a teacher's entries, whose barriers nothing hides there, and for
// log probabilities, which are not written, reading twice is better: 2048 x 131072, 64 entries, 253 and 274 us; log probabilities 96
// and 118.  (The rule does not ask whether a gradient is wanted: a loss has the same bits with and without.)
gx_status run_rows(const gx_logits_cfg& c, RowArgs a, bool again, hipStream_t s, const TopArgs& teacher = TopArgs{}) {
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  const bool bf = c.dtype == GX_BF16, top = a.kind == DISTILL;
  const int per_row = chunks_of(c, a.z, c.stride);
  bool refused = false;
  auto go = [&](auto kernel, int threads, auto more) {
    const int rows = threads < 256 ? 256 / threads : 1;
    size_t lds = 0;
    if (top) {                                                 // what reads the teacher and what keeps the entries, one after the other
      a.words = per_row > 0 ? cdiv(cdiv(per_row, threads), 32) : 1;
      a.lds_bytes = top_bytes(a.top, a.words, threads);
      if (!a.top_rows && a.lds_bytes < 4 * top_words(teacher)) a.lds_bytes = 4 * top_words(teacher);
      lds = (size_t)rows * a.lds_bytes;
    }
    if (lds > 65536 &&
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
      refused = true;
      return;
    }
    hipLaunchKernelGGL(kernel, dim3(cdiv(a.rows, rows)), dim3(threads < 256 ? 256 : threads), lds, s, a, more);
  };
  // which of them a shape has instances of: entries, a row that is read again
  auto with = [&](auto threads, auto ch, auto stream, auto has_top, auto has_again) {
    constexpr int TH = decltype(threads)::value, CH = decltype(ch)::value;
    constexpr bool ST = decltype(stream)::value;
    auto run = [&](auto of_bf16, auto of_f32, auto more) { bf ? go(of_bf16, TH, more) : go(of_f32, TH, more); };
    if constexpr (decltype(has_top)::value) {
      if (top) return run(loss_row_kernel<bf16, TH, CH, ST, true, false>, loss_row_kernel<float, TH, CH, ST, true, false>, teacher);
    }
    if constexpr (decltype(has_again)::value) {
      if (again) return run(loss_row_kernel<bf16, TH, CH, ST, false, true>, loss_row_kernel<float, TH, CH, ST, false, true>, None());
    }
    run(loss_row_kernel<bf16, TH, CH, ST, false, false>, loss_row_kernel<float, TH, CH, ST, false, false>, None());
  };
  const Flag<false> no;
  const Flag<true> yes;
  if (per_row <= 256) with(Int<64>(), Int<4>(), no, yes, yes);
  else if (per_row <= 512) with(Int<64>(), Int<8>(), no, yes, yes);
  else if (per_row <= 1024) with(Int<256>(), Int<4>(), no, yes, yes);
  else if (per_row <= 2048) with(Int<256>(), Int<8>(), no, yes, yes);
  else if (per_row <= 4096) with(Int<512>(), Int<8>(), no, yes, yes);
  else if (per_row <= 8192) with(Int<512>(), Int<16>(), no, yes, yes);
  else if (top || a.kind == SCORE) with(Int<512>(), Int<8>(), yes, yes, no);
  else if (per_row <= 16384) with(Int<1024>(), Int<16>(), no, no, no);
  else with(Int<1024>(), Int<4>(), yes, no, no);
  return refused ? GX_ERR_LAUNCH : launched();
}

// Pieces of 256 * GRAD_CH chunks that the gradient's workgroups cut a row into
constexpr int GRAD_CH = 4;
int grad_parts(const gx_logits_cfg& c, const void* z) { return std::max(1, cdiv(chunks_of(c, z, c.stride), 256 * GRAD_CH)); }
bool too_many_parts(const gx_logits_cfg& c, const void* z) { return (long)c.rows * grad_parts(c, z) > MAX_GRID; }

// Whether rows read their teachers in the launch that does the rest.  Many have a launch before it, which is quicker at it where workgroups
// wait for one another.  us, one launch and two, 64 entries, bf16: rows of a wavefront (1000 columns), 1024 of them 10.5 and 13.7, 16384
// 41.8 and 45.3 (256 entries, 65536 rows, 435 and 406); of 256 threads (8000), 2048 24.2 and 25.8, 4096 41.4 and 41.2; of 512 (32000), 512
// 20.0 and 21.9, 1024 35.2 and 32.5.  The rule does not ask for the number of entries; between 64 and 256 the sides of short rows come closer, and
// more than 256 were not timed.
bool reads_here(const gx_logits_cfg& c, const void* z) {
  const int per_row = chunks_of(c, z, c.stride);
  return c.rows <= (per_row <= 512 ? 1 << 15 : per_row <= 2048 ? 2048 : 512);
}

gx_status run_grad(const gx_logits_cfg& c, GradArgs a, const PairArgs* pairs, hipStream_t s) {
  constexpr int CH = GRAD_CH;
  const bool bf = c.dtype == GX_BF16;
  a.stride = (long)c.stride;
  a.grad_stride = (long)c.grad_stride;
  a.rows = c.rows;
  a.vocab = c.vocab;
  a.scale = c.scale;
  // short rows go one to a wavefront (the gradient of log probabilities, bf16: 16384 x 300 9.3 us, 19.3 with a workgroup each; x 1000 15.5
  // and 20.1)
  const bool wave = !pairs && chunks_of(c, a.z, c.stride) <= 64 * CH;
  a.parts = grad_parts(c, a.z);
  const dim3 grid((unsigned)(wave ? cdiv(c.rows, 4) : c.rows * a.parts + (pairs ? pairs->pairs : 0)));
  auto go = [&](auto kernel, auto more) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, more); };
  if (pairs) bf ? go(loss_grad_kernel<bf16, 256, CH, true>, *pairs) : go(loss_grad_kernel<float, 256, CH, true>, *pairs);
  else if (wave) bf ? go(loss_grad_kernel<bf16, 64, CH, false>, None()) : go(loss_grad_kernel<float, 64, CH, false>, None());
  else bf ? go(loss_grad_kernel<bf16, 256, CH, false>, None()) : go(loss_grad_kernel<float, 256, CH, false>, None());
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
  if (too_many_parts(*cfg, logits)) return GX_ERR_SHAPE;
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
  if (dlogits && too_many_parts(*cfg, logits)) return GX_ERR_SHAPE;
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
  if (cfg->rows > 0 && (st = run_rows(*cfg, a, true, s)) != GX_OK) return st;
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
  g.logp = a.logp64;
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
  if (!reads_here(*cfg, logits)) {
    a.top_rows = t.out;
    const int rows = t.top <= 64 ? 4 : 1;                      // of a workgroup
    auto read = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(cdiv(t.rows, rows)), dim3(256), rows * 4 * (size_t)top_words(t), s, t); };
    rows == 4 ? read(top_kernel<64>) : read(top_kernel<256>);
    if ((st = launched()) != GX_OK) return st;
  }
  return run_rows(*cfg, a, false, s, t);
}

}  // extern "C"
