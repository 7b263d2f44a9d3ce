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

namespace {

using namespace gx;

constexpr int MAX_ROWS = 1 << 21, MAX_VOCAB = 1 << 19, MAX_TOP = 1024, MAX_PAIRS = 1 << 20;
constexpr long MAX_GRID = (1 << 24) - 1;                       // workgroups of 256: a launch has less than 2^32 threads
constexpr float NO_LOGIT = -INFINITY, MIN_SCALE = 1.f / (1 << 20);

template <typename T> struct Lanes;                            // elements of 16 bytes
template <> struct Lanes<float> { static constexpr int N = 4; typedef f32x4 type; };
template <> struct Lanes<bf16> { static constexpr int N = 8; typedef bf16x8 type; };

// A row cut at the borders of 16 bytes: `head` elements before the first, `body` chunks, `tail` elements behind the last.  The
// elements at the ends (fewer than two chunks) go one to a thread.
template <typename T>
struct Cut {
  static constexpr int N = Lanes<T>::N;
  int head, body, ends, vocab;
  GX_DEVINL Cut(const void* row, int v) : vocab(v) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = min(v, (N - off) % N);
    body = (v - head) / N;
    ends = v - body * N;                                       // head and tail together
  }
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
  const void *top_ids, *top_logits;
  const float* top_lse;
  int top, top_id_bytes, top_bf16;
};

// exp(scale d) for d = z - maximum.  c_lo: the rounding of the constant would shift every term of a sum the same way.  It is
// positive, so that d = -inf gives 0.
GX_DEVINL float exp_scaled(float d, float c_hi, float c_lo) { return __builtin_amdgcn_exp2f(fmaf(d, c_lo, d * c_hi)); }

GX_DEVINL double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Maximum and sum of exponentials (relative to the maximum) of a set of logits; the empty set has -inf and 0
struct Sums {
  float m;
  double s;
};
GX_DEVINL float reference(float m) { return m == NO_LOGIT ? 0.f : m; }
GX_DEVINL double rescaled(Sums x, float m, const RowArgs& a) {
  return x.s == 0.0 ? 0.0 : x.s * (double)exp_scaled(x.m - m, a.c_hi, a.c_lo);
}
GX_DEVINL Sums joined(Sums x, Sums y, const RowArgs& a) {
  const float m = fmaxf(x.m, y.m);
  return {m, rescaled(x, m, a) + rescaled(y, m, a)};
}
GX_DEVINL double log_sum(Sums x, const RowArgs& a) { return (double)a.scale * (double)x.m + log(x.s); }

template <typename T>
GX_DEVINL void clear_row(T* row, int vocab, int tid, int threads) {
  typedef typename Lanes<T>::type Raw;
  const Cut<T> k(row, vocab);
  for (int c = tid; c < k.body; c += threads) reinterpret_cast<Raw*>(row + k.head)[c] = Raw{};
  if (tid < k.ends) row[k.end_at(tid)] = from_f32<T>(0.f);
}

template <typename T>
GX_DEVINL void store_chunk(T* p, const float (&x)[Lanes<T>::N], bool aligned) {
  typename Lanes<T>::type v;
#pragma unroll
  for (int e = 0; e < Lanes<T>::N; e++) v[e] = from_f32<T>(x[e]);
  if (aligned) {
    *reinterpret_cast<typename Lanes<T>::type*>(p) = v;
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
  const double r = exp(logp - (double)old);
  double l = 0.0;
  if (adv != 0.f) {
    const double cut = fmin(fmax(r, 1.0 - (double)a.low), 1.0 + (double)a.high), gain = r * (double)adv;
    l = gain <= cut * (double)adv ? -gain : -cut * (double)adv;
    if (r != r) l = r;
  }
  if (a.kl != 0.f) {
    const double d = (double)ref - logp;
    l += (double)a.kl * (exp(d) - d - 1.0);
  }
  return l;
}

// What a row's teacher says, in LDS: which columns have an entry (bit column - head + N), and the entries
struct Top {
  unsigned* mask;
  int* col;                                                    // -1: the entry does not count
  float *z, *t, *q;                                            // the student's logit, the teacher's scaled one, its probability
  struct Shared {
    double q_sum, terms, rest;                                 // sum of q; of q (log q - scale (z - m)); 1 - sum of q, or 0
    Sums k;                                                    // of the student's logits that have an entry
    int repeated;
  }* sh;
};
template <typename T>
GX_DEVINL int top_bit(const Cut<T>& k, int col) { return col - k.head + Lanes<T>::N; }
__host__ __device__ inline int top_words(int vocab) { return (vocab + 16) / 32 + 1; }
inline size_t top_lds(int vocab, int top) { return (size_t)4 * top_words(vocab) + 16 * (size_t)top + 64; }

GX_DEVINL int top_id(const RowArgs& a, long i) {
  const long id = a.top_id_bytes == 8 ? static_cast<const long*>(a.top_ids)[i] : static_cast<const int*>(a.top_ids)[i];
  return id >= 0 && id < a.vocab ? (int)id : -1;
}

// The first wavefront reads a row's entries.  An index that comes twice is one column with two entries: the first of them
// stands for the column.
template <typename T>
GX_DEVINL void read_top(const RowArgs& a, const Cut<T>& k, const T* zr, int row, int lane, const Top& t) {
  float mz = NO_LOGIT, mt = NO_LOGIT;
  int repeated = 0;
  for (int i = lane; i < a.top; i += 64) {
    const long at = (long)row * a.top + i;
    const int col = top_id(a, at);
    const float tl = a.top_bf16 ? (float)static_cast<const bf16*>(a.top_logits)[at] : static_cast<const float*>(a.top_logits)[at];
    t.col[i] = col;
    t.t[i] = tl;
    if (col < 0) continue;
    const float z = to_f32(zr[col]);
    t.z[i] = z;
    mz = fmaxf(mz, z);
    mt = fmaxf(mt, tl);
    const int bit = top_bit(k, col);
    repeated |= (atomicOr(&t.mask[bit >> 5], 1u << (bit & 31)) >> (bit & 31)) & 1;
  }
  repeated = __any(repeated);
  __threadfence_block();
  mz = wave_max(mz);
  mt = wave_max(mt);
  double lse;
  if (a.top_lse) {
    lse = (double)a.top_lse[row];
  } else {
    double s = 0.0;
    for (int i = lane; i < a.top; i += 64)
      if (t.col[i] >= 0) s += exp((double)a.scale * ((double)t.t[i] - (double)mt));
    lse = (double)a.scale * (double)mt + log(wave_sum_f64(s));
  }
  double q_sum = 0.0, terms = 0.0, sz = 0.0;
  for (int i = lane; i < a.top; i += 64) {
    const int col = t.col[i];
    if (col < 0) continue;
    const double logq = (double)a.scale * (double)t.t[i] - lse, q = exp(logq), az = (double)a.scale * ((double)t.z[i] - (double)reference(mz));
    q_sum += q;
    if (q != 0.0) terms += q * (logq - az);
    t.q[i] = (float)q;
    bool first = true;
    if (repeated)
      for (int j = 0; j < i; j++) first &= t.col[j] != col;
    if (first) sz += exp(az);
  }
  q_sum = wave_sum_f64(q_sum);
  terms = wave_sum_f64(terms);
  sz = wave_sum_f64(sz);
  if (lane == 0) *t.sh = {q_sum, terms, a.top_lse ? fmax(0.0, 1.0 - q_sum) : 0.0, {mz, sz}, repeated};
}

// A row to a workgroup of THREADS, or with 64 one to each of a workgroup's four wavefronts.  A thread has CH chunks in flight; with
// STREAM as many of those steps as the row needs, and reads them again for the gradient, without it one.
template <typename T, int THREADS, int CH, bool STREAM, bool TOP>
__global__ void __launch_bounds__(THREADS < 256 ? 256 : THREADS) loss_row_kernel(RowArgs a) {
  constexpr int N = Lanes<T>::N, WAVES = THREADS / 64, ROWS = THREADS < 256 ? 256 / THREADS : 1;
  static_assert(!TOP || ROWS == 1, "");
  typedef typename Lanes<T>::type Raw;
  extern __shared__ double lds[];
  __shared__ Sums part[WAVES];
  const int row = ROWS == 1 ? blockIdx.x : blockIdx.x * ROWS + (threadIdx.x >> 6);
  if (ROWS > 1 && row >= a.rows) return;
  const int tid = ROWS == 1 ? threadIdx.x : threadIdx.x & 63, lane = threadIdx.x & 63, wave = ROWS == 1 ? threadIdx.x >> 6 : 0;
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
  const Cut<T> k(zr, a.vocab);
  const Raw* body = reinterpret_cast<const Raw*>(zr + k.head);
  Raw v[CH];
  auto load = [&](int base) {
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int c = base + j * THREADS + tid;
      v[j] = splat<T>(NO_LOGIT);
      if (c < k.body) v[j] = body[c];
    }
  };
  load(0);
  const bool has_end = tid < k.ends;
  const int end_col = k.end_at(tid);
  float end = has_end ? to_f32(zr[end_col]) : NO_LOGIT;
  float zy = 0.f;
  if (!TOP && y >= 0) zy = to_f32(zr[y]);

  Top top;
  if (TOP) {
    top.sh = reinterpret_cast<Top::Shared*>(lds);
    top.mask = reinterpret_cast<unsigned*>(lds + 8);
    const int words = top_words(a.vocab);
    top.col = reinterpret_cast<int*>(top.mask + words);
    top.z = reinterpret_cast<float*>(top.col + a.top);
    top.t = top.z + a.top;
    top.q = top.t + a.top;
    for (int i = tid; i < words; i += THREADS) top.mask[i] = 0;
    __syncthreads();
    if (wave == 0) read_top(a, k, zr, row, lane, top);
    __syncthreads();
    if (has_end) {
      const int bit = top_bit(k, end_col);
      if (top.mask[bit >> 5] >> (bit & 31) & 1) end = NO_LOGIT;
    }
  }
  // with TOP, the logits that have an entry of their own are taken out
  auto take_out = [&](int base) {
    if (!TOP) return;
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int c = base + j * THREADS + tid;
      if (c >= k.body) continue;
      const int bit = (c + 1) * N;
      const unsigned on = top.mask[bit >> 5] >> (bit & 31) & ((1u << N) - 1);
      if (on) {
#pragma unroll
        for (int e = 0; e < N; e++)
          if (on >> e & 1) v[j][e] = from_f32<T>(NO_LOGIT);
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
    for (int j = 0; j < CH; j++)
#pragma unroll
      for (int e = 0; e < N; e++) top_here = fmaxf(top_here, to_f32(v[j][e]));
    const float ref = reference(top_here);
    if (s != 0.f) s *= exp_scaled(m - ref, a.c_hi, a.c_lo);
    m = top_here;
#pragma unroll
    for (int j = 0; j < CH; j++)
#pragma unroll
      for (int e = 0; e < N; e++) s += exp_scaled(to_f32(v[j][e]) - ref, a.c_hi, a.c_lo);
    if (!STREAM) break;
    base += THREADS * CH;
    if (base >= k.body) break;
    load(base);
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
  float ref = all.m, slope = 0.f;
  float own = 0.f;                                             // g scale
  float p_top = 0.f, ref_top = 0.f, mass = 0.f;                // TOP: p of an entry's column is p_top exp(scale (z - ref_top))
  if (TOP) {
    const Top::Shared sh = *top.sh;
    const bool others = all.m != NO_LOGIT || all.s != 0.0;     // columns without an entry
    const double r = others ? sh.rest : 0.0, total = sh.q_sum + r;
    const Sums row_sums = joined(all, sh.k, a);
    const double log_all = log_sum(row_sums, a);
    if (tid == 0 && a.loss) {
      double l = sh.terms + sh.q_sum * (log_all - (double)a.scale * (double)reference(sh.k.m));
      if (r > 0.0) l += r * (log(r) - (log_sum(all, a) - log_all));
      a.loss[row] = (float)((double)w * l);
    }
    if (!dr) return;
    // total p - r exp(a - lse of the others), and what that is relative to the others' own sum
    const double p_others = rescaled(all, row_sums.m, a) / row_sums.s;
    const double ws = (double)w * (double)a.scale;
    slope = others ? (float)(ws * (total * p_others - r) / all.s) : 0.f;
    ref = reference(all.m);
    ref_top = row_sums.m;
    p_top = (float)(1.0 / row_sums.s);
    mass = (float)total;
  } else {
    // of the cross entropy's wavefronts only the first has a use for it
    const double log_s = a.kind == TOKEN && wave > 0 ? 0.0 : log(all.s);
    double logp = (double)a.scale * ((double)zy - (double)all.m) - log_s;
    if (y == ELSEWHERE) logp = -((double)a.scale * (double)all.m + log_s);
    if (y == INVALID) logp = __builtin_nan("");
    if (tid == 0) {
      if (a.logp) a.logp[row] = (float)logp;
      if (a.lse) a.lse[row] = (float)((double)a.scale * (double)all.m + log_s);
      if (a.logp64) {
        a.logp64[row] = logp;
        a.stats[row] = f32x2{all.m, (float)(1.0 / all.s)};
        a.counted[row] = w;
      }
      if (a.kind == TOKEN) a.loss[row] = (float)(-(double)w * logp);
    }
    float g = -w;
    if (a.kind == POLICY) {
      const float old = a.old_logp[row], refp = a.kl != 0.f ? a.ref_logp[row] : 0.f, adv = a.adv[row];
      g = w * policy_slope(a, logp, old, refp, adv);
      if (tid == 0) a.loss[row] = (float)((double)w * policy_loss(a, logp, old, refp, adv));
    }
    if (!dr) return;
    if (y == INVALID) g = __builtin_nanf("");
    slope = (float)(-(double)g * (double)a.scale / all.s);
    own = g * a.scale;
  }
  // g scale (1 - p) at y, without the difference
  auto at_y = [&]() { return own * -expm1f((float)((double)a.scale * ((double)zy - (double)all.m) - log(all.s))); };

  const bool aligned = ((reinterpret_cast<uintptr_t>(dr) ^ reinterpret_cast<uintptr_t>(zr)) & 15) == 0;
  for (int base = 0;;) {
    if (STREAM) {
      load(base);
      take_out(base);
    }
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int c = base + j * THREADS + tid;
      if (c >= k.body) continue;
      float x[N];
#pragma unroll
      for (int e = 0; e < N; e++) x[e] = slope * exp_scaled(to_f32(v[j][e]) - ref, a.c_hi, a.c_lo);
      store_chunk(dr + k.head + (size_t)c * N, x, aligned);
    }
    if (!STREAM) break;
    base += THREADS * CH;
    if (base >= k.body) break;
  }
  if (has_end) {
    float x = slope * exp_scaled(end - ref, a.c_hi, a.c_lo);
    if (!TOP && end_col == y) x = at_y();
    dr[end_col] = from_f32<T>(x);
  }
  if (!TOP) {
    // by the thread that has stored the chunk around it, after that
    const int at = y - k.head;
    if (y >= k.head && at < k.body * N && (at / N) % THREADS == tid) dr[y] = from_f32<T>(at_y());
  } else {
    __syncthreads();                                           // the chunks are stored
    const float ws = w * a.scale;
    for (int i = tid; i < a.top; i += THREADS) {
      const int col = top.col[i];
      if (col < 0) continue;
      float q = top.q[i];
      if (top.sh->repeated) {                                  // the first entry of a column writes for all of them
        bool first = true;
        for (int j = 0; j < i; j++) first &= top.col[j] != col;
        if (!first) continue;
        for (int j = i + 1; j < a.top; j++)
          if (top.col[j] == col) q += top.q[j];
      }
      dr[col] = from_f32<T>(ws * (mass * p_top * exp_scaled(top.z[i] - ref_top, a.c_hi, a.c_lo) - q));
    }
  }
}

// dz = g scale (1_y - p) where p = f exp(c (u z - m)): m = lse of the whole vocabulary (u = scale, c = 1, f = 1), or what the row
// kernel has left (u = 1, c = scale, m the maximum, f = 1 / sum).  A workgroup takes 256 * CH chunks of a row.
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
template <typename T, int CH>
__global__ void __launch_bounds__(256) loss_grad_kernel(GradArgs a) {
  constexpr int N = Lanes<T>::N;
  typedef typename Lanes<T>::type Raw;
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts, tid = threadIdx.x;
  const T* zr = static_cast<const T*>(a.z) + (size_t)row * a.stride;
  T* dr = static_cast<T*>(a.dz) + (size_t)row * a.grad_stride;
  const Cut<T> k(zr, a.vocab);
  const int y = a.ids.column(row, a.vocab), first = part * 256 * CH;
  float g = a.dlogp[row] * a.scale;
  const bool aligned = ((reinterpret_cast<uintptr_t>(dr) ^ reinterpret_cast<uintptr_t>(zr)) & 15) == 0;
  const bool counts = y != IGNORED && g != 0.f;
  if (counts && y == INVALID) g = __builtin_nanf("");
  const f32x2 st = !counts ? f32x2{0.f, 0.f} : a.stats ? a.stats[row] : f32x2{a.lse[row], 1.f};
  const float slope = -g * st[1];
  auto at = [&](float z) { return slope * exp_scaled(fmaf(z, a.unit, -st[0]), a.c_hi, a.c_lo); };
  Raw v[CH];
  if (counts) {
#pragma unroll
    for (int j = 0; j < CH; j++) {
      const int c = first + j * 256 + tid;
      if (c < k.body) v[j] = reinterpret_cast<const Raw*>(zr + k.head)[c];
    }
  }
#pragma unroll
  for (int j = 0; j < CH; j++) {
    const int c = first + j * 256 + tid;
    if (c >= k.body) continue;
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

// Pairs of sequences: sequence j's reward is beta times the sum of w (logp - ref) over its tokens, the pair's loss a function of the
// difference of two rewards, and a token's share of the gradient its weight times the pair's slope.  A workgroup takes a pair, one
// more the tokens of no sequence.
struct PairArgs {
  const void* logp;
  const float *ref, *weights, *pair_weights;
  const int* starts;
  float *loss, *rewards, *dlogp;
  int pairs, rows;
  float beta, margin, smoothing;
};
template <typename L>
__global__ void __launch_bounds__(256) pairs_kernel(PairArgs a) {
  __shared__ double part[2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pair = blockIdx.x;
  auto start = [&](int i) { return min(max(a.starts[i], 0), a.rows); };
  if (pair == a.pairs) {
    for (int t = tid; t < start(0); t += 256) a.dlogp[t] = 0.f;
    for (int t = start(2 * a.pairs) + tid; t < a.rows; t += 256) a.dlogp[t] = 0.f;
    return;
  }
  const int at[3] = {start(2 * pair), start(2 * pair + 1), start(2 * pair + 2)};
#pragma unroll
  for (int h = 0; h < 2; h++) {
    double s = 0.0;
    for (int t = at[h] + tid; t < at[h + 1]; t += 256) {
      const float w = a.weights ? a.weights[t] : 1.f;
      if (w != 0.f) s += (double)w * ((double)static_cast<const L*>(a.logp)[t] - (a.ref ? (double)a.ref[t] : 0.0));
    }
    s = wave_sum_f64(s);
    if (lane == 0) part[h][wave] = s;
  }
  __syncthreads();
  double reward[2];
#pragma unroll
  for (int h = 0; h < 2; h++) reward[h] = (double)a.beta * ((part[h][0] + part[h][1]) + (part[h][2] + part[h][3]));
  const float pw = a.pair_weights ? a.pair_weights[pair] : 1.f;
  const double x = reward[0] - reward[1] - (double)a.margin, sm = (double)a.smoothing;
  if (tid == 0) {
    const double low = log1p(exp(-fabs(x)));                   // -log sigmoid(|x|)
    const double l = (1.0 - sm) * (low + fmax(-x, 0.0)) + sm * (low + fmax(x, 0.0));
    a.loss[pair] = pw != 0.f ? (float)((double)pw * l) : 0.f;
    if (a.rewards) {
      a.rewards[2 * pair] = (float)reward[0];
      a.rewards[2 * pair + 1] = (float)reward[1];
    }
  }
  if (!a.dlogp) return;
  // the derivative by x is smoothing - sigmoid(-x), formed without a difference of numbers near 1
  const double slope = (double)a.beta * (double)pw * (sm - 1.0 / (1.0 + exp(x)));
#pragma unroll
  for (int h = 0; h < 2; h++)
    for (int t = at[h] + tid; t < at[h + 1]; t += 256) {
      const float w = a.weights ? a.weights[t] : 1.f;
      a.dlogp[t] = w != 0.f && pw != 0.f ? (float)((h ? -slope : slope) * (double)w) : 0.f;
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

gx_status run_rows(const gx_logits_cfg& c, const RowArgs& a, hipStream_t s) {
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  const bool bf = c.dtype == GX_BF16, top = a.kind == DISTILL;
  const size_t lds = top ? top_lds(a.vocab, a.top) : 0;
  auto go = [&](auto kernel, int threads, int rows) {
    if (lds > 65536 && hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
      return;
    hipLaunchKernelGGL(kernel, dim3(cdiv(a.rows, rows)), dim3(threads), lds, s, a);
  };
  if (top) bf ? go(loss_row_kernel<bf16, 256, 4, true, true>, 256, 1) : go(loss_row_kernel<float, 256, 4, true, true>, 256, 1);
  else bf ? go(loss_row_kernel<bf16, 256, 4, true, false>, 256, 1) : go(loss_row_kernel<float, 256, 4, true, false>, 256, 1);
  return launched();
}

gx_status run_grad(const gx_logits_cfg& c, GradArgs a, hipStream_t s) {
  constexpr int CH = 4;
  const bool bf = c.dtype == GX_BF16;
  a.stride = (long)c.stride;
  a.grad_stride = (long)c.grad_stride;
  a.rows = c.rows;
  a.vocab = c.vocab;
  a.scale = c.scale;
  const int chunks = c.vocab / (bf ? 8 : 4);
  a.parts = chunks > 0 ? cdiv(chunks, 256 * CH) : 1;
  if ((long)c.rows * a.parts > MAX_GRID) return GX_ERR_SHAPE;
  const dim3 grid((unsigned)c.rows * (unsigned)a.parts);
  if (bf) hipLaunchKernelGGL((loss_grad_kernel<bf16, CH>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((loss_grad_kernel<float, CH>), grid, dim3(256), 0, s, a);
  return launched();
}

template <typename L>
gx_status run_pairs(const gx_pairs_cfg& c, const gx_pairs_in& in, const float* weights, const void* logp, float* loss, float* rewards,
                    float* dlogp, hipStream_t s) {
  const PairArgs a{logp, in.ref_logp, weights, in.pair_weights, in.starts, loss, rewards, dlogp, c.pairs, c.rows,
                   c.beta, c.margin, c.smoothing};
  hipLaunchKernelGGL(pairs_kernel<L>, dim3(c.pairs + (dlogp ? 1 : 0)), dim3(256), 0, s, a);
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
  return run_rows(*cfg, a, static_cast<hipStream_t>(hip_stream));
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
  return run_grad(*cfg, a, static_cast<hipStream_t>(hip_stream));
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
  return run_rows(*cfg, a, static_cast<hipStream_t>(hip_stream));
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
  return run_rows(*cfg, a, static_cast<hipStream_t>(hip_stream));
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
  return run_pairs<float>(*pairs, *in, in->weights, logp, loss, rewards, dlogp, static_cast<hipStream_t>(hip_stream));
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
  if (cfg->rows > 0 && (st = run_rows(*cfg, a, s)) != GX_OK) return st;
  st = run_pairs<double>(*pairs, *in, a.counted, a.logp64, loss, rewards, dlogits ? dlogp : nullptr, s);
  if (st != GX_OK || !dlogits || cfg->rows == 0) return st;
  GradArgs g = {};
  g.z = logits;
  g.dz = dlogits;
  g.unit = 1.f;
  set_scale(cfg->scale, g.c_hi, g.c_lo);
  g.ids = a.ids;
  g.stats = a.stats;
  g.dlogp = dlogp;
  return run_grad(*cfg, g, s);
}

gx_status gx_distill_loss(const gx_logits_cfg* cfg, const gx_distill_cfg* distill, const gx_distill_in* in, const void* logits,
                          float* loss, void* dlogits, void* hip_stream) {
  const gx_status st = check_whole(cfg);
  if (st != GX_OK) return st;
  if (!distill || !in) return GX_ERR_NULL;
  if (distill->top_dtype != GX_F32 && distill->top_dtype != GX_BF16) return GX_ERR_DTYPE;
  if (distill->flags) return GX_ERR_FLAGS;
  if (distill->top <= 0 || distill->top > MAX_TOP) return GX_ERR_SHAPE;
  if (cfg->rows == 0) return GX_OK;
  if (!logits || !loss || !in->top_ids || !in->top_logits) return GX_ERR_NULL;
  if (logits_misaligned(*cfg, logits) || logits_misaligned(*cfg, dlogits) || misaligned(in->top_ids, cfg->id_bytes) ||
      misaligned(in->top_logits, distill->top_dtype == GX_BF16 ? 2 : 4) || misaligned(in->top_lse, 4) || misaligned(in->weights, 4) ||
      misaligned(loss, 4))
    return GX_ERR_ALIGN;
  RowArgs a = row_args(*cfg, DISTILL, logits, dlogits, in->weights, loss);
  a.top_ids = in->top_ids;
  a.top_logits = in->top_logits;
  a.top_lse = in->top_lse;
  a.top = distill->top;
  a.top_id_bytes = cfg->id_bytes;
  a.top_bf16 = distill->top_dtype == GX_BF16;
  return run_rows(*cfg, a, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
