// Token embedding: lookup with scaling, and the gradient of the table by sorted tokens.
//
// y[t] = s E[id_t - first] is a gather of rows, bound by memory.  Its transpose, dE[v] = s sum_{id_t = first + v} dy[t], has
// outputs of very uneven length: text repeats few tokens very often.  So the tokens are sorted by row first (stable, so that
// a row's tokens keep their order), the sorted tokens are cut into pieces of equal length, whoever they belong to,
// and every piece adds up its runs of equal rows: a run that lies inside a piece is stored, one that crosses the piece's ends leaves
// a partial sum, and the partial sums of a run are added in order afterwards.  No floating-point atomics; the order of every
// sum depends on sizes and ids alone.
#include "../../include/gx.h"
#include "gx_kernels.h"

namespace {

using namespace gx;

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

constexpr int MAX_TOKENS = 1 << 24, MAX_ROWS = 1 << 24, MAX_HIDDEN = 65536;

template <typename T> struct Lanes;                            // elements of 16 bytes
template <> struct Lanes<float> { static constexpr int N = 4; typedef f32x4 type; };
template <> struct Lanes<bf16> { static constexpr int N = 8; typedef bf16x8 type; };

// The row of this shard that token t points to, or -1
struct Ids {
  const void* p;
  int bytes;
  long first, rows;
  GX_DEVINL long row(int t) const {
    const long id = bytes == 8 ? static_cast<const long*>(p)[t] : (long)static_cast<const int*>(p)[t];
    const unsigned long r = (unsigned long)id - (unsigned long)first;
    return r < (unsigned long)rows ? (long)r : -1;
  }
};

// ------------------------------------------------------------------------------- forward
// `lpr` lanes (a power of two) to a row, 16 bytes each at a time
template <typename T>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const T* __restrict__ table, Ids ids, T* __restrict__ y, int tokens,
                                                        int hidden, int lpr_log, float scale) {
  constexpr int V = Lanes<T>::N;
  typedef typename Lanes<T>::type Raw;
  const int lpr = 1 << lpr_log, c0 = threadIdx.x & (lpr - 1), chunks = hidden / V;
  const int t = (blockIdx.x << (8 - lpr_log)) + (threadIdx.x >> lpr_log);
  if (t >= tokens) return;
  const long r = ids.row(t);
  const T* src = table + (size_t)(r < 0 ? 0 : r) * hidden;
  T* dst = y + (size_t)t * hidden;
  for (int c = c0 + blockIdx.y * lpr; c < chunks; c += lpr * gridDim.y) {
    Raw v = {};
    if (r >= 0) {
      v = *reinterpret_cast<const Raw*>(src + (size_t)c * V);
#pragma unroll
      for (int e = 0; e < V; e++) v[e] = from_f32<T>(to_f32(v[e]) * scale);
    }
    *reinterpret_cast<Raw*>(dst + (size_t)c * V) = v;
  }
}

// ------------------------------------------------------------------------------- backward: sort
// Stable radix sort of (row, token) by row, digits of up to 9 bits from the lowest up; tokens without a gradient sort behind
// the last row.  A block owns TPB consecutive tokens, its wavefronts consecutive parts of them, 64 at a time: a token's place among
// those of its digit is the count of earlier ones in the wavefront (kept in LDS, one counter per wavefront and
// digit), plus those of earlier wavefronts, plus those of earlier blocks, plus those of lower digits.
constexpr int DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS;
constexpr int SORT_WAVES = 8, SORT_THREADS = 64 * SORT_WAVES, ROUNDS = 8, TPB = SORT_THREADS * ROUNDS;
static_assert(SORT_THREADS == DIGITS, "one thread to a digit");

struct SortArgs {
  Ids ids;
  long pad_row;                    // relative to the shard, -1: none
  int tokens, shift, mask;
  const unsigned *key_in, *tok_in; // null in the first pass: keys come from the ids, tokens are in order
  unsigned *key_out, *tok_out;
  unsigned* hist;                  // [blocks][DIGITS]
};
GX_DEVINL unsigned key_of(const SortArgs& a, int i) {
  if (a.key_in) return a.key_in[i];
  const long r = a.ids.row(i);
  return r < 0 || r == a.pad_row ? (unsigned)a.ids.rows : (unsigned)r;
}

__global__ void __launch_bounds__(SORT_THREADS) embed_count_kernel(SortArgs a) {
  __shared__ unsigned n[DIGITS];
  n[threadIdx.x] = 0;
  __syncthreads();
  const int i0 = blockIdx.x * TPB + threadIdx.x;
#pragma unroll
  for (int r = 0; r < ROUNDS; r++) {
    const int i = i0 + r * SORT_THREADS;
    if (i < a.tokens) atomicAdd(&n[(key_of(a, i) >> a.shift) & a.mask], 1u);      // whole numbers: any order gives the same
  }
  __syncthreads();
  a.hist[(size_t)blockIdx.x * DIGITS + threadIdx.x] = n[threadIdx.x];
}

__global__ void __launch_bounds__(SORT_THREADS) embed_place_kernel(SortArgs a, int blocks) {
  __shared__ unsigned count[SORT_WAVES][DIGITS];
  __shared__ unsigned wave_total[SORT_WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int d0 = threadIdx.x;
  // this thread's digit: how many in the whole, how many in the blocks before this one
  unsigned before = 0, total = 0;
  for (int b = 0; b < blocks; b++) {
    const unsigned c = a.hist[(size_t)b * DIGITS + d0];
    if (b < (int)blockIdx.x) before += c;
    total += c;
  }
#pragma unroll
  for (int w = 0; w < SORT_WAVES; w++) count[w][d0] = 0;
  __syncthreads();
  unsigned key[ROUNDS], tok[ROUNDS], rank[ROUNDS];
  const int i0 = blockIdx.x * TPB + wave * (64 * ROUNDS) + lane;
#pragma unroll
  for (int r = 0; r < ROUNDS; r++) {
    const int i = i0 + 64 * r;
    key[r] = i < a.tokens ? key_of(a, i) : 0u;
    tok[r] = i < a.tokens ? (a.tok_in ? a.tok_in[i] : (unsigned)i) : 0u;
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; r++) {
    const bool live = i0 + 64 * r < a.tokens;
    const unsigned d = (key[r] >> a.shift) & a.mask;
    unsigned long long same = __builtin_amdgcn_ballot_w64(live);
#pragma unroll
    for (int bit = 0; bit < DIGIT_BITS; bit++) {
      const unsigned long long set = __builtin_amdgcn_ballot_w64((d >> bit) & 1u);
      same &= ((d >> bit) & 1u) ? set : ~set;
    }
    const unsigned earlier = __popcll(same & ((1ull << lane) - 1ull));
    volatile unsigned* n = &count[wave][d];
    const unsigned old = *n;
    rank[r] = old + earlier;
    if (live && earlier == 0) *n = old + (unsigned)__popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  // places: exclusive sum of the totals over the digits, the earlier blocks, then wavefront by wavefront
  unsigned run = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned up = __shfl_up(run, o, 64);
    if (lane >= o) run += up;
  }
  if (lane == 63) wave_total[wave] = run;
  __syncthreads();
  unsigned place = run - total + before;
  for (int w = 0; w < wave; w++) place += wave_total[w];
#pragma unroll
  for (int w = 0; w < SORT_WAVES; w++) {
    const unsigned c = count[w][d0];
    count[w][d0] = place;
    place += c;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < ROUNDS; r++)
    if (i0 + 64 * r < a.tokens) {
      const unsigned at = count[wave][(key[r] >> a.shift) & a.mask] + rank[r];
      a.key_out[at] = key[r];
      a.tok_out[at] = tok[r];
    }
}

// ------------------------------------------------------------------------------- backward: sums
__global__ void __launch_bounds__(256) embed_zero_kernel(f32x4* __restrict__ p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
}

struct SumArgs {
  const unsigned *key, *tok;       // sorted
  const void* dy;
  float* dtable;
  float* part;                     // [piece][2][hidden]: a run that began before the piece, a run that goes on behind it
  int tokens, hidden, rows, piece, pieces, accumulate;
  float scale;
};

// Stores or adds a run's sum: 16 bytes of fp32 per lane and half of a bf16 chunk
template <int V>
GX_DEVINL void put_row(float* dst, const float (&s)[V], float scale, bool accumulate) {
#pragma unroll
  for (int h = 0; h < V / 4; h++) {
    f32x4* p = reinterpret_cast<f32x4*>(dst) + h;
    f32x4 v = {s[4 * h] * scale, s[4 * h + 1] * scale, s[4 * h + 2] * scale, s[4 * h + 3] * scale};
    if (accumulate) v += *p;
    *p = v;
  }
}

// `lpr` lanes own a piece of the sorted tokens and 16 bytes of every row each
template <typename T>
__global__ void __launch_bounds__(256) embed_sum_kernel(SumArgs a, int lpr_log) {
  constexpr int V = Lanes<T>::N, AHEAD = 4;
  typedef typename Lanes<T>::type Raw;
  const int lpr = 1 << lpr_log;
  const int p = (blockIdx.x << (8 - lpr_log)) + (threadIdx.x >> lpr_log);
  const int c = (threadIdx.x & (lpr - 1)) + blockIdx.y * lpr;
  if (p >= a.pieces || c >= a.hidden / V) return;
  const int i0 = p * a.piece, i1 = min(i0 + a.piece, a.tokens);
  const T* dy = static_cast<const T*>(a.dy) + (size_t)c * V;
  const unsigned none = (unsigned)a.rows;
  const bool from_before = i0 > 0 && a.key[i0 - 1] == a.key[i0];
  const bool goes_on = i1 < a.tokens && a.key[i1] == a.key[i1 - 1];
  bool first_run = true;
  float s[V];
#pragma unroll
  for (int e = 0; e < V; e++) s[e] = 0.f;
  for (int i = i0; i < i1; i += AHEAD) {
    Raw x[AHEAD];
    unsigned k[AHEAD + 1];
#pragma unroll
    for (int u = 0; u <= AHEAD; u++) k[u] = i + u < i1 ? a.key[i + u] : none;
    if (k[0] == none) break;                           // sorted: nothing that counts follows
#pragma unroll
    for (int u = 0; u < AHEAD; u++)
      if (k[u] != none) x[u] = *reinterpret_cast<const Raw*>(dy + (size_t)a.tok[i + u] * a.hidden);
#pragma unroll
    for (int u = 0; u < AHEAD; u++) {
      if (k[u] == none) break;
#pragma unroll
      for (int e = 0; e < V; e++) s[e] += to_f32(x[u][e]);
      const bool piece_end = i + u + 1 == i1;
      if (piece_end || k[u + 1] != k[u]) {             // the run ends here, or is cut
        if (first_run && from_before) put_row<V>(a.part + ((size_t)p * 2) * a.hidden + (size_t)c * V, s, 1.f, false);
        else if (piece_end && goes_on) put_row<V>(a.part + ((size_t)p * 2 + 1) * a.hidden + (size_t)c * V, s, 1.f, false);
        else put_row<V>(a.dtable + (size_t)k[u] * a.hidden + (size_t)c * V, s, a.scale, a.accumulate);
        first_run = false;
#pragma unroll
        for (int e = 0; e < V; e++) s[e] = 0.f;
      }
    }
  }
}

// One block per piece: if a run begins in it and goes on behind it, adds the run's partial sums, piece by piece
__global__ void __launch_bounds__(256) embed_join_kernel(SumArgs a) {
  const int p = blockIdx.x, c = blockIdx.y * 256 + threadIdx.x;
  const int i0 = p * a.piece, i1 = min(i0 + a.piece, a.tokens);
  if (i1 >= a.tokens) return;
  const unsigned key = a.key[i1 - 1];
  if (key >= (unsigned)a.rows || a.key[i1] != key) return;                 // nothing goes on
  if (i0 > 0 && a.key[i0 - 1] == key) return;                              // it began in an earlier piece
  // the run's last piece: the last one whose first token has this key
  int lo = p + 1, hi = a.pieces - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.key[mid * a.piece] == key) lo = mid;
    else hi = mid - 1;
  }
  if (c >= a.hidden / 4) return;
  f32x4 s = reinterpret_cast<const f32x4*>(a.part + ((size_t)p * 2 + 1) * a.hidden)[c];
  for (int q = p + 1; q <= lo; q++) s += reinterpret_cast<const f32x4*>(a.part + ((size_t)q * 2) * a.hidden)[c];
  const float v[4] = {s[0], s[1], s[2], s[3]};
  put_row<4>(a.dtable + (size_t)key * a.hidden + (size_t)c * 4, v, a.scale, a.accumulate);
}

// ------------------------------------------------------------------------------- host
int lanes_log(int chunks) {
  int l = 3;
  while (l < 8 && (1 << l) < chunks) l++;
  return l;
}

constexpr int PIECE = 16;          // tokens of a piece

size_t align_up(size_t v) { return (v + 255) & ~(size_t)255; }

struct Plan {
  int pieces, blocks, passes, digit;
  size_t key[2], tok[2], hist, part, bytes;
};
Plan plan_of(const gx_embed_cfg& c) {
  Plan p;
  p.pieces = cdiv(c.tokens, PIECE);
  p.blocks = cdiv(c.tokens, TPB);
  int bits = 1;
  while (((unsigned)c.rows >> bits) != 0) bits++;              // keys are 0 .. rows
  p.passes = cdiv(bits, DIGIT_BITS);
  p.digit = cdiv(bits, p.passes);
  size_t at = 0;
  auto take = [&](size_t n) { const size_t was = at; at += align_up(n); return was; };
  for (int k = 0; k < 2; k++) {
    p.key[k] = take((size_t)c.tokens * 4);
    p.tok[k] = take((size_t)c.tokens * 4);
  }
  p.hist = take((size_t)p.blocks * DIGITS * 4);
  p.part = take((size_t)p.pieces * 2 * c.hidden * 4);
  p.bytes = at;
  return p;
}

gx_status check(const gx_embed_cfg* c) {
  if (!c) return GX_ERR_NULL;
  if (c->dtype != GX_F32 && c->dtype != GX_BF16) return GX_ERR_DTYPE;
  if (c->id_bytes != 4 && c->id_bytes != 8) return GX_ERR_DTYPE;
  if (c->flags & ~GX_ACCUM_WGRAD) return GX_ERR_FLAGS;
  if (c->tokens < 0 || c->tokens > MAX_TOKENS || c->rows <= 0 || c->rows > MAX_ROWS || c->hidden <= 0 || c->hidden > MAX_HIDDEN ||
      c->first_row < 0 || c->pad_id < -1)
    return GX_ERR_SHAPE;
  if (c->hidden % (c->dtype == GX_BF16 ? 8 : 4)) return GX_ERR_DIVIS;
  return GX_OK;
}
bool ids_misaligned(const gx_embed_cfg& c, const void* ids) { return reinterpret_cast<uintptr_t>(ids) % c.id_bytes != 0; }
Ids ids_of(const gx_embed_cfg& c, const void* ids) { return Ids{ids, c.id_bytes, (long)c.first_row, (long)c.rows}; }

gx_status launched() { return hipGetLastError() == hipSuccess ? GX_OK : GX_ERR_LAUNCH; }

}  // namespace

extern "C" {

size_t gx_embed_workspace_bytes(const gx_embed_cfg* cfg) { return check(cfg) == GX_OK ? plan_of(*cfg).bytes : 0; }

gx_status gx_embed_fwd(const gx_embed_cfg* cfg, const void* table, const void* ids, void* y, void* hip_stream) {
  const gx_status st = check(cfg);
  if (st != GX_OK) return st;
  if (cfg->tokens == 0) return GX_OK;
  if (!table || !ids || !y) return GX_ERR_NULL;
  if (misaligned(table) || misaligned(y) || ids_misaligned(*cfg, ids)) return GX_ERR_ALIGN;
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  const bool bf = cfg->dtype == GX_BF16;
  const int chunks = cfg->hidden / (bf ? 8 : 4), log = lanes_log(chunks);
  const dim3 grid(cdiv(cfg->tokens, 256 >> log), 1);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (bf)
    hipLaunchKernelGGL((embed_fwd_kernel<bf16>), grid, dim3(256), 0, s, static_cast<const bf16*>(table), ids_of(*cfg, ids),
                       static_cast<bf16*>(y), cfg->tokens, cfg->hidden, log, cfg->scale);
  else
    hipLaunchKernelGGL((embed_fwd_kernel<float>), grid, dim3(256), 0, s, static_cast<const float*>(table), ids_of(*cfg, ids),
                       static_cast<float*>(y), cfg->tokens, cfg->hidden, log, cfg->scale);
  return launched();
}

gx_status gx_embed_bwd(const gx_embed_cfg* cfg, const void* ids, const void* dy, float* dtable, void* workspace,
                       void* hip_stream) {
  const gx_status st = check(cfg);
  if (st != GX_OK) return st;
  if (!dtable || (cfg->tokens > 0 && (!ids || !dy || !workspace))) return GX_ERR_NULL;
  if (misaligned(dtable) || ids_misaligned(*cfg, ids) || misaligned(dy) || misaligned(workspace)) return GX_ERR_ALIGN;
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool accumulate = cfg->flags & GX_ACCUM_WGRAD, bf = cfg->dtype == GX_BF16;
  if (!accumulate) {
    const size_t n = (size_t)cfg->rows * cfg->hidden / 4;
    const size_t wgs = (n + 256 * 4 - 1) / (256 * 4);
    hipLaunchKernelGGL(embed_zero_kernel, dim3((unsigned)(wgs > 65536 ? 65536 : wgs)), dim3(256), 0, s,
                       reinterpret_cast<f32x4*>(dtable), n);
  }
  if (cfg->tokens == 0) return launched();
  const Plan p = plan_of(*cfg);
  char* ws = static_cast<char*>(workspace);
  auto u32 = [&](size_t at) { return reinterpret_cast<unsigned*>(ws + at); };
  SortArgs a{ids_of(*cfg, ids), cfg->pad_id < 0 ? -1 : (long)(cfg->pad_id - cfg->first_row), cfg->tokens, 0, (1 << p.digit) - 1,
             nullptr, nullptr, nullptr, nullptr, u32(p.hist)};
  for (int k = 0; k < p.passes; k++) {
    a.shift = k * p.digit;
    a.key_in = k ? u32(p.key[(k - 1) & 1]) : nullptr;
    a.tok_in = k ? u32(p.tok[(k - 1) & 1]) : nullptr;
    a.key_out = u32(p.key[k & 1]);
    a.tok_out = u32(p.tok[k & 1]);
    hipLaunchKernelGGL(embed_count_kernel, dim3(p.blocks), dim3(SORT_THREADS), 0, s, a);
    hipLaunchKernelGGL(embed_place_kernel, dim3(p.blocks), dim3(SORT_THREADS), 0, s, a, p.blocks);
  }
  SumArgs m{a.key_out, a.tok_out, dy, dtable, reinterpret_cast<float*>(ws + p.part), cfg->tokens, cfg->hidden, cfg->rows, PIECE,
            p.pieces, accumulate, cfg->scale};
  const int chunks = cfg->hidden / (bf ? 8 : 4), log = lanes_log(chunks);
  const dim3 grid(cdiv(p.pieces, 256 >> log), cdiv(chunks, 1 << log));
  if (bf) hipLaunchKernelGGL((embed_sum_kernel<bf16>), grid, dim3(256), 0, s, m, log);
  else hipLaunchKernelGGL((embed_sum_kernel<float>), grid, dim3(256), 0, s, m, log);
  if (p.pieces > 1)
    hipLaunchKernelGGL(embed_join_kernel, dim3(p.pieces, cdiv(cfg->hidden / 4, 256)), dim3(256), 0, s, m);
  return launched();
}

}  // extern "C"
