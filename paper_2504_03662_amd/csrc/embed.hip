// Token embedding: lookup with scaling, and the gradient of the table by sorted tokens.
//
// y[t] = s E[id_t - first] is a gather of rows, bound by memory.  Its transpose, dE[v] = s sum_{id_t = first + v} dy[t], has
// outputs of very uneven length: text repeats few tokens very often.  So the tokens are sorted by row first (stably: a row's
// tokens keep their order), the sorted tokens are cut into pieces of equal length, whoever they belong to,
// and every piece adds up its runs of equal rows: a run that lies inside a piece is stored, one that crosses the piece's ends leaves
// a partial sum, and the partial sums of a run are added in order afterwards.  No floating-point atomics; the order of every
// sum depends on sizes and ids alone.
// Both directions are bound by memory (a large copy moves 5.7 TB/s on these chips, read and written): 8192 tokens of 2048 columns
// (bf16) look up in 15 us (4.4 TB/s) and, with 32768 rows of which most are cleared, get their gradient in 69 us (268 MB of
// fp32 gradient alone take 47); 16385 tokens of 4096, half of them of this shard, a quarter padding, 64013 rows: 34 to 41 and 217 us
// (1.05 GB of gradient take 185).  Few tokens cost the launches: 257 tokens, 1001 rows of 256 (fp32) 2.5 and 4.7 us.
#include "../../include/gx.h"
#include "gx_kernels.h"

namespace {

using namespace gx;

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

constexpr int MAX_TOKENS = 1 << 24, MAX_ROWS = 1 << 24, MAX_HIDDEN = 65536;

template <typename T> struct Lanes;                            // elements of 16 bytes
template <> struct Lanes<float> { static constexpr int N = 4; typedef f32x4 type; };
template <> struct Lanes<bf16> { static constexpr int N = 8; typedef bf16x8 type; };

// Ids of type I (a template argument throughout: a choice at run time keeps loads from being issued together); the row
// of this shard that token t points to, or -1
template <typename I>
struct Ids {
  const I* p;
  long first, rows;
  GX_DEVINL long row_of(I id) const {
    const unsigned long r = (unsigned long)(long)id - (unsigned long)first;
    return r < (unsigned long)rows ? (long)r : -1;
  }
  GX_DEVINL long row(int t) const { return row_of(p[t]); }
};

// ------------------------------------------------------------------------------- forward
// `lpr` lanes (a power of two) to a row, 16 bytes each at a time; a lane's ROWS tokens are looked up together, so that as many
// dependent pairs of loads (id, then row) are in flight.  Few tokens take one a lane and spread their columns over blockIdx.y.
template <typename T, typename I, int ROWS>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const T* __restrict__ table, Ids<I> ids, T* __restrict__ y, int tokens,
                                                        int hidden, int lpr_log, float scale) {
  constexpr int V = Lanes<T>::N;
  typedef typename Lanes<T>::type Raw;
  const int lpr = 1 << lpr_log, chunks = hidden / V, step = 256 >> lpr_log;
  const int t0 = blockIdx.x * (step * ROWS) + (threadIdx.x >> lpr_log);
  long r[ROWS];
#pragma unroll
  for (int k = 0; k < ROWS; k++) r[k] = t0 + k * step < tokens ? ids.row(t0 + k * step) : -1;
  for (int c = (threadIdx.x & (lpr - 1)) + blockIdx.y * lpr; c < chunks; c += lpr * gridDim.y) {
    Raw v[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; k++) {
      v[k] = Raw{};
      if (r[k] >= 0) v[k] = *reinterpret_cast<const Raw*>(table + (size_t)r[k] * hidden + (size_t)c * V);
    }
#pragma unroll
    for (int k = 0; k < ROWS; k++) {
      if (r[k] >= 0)
#pragma unroll
        for (int e = 0; e < V; e++) v[k][e] = from_f32<T>(to_f32(v[k][e]) * scale);
      if (t0 + k * step < tokens) *reinterpret_cast<Raw*>(y + (size_t)(t0 + k * step) * hidden + (size_t)c * V) = v[k];
    }
  }
}

// ------------------------------------------------------------------------------- backward: sort
// Every workgroup owns `span` consecutive rows of the table and sorts the tokens that point to them, all by itself: it looks
// at all the ids, counts those of earlier rows (its place in the result) and its own, lists its own in order, and sorts the list by
// row, stably.  A wavefront takes a consecutive part of what is gone over each time, 64 at a time: a token's place is that of its
// row's first one, plus the count of that row's tokens in earlier wavefronts, plus those before it in its own (the lanes with the
// same row, found by ballots over the row's bits).
// The ids are read once by each workgroup, from L2: 64 workgroups and 8192 ids 4 MB, for which the rest of the pass moves hundreds.
// 8192 tokens, 32768 rows: 9 us (a radix sort over blocks of tokens, two launches to a digit, took 28).  Ids that are not all requested
// before the first is looked at cost another 5.
constexpr int SORT_WAVES = 8, SORT_THREADS = 64 * SORT_WAVES, MAX_SPAN = 2048;

template <typename I>
struct SortArgs {
  Ids<I> ids;
  long pad_row;                    // relative to the shard, -1: none
  int tokens, span, span_log;
  unsigned *list_key, *list_tok;   // the workgroups' lists, unsorted
  unsigned *key, *tok;             // the result: rows and tokens, sorted
  unsigned* start;                 // [rows + 1]: where a row's tokens start; the last one says how many there are in all
};

template <typename I>
__global__ void __launch_bounds__(SORT_THREADS) embed_sort_kernel(SortArgs<I> a) {
  __shared__ unsigned count[SORT_WAVES][MAX_SPAN];
  __shared__ unsigned lower[SORT_WAVES], mine[SORT_WAVES], sums[SORT_WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long lo = (long)blockIdx.x * a.span;
  const int own_rows = (int)(a.ids.rows - lo < a.span ? a.ids.rows - lo : a.span);
  const unsigned long long before_me = (1ull << lane) - 1ull;
  for (int i = threadIdx.x; i < SORT_WAVES * a.span; i += SORT_THREADS) count[i >> a.span_log][i & (a.span - 1)] = 0;
  // rows among this workgroup's, or beyond them, of tokens t, t + 64, ...: negative if it is an earlier one.  The loads are
  // unconditional, so that all of them are in flight
  constexpr int NONE = 1 << 30, AHEAD = 16;
  auto rows_from = [&](int t, int end, int (&r)[AHEAD]) {
    I id[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; u++) id[u] = a.ids.p[min(t + 64 * u, end - 1)];
#pragma unroll
    for (int u = 0; u < AHEAD; u++) {
      const long x = a.ids.row_of(id[u]);
      r[u] = x < 0 || x == a.pad_row || t + 64 * u >= end ? NONE : (int)x - (int)lo;
    }
  };
  // this wavefront's part of the tokens
  const int per = ((a.tokens + SORT_THREADS - 1) / SORT_THREADS) * 64;
  const int t0 = min(wave * per, a.tokens), t1 = min(t0 + per, a.tokens);
  unsigned below = 0, own = 0;
  for (int t = t0 + lane; t < t1; t += 64 * AHEAD) {
    int r[AHEAD];
    rows_from(t, t1, r);
#pragma unroll
    for (int u = 0; u < AHEAD; u++) {
      below += r[u] < 0;
      own += (unsigned)r[u] < (unsigned)own_rows;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    below += __shfl_xor(below, o, 64);
    own += __shfl_xor(own, o, 64);
  }
  if (lane == 0) {
    lower[wave] = below;
    mine[wave] = own;
  }
  __syncthreads();
  unsigned base = 0, n = 0, before = 0;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; w++) {
    base += lower[w];
    if (w < wave) before += mine[w];
    n += mine[w];
  }
  // this wavefront's part of the list, in the order of the tokens, and the count of every row in it
  unsigned* const list_key = a.list_key + base + before;
  unsigned* const list_tok = a.list_tok + base + before;
  if (own > 0) {
    unsigned at = 0;
    for (int t = t0 + lane; t < t0 + per; t += 64 * AHEAD) {
      int r[AHEAD];
      rows_from(t, t1, r);
#pragma unroll
      for (int u = 0; u < AHEAD; u++) {
        const bool in = (unsigned)r[u] < (unsigned)own_rows;
        const unsigned long long all = __builtin_amdgcn_ballot_w64(in);
        if (in) {
          const unsigned p = at + __popcll(all & before_me);
          list_key[p] = (unsigned)r[u];
          list_tok[p] = (unsigned)(t + 64 * u);
          atomicAdd(&count[wave][r[u]], 1u);                       // whole numbers: any order gives the same
        }
        at += __popcll(all);
      }
    }
  }
  __syncthreads();
  // places: a thread takes consecutive rows
  const int rpt = (a.span + SORT_THREADS - 1) / SORT_THREADS, r0 = threadIdx.x * rpt;
  unsigned total = 0;
  for (int r = r0; r < r0 + rpt && r < a.span; r++)
#pragma unroll
    for (int w = 0; w < SORT_WAVES; w++) total += count[w][r];
  unsigned run = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned up = __shfl_up(run, o, 64);
    if (lane >= o) run += up;
  }
  if (lane == 63) sums[wave] = run;
  __syncthreads();
  unsigned place = base + run - total;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; w++)
    if (w < wave) place += sums[w];
  for (int r = r0; r < r0 + rpt && r < a.span; r++) {
    if (r < own_rows) a.start[lo + r] = place;
#pragma unroll
    for (int w = 0; w < SORT_WAVES; w++) {
      const unsigned c = count[w][r];
      count[w][r] = place;
      place += c;
    }
  }
  if (lo + own_rows == a.ids.rows && threadIdx.x == 0) a.start[a.ids.rows] = base + n;
  __syncthreads();
  for (int i = lane; i < (int)((own + 63) & ~63u); i += 64 * 8) {
    unsigned key[8], tok[8];
#pragma unroll
    for (int u = 0; u < 8; u++) {
      const bool live = i + 64 * u < (int)own;
      key[u] = live ? list_key[i + 64 * u] : 0u;
      tok[u] = live ? list_tok[i + 64 * u] : 0u;
    }
#pragma unroll
    for (int u = 0; u < 8; u++) {
      const bool live = i + 64 * u < (int)own;
      const unsigned d = key[u];
      unsigned long long same = __builtin_amdgcn_ballot_w64(live);
      if (same == 0) break;
      for (int bit = 0; bit < a.span_log; bit++) {
        const unsigned long long set = __builtin_amdgcn_ballot_w64((d >> bit) & 1u);
        same &= ((d >> bit) & 1u) ? set : ~set;
      }
      const unsigned earlier = __popcll(same & before_me);
      volatile unsigned* next = &count[wave][d];
      const unsigned first = *next;
      if (live) {
        a.key[first + earlier] = (unsigned)lo + d;
        a.tok[first + earlier] = tok[u];
        if (earlier == 0) *next = first + (unsigned)__popcll(same);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// ------------------------------------------------------------------------------- backward: sums
struct SumArgs {
  const unsigned *key, *tok;       // sorted
  const unsigned* start;           // [rows + 1]
  const void* dy;
  float* dtable;
  float* part;                     // [piece][2][hidden]: a run that began before the piece, a run that goes on behind it
  int tokens, hidden, rows, pieces, accumulate;
  int sum_blocks, fill_rows;       // workgroups that add; rows of the table that each of the others clears
  float scale;
};
constexpr int PIECE = 16;          // tokens of a piece: as many row loads in flight as a lane has registers for

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

// The first workgroups: `lpr` lanes own a piece of the sorted tokens and 16 bytes of every row each.  The others clear the
// rows to which no token points, so that the one's reads and the other's writes share the memory's time (8192 tokens of 2048
// columns, 32768 rows: 43 to 55 us).
template <typename T>
__global__ void __launch_bounds__(256) embed_sum_kernel(SumArgs a, int lpr_log, int col_blocks) {
  constexpr int V = Lanes<T>::N;
  typedef typename Lanes<T>::type Raw;
  if ((int)blockIdx.x >= a.sum_blocks) {
    const int first = (blockIdx.x - a.sum_blocks) * a.fill_rows, chunks = a.hidden / 4;
    const int log = min(8, 32 - __clz(chunks - 1)), lanes = 1 << log, c0 = threadIdx.x & (lanes - 1);
    for (int r = first + (threadIdx.x >> log); r < min(first + a.fill_rows, a.rows); r += 256 >> log)
      if (a.start[r] == a.start[r + 1]) {
        f32x4* row = reinterpret_cast<f32x4*>(a.dtable + (size_t)r * a.hidden);
        for (int c = c0; c < chunks; c += lanes) row[c] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    return;
  }
  const int lpr = 1 << lpr_log, pb = blockIdx.x / col_blocks, cb = blockIdx.x - pb * col_blocks;
  const int p = (pb << (8 - lpr_log)) + (threadIdx.x >> lpr_log);
  const int c = (threadIdx.x & (lpr - 1)) + cb * lpr;
  const int i0 = p * PIECE;
  if (p >= a.pieces || c >= a.hidden / V) return;
  const T* dy = static_cast<const T*>(a.dy) + (size_t)c * V;
  unsigned k[PIECE + 1];
  Raw x[PIECE];
  const unsigned earlier = a.key[max(i0 - 1, 0)];
  const int n = (int)a.start[a.rows];
  int left;
  {
    unsigned t[PIECE];
#pragma unroll
    for (int u = 0; u <= PIECE; u++) {                 // all of them before n is known: what lies beyond is not used
      const int i = min(i0 + u, a.tokens - 1);
      k[u] = a.key[i];
      if (u < PIECE) t[u] = a.tok[i];
    }
    left = min(PIECE, n - i0);
    if (left <= 0) return;
#pragma unroll
    for (int u = 0; u < PIECE; u++) x[u] = *reinterpret_cast<const Raw*>(dy + (size_t)(u < left ? t[u] : t[0]) * a.hidden);
  }
  const bool from_before = i0 > 0 && earlier == k[0];
  const bool goes_on = i0 + left < n && k[left] == k[left - 1];
  bool first_run = true;
  float s[V];
#pragma unroll
  for (int e = 0; e < V; e++) s[e] = 0.f;
#pragma unroll
  for (int u = 0; u < PIECE; u++) {
    if (u < left) {
#pragma unroll
      for (int e = 0; e < V; e++) s[e] += to_f32(x[u][e]);
      const bool piece_end = u + 1 == left;
      if (piece_end || k[u + 1] != k[u]) {             // the run ends here, or is cut
        float* const part = a.part + (size_t)p * 2 * a.hidden + (size_t)c * V;
        if (first_run && from_before) put_row<V>(part, s, 1.f, false);
        else if (piece_end && goes_on) put_row<V>(part + a.hidden, s, 1.f, false);
        else put_row<V>(a.dtable + (size_t)k[u] * a.hidden + (size_t)c * V, s, a.scale, a.accumulate);
        first_run = false;
#pragma unroll
        for (int e = 0; e < V; e++) s[e] = 0.f;
      }
    }
  }
}

// One workgroup per piece and 256 columns: if a run begins in the piece and goes on behind it, adds the run's partial sums.  Each
// wavefront takes a consecutive quarter of them, and the quarters are added in order.  The most frequent token of a text has hundreds
// of pieces: 7 us at 8192 tokens.
__global__ void __launch_bounds__(256) embed_join_kernel(SumArgs a) {
  __shared__ f32x4 red[3][64];
  const int p = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.y * 64 + lane;
  const int i1 = (p + 1) * PIECE;
  if (i1 >= a.tokens) return;
  const int n = (int)a.start[a.rows];
  const unsigned key = a.key[i1 - 1], next = a.key[i1];
  if (i1 >= n || next != key) return;                                      // nothing goes on
  const int first = (int)a.start[key], end = (int)a.start[key + 1];
  if (first < p * PIECE) return;                                           // it began in an earlier piece
  const int last = (end - 1) / PIECE, rows = last - p + 1, per = (rows + 3) / 4;
  const int q0 = p + min(wave * per, rows), q1 = min(q0 + per, last + 1);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (c < a.hidden / 4) {
#pragma unroll 8
    for (int q = q0; q < q1; q++) s += reinterpret_cast<const f32x4*>(a.part + ((size_t)q * 2 + (q == p)) * a.hidden)[c];
  }
  if (wave > 0) red[wave - 1][lane] = s;
  __syncthreads();
  if (wave > 0 || c >= a.hidden / 4) return;
#pragma unroll
  for (int w = 0; w < 3; w++) s += red[w][lane];
  const float v[4] = {s[0], s[1], s[2], s[3]};
  put_row<4>(a.dtable + (size_t)key * a.hidden + (size_t)c * 4, v, a.scale, a.accumulate);
}

// ------------------------------------------------------------------------------- backward: few tokens
// One launch: every workgroup owns `span` consecutive rows of the table, 64 lanes' columns of them, and looks at all ids.  A wavefront
// takes every 4th row: it lists the row's tokens in order (ballots over the ids that its lanes hold) and adds them up, or clears the row; rows
// with more than HOT tokens come after that, a quarter of the tokens to a wavefront, and the quarters are added in order.
// us of the kernels, this / by sorted tokens: 257 tokens, 1001 rows of 256 (fp32) 4.7 / 15.3; 48 tokens, 97749 x 576 (bf16) 33.7 / 46.8;
// 512 tokens, 300000 x 64 21.6 / 30.4; 512 tokens, 32000 x 4096 109.8 / 109.8 (a copy's rate for the table's gradient); 512 tokens all
// alike, 500 x 8192 (fp32) 23.3 / 17.5, 1001 x 256 11.3 / 13.8.  More tokens would make rows that all of them share a long sum, and ids a long list.
constexpr int FEW_TOKENS = 512, FEW_CHUNKS = FEW_TOKENS / 64, FEW_ROWS = 32, HOT = 16;
template <typename I>
struct FewArgs {
  Ids<I> ids;
  long pad_row;                    // relative to the shard, -1: none
  const void* dy;
  float* dtable;
  int tokens, hidden, rows, span, accumulate;
  float scale;
};
// adds chunk c of the tokens list[from .. to), AT_ONCE of them requested together
template <typename T, int AT_ONCE>
GX_DEVINL void sum_listed(float (&s)[Lanes<T>::N], const T* dy, const unsigned short* list, int from, int to, int hidden, int c) {
  constexpr int V = Lanes<T>::N;
  typedef typename Lanes<T>::type Raw;
#pragma unroll
  for (int e = 0; e < V; e++) s[e] = 0.f;
  for (int i = from; i < to; i += AT_ONCE) {
    Raw x[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; u++)
      x[u] = *reinterpret_cast<const Raw*>(dy + (size_t)list[min(i + u, to - 1)] * hidden + (size_t)c * V);
#pragma unroll
    for (int u = 0; u < AT_ONCE; u++)
      if (i + u < to)
#pragma unroll
        for (int e = 0; e < V; e++) s[e] += to_f32(x[u][e]);
  }
}
template <typename T, typename I>
__global__ void __launch_bounds__(256) embed_few_kernel(FewArgs<I> a) {
  constexpr int V = Lanes<T>::N;
  __shared__ int row_of[FEW_TOKENS];
  __shared__ unsigned short lists[4][FEW_TOKENS];
  __shared__ int counts[FEW_ROWS];
  __shared__ float red[3][V][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long first = (long)blockIdx.x * a.span;
  const int rows = (int)min((long)a.span, a.rows - first), chunks = a.hidden / V, c = blockIdx.y * 64 + lane;
  bool some = false;
#pragma unroll
  for (int k = 0; k < FEW_TOKENS / 256; k++) {
    const int t = threadIdx.x + 256 * k;
    long r = -1;
    if (t < a.tokens) {
      r = a.ids.row(t);
      if (r == a.pad_row) r = -1;
    }
    const bool own = r >= first && r < first + rows;
    row_of[t] = own ? (int)(r - first) : -1;
    some |= own;
  }
  float* const table = a.dtable + first * a.hidden;
  if (!__syncthreads_or(some)) {
    if (a.accumulate) return;
    if (gridDim.y == 1) {
      for (int i = threadIdx.x; i < rows * (a.hidden / 4); i += 256) reinterpret_cast<f32x4*>(table)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      return;
    }
    constexpr int W = 64 * V / 4;                                // 16 bytes of fp32 at a time
    const int at = blockIdx.y * W + threadIdx.x % W;
    if (at < a.hidden / 4)
      for (int r = threadIdx.x / W; r < rows; r += 256 / W)
        reinterpret_cast<f32x4*>(table + (size_t)r * a.hidden)[at] = f32x4{0.f, 0.f, 0.f, 0.f};
    return;
  }
  int mine[FEW_CHUNKS];
#pragma unroll
  for (int k = 0; k < FEW_CHUNKS; k++) mine[k] = row_of[64 * k + lane];
  unsigned short* const list = lists[wave];
  auto list_tokens = [&](int r) __attribute__((always_inline)) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < FEW_CHUNKS; k++) {
      const bool it = mine[k] == r;
      const unsigned long long m = __builtin_amdgcn_ballot_w64(it);
      if (it) list[n + __popcll(m & ((1ull << lane) - 1))] = (unsigned short)(64 * k + lane);
      n += __popcll(m);
    }
    __builtin_amdgcn_wave_barrier();
    return n;
  };
  const T* const dy = static_cast<const T*>(a.dy);
  float s[V];
  for (int r = wave; r < rows; r += 4) {
    const int n = list_tokens(r);
    if (lane == 0) counts[r] = n;
    if (n > HOT || (n == 0 && a.accumulate)) continue;
    if (c >= chunks) continue;
    sum_listed<T, 4>(s, dy, list, 0, n, a.hidden, c);               // of no token: zeros
    put_row<V>(table + (size_t)r * a.hidden + (size_t)c * V, s, a.scale, a.accumulate);
  }
  __syncthreads();
  for (int r = 0; r < rows; r++) {
    if (counts[r] <= HOT) continue;                              // the same for all
    const int n = list_tokens(r), per = (n + 3) / 4, from = min(wave * per, n), to = min(from + per, n);
    sum_listed<T, 16>(s, dy, list, from, to, a.hidden, min(c, chunks - 1));
    if (wave > 0)
#pragma unroll
      for (int e = 0; e < V; e++) red[wave - 1][e][lane] = s[e];
    __syncthreads();
    if (wave == 0 && c < chunks) {
#pragma unroll
      for (int w = 0; w < 3; w++)
#pragma unroll
        for (int e = 0; e < V; e++) s[e] += red[w][e][lane];
      put_row<V>(table + (size_t)r * a.hidden + (size_t)c * V, s, a.scale, a.accumulate);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------- host
int lanes_log(int chunks) {
  int l = 3;
  while (l < 8 && (1 << l) < chunks) l++;
  return l;
}

constexpr long FEW_WGS = 2048;             // workgroups of a lookup with one token a lane: all on the chip at once
constexpr long FILL_BYTES = 32 << 10;      // of the table, for each workgroup that clears

size_t align_up(size_t v) { return (v + 255) & ~(size_t)255; }

struct Plan {
  int pieces, span, span_log;
  size_t list_key, list_tok, key, tok, start, part, bytes;
};
// Rows of the table that a workgroup of the sort owns: about 128 workgroups, which each look at all ids
Plan plan_of(const gx_embed_cfg& c) {
  Plan p;
  p.pieces = cdiv(c.tokens, PIECE);
  p.span_log = 6;
  while ((1 << p.span_log) < MAX_SPAN && ((long)128 << p.span_log) < c.rows) p.span_log++;
  p.span = 1 << p.span_log;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t was = at; at += align_up(n); return was; };
  p.list_key = take((size_t)c.tokens * 4);
  p.list_tok = take((size_t)c.tokens * 4);
  p.key = take((size_t)c.tokens * 4);
  p.tok = take((size_t)c.tokens * 4);
  p.start = take(((size_t)c.rows + 1) * 4);
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
template <typename I>
Ids<I> ids_of(const gx_embed_cfg& c, const void* ids) { return Ids<I>{static_cast<const I*>(ids), (long)c.first_row, (long)c.rows}; }

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
  const long wgs = cdiv(cfg->tokens, 256 >> log);              // with one token a lane
  const bool few = wgs * cdiv(chunks, 256) < FEW_WGS;
  const dim3 grid(few ? (unsigned)wgs : (unsigned)cdiv(cfg->tokens, (256 >> log) * 4), few ? cdiv(chunks, 1 << log) : 1);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  auto go = [&](auto type, auto id) {
    typedef decltype(type) T;
    typedef decltype(id) I;
    if (few)
      hipLaunchKernelGGL((embed_fwd_kernel<T, I, 1>), grid, dim3(256), 0, s, static_cast<const T*>(table), ids_of<I>(*cfg, ids),
                         static_cast<T*>(y), cfg->tokens, cfg->hidden, log, cfg->scale);
    else
      hipLaunchKernelGGL((embed_fwd_kernel<T, I, 4>), grid, dim3(256), 0, s, static_cast<const T*>(table), ids_of<I>(*cfg, ids),
                         static_cast<T*>(y), cfg->tokens, cfg->hidden, log, cfg->scale);
  };
  if (cfg->id_bytes == 8) bf ? go(bf16(), 0l) : go(0.f, 0l);
  else bf ? go(bf16(), 0) : go(0.f, 0);
  return launched();
}

gx_status gx_embed_bwd(const gx_embed_cfg* cfg, const void* ids, const void* dy, float* dtable, void* workspace,
                       void* hip_stream) {
  const gx_status st = check(cfg);
  if (st != GX_OK) return st;
  if (!dtable || !workspace || (cfg->tokens > 0 && (!ids || !dy))) return GX_ERR_NULL;
  if (misaligned(dtable) || ids_misaligned(*cfg, ids) || misaligned(dy) || misaligned(workspace)) return GX_ERR_ALIGN;
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool accumulate = cfg->flags & GX_ACCUM_WGRAD, bf = cfg->dtype == GX_BF16;
  const long pad_row = cfg->pad_id < 0 ? -1 : (long)(cfg->pad_id - cfg->first_row);
  if (cfg->tokens <= FEW_TOKENS) {
    // about 2048 workgroups, or more of 32 rows
    const int cols = cdiv(cfg->hidden, bf ? 512 : 256);
    const long even = (long)cfg->rows * cols / 2048;
    const int span = even < 1 ? 1 : even > FEW_ROWS ? FEW_ROWS : (int)even;
    auto go = [&](auto type, auto id) {
      typedef decltype(type) T;
      typedef decltype(id) I;
      const FewArgs<I> a{ids_of<I>(*cfg, ids), pad_row, dy, dtable, cfg->tokens, cfg->hidden, cfg->rows, span, accumulate, cfg->scale};
      hipLaunchKernelGGL((embed_few_kernel<T, I>), dim3(cdiv(cfg->rows, span), cols), dim3(256), 0, s, a);
    };
    if (cfg->id_bytes == 8) bf ? go(bf16(), 0l) : go(0.f, 0l);
    else bf ? go(bf16(), 0) : go(0.f, 0);
    return launched();
  }
  const Plan p = plan_of(*cfg);
  char* ws = static_cast<char*>(workspace);
  auto u32 = [&](size_t at) { return reinterpret_cast<unsigned*>(ws + at); };
  auto sort = [&](auto id) {
    typedef decltype(id) I;
    const SortArgs<I> a{ids_of<I>(*cfg, ids), pad_row, cfg->tokens, p.span, p.span_log,
                        u32(p.list_key), u32(p.list_tok), u32(p.key), u32(p.tok), u32(p.start)};
    hipLaunchKernelGGL(embed_sort_kernel<I>, dim3(cdiv(cfg->rows, p.span)), dim3(SORT_THREADS), 0, s, a);
  };
  cfg->id_bytes == 8 ? sort(0l) : sort(0);
  SumArgs m{u32(p.key), u32(p.tok), u32(p.start), dy, dtable, reinterpret_cast<float*>(ws + p.part), cfg->tokens, cfg->hidden, cfg->rows,
            p.pieces, accumulate, 0, 0, cfg->scale};
  const int chunks = cfg->hidden / (bf ? 8 : 4), log = lanes_log(chunks), cols = cdiv(chunks, 1 << log);
  m.sum_blocks = cdiv(p.pieces, 256 >> log) * cols;
  m.fill_rows = cdiv(FILL_BYTES, (long)cfg->hidden * 4);
  const dim3 grid(m.sum_blocks + (accumulate ? 0 : cdiv(cfg->rows, m.fill_rows)));
  if (grid.x > 0) {
    if (bf) hipLaunchKernelGGL((embed_sum_kernel<bf16>), grid, dim3(256), 0, s, m, log, cols);
    else hipLaunchKernelGGL((embed_sum_kernel<float>), grid, dim3(256), 0, s, m, log, cols);
  }
  if (p.pieces > 1)
    hipLaunchKernelGGL(embed_join_kernel, dim3(p.pieces, cdiv(cfg->hidden / 4, 64)), dim3(256), 0, s, m);
  return launched();
}

}  // extern "C"
