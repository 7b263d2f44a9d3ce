// Per-head RMS norm of queries and keys with the position rotation, forward and backward: one pass over each tensor, bound
// by memory.
//
// A lane owns two chunks of 8 columns of a head: in the rotated part those at columns 8 c and 8 c + rot / 2 (or, for
// neighbouring pairs, 8 c and 8 c + rot / 2 as well: either chunk then turns in itself), so that a rotation needs no other lane's
// columns; in the rest two neighbouring chunks.  LPH lanes (a power of two) share a head, 64 / LPH heads a wavefront; the
// mean of squares is a sum over LPH lanes.  A lane's columns are the same for every head and token it meets: the gain
// stays in registers, the token's cosines and sines are read once for all the heads that a wavefront takes of it, and the gain's
// gradient is a sum in registers, added up over lanes, wavefronts and blocks in a fixed order at the end.
// A unit of work is 64 / LPH heads of a token; a wavefront takes a run of units, and queries and keys get workgroups in proportion.
// 4096 tokens of 40 heads of 128 (bf16): forward 17 to 19 us (84 MB: 4.5 to 4.9 of the 5.7 TB/s that a copy moves), backward
// 32 (126 MB, 4.0 TB/s) and 4 for the gains; 3003 tokens of 32 heads of 64 (fp32): 14 (3.5 TB/s), 19 (3.8) and 4; one token of
// 64 samples 4, all of it latency (position, angles, heads).
#include "../../include/gx.h"
#include "gx_kernels.h"

namespace {

using namespace gx;

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

typedef float Chunk[8];

// Eight columns as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<bf16> {
  bf16x8 v;
  GX_DEVINL void load(const bf16* p) { v = *reinterpret_cast<const bf16x8*>(p); }
  GX_DEVINL void zero() { v = bf16x8{}; }
  GX_DEVINL void widen(Chunk& o) const {
#pragma unroll
    for (int e = 0; e < 8; e++) o[e] = (float)v[e];
  }
};
template <> struct Raw8<float> {
  f32x4 v[2];
  GX_DEVINL void load(const float* p) {
#pragma unroll
    for (int h = 0; h < 2; h++) v[h] = reinterpret_cast<const f32x4*>(p)[h];
  }
  GX_DEVINL void zero() { v[0] = v[1] = f32x4{0.f, 0.f, 0.f, 0.f}; }
  GX_DEVINL void widen(Chunk& o) const {
#pragma unroll
    for (int e = 0; e < 8; e++) o[e] = v[e >> 2][e & 3];
  }
};
GX_DEVINL void store8(bf16* p, const Chunk& x) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; e++) v[e] = (bf16)x[e];
  *reinterpret_cast<bf16x8*>(p) = v;
}
GX_DEVINL void store8(float* p, const Chunk& x) {
#pragma unroll
  for (int h = 0; h < 2; h++) reinterpret_cast<f32x4*>(p)[h] = f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
}

struct Heads {
  char* p;
  long batch, token, head;         // strides in bytes
};
struct Side {
  Heads x, dy, out;                // dy: backward only
  const void* gain;
  const int* pos;
  float* part;                     // backward: partial gain gradients, [blocks of this side][head_dim], or null
  int len, heads, blocks;          // blocks: how many of the launch work on this side
  int per_token;                   // units of a token
  long units;
};
struct NormArgs {
  Side side[2];                    // queries, keys: the first side[0].blocks blocks take queries
  const float *cos, *sin;
  int batch, dh, rot, max_pos, lph_log;
  float eps;
};

// The two chunks of a lane: columns of chunk a and b; has_a, has_b; turned: they are rotated, by angles at ang_a / ang_b
struct Place {
  int a, b, ang_a, ang_b;
  bool has_a, has_b, turned;
  template <bool PAIRS>
  GX_DEVINL static Place of(int sub, int dh, int rot) {
    Place p;
    const int np = rot / 16;                         // chunk pairs in the rotated part
    p.turned = sub < np;
    if (p.turned) {
      p.a = 8 * sub;
      p.b = 8 * sub + rot / 2;
      p.ang_a = PAIRS ? p.a / 2 : p.a;
      p.ang_b = PAIRS ? p.b / 2 : p.a;
      p.has_a = p.has_b = true;
    } else {
      p.a = rot + 16 * (sub - np);
      p.b = p.a + 8;
      p.ang_a = p.ang_b = 0;
      p.has_a = p.a < dh;
      p.has_b = p.b < dh;
    }
    return p;
  }
};

// Whether a token can be turned: the tables have its position
GX_DEVINL bool has_position(const NormArgs& a, int pos) { return a.rot == 0 || (pos >= 0 && pos < a.max_pos); }

// The angles of a lane's columns at a token.  PAIRS: four for each chunk; else the same eight for both.
struct Angles {
  f32x4 c[2], s[2];
  template <bool PAIRS>
  GX_DEVINL void load(const NormArgs& a, const Place& p, int pos) {
    if (!p.turned || !has_position(a, pos)) return;       // (a token without its position is NaN whatever the angles are)
    const float* cr = a.cos + (size_t)pos * (a.rot / 2);
    const float* sr = a.sin + (size_t)pos * (a.rot / 2);
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int at = PAIRS ? (h ? p.ang_b : p.ang_a) : p.ang_a + 4 * h;
      c[h] = *reinterpret_cast<const f32x4*>(cr + at);
      s[h] = *reinterpret_cast<const f32x4*>(sr + at);
    }
  }
  // x -> R x, or with BACK R^T x
  template <bool PAIRS, bool BACK>
  GX_DEVINL void turn(Chunk& a, Chunk& b) const {
    if (PAIRS) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        one<BACK>(a[2 * i], a[2 * i + 1], c[0][i], s[0][i]);
        one<BACK>(b[2 * i], b[2 * i + 1], c[1][i], s[1][i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) one<BACK>(a[i], b[i], c[i >> 2][i & 3], s[i >> 2][i & 3]);
    }
  }
  template <bool BACK>
  GX_DEVINL static void one(float& x, float& y, float cv, float sv) {
    const float t = BACK ? fmaf(y, sv, x * cv) : fmaf(-y, sv, x * cv);
    y = BACK ? fmaf(-x, sv, y * cv) : fmaf(x, sv, y * cv);
    x = t;
  }
};

GX_DEVINL float head_sum(float v, int lph) {
  for (int o = lph >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <typename T>
struct RawPair {
  Raw8<T> a, b;
  GX_DEVINL void load(const char* head, const Place& p) {
    const T* row = reinterpret_cast<const T*>(head);
    a.zero();
    b.zero();
    if (p.has_a) a.load(row + p.a);
    if (p.has_b) b.load(row + p.b);
  }
};
template <typename T>
GX_DEVINL void store_pair(char* head, const Place& p, const Chunk& a, const Chunk& b) {
  T* row = reinterpret_cast<T*>(head);
  if (p.has_a) store8(row + p.a, a);
  if (p.has_b) store8(row + p.b, b);
}

// What a wavefront works on next: unit after unit, token after token
struct Cursor {
  long t;
  int b, i, hb;
  GX_DEVINL void start(const Side& s, long u) {
    t = u / s.per_token;
    hb = (int)(u - t * s.per_token);
    b = (int)(t / s.len);
    i = (int)(t - (long)b * s.len);
  }
  GX_DEVINL void next(const Side& s) {
    if (++hb < s.per_token) return;
    hb = 0;
    t++;
    if (++i == s.len) {
      i = 0;
      b++;
    }
  }
  GX_DEVINL long at(const Heads& x, int h) const { return b * x.batch + i * x.token + h * x.head; }
};

// A unit's loads are issued before the unit before it is worked on; its angles with them, for which the position has
// been read one unit earlier still.  A unit is of one token, so that it takes one scalar comparison to make all of a token's
// columns NaN whose position is not in the tables: its heads' factor r is.
template <typename T, bool PAIRS, bool BACK>
GX_DEVINL void work_on(const NormArgs& a, const Side& s, int blk, float (&red)[4][256]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lph = 1 << a.lph_log, sub = lane & (lph - 1), slot = lane >> a.lph_log, slots = 64 >> a.lph_log;
  const Place p = Place::of<PAIRS>(sub, a.dh, a.rot);
  Chunk ga, gb, sum_a, sum_b;
#pragma unroll
  for (int e = 0; e < 8; e++) {
    ga[e] = gb[e] = 1.f;
    sum_a[e] = sum_b[e] = 0.f;
  }
  const int w = blk * 4 + wave, waves = s.blocks * 4;
  const long u0 = s.units * w / waves, u1 = s.units * (w + 1) / waves;
  Cursor now;
  now.start(s, u0 < s.units ? u0 : 0);
  Cursor ahead = now;
  auto pos_of = [&](const Cursor& c) { return s.pos ? s.pos[c.t] : c.i; };
  RawPair<T> x, d;
  Angles ang;
  auto fetch = [&](const Cursor& c, int pos, RawPair<T>& xr, RawPair<T>& dr, Angles& an) {
    const int h = min(c.hb * slots + slot, s.heads - 1);      // a lane without a head reads another one's
    xr.load(s.x.p + c.at(s.x, h), p);
    if (BACK) dr.load(s.dy.p + c.at(s.dy, h), p);
    an.load<PAIRS>(a, p, pos);
  };
  const int pos_first = __builtin_amdgcn_readfirstlane(pos_of(now));
  bool there = has_position(a, pos_first);
  fetch(now, pos_first, x, d, ang);
  if (s.gain) {
    RawPair<T> g;
    g.load(static_cast<const char*>(s.gain), p);
    g.a.widen(ga);
    g.b.widen(gb);
  }
  const float inv = 1.0f / (float)a.dh;
  if (u0 + 1 < u1) ahead.next(s);
  int pos = pos_of(ahead);
  for (long u = u0; u < u1; u++) {
    RawPair<T> xn = x, dn = d;
    Angles an = ang;
    const Cursor then = ahead;
    bool there_then = there;
    if (u + 1 < u1) {
      const int pos_then = __builtin_amdgcn_readfirstlane(pos);
      there_then = has_position(a, pos_then);
      fetch(ahead, pos_then, xn, dn, an);
      if (u + 2 < u1) ahead.next(s);
      pos = pos_of(ahead);
    }
    const int h = now.hb * slots + slot;
    const bool live = h < s.heads;                    // the same for all lanes of a head
    Chunk xa, xb;
    x.a.widen(xa);
    x.b.widen(xb);
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e++) q = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], q));
    float r = rsqrtf(fmaf(head_sum(q, lph), inv, a.eps));
    if (!there) r = __builtin_nanf("");
    char* const out = s.out.p + now.at(s.out, h);
    if (!BACK) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        xa[e] *= r * ga[e];
        xb[e] *= r * gb[e];
      }
      if (p.turned) ang.turn<PAIRS, false>(xa, xb);
      if (live) store_pair<T>(out, p, xa, xb);
    } else {
      Chunk da, db;
      d.a.widen(da);
      d.b.widen(db);
      if (p.turned) ang.turn<PAIRS, true>(da, db);
      float m = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        xa[e] *= r;                                   // u
        xb[e] *= r;
        if (live) {
          sum_a[e] = fmaf(da[e], xa[e], sum_a[e]);
          sum_b[e] = fmaf(db[e], xb[e], sum_b[e]);
        }
        da[e] *= ga[e];                               // the gradient reaching u
        db[e] *= gb[e];
        m = fmaf(da[e], xa[e], fmaf(db[e], xb[e], m));
      }
      m = head_sum(m, lph) * inv;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        da[e] = r * fmaf(-xa[e], m, da[e]);
        db[e] = r * fmaf(-xb[e], m, db[e]);
      }
      if (live) store_pair<T>(out, p, da, db);
    }
    x = xn;
    d = dn;
    ang = an;
    now = then;
    there = there_then;
  }
  if (BACK && s.part) {
#pragma unroll
    for (int e = 0; e < 8; e++)
      for (int o = lph; o < 64; o <<= 1) {
        sum_a[e] += __shfl_xor(sum_a[e], o, 64);
        sum_b[e] += __shfl_xor(sum_b[e], o, 64);
      }
    if (slot == 0) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        if (p.has_a) red[wave][p.a + e] = sum_a[e];
        if (p.has_b) red[wave][p.b + e] = sum_b[e];
      }
    }
    __syncthreads();
    const int d = threadIdx.x;
    if (d < a.dh) s.part[(size_t)blk * a.dh + d] = (red[0][d] + red[1][d]) + (red[2][d] + red[3][d]);
  }
}

// Queries first; two calls, so that neither side's record is picked by an index (and copied to memory for that)
template <typename T, bool PAIRS, bool BACK>
__global__ void __launch_bounds__(256) heads_norm_kernel(NormArgs a) {
  __shared__ float red[4][256];
  const int blk = blockIdx.x;
  if (blk < a.side[0].blocks) work_on<T, PAIRS, BACK>(a, a.side[0], blk, red);
  else work_on<T, PAIRS, BACK>(a, a.side[1], blk - a.side[0].blocks, red);
}

// Sum of a side's partial rows (there may be none), in order: 8 lanes of 4 columns, 32 runs of rows
struct GainArgs {
  struct { const float* part; float* out; int blocks; } side[2];
  int dh, accumulate;
};
__global__ void __launch_bounds__(256) heads_gain_kernel(GainArgs a) {
  __shared__ f32x4 red[32][8];
  const float* part = blockIdx.y ? a.side[1].part : a.side[0].part;
  float* out = blockIdx.y ? a.side[1].out : a.side[0].out;
  const int blocks = blockIdx.y ? a.side[1].blocks : a.side[0].blocks;
  const int x = threadIdx.x & 7, y = threadIdx.x >> 3, c = blockIdx.x * 32 + x * 4;
  if (!out) return;
  const int per = (blocks + 31) / 32, r0 = min(y * per, blocks), r1 = min(r0 + per, blocks);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (c < a.dh) {
#pragma unroll 8
    for (int r = r0; r < r1; r++) s += *reinterpret_cast<const f32x4*>(part + (size_t)r * a.dh + c);
  }
  red[y][x] = s;
  __syncthreads();
  if (y > 0 || c >= a.dh) return;
#pragma unroll
  for (int k = 1; k < 32; k++) s += red[k][x];
  f32x4* o = reinterpret_cast<f32x4*>(out + c);
  if (a.accumulate) s += *o;
  *o = s;
}

// ------------------------------------------------------------------------------- host
// Workgroups of a pass with more units than they have wavefronts (backward: as many partial rows of the gains' gradients).  Two to
// four wavefronts per SIMD, each with the next unit's loads in flight, are enough; more of them have shorter runs, and read a
// token's angles more often.  Forward and backward, us, 4096 tokens of 40 heads of 128 (bf16) / 3003 of 32 of 64 (fp32): 1024 and 512
// workgroups 58.6 / 35.1, 2048 and 512 59.2 / 36.1, 2560 and 640 57.3 / 39.3, 4096 and 384 66.2 / 39.1, 2560 and 256 75.9 / 37.4,
// 5120 and 1536 67.1 / 43.2.  Without the loads ahead of the unit before, 2048 and 1024: 81.9 / 38.9.
constexpr int FWD_BLOCKS = 1024, BACK_BLOCKS = 512;

struct Shares {
  int lph_log, per_token[2], blocks[2];
  long units[2];
};
Shares shares_of(const gx_heads_norm_cfg& c, bool backward) {
  Shares l = {};
  const int lanes = c.rot_dim / 16 + cdiv(c.head_dim - c.rot_dim, 16);
  while ((1 << l.lph_log) < lanes) l.lph_log++;
  for (int k = 0; k < 2; k++) {
    l.per_token[k] = cdiv(k ? c.k_heads : c.q_heads, 64 >> l.lph_log);
    l.units[k] = (long)c.batch * (k ? c.k_len : c.q_len) * l.per_token[k];
  }
  const long all = l.units[0] + l.units[1];
  // one unit a wavefront while all of them find a place together; then runs of units, which read a token's angles once
  const long most = backward ? BACK_BLOCKS : FWD_BLOCKS;
  for (int k = 0; k < 2; k++) {
    if (l.units[k] == 0) continue;
    const long one_each = (l.units[k] + 3) / 4, share = (most * l.units[k] + all - 1) / all;
    l.blocks[k] = (int)(one_each < share ? one_each : share);
  }
  return l;
}

gx_status check(const gx_heads_norm_cfg* c) {
  if (!c) return GX_ERR_NULL;
  if (c->dtype != GX_F32 && c->dtype != GX_BF16) return GX_ERR_DTYPE;
  if (c->flags & ~(GX_ROPE_PAIRS | GX_ACCUM_WGRAD)) return GX_ERR_FLAGS;
  if (c->batch <= 0 || c->q_len < 0 || c->k_len < 0 || c->q_heads < 0 || c->k_heads < 0 || c->head_dim <= 0 || c->head_dim > 256 ||
      c->rot_dim < 0 || c->rot_dim > c->head_dim || c->max_pos < 0 || !(c->eps >= 0.f) || !(c->eps < INFINITY))
    return GX_ERR_SHAPE;
  if (c->head_dim % 8 || c->rot_dim % 16) return GX_ERR_DIVIS;
  return GX_OK;
}

// Whether a tensor's pointer and the strides that are used keep 16-byte alignment and a written one's elements are apart
gx_status check_heads(const gx_heads* t, long batch, long len, long heads, long dh, long e, bool written) {
  if (!t || !t->data) return GX_ERR_NULL;
  if (misaligned(t->data)) return GX_ERR_ALIGN;
  const long stride[3] = {(long)t->batch, (long)t->token, (long)t->head}, extent[3] = {batch, len, heads};
  for (int k = 0; k < 3; k++) {
    if (extent[k] == 1) continue;
    if (stride[k] < 0 || stride[k] > ((long)1 << 40) || (written && stride[k] < dh)) return GX_ERR_SHAPE;
    if ((stride[k] * e) & 15) return GX_ERR_ALIGN;
  }
  return GX_OK;
}
Heads heads_of(const gx_heads* t, long e) {
  return Heads{static_cast<char*>(t->data), (long)t->batch * e, (long)t->token * e, (long)t->head * e};
}

gx_status run(const gx_heads_norm_cfg* c, const gx_heads_norm_in* in, const gx_heads* dy[2], const gx_heads* out[2],
              float* dgain[2], void* workspace, bool backward, hipStream_t st) {
  gx_status bad = check(c);
  if (bad != GX_OK) return bad;
  if (!in) return GX_ERR_NULL;
  const long e = c->dtype == GX_BF16 ? 2 : 4;
  NormArgs a = {};
  a.cos = in->cos_table;
  a.sin = in->sin_table;
  a.batch = c->batch;
  a.dh = c->head_dim;
  a.rot = c->rot_dim;
  a.max_pos = c->max_pos;
  a.eps = c->eps;
  if (c->rot_dim > 0) {
    if (!a.cos || !a.sin) return GX_ERR_NULL;
    if (misaligned(a.cos) || misaligned(a.sin)) return GX_ERR_ALIGN;
  }
  const Shares l = shares_of(*c, backward);
  a.lph_log = l.lph_log;
  GainArgs gains = {};
  gains.dh = c->head_dim;
  gains.accumulate = (c->flags & GX_ACCUM_WGRAD) != 0;
  bool any_gain = false;
  float* part = static_cast<float*>(workspace);
  for (int k = 0; k < 2; k++) {
    Side& s = a.side[k];
    const gx_heads& x = k ? in->k : in->q;
    s.len = k ? c->k_len : c->q_len;
    s.heads = k ? c->k_heads : c->q_heads;
    s.blocks = l.blocks[k];
    s.per_token = l.per_token[k];
    s.units = l.units[k];
    if (s.blocks == 0) {                             // no token or no head: the gain's gradient is a sum of nothing
      if (!backward || !dgain[k]) continue;
      if (misaligned(dgain[k])) return GX_ERR_ALIGN;
      gains.side[k] = {nullptr, dgain[k], 0};
      any_gain = true;
      continue;
    }
    bad = check_heads(&x, c->batch, s.len, s.heads, c->head_dim, e, false);
    if (bad == GX_OK) bad = check_heads(out[k], c->batch, s.len, s.heads, c->head_dim, e, true);
    if (bad == GX_OK && backward) bad = check_heads(dy[k], c->batch, s.len, s.heads, c->head_dim, e, false);
    if (bad != GX_OK) return bad;
    s.x = heads_of(&x, e);
    s.out = heads_of(out[k], e);
    if (backward) s.dy = heads_of(dy[k], e);
    s.gain = k ? in->k_gain : in->q_gain;
    s.pos = k ? in->k_pos : in->q_pos;
    if (misaligned(s.gain) || (reinterpret_cast<uintptr_t>(s.pos) & 3)) return GX_ERR_ALIGN;
    if (backward && dgain[k]) {
      if (!s.gain || !workspace) return GX_ERR_NULL;
      if (misaligned(dgain[k]) || misaligned(workspace)) return GX_ERR_ALIGN;
      s.part = part;
      part += (size_t)s.blocks * c->head_dim;
      gains.side[k] = {s.part, dgain[k], s.blocks};
      any_gain = true;
    }
  }
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  const int blocks = a.side[0].blocks + a.side[1].blocks;
  if (blocks == 0 && !any_gain) return GX_OK;
  const bool bf = c->dtype == GX_BF16, pairs = c->flags & GX_ROPE_PAIRS;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, a); };
  if (backward && blocks > 0) {
    if (bf) pairs ? go(heads_norm_kernel<bf16, true, true>) : go(heads_norm_kernel<bf16, false, true>);
    else pairs ? go(heads_norm_kernel<float, true, true>) : go(heads_norm_kernel<float, false, true>);
  } else if (blocks > 0) {
    if (bf) pairs ? go(heads_norm_kernel<bf16, true, false>) : go(heads_norm_kernel<bf16, false, false>);
    else pairs ? go(heads_norm_kernel<float, true, false>) : go(heads_norm_kernel<float, false, false>);
  }
  if (hipGetLastError() != hipSuccess) return GX_ERR_LAUNCH;
  if (any_gain) hipLaunchKernelGGL(heads_gain_kernel, dim3(cdiv(c->head_dim, 32), 2), dim3(256), 0, st, gains);
  return hipGetLastError() == hipSuccess ? GX_OK : GX_ERR_LAUNCH;
}

}  // namespace

extern "C" {

size_t gx_heads_norm_workspace_bytes(const gx_heads_norm_cfg* cfg) {
  if (check(cfg) != GX_OK) return 0;
  const Shares l = shares_of(*cfg, true);
  return (size_t)(l.blocks[0] + l.blocks[1]) * cfg->head_dim * 4;
}

gx_status gx_heads_norm_fwd(const gx_heads_norm_cfg* cfg, const gx_heads_norm_in* in, const gx_heads* q_out,
                            const gx_heads* k_out, void* hip_stream) {
  const gx_heads *dy[2] = {nullptr, nullptr}, *out[2] = {q_out, k_out};
  float* dgain[2] = {nullptr, nullptr};
  return run(cfg, in, dy, out, dgain, nullptr, false, static_cast<hipStream_t>(hip_stream));
}

gx_status gx_heads_norm_bwd(const gx_heads_norm_cfg* cfg, const gx_heads_norm_in* in, const gx_heads* dq_out,
                            const gx_heads* dk_out, const gx_heads* dq, const gx_heads* dk, float* dq_gain, float* dk_gain,
                            void* workspace, void* hip_stream) {
  const gx_heads *dy[2] = {dq_out, dk_out}, *out[2] = {dq, dk};
  float* dgain[2] = {dq_gain, dk_gain};
  return run(cfg, in, dy, out, dgain, workspace, true, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
