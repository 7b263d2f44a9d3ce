// Per-head RMS norm of queries and keys with the position rotation, forward and backward: one pass over each tensor, bound
// by memory.
//
// A lane owns two chunks of 8 columns of a head: in the rotated part those at columns 8 c and 8 c + rot / 2 (or, for
// neighbouring pairs, 8 c and 8 c + rot / 2 as well: either chunk then turns in itself), so that a rotation needs no other lane's
// columns; in the rest two neighbouring chunks.  LPH lanes (a power of two) share a head, 64 / LPH heads a wavefront; the
// mean of squares is a sum over LPH lanes.  A lane's columns are the same for every head and token it meets: the gain
// stays in registers, the token's cosines and sines are read once for all of its heads, and the gain's gradient is a sum in
// registers, added up over lanes, wavefronts and blocks in a fixed order at the end.
#include "../../include/gx.h"
#include "gx_kernels.h"

namespace {

using namespace gx;

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

typedef float Chunk[8];

template <typename T> GX_DEVINL void load8(const T* p, Chunk& o);
template <> GX_DEVINL void load8<bf16>(const bf16* p, Chunk& o) {
  const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
  for (int e = 0; e < 8; e++) o[e] = (float)v[e];
}
template <> GX_DEVINL void load8<float>(const float* p, Chunk& o) {
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const f32x4 v = reinterpret_cast<const f32x4*>(p)[h];
#pragma unroll
    for (int e = 0; e < 4; e++) o[4 * h + e] = v[e];
  }
}
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

// The angles of a lane's columns at a token.  PAIRS: four for each chunk; else the same eight for both.
struct Angles {
  Chunk c, s;
  template <bool PAIRS>
  GX_DEVINL void load(const NormArgs& a, const Place& p, int pos) {
    if (!p.turned) return;
    if (pos < 0 || pos >= a.max_pos) {
#pragma unroll
      for (int e = 0; e < 8; e++) c[e] = s[e] = __builtin_nanf("");
      return;
    }
    const float* cr = a.cos + (size_t)pos * (a.rot / 2);
    const float* sr = a.sin + (size_t)pos * (a.rot / 2);
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int at = PAIRS ? (h ? p.ang_b : p.ang_a) : p.ang_a + 4 * h;
      const f32x4 x = *reinterpret_cast<const f32x4*>(cr + at), y = *reinterpret_cast<const f32x4*>(sr + at);
#pragma unroll
      for (int e = 0; e < 4; e++) {
        c[4 * h + e] = x[e];
        s[4 * h + e] = y[e];
      }
    }
  }
  // x -> R x, or with BACK R^T x
  template <bool PAIRS, bool BACK>
  GX_DEVINL void turn(Chunk& a, Chunk& b) const {
    if (PAIRS) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        one<BACK>(a[2 * i], a[2 * i + 1], c[i], s[i]);
        one<BACK>(b[2 * i], b[2 * i + 1], c[4 + i], s[4 + i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) one<BACK>(a[i], b[i], c[i], s[i]);
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
GX_DEVINL void load_pair(const char* head, const Place& p, Chunk& a, Chunk& b) {
  const T* row = reinterpret_cast<const T*>(head);
#pragma unroll
  for (int e = 0; e < 8; e++) a[e] = b[e] = 0.f;
  if (p.has_a) load8<T>(row + p.a, a);
  if (p.has_b) load8<T>(row + p.b, b);
}
template <typename T>
GX_DEVINL void store_pair(char* head, const Place& p, const Chunk& a, const Chunk& b) {
  T* row = reinterpret_cast<T*>(head);
  if (p.has_a) store8(row + p.a, a);
  if (p.has_b) store8(row + p.b, b);
}

// A wavefront takes tokens in a grid stride and goes over all heads of each.
template <typename T, bool PAIRS, bool BACK>
__global__ void __launch_bounds__(256) heads_norm_kernel(NormArgs a) {
  __shared__ float red[4][256];
  const bool keys = (int)blockIdx.x >= a.side[0].blocks;
  const Side& s = a.side[keys];
  const int blk = blockIdx.x - (keys ? a.side[0].blocks : 0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lph = 1 << a.lph_log, sub = lane & (lph - 1), slot = lane >> a.lph_log, slots = 64 >> a.lph_log;
  const Place p = Place::of<PAIRS>(sub, a.dh, a.rot);
  Chunk ga, gb, sum_a, sum_b;
#pragma unroll
  for (int e = 0; e < 8; e++) {
    ga[e] = gb[e] = 1.f;
    sum_a[e] = sum_b[e] = 0.f;
  }
  if (s.gain) load_pair<T>(static_cast<const char*>(s.gain), p, ga, gb);
  const float inv = 1.0f / (float)a.dh;
  const long tokens = (long)a.batch * s.len;
  for (long t = (long)blk * 4 + wave; t < tokens; t += (long)s.blocks * 4) {
    const long b = t / s.len, i = t - b * s.len;
    Angles ang;
    ang.load<PAIRS>(a, p, s.pos ? s.pos[t] : (int)i);
    for (int h = slot; h < s.heads; h += slots) {
      Chunk xa, xb;
      load_pair<T>(s.x.p + b * s.x.batch + i * s.x.token + h * s.x.head, p, xa, xb);
      float q = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) q = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], q));
      const float r = rsqrtf(fmaf(head_sum(q, lph), inv, a.eps));
      char* const out = s.out.p + b * s.out.batch + i * s.out.token + h * s.out.head;
      if (!BACK) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
          xa[e] *= r * ga[e];
          xb[e] *= r * gb[e];
        }
        if (p.turned) ang.turn<PAIRS, false>(xa, xb);
        store_pair<T>(out, p, xa, xb);
      } else {
        Chunk da, db;
        load_pair<T>(s.dy.p + b * s.dy.batch + i * s.dy.token + h * s.dy.head, p, da, db);
        if (p.turned) ang.turn<PAIRS, true>(da, db);
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) {
          xa[e] *= r;                                 // u
          xb[e] *= r;
          sum_a[e] = fmaf(da[e], xa[e], sum_a[e]);
          sum_b[e] = fmaf(db[e], xb[e], sum_b[e]);
          da[e] *= ga[e];                             // the gradient reaching u
          db[e] *= gb[e];
          m = fmaf(da[e], xa[e], fmaf(db[e], xb[e], m));
        }
        m = head_sum(m, lph) * inv;
#pragma unroll
        for (int e = 0; e < 8; e++) {
          da[e] = r * fmaf(-xa[e], m, da[e]);
          db[e] = r * fmaf(-xb[e], m, db[e]);
        }
        store_pair<T>(out, p, da, db);
      }
    }
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

// ------------------------------------------------------------------------------- host
constexpr int MAX_BLOCKS = 1024;           // of a side, backward: as many partial rows of the gain's gradient

int blocks_of(const gx_heads_norm_cfg& c, bool keys, bool backward) {
  const long len = keys ? c.k_len : c.q_len, heads = keys ? c.k_heads : c.q_heads;
  if (len == 0 || heads == 0) return 0;
  const long wgs = ((long)c.batch * len + 3) / 4, most = backward ? MAX_BLOCKS : 65536;
  return (int)(wgs < most ? wgs : most);
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
  const int lanes = c->rot_dim / 16 + cdiv(c->head_dim - c->rot_dim, 16);
  while ((1 << a.lph_log) < lanes) a.lph_log++;
  FinishSeg seg[2];
  int nseg = 0;
  float* part = static_cast<float*>(workspace);
  for (int k = 0; k < 2; k++) {
    Side& s = a.side[k];
    const gx_heads& x = k ? in->k : in->q;
    s.len = k ? c->k_len : c->q_len;
    s.heads = k ? c->k_heads : c->q_heads;
    s.blocks = blocks_of(*c, k, backward);
    if (s.blocks == 0) continue;
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
      seg[nseg++] = FinishSeg{s.part, dgain[k], s.blocks, c->head_dim, (c->flags & GX_ACCUM_WGRAD) != 0, 0};
    }
  }
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  const int blocks = a.side[0].blocks + a.side[1].blocks;
  if (blocks == 0) return GX_OK;
  const bool bf = c->dtype == GX_BF16, pairs = c->flags & GX_ROPE_PAIRS;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, a); };
  if (backward) {
    if (bf) pairs ? go(heads_norm_kernel<bf16, true, true>) : go(heads_norm_kernel<bf16, false, true>);
    else pairs ? go(heads_norm_kernel<float, true, true>) : go(heads_norm_kernel<float, false, true>);
  } else {
    if (bf) pairs ? go(heads_norm_kernel<bf16, true, false>) : go(heads_norm_kernel<bf16, false, false>);
    else pairs ? go(heads_norm_kernel<float, true, false>) : go(heads_norm_kernel<float, false, false>);
  }
  if (hipGetLastError() != hipSuccess) return GX_ERR_LAUNCH;
  if (nseg > 0 && colsum_finish(seg, nseg, st) != hipSuccess) return GX_ERR_LAUNCH;
  return GX_OK;
}

}  // namespace

extern "C" {

size_t gx_heads_norm_workspace_bytes(const gx_heads_norm_cfg* cfg) {
  if (check(cfg) != GX_OK) return 0;
  return (size_t)(blocks_of(*cfg, false, true) + blocks_of(*cfg, true, true)) * cfg->head_dim * 4;
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
