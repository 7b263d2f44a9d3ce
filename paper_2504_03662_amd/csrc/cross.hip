// Cross attention: C-ABI entry points, and the launches that join the parts of one that was split (deterministic: parts are added
// in order).
#include "../../include/gx.h"
#include "cross.h"

namespace gx {
namespace {

template <typename T> GX_DEVINL void store4(T* p, const f32x4& v);
template <> GX_DEVINL void store4<float>(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }
template <> GX_DEVINL void store4<bf16>(bf16* p, const f32x4& v) {
  bf16x4 o;
#pragma unroll
  for (int e = 0; e < 4; e++) o[e] = (bf16)v[e];
  *reinterpret_cast<bf16x4*>(p) = o;
}

// `lpr` lanes (a power of two) to a row of dh columns, 4 columns each
struct Lane {
  long row;
  int c;
  GX_DEVINL Lane(int lpr_log) {
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    row = i >> lpr_log;
    c = ((int)i & ((1 << lpr_log) - 1)) * 4;
  }
};

// Parts are requested AHEAD at a time (one after the other, each costs a load's latency: 16 parts 8.6 us instead of 4) and
// added in order; beyond the last one the last is read again and counts for nothing.
constexpr int AHEAD = 8;

// T bf16: exponentials of base 2
template <typename T>
__global__ void __launch_bounds__(256) cross_join_fwd_kernel(CrossArgs a, int lpr_log) {
  const Lane x(lpr_log);
  const long all = (long)a.B * a.hk * a.rows;
  if (x.row >= all || x.c >= a.dh) return;
  const f32x2* ml = reinterpret_cast<const f32x2*>(a.part + a.splits * all * a.dh);
  constexpr bool BASE2 = sizeof(T) == 2;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.splits; s0 += AHEAD) {
    f32x2 p[AHEAD];
    f32x4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; u++) {
      const long at = min(s0 + u, a.splits - 1) * all + x.row;
      p[u] = ml[at];
      v[u] = *reinterpret_cast<const f32x4*>(a.part + at * a.dh + x.c);
    }
    float mm = m;
#pragma unroll
    for (int u = 0; u < AHEAD; u++) mm = fmaxf(mm, p[u][0]);
    const float to = mm == -INFINITY ? 0.f : mm, old = BASE2 ? __builtin_amdgcn_exp2f(m - to) : expf(m - to);
    l *= old;
    o *= old;
#pragma unroll
    for (int u = 0; u < AHEAD; u++) {
      const float e = BASE2 ? __builtin_amdgcn_exp2f(p[u][0] - to) : expf(p[u][0] - to), w = s0 + u < a.splits ? e : 0.f;
      l += p[u][1] * w;
      o += v[u] * w;
    }
    m = mm;
  }
  const float ref = m == -INFINITY ? 0.f : m;
  const int pair = (int)(x.row / a.rows), r = (int)(x.row - (long)pair * a.rows), kh = pair % a.hk, b = pair / a.hk;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  store4<T>(static_cast<T*>(a.out) + pair_offset(a.so, b, kh * a.group) + row_offset(a.so, a.group, r) + x.c, o * inv);
  if (a.lse && x.c == 0) {
    const int i = r / a.group, h = kh * a.group + (r - i * a.group);
    const float lse = BASE2 ? (ref + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : ref + logf(l);
    a.lse[((long)b * a.hk * a.group + h) * a.Sq + i] = l == 0.f ? -INFINITY : lse;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) cross_join_dq_kernel(CrossArgs a, int lpr_log) {
  const Lane x(lpr_log);
  const long all = (long)a.B * a.hk * a.rows;
  if (x.row >= all || x.c >= a.dh) return;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.splits; s0 += AHEAD) {
    f32x4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; u++)
      v[u] = *reinterpret_cast<const f32x4*>(a.part + (min(s0 + u, a.splits - 1) * all + x.row) * a.dh + x.c);
#pragma unroll
    for (int u = 0; u < AHEAD; u++)
      if (s0 + u < a.splits) o += v[u];
  }
  const int pair = (int)(x.row / a.rows), r = (int)(x.row - (long)pair * a.rows), kh = pair % a.hk, b = pair / a.hk;
  store4<T>(static_cast<T*>(a.dq) + pair_offset(a.sdq, b, kh * a.group) + row_offset(a.sdq, a.group, r) + x.c, o * a.scale);
}

// keys that do not count have no parts: zeros
template <typename T>
__global__ void __launch_bounds__(256) cross_join_dkv_kernel(CrossArgs a, int lpr_log) {
  const Lane x(lpr_log);
  const long all = (long)a.B * a.hk * a.Sk;
  if (x.row >= all || x.c >= a.dh) return;
  const int pair = (int)(x.row / a.Sk), j = (int)(x.row - (long)pair * a.Sk), kh = pair % a.hk, b = pair / a.hk;
  const int n = a.key_lens ? a.key_lens[b] : a.Sk;
  f32x4 dk = {0.f, 0.f, 0.f, 0.f}, dv = dk;
  if (j < n && (!a.key_mask || a.key_mask[(long)b * a.Sk + j] != 0)) {
    for (int s0 = 0; s0 < a.splits; s0 += AHEAD) {
      f32x4 v[AHEAD][2];
#pragma unroll
      for (int u = 0; u < AHEAD; u++) {
        const float* p = a.part + (min(s0 + u, a.splits - 1) * all + x.row) * 2 * a.dh + x.c;
        v[u][0] = *reinterpret_cast<const f32x4*>(p);
        v[u][1] = *reinterpret_cast<const f32x4*>(p + a.dh);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; u++)
        if (s0 + u < a.splits) {
          dk += v[u][0];
          dv += v[u][1];
        }
    }
  }
  store4<T>(static_cast<T*>(a.dk) + pair_offset(a.sdk, b, kh) + (long)j * a.sdk.t + x.c, dk);
  store4<T>(static_cast<T*>(a.dv) + pair_offset(a.sdv, b, kh) + (long)j * a.sdv.t + x.c, dv);
}

template <class K16, class K32>
hipError_t join(bool bf, K16 k16, K32 k32, const CrossArgs& a, long rows, hipStream_t s) {
  int log = 0;
  while ((4 << log) < a.dh) log++;
  const dim3 grid((unsigned)(((rows << log) + 255) / 256));
  if (bf) hipLaunchKernelGGL(k16, grid, dim3(256), 0, s, a, log);
  else hipLaunchKernelGGL(k32, grid, dim3(256), 0, s, a, log);
  return hipGetLastError();
}

}  // namespace

hipError_t cross_join_fwd(bool bf, const CrossArgs& a, hipStream_t s) {
  return join(bf, cross_join_fwd_kernel<bf16>, cross_join_fwd_kernel<float>, a, (long)a.B * a.hk * a.rows, s);
}
hipError_t cross_join_dq(bool bf, const CrossArgs& a, hipStream_t s) {
  return join(bf, cross_join_dq_kernel<bf16>, cross_join_dq_kernel<float>, a, (long)a.B * a.hk * a.rows, s);
}
hipError_t cross_join_dkv(bool bf, const CrossArgs& a, hipStream_t s) {
  return join(bf, cross_join_dkv_kernel<bf16>, cross_join_dkv_kernel<float>, a, (long)a.B * a.hk * a.Sk, s);
}

}  // namespace gx

namespace {

using namespace gx;

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

constexpr long MAX_TOKEN_STRIDE = 1 << 22, MAX_GROUP_SPAN = 1 << 28, MAX_COUNT = 1 << 30, MAX_KEYS = 1 << 22;

gx_status check(const gx_cross_cfg* c) {
  if (!c) return GX_ERR_NULL;
  if (c->dtype != GX_F32 && c->dtype != GX_BF16) return GX_ERR_DTYPE;
  if (c->flags != 0) return GX_ERR_FLAGS;
  if (c->batch <= 0 || c->q_len < 0 || c->k_len < 0 || c->q_heads <= 0 || c->k_heads <= 0 || c->head_dim <= 0 ||
      c->head_dim > 128 || !(c->scale > 0.f) || !(c->scale < INFINITY))
    return GX_ERR_SHAPE;
  if (c->q_heads % c->k_heads) return GX_ERR_DIVIS;
  if (c->dtype == GX_BF16 && c->head_dim != 64 && c->head_dim != 128) return GX_ERR_SHAPE;
  if (c->head_dim % 4) return GX_ERR_DIVIS;
  const long pairs = (long)c->batch * c->k_heads;
  if ((long)c->batch * c->q_heads >= MAX_COUNT || (long)c->q_len * c->q_heads >= MAX_COUNT || c->k_len > MAX_KEYS ||
      // workgroups of any launch, and rows of one that joins, fit a grid
      pairs * (cdiv((long)c->q_len * (c->q_heads / c->k_heads), 32) + 1L) * 64 >= (1L << 31) ||
      pairs * (cdiv(c->k_len, 32) + 1L) * 64 >= (1L << 31))
    return GX_ERR_SHAPE;
  return GX_OK;
}

CrossArgs args_of(const gx_cross_cfg& c) {
  CrossArgs a = {};
  a.B = c.batch;
  a.Sq = c.q_len;
  a.Sk = c.k_len;
  a.hk = c.k_heads;
  a.group = c.q_heads / c.k_heads;
  a.rows = c.q_len * a.group;
  a.dh = c.head_dim;
  a.scale = c.scale;
  a.splits = 1;
  return a;
}
long parts_of(const gx_cross_cfg& c, const CrossArgs& a, int pass) {
  return c.dtype == GX_BF16 ? cross_parts_bf16(a, pass) : cross_parts_f32(a, pass);
}
size_t align_up(size_t v) { return (v + 255) & ~(size_t)255; }
size_t rows_bytes(const CrossArgs& a) { return align_up((size_t)a.B * a.hk * a.rows * 4); }

// One tensor of heads: pointer and the strides that are used
gx_status take(const gx_heads* t, long batch, long len, long heads, long dh, long e, bool written, bool keys, HeadStrides& s,
               const void*& p) {
  if (len == 0) return GX_OK;
  if (!t || !t->data) return GX_ERR_NULL;
  if (misaligned(t->data)) return GX_ERR_ALIGN;
  const long stride[3] = {(long)t->batch, (long)t->token, (long)t->head}, extent[3] = {batch, len, heads};
  long used[3];
  for (int k = 0; k < 3; k++) {
    used[k] = extent[k] == 1 ? 0 : stride[k];
    if (used[k] < 0 || used[k] > (1L << 40) || (written && extent[k] > 1 && used[k] < dh)) return GX_ERR_SHAPE;
    if ((used[k] * e) & 15) return GX_ERR_ALIGN;
  }
  if (used[1] > MAX_TOKEN_STRIDE) return GX_ERR_SHAPE;
  if (keys) {                                  // rows of a tile end where their keys do
    if (len == 1) used[1] = dh;
    else if (used[1] < dh) return GX_ERR_SHAPE;
  }
  s = HeadStrides{used[0], used[1], used[2]};
  p = t->data;
  return GX_OK;
}

gx_status inputs(const gx_cross_cfg& c, const gx_cross_in* in, CrossArgs& a) {
  if (!in) return GX_ERR_NULL;
  const long e = c.dtype == GX_BF16 ? 2 : 4;
  gx_status st = take(&in->q, c.batch, c.q_len, c.q_heads, c.head_dim, e, false, false, a.sq, a.q);
  if (st == GX_OK) st = take(&in->k, c.batch, c.k_len, c.k_heads, c.head_dim, e, false, true, a.sk, a.k);
  if (st == GX_OK) st = take(&in->v, c.batch, c.k_len, c.k_heads, c.head_dim, e, false, true, a.sv, a.v);
  if (st != GX_OK) return st;
  if ((long)(a.group - 1) * a.sq.h >= MAX_GROUP_SPAN) return GX_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(in->key_lens) & 3) return GX_ERR_ALIGN;
  a.key_lens = in->key_lens;
  a.key_mask = in->key_mask;
  return GX_OK;
}

}  // namespace

extern "C" {

size_t gx_cross_workspace_bytes(const gx_cross_cfg* cfg, int is_backward) {
  if (check(cfg) != GX_OK) return 0;
  const CrossArgs a = args_of(*cfg);
  const size_t rows = (size_t)a.B * a.hk * a.rows, keys = (size_t)a.B * a.hk * a.Sk;
  // what `parts` parts of `one` bytes each need; one part is none
  auto room = [](long parts, size_t one) { return parts > 1 ? parts * one : 0; };
  if (!is_backward) return room(parts_of(*cfg, a, 0), rows * (a.dh + 2) * 4);
  const size_t dq = room(parts_of(*cfg, a, 1), rows * a.dh * 4), dkv = room(parts_of(*cfg, a, 2), keys * 2 * a.dh * 4);
  return 2 * rows_bytes(a) + (dq > dkv ? dq : dkv);
}

gx_status gx_cross_fwd(const gx_cross_cfg* cfg, const gx_cross_in* in, const gx_heads* o, float* lse, void* workspace,
                       void* hip_stream) {
  gx_status st = check(cfg);
  if (st != GX_OK) return st;
  CrossArgs a = args_of(*cfg);
  const bool bf = cfg->dtype == GX_BF16;
  st = inputs(*cfg, in, a);
  const void* out = nullptr;
  if (st == GX_OK) st = take(o, cfg->batch, cfg->q_len, cfg->q_heads, cfg->head_dim, bf ? 2 : 4, true, false, a.so, out);
  if (st != GX_OK) return st;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return GX_ERR_ALIGN;
  if (gx_cross_workspace_bytes(cfg, 0) > 0) {
    if (!workspace) return GX_ERR_NULL;
    if (misaligned(workspace)) return GX_ERR_ALIGN;
  }
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  if (a.rows == 0) return GX_OK;
  a.out = const_cast<void*>(out);
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  return (bf ? cross_fwd_bf16(a, s) : cross_fwd_f32(a, s)) == hipSuccess ? GX_OK : GX_ERR_LAUNCH;
}

gx_status gx_cross_bwd(const gx_cross_cfg* cfg, const gx_cross_in* in, const gx_heads* o, const float* lse, const gx_heads* d_o,
                       const gx_heads* dq, const gx_heads* dk, const gx_heads* dv, void* workspace, void* hip_stream) {
  gx_status st = check(cfg);
  if (st != GX_OK) return st;
  CrossArgs a = args_of(*cfg);
  const bool bf = cfg->dtype == GX_BF16;
  const long e = bf ? 2 : 4, B = cfg->batch, dh = cfg->head_dim;
  st = inputs(*cfg, in, a);
  const void *pq = nullptr, *pk = nullptr, *pv = nullptr;
  if (st == GX_OK) st = take(o, B, cfg->q_len, cfg->q_heads, dh, e, false, false, a.so, a.o);
  if (st == GX_OK) st = take(d_o, B, cfg->q_len, cfg->q_heads, dh, e, false, false, a.sdo, a.d_o);
  if (st == GX_OK) st = take(dq, B, cfg->q_len, cfg->q_heads, dh, e, true, false, a.sdq, pq);
  if (st == GX_OK) st = take(dk, B, cfg->k_len, cfg->k_heads, dh, e, true, false, a.sdk, pk);
  if (st == GX_OK) st = take(dv, B, cfg->k_len, cfg->k_heads, dh, e, true, false, a.sdv, pv);
  if (st != GX_OK) return st;
  if ((long)(a.group - 1) * a.sdo.h >= MAX_GROUP_SPAN) return GX_ERR_SHAPE;
  if (a.rows > 0 && (!lse || !workspace)) return GX_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(lse) & 3) || misaligned(workspace)) return GX_ERR_ALIGN;
  if (!device_is_gfx950()) return GX_ERR_ARCH;
  a.dq = const_cast<void*>(pq);
  a.dk = const_cast<void*>(pk);
  a.dv = const_cast<void*>(pv);
  a.lse = const_cast<float*>(lse);
  char* ws = static_cast<char*>(workspace);
  a.lrow = reinterpret_cast<float*>(ws);
  a.drow = reinterpret_cast<float*>(ws + rows_bytes(a));
  a.part = reinterpret_cast<float*>(ws + 2 * rows_bytes(a));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  return (bf ? cross_bwd_bf16(a, s) : cross_bwd_f32(a, s)) == hipSuccess ? GX_OK : GX_ERR_LAUNCH;
}

}  // extern "C"
