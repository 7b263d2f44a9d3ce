// fp32 cross attention on v_mfma_f32_32x32x2_f32: every product and sum is a full fp32 one, in a fixed order.
//
// As in the causal fp32 kernels a workgroup owns 32 rows (forward, dQ) or 32 keys (dK / dV) of a (sample, key head) pair and
// its 4 wavefronts take every 4th 32-wide tile of the other side, or every wavefront owns 32 and takes all the tiles.  Scores
// are taken transposed to the owner, so that an accumulator register is, as it stands, an operand of the next product (register
// v of a lane in half g holds tile row 8 (v / 4) + 4 g + v % 4).
// Operands come from global memory, requested while the tile before is worked on; where a tile's rows are the second operand of
// one product and the first of another (dQ, dK / dV) a wavefront puts what it holds of them into LDS and reads columns.  The parts'
// results are merged through LDS in wavefront order.  Head dimensions up to 128 (multiples of 4) are padded with zeros to 32, 64 or 128.
// Keys that do not count have bits of a 32-bit word per tile: their scores are left out by selection, and what is read of them
// is replaced by zeros before it becomes an operand.
// Bound by the matrix pipe where there are many tiles (2048 x 2048, 16 heads of 128: forward 365 us, 94 TFLOP/s of the 145 that a
// library product of fp32 reaches; a lone wavefront per SIMD does not overlap its exponentials), by latency where there are few:
// 3 x 257 x 333, 8 / 4 heads of 64: 17 us, 24 us (dQ) and 29 us (dK / dV in three parts, 4.5 to join them; whole 40).
#include "cross.h"

namespace gx {
namespace {

constexpr int PARTS = 4;          // wavefronts of a workgroup
constexpr unsigned ALL = 0xFFFFFFFFu;

GX_DEVINL f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; v++) z[v] = 0.f;
  return z;
}
GX_DEVINL int acc_row(int v, int g) { return 8 * (v >> 2) + 4 * g + (v & 3); }
GX_DEVINL bool bit_of(unsigned bits, int v, int g) { return (bits >> acc_row(v, g)) & 1u; }
GX_DEVINL f32x16 mfma(float a, float b, const f32x16& c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// One lane's share of 32 rows by DHP columns whose reduction index is the column: chunk c holds columns 8 c + 4 g .. + 3
template <int DHP>
GX_DEVINL void load_rows(const float* row, int dh, int g, f32x4 (&out)[DHP / 8]) {
#pragma unroll
  for (int c = 0; c < DHP / 8; c++) {
    const int d = 8 * c + 4 * g;
    out[c] = d < dh ? *reinterpret_cast<const f32x4*>(row + d) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
}
// 32 x 32 scores: sum over columns of a[row] * b[col]
template <int DHP>
GX_DEVINL f32x16 row_product(const f32x4 (&a)[DHP / 8], const f32x4 (&b)[DHP / 8]) {
  f32x16 s = zero16();
#pragma unroll
  for (int c = 0; c < DHP / 8; c++)
#pragma unroll
    for (int e = 0; e < 4; e++) s = mfma(a[c][e], b[c][e], s);
  return s;
}
// A tile's rows as the other operand of a product over them: a wavefront puts the rows that its lanes hold into LDS (zeros for
// rows that do not count) and reads columns.  A row's 16 spare bytes put rows that are written together into different banks.
template <int DHP>
constexpr int STRIDE = DHP + 4;
template <int DHP>
GX_DEVINL void put_rows(float* tile, const f32x4 (&x)[DHP / 8], bool on, int g, int l32) {
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int c = 0; c < DHP / 8; c++) {
    f32x4 y = x[c];
#pragma unroll
    for (int e = 0; e < 4; e++) y[e] = on ? y[e] : 0.f;
    *reinterpret_cast<f32x4*>(tile + l32 * STRIDE<DHP> + 8 * c + 4 * g) = y;
  }
  __builtin_amdgcn_wave_barrier();
}
// acc[dt][d][col] += sum over the tile's rows of x[row][d] * w[row][col]
template <int DHP>
GX_DEVINL void col_product(f32x16 (&acc)[DHP / 32], const f32x16& w, const float* tile, int g, int l32) {
  constexpr int AHEAD = DHP <= 32 ? 4 : 2;                   // rows read ahead of the products
  float x[AHEAD][DHP / 32];
  const float* const mine = tile + 4 * g * STRIDE<DHP> + l32;
  auto read = [&](int v) __attribute__((always_inline)) {
#pragma unroll
    for (int dt = 0; dt < DHP / 32; dt++) x[v % AHEAD][dt] = mine[acc_row(v, 0) * STRIDE<DHP> + 32 * dt];
  };
#pragma unroll
  for (int v = 0; v < AHEAD; v++) read(v);
#pragma unroll
  for (int v = 0; v < 16; v++) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int dt = 0; dt < DHP / 32; dt++) acc[dt] = mfma(x[v % AHEAD][dt], w[v], acc[dt]);
    if (v + AHEAD < 16) read(v + AHEAD);
  }
}
// Adds the parts' accumulators in the order of the wavefronts; the sum is complete in wavefront 0.
template <int DT>
GX_DEVINL void merge_parts(f32x16 (&acc)[DT], float* park, int part, int lane) {
  __syncthreads();
  if (part > 0)
#pragma unroll
    for (int dt = 0; dt < DT; dt++)
#pragma unroll
      for (int v = 0; v < 16; v++) park[((part - 1) * DT * 16 + 16 * dt + v) * 64 + lane] = acc[dt][v];
  __syncthreads();
  if (part == 0)
    for (int p = 0; p < PARTS - 1; p++)
#pragma unroll
      for (int dt = 0; dt < DT; dt++)
#pragma unroll
        for (int v = 0; v < 16; v++) acc[dt][v] += park[(p * DT * 16 + 16 * dt + v) * 64 + lane];
}
// one column (= one row of the tensor) of a transposed result: dst[d] = acc * scale
template <int DHP>
GX_DEVINL void store_column(const f32x16 (&acc)[DHP / 32], float* dst, float scale, int dh, int g) {
#pragma unroll
  for (int dt = 0; dt < DHP / 32; dt++)
#pragma unroll
    for (int q = 0; q < 4; q++) {
      const int d = 32 * dt + 8 * q + 4 * g;
      if (d < dh)
        *reinterpret_cast<f32x4*>(dst + d) = f32x4{acc[dt][4 * q] * scale, acc[dt][4 * q + 1] * scale, acc[dt][4 * q + 2] * scale,
                                                   acc[dt][4 * q + 3] * scale};
    }
}

// the pair, tile and split of a workgroup, and the keys that count
struct Where {
  int b, kh, pair, tile, split, len;
  GX_DEVINL Where(const CrossArgs& a, int tiles) {
    const Share x = share_of(a, blockIdx.x, tiles);
    b = x.b;
    kh = x.kh;
    pair = x.pair;
    tile = x.block;
    split = x.split;
    len = keys_of(a, b);
  }
};
// the mask's byte of this lane's key of the 32 from key j0 on, read a tile early, and the bits of the 32, the same in every lane
GX_DEVINL unsigned key_byte(const CrossArgs& a, int b, int j0, int l32) {
  return a.key_mask ? a.key_mask[(long)b * a.Sk + min(j0 + l32, a.Sk - 1)] : 1u;
}
GX_DEVINL unsigned key_bits(unsigned byte, int j0, int len, int l32) {
  return (unsigned)__builtin_amdgcn_ballot_w64(byte != 0 && j0 + l32 < len);
}
GX_DEVINL const float* f32_of(const void* p) { return static_cast<const float*>(p); }

// what exponents are taken relative to while a row has seen no key, or only scores of -inf
GX_DEVINL float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }

// EACH: every wavefront has 32 rows of its own and goes over all of the keys
template <int DHP, bool EACH>
__global__ void __launch_bounds__(64 * PARTS, DHP <= 64 ? 2 : 1) cross_fwd_f32_kernel(CrossArgs a) {
  constexpr int VALS = DHP / 2 + 2;
  __shared__ float lds[EACH ? 1 : (PARTS - 1) * VALS * 64];
  const int lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  constexpr int ROWS = EACH ? 32 * PARTS : 32, STEP = EACH ? 1 : PARTS;
  const Where w(a, (a.rows + ROWS - 1) / ROWS);
  const int first = EACH ? 0 : part, r = ROWS * w.tile + (EACH ? 32 * part : 0) + l32, rc = r < a.rows ? r : a.rows - 1;
  f32x4 qf[DHP / 8];
  load_rows<DHP>(f32_of(a.q) + pair_offset(a.sq, w.b, w.kh * a.group) + row_offset(a.sq, a.group, rc), a.dh, g, qf);
  f32x16 o[DHP / 32];
#pragma unroll
  for (int dt = 0; dt < DHP / 32; dt++) o[dt] = zero16();
  float m = -INFINITY, l = 0.f;
  const float* const kb = f32_of(a.k) + pair_offset(a.sk, w.b, w.kh);
  const float* const vb = f32_of(a.v) + pair_offset(a.sv, w.b, w.kh);
  const int nt = (w.len + 31) / 32;
  const int t0 = (int)((long)nt * w.split / a.splits), t1 = (int)((long)nt * (w.split + 1) / a.splits);
  f32x4 kf[DHP / 8];
  auto load_k = [&](int t) __attribute__((always_inline)) {
    load_rows<DHP>(kb + (long)min(32 * t + l32, w.len - 1) * a.sk.t, a.dh, g, kf);
  };
  unsigned byte = 0;
  if (t0 + first < t1) {
    byte = key_byte(a, w.b, 32 * (t0 + first), l32);
    load_k(t0 + first);
  }
  for (int t = t0 + first; t < t1; t += STEP) {
    const int j0 = 32 * t;
    const unsigned bits = key_bits(byte, j0, w.len, l32);
    float vf[DHP / 32][16];                                      // columns of the tile's rows, on their way while the scores are taken
#pragma unroll
    for (int v = 0; v < 16; v++) {
      const float* const row = vb + (long)min(j0 + acc_row(v, g), w.len - 1) * a.sv.t;
#pragma unroll
      for (int dt = 0; dt < DHP / 32; dt++) vf[dt][v] = row[min(32 * dt + l32, a.dh - 1)];    // columns beyond dh are never stored
    }
    __builtin_amdgcn_sched_barrier(0);
    f32x16 s = row_product<DHP>(kf, qf);                         // S^T[j][i]
    __builtin_amdgcn_sched_barrier(0);
    if (t + STEP < t1) {                                        // and these while the output is
      byte = key_byte(a, w.b, 32 * (t + STEP), l32);
      load_k(t + STEP);
    }
    __builtin_amdgcn_sched_barrier(0);
    float mx = -INFINITY;
    const float mold = m;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      s[v] = bit_of(bits, v, g) ? s[v] * a.scale : -INFINITY;
      mx = fmaxf(mx, s[v]);
    }
    m = fmaxf(m, max_across_halves(mx));
    const float ref = finite_ref(m), alpha = expf(mold - ref);
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; v++) {
      s[v] = expf(s[v] - ref);
      sum += s[v];
    }
    l = l * alpha + sum;
#pragma unroll
    for (int dt = 0; dt < DHP / 32; dt++)
#pragma unroll
      for (int v = 0; v < 16; v++) o[dt][v] *= alpha;
    if (bits != ALL) {
#pragma unroll
      for (int v = 0; v < 16; v++)
        if (!bit_of(bits, v, g)) {
#pragma unroll
          for (int dt = 0; dt < DHP / 32; dt++) vf[dt][v] = 0.f;
        }
    }
#pragma unroll
    for (int v = 0; v < 16; v++)
#pragma unroll
      for (int dt = 0; dt < DHP / 32; dt++) o[dt] = mfma(vf[dt][v], s[v], o[dt]);
  }
  if constexpr (!EACH) {
    // merge the parts' (m, l, O); a part without a key has m = -inf, l = 0, O = 0 and adds nothing
    if (part > 0) {
      float* p = lds + (part - 1) * VALS * 64 + lane;
      p[0] = m;
      p[64] = l;
#pragma unroll
      for (int dt = 0; dt < DHP / 32; dt++)
#pragma unroll
        for (int v = 0; v < 16; v++) p[(2 + 16 * dt + v) * 64] = o[dt][v];
    }
    __syncthreads();
    if (part > 0) return;
    for (int pp = 0; pp < PARTS - 1; pp++) {
      const float* p = lds + pp * VALS * 64 + lane;
      const float mm = fmaxf(m, p[0]), ref = finite_ref(mm), a0 = expf(m - ref), a1 = expf(p[0] - ref);
      l = l * a0 + p[64] * a1;
      m = mm;
#pragma unroll
      for (int dt = 0; dt < DHP / 32; dt++)
#pragma unroll
        for (int v = 0; v < 16; v++) o[dt][v] = o[dt][v] * a0 + p[(2 + 16 * dt + v) * 64] * a1;
    }
  }
  l += __shfl_xor(l, 32, 64);
  if (r >= a.rows) return;
  if (a.splits > 1) {
    const long npair = (long)a.B * a.hk, at = (w.split * npair + w.pair) * a.rows + r;
    store_column<DHP>(o, a.part + at * a.dh, 1.0f, a.dh, g);
    if (g == 0) *reinterpret_cast<f32x2*>(a.part + a.splits * npair * a.rows * a.dh + at * 2) = f32x2{m, l};
    return;
  }
  store_column<DHP>(o, static_cast<float*>(a.out) + pair_offset(a.so, w.b, w.kh * a.group) + row_offset(a.so, a.group, r),
                    l == 0.f ? 0.f : 1.0f / l, a.dh, g);
  if (a.lse && g == 0) {
    const int i = r / a.group, h = w.kh * a.group + (r - i * a.group);
    a.lse[((long)w.b * a.hk * a.group + h) * a.Sq + i] = l == 0.f ? -INFINITY : m + logf(l);
  }
}

// D = rowsum(dO * O), dS = P (dP - D), dQ = scale dS K; leaves D and lse in row order (+inf for a row without a key or with scores of
// -inf only, whose dQ is zeros)
template <int DHP, bool EACH>
__global__ void __launch_bounds__(64 * PARTS, DHP <= 64 ? 2 : 1) cross_dq_f32_kernel(CrossArgs a) {
  constexpr int TILE = 32 * STRIDE<DHP>;
  __shared__ alignas(16) float lds[PARTS * TILE];
  const int lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  constexpr int ROWS = EACH ? 32 * PARTS : 32, STEP = EACH ? 1 : PARTS;
  const Where w(a, (a.rows + ROWS - 1) / ROWS);
  const int first = EACH ? 0 : part, r = ROWS * w.tile + (EACH ? 32 * part : 0) + l32, rc = r < a.rows ? r : a.rows - 1;
  const int head0 = w.kh * a.group;
  f32x4 qf[DHP / 8], dof[DHP / 8];
  load_rows<DHP>(f32_of(a.q) + pair_offset(a.sq, w.b, head0) + row_offset(a.sq, a.group, rc), a.dh, g, qf);
  load_rows<DHP>(f32_of(a.d_o) + pair_offset(a.sdo, w.b, head0) + row_offset(a.sdo, a.group, rc), a.dh, g, dof);
  // D in dP's own order of summation: a row with one key has o = v to the bit, and its dS is exactly zero
  float dd = 0.f;
  {
    f32x4 of[DHP / 8];
    load_rows<DHP>(f32_of(a.o) + pair_offset(a.so, w.b, head0) + row_offset(a.so, a.group, rc), a.dh, g, of);
    const f32x16 all = row_product<DHP>(of, dof);
#pragma unroll
    for (int v = 0; v < 16; v++) dd = acc_row(v, g) == l32 ? all[v] : dd;       // the diagonal, in one of a column's lanes
  }
  dd += __shfl_xor(dd, 32, 64);
  const int i = rc / a.group, h = head0 + (rc - i * a.group);
  float lse = a.lse[((long)w.b * a.hk * a.group + h) * a.Sq + i];
  const bool none = lse == -INFINITY;
  if (none) lse = INFINITY;
  if (w.split == 0 && first == 0 && g == 0 && r < a.rows) {
    a.drow[(long)w.pair * a.rows + r] = dd;
    a.lrow[(long)w.pair * a.rows + r] = lse;
  }
  f32x16 dq[DHP / 32];
#pragma unroll
  for (int dt = 0; dt < DHP / 32; dt++) dq[dt] = zero16();
  const float* const kb = f32_of(a.k) + pair_offset(a.sk, w.b, w.kh);
  const float* const vb = f32_of(a.v) + pair_offset(a.sv, w.b, w.kh);
  const int nt = (w.len + 31) / 32;
  const int t0 = (int)((long)nt * w.split / a.splits), t1 = (int)((long)nt * (w.split + 1) / a.splits);
  float* const tile = lds + part * TILE;
  f32x4 kf[DHP / 8], vf[DHP / 8];
  auto row_of = [&](int t) __attribute__((always_inline)) { return (long)min(32 * t + l32, w.len - 1); };
  unsigned byte = 0;
  if (t0 + first < t1) {
    byte = key_byte(a, w.b, 32 * (t0 + first), l32);
    load_rows<DHP>(kb + row_of(t0 + first) * a.sk.t, a.dh, g, kf);
    load_rows<DHP>(vb + row_of(t0 + first) * a.sv.t, a.dh, g, vf);
  }
  for (int t = t0 + first; t < t1; t += STEP) {
    const unsigned bits = key_bits(byte, 32 * t, w.len, l32);
    const bool more = t + STEP < t1;
    f32x16 s = row_product<DHP>(kf, qf);                         // S^T[j][i]
    __builtin_amdgcn_sched_barrier(0);
    put_rows<DHP>(tile, kf, (bits >> l32) & 1u, g, l32);
    if (more) {                                                  // on their way during the rest of this tile
      byte = key_byte(a, w.b, 32 * (t + STEP), l32);
      load_rows<DHP>(kb + row_of(t + STEP) * a.sk.t, a.dh, g, kf);
    }
    __builtin_amdgcn_sched_barrier(0);
    const f32x16 dp = row_product<DHP>(vf, dof);                 // dP^T[j][i]
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_rows<DHP>(vb + row_of(t + STEP) * a.sv.t, a.dh, g, vf);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int v = 0; v < 16; v++) s[v] = bit_of(bits, v, g) ? expf(s[v] * a.scale - lse) * (dp[v] - dd) : 0.f;
    col_product<DHP>(dq, s, tile, g, l32);
  }
  if constexpr (!EACH) merge_parts(dq, lds, part, lane);
  if (first != 0 || r >= a.rows) return;
  if (none) {                                                    // its sum may hold 0 times a key's infinity
#pragma unroll
    for (int dt = 0; dt < DHP / 32; dt++) dq[dt] = zero16();
  }
  if (a.splits > 1) store_column<DHP>(dq, a.part + (((long)w.split * a.B * a.hk + w.pair) * a.rows + r) * a.dh, 1.0f, a.dh, g);
  else store_column<DHP>(dq, static_cast<float*>(a.dq) + pair_offset(a.sdq, w.b, head0) + row_offset(a.sdq, a.group, r), a.scale,
                         a.dh, g);
}

// dV_j = sum_i P_ij dO_i, dK_j = scale sum_i dS_ij Q_i over the pair's rows.  A lane owns a key; what the lanes of keys that do not
// count compute stays in their columns, and zeros are stored for them.
template <int DHP, bool EACH>
__global__ void __launch_bounds__(64 * PARTS, DHP <= 64 ? 2 : 1) cross_dkv_f32_kernel(CrossArgs a) {
  constexpr int TILE = 32 * STRIDE<DHP>;
  __shared__ alignas(16) float lds[PARTS * TILE + PARTS * 64];
  const int lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  constexpr int KEYS = EACH ? 32 * PARTS : 32, STEP = EACH ? 1 : PARTS;
  const Where w(a, (a.Sk + KEYS - 1) / KEYS);
  const int first = EACH ? 0 : part, j0 = KEYS * w.tile + (EACH ? 32 * part : 0), j = j0 + l32, head0 = w.kh * a.group;
  const long jc = min(j, a.Sk - 1);
  const unsigned bits = key_bits(key_byte(a, w.b, j0, l32), j0, w.len, l32);
  const bool on = (bits >> l32) & 1u;
  f32x16 dk[DHP / 32], dv[DHP / 32];
#pragma unroll
  for (int dt = 0; dt < DHP / 32; dt++) dk[dt] = dv[dt] = zero16();
  if (bits) {
    f32x4 kf[DHP / 8], vf[DHP / 8];
    load_rows<DHP>(f32_of(a.k) + pair_offset(a.sk, w.b, w.kh) + jc * a.sk.t, a.dh, g, kf);
    load_rows<DHP>(f32_of(a.v) + pair_offset(a.sv, w.b, w.kh) + jc * a.sv.t, a.dh, g, vf);
    const float* const qb = f32_of(a.q) + pair_offset(a.sq, w.b, head0);
    const float* const dob = f32_of(a.d_o) + pair_offset(a.sdo, w.b, head0);
    const float* const lrow = a.lrow + (long)w.pair * a.rows;
    const float* const drow = a.drow + (long)w.pair * a.rows;
    const int nt = (a.rows + 31) / 32;
    const int t0 = (int)((long)nt * w.split / a.splits), t1 = (int)((long)nt * (w.split + 1) / a.splits);
    float* const tile = lds + part * TILE;
    float* const values = lds + PARTS * TILE + part * 64;        // lse of the tile's rows, then D
    f32x4 qf[DHP / 8], dof[DHP / 8];
    auto row_of = [&](int t) __attribute__((always_inline)) { return min(32 * t + l32, a.rows - 1); };
    float value = 0.f;                                           // lane l: lse of row l, lane 32 + l: D
    if (t0 + first < t1) {
      const int i = row_of(t0 + first);
      value = (g ? drow : lrow)[i];
      load_rows<DHP>(qb + row_offset(a.sq, a.group, i), a.dh, g, qf);
      load_rows<DHP>(dob + row_offset(a.sdo, a.group, i), a.dh, g, dof);
    }
    for (int t = t0 + first; t < t1; t += STEP) {
      const int left = a.rows - 32 * t;
      const bool more = t + STEP < t1, counts = l32 < left;
      values[lane] = value;
      f32x16 p = row_product<DHP>(qf, kf);                       // S[i][j]
      __builtin_amdgcn_sched_barrier(0);
      f32x16 ds = row_product<DHP>(dof, vf);                     // dP[i][j]
      __builtin_amdgcn_sched_barrier(0);
      put_rows<DHP>(tile, dof, counts, g, l32);
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const f32x4 lse = *reinterpret_cast<const f32x4*>(values + 8 * q + 4 * g);
        const f32x4 dd = *reinterpret_cast<const f32x4*>(values + 32 + 8 * q + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const int v = 4 * q + e, i = acc_row(v, g);
          p[v] = i < left ? expf(p[v] * a.scale - lse[e]) : 0.f;
          ds[v] = i < left ? p[v] * (ds[v] - dd[e]) : 0.f;
        }
      }
      col_product<DHP>(dv, p, tile, g, l32);
      __builtin_amdgcn_sched_barrier(0);
      put_rows<DHP>(tile, qf, counts, g, l32);
      if (more) {                                                // the next tile's are on their way during the rest of this one
        const int next = row_of(t + STEP);
        value = (g ? drow : lrow)[next];
        load_rows<DHP>(dob + row_offset(a.sdo, a.group, next), a.dh, g, dof);
        load_rows<DHP>(qb + row_offset(a.sq, a.group, next), a.dh, g, qf);
      }
      __builtin_amdgcn_sched_barrier(0);
      col_product<DHP>(dk, ds, tile, g, l32);
    }
  }
  if constexpr (!EACH) {
    merge_parts(dk, lds, part, lane);
    merge_parts(dv, lds, part, lane);
  }
  if (first != 0 || j >= a.Sk) return;
  if (a.splits > 1) {
    if (!on) return;                                             // the launch that joins the splits stores zeros
    float* dst = a.part + (((long)w.split * a.B * a.hk + w.pair) * a.Sk + j) * 2 * a.dh;
    store_column<DHP>(dk, dst, a.scale, a.dh, g);
    store_column<DHP>(dv, dst + a.dh, 1.0f, a.dh, g);
    return;
  }
  if (!on) {
#pragma unroll
    for (int dt = 0; dt < DHP / 32; dt++) dk[dt] = dv[dt] = zero16();
  }
  store_column<DHP>(dk, static_cast<float*>(a.dk) + pair_offset(a.sdk, w.b, w.kh) + (long)j * a.sdk.t, a.scale, a.dh, g);
  store_column<DHP>(dv, static_cast<float*>(a.dv) + pair_offset(a.sdv, w.b, w.kh) + (long)j * a.sdv.t, 1.0f, a.dh, g);
}

// How a launch is cut, by an estimate in microseconds: a workgroup takes 4 and `alone` for each 32 x 32 tile of a wavefront's share,
// `pair` where two share a compute unit (0: one at a time); a launch of its own joins parts, which are written and read.  A workgroup
// works on 32 rows (dK / dV: keys) together, or on 32 for each wavefront, which few keys (rows) or many rows (keys) need.
// us, forward + backward, head dim 128, each / together: 3 x 6231 x 7, 8 / 1 heads 283 / 672; 2048 x 2048, 16 / 4 heads 1558 / 1603;
// one query, 8192 keys of 8 heads 113 / 213.
struct Tile { double alone, pair; };
struct Cut { int parts; bool each; double us; };
Cut best_cut(const Tile& c, long blocks, long units, int share, double part_mb) {
  Cut best{0, share == 1, 0.0};
  for (const int p : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
    if (p > 1 && units < 2 * p) break;
    const long n = cdiv(blocks * p, 256), per = cdiv(cdiv(units, p), share);
    double t = c.pair > 0 ? (n / 2) * (4.0 + per * c.pair) + (n % 2) * (4.0 + per * c.alone) : n * (4.0 + per * c.alone);
    if (p > 1) t += 3.5 + 0.04 * p + p * part_mb / 4.0;
    if (p == 1 || t < best.us) {
      best.parts = p;
      best.us = t;
    }
  }
  return best;
}
// pass 0: forward, 1: dQ, 2: dK / dV
Cut cut_of(const CrossArgs& a, int pass) {
  constexpr Tile COST[3][3] = {{{2.3, 3.3}, {3.0, 4.5}, {3.6, 5.5}},           // forward, dQ, dK / dV at head dims up to 32
                               {{4.5, 6.5}, {6.0, 9.0}, {7.2, 11.0}},          // 64
                               {{5.7, 0.0}, {7.5, 0.0}, {11.0, 0.0}}};         // 128
  const long pairs = (long)a.B * a.hk;
  const Tile& c = COST[a.dh <= 32 ? 0 : a.dh <= 64 ? 1 : 2][pass];
  const int own = pass == 2 ? a.Sk : a.rows, units = cdiv(pass == 2 ? a.rows : a.Sk, 32);
  const double mb = pairs * own * a.dh * (pass == 2 ? 16e-6 : 8e-6);
  const Cut together = best_cut(c, pairs * cdiv(own, 32), units, PARTS, mb);
  const Cut each = best_cut(c, pairs * cdiv(own, 32 * PARTS), units, 1, mb);
  return each.us < together.us ? each : together;
}

#define GX_CROSS_F32(KERNEL, TILES, EACH)                                                  \
  do {                                                                                     \
    const dim3 grid((unsigned)((long)a.B * a.hk * (TILES) * a.splits)), block(64 * PARTS); \
    if (a.dh <= 32) hipLaunchKernelGGL((KERNEL<32, EACH>), grid, block, 0, s, a);          \
    else if (a.dh <= 64) hipLaunchKernelGGL((KERNEL<64, EACH>), grid, block, 0, s, a);     \
    else hipLaunchKernelGGL((KERNEL<128, EACH>), grid, block, 0, s, a);                    \
  } while (0)

}  // namespace

int cross_parts_f32(const CrossArgs& a, int pass) { return cut_of(a, pass).parts; }

hipError_t cross_fwd_f32(const CrossArgs& args, hipStream_t s) {
  CrossArgs a = args;
  const Cut c = cut_of(a, 0);
  a.splits = c.parts;
  if (c.each) GX_CROSS_F32(cross_fwd_f32_kernel, cdiv(a.rows, 32 * PARTS), true);
  else GX_CROSS_F32(cross_fwd_f32_kernel, cdiv(a.rows, 32), false);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.splits == 1 ? e : cross_join_fwd(false, a, s);
}

hipError_t cross_bwd_f32(const CrossArgs& args, hipStream_t s) {
  CrossArgs a = args;
  hipError_t e = hipSuccess;
  if (a.rows > 0) {
    const Cut c = cut_of(a, 1);
    a.splits = c.parts;
    if (c.each) GX_CROSS_F32(cross_dq_f32_kernel, cdiv(a.rows, 32 * PARTS), true);
    else GX_CROSS_F32(cross_dq_f32_kernel, cdiv(a.rows, 32), false);
    e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) e = cross_join_dq(false, a, s);
  }
  if (e != hipSuccess || a.Sk == 0) return e;
  const Cut c = cut_of(a, 2);
  a.splits = c.parts;
  if (c.each) GX_CROSS_F32(cross_dkv_f32_kernel, cdiv(a.Sk, 32 * PARTS), true);
  else GX_CROSS_F32(cross_dkv_f32_kernel, cdiv(a.Sk, 32), false);
  e = hipGetLastError();
  return e != hipSuccess || a.splits == 1 ? e : cross_join_dkv(false, a, s);
}

}  // namespace gx
