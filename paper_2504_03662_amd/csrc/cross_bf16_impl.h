// Body of the bf16 cross-attention kernels for one head dimension.  Included by cross_bf16.hip once per supported head
// dimension, inside a namespace of its own, with GX_ATTN_DH defined.
#include "attn_bf16_tiles.h"

// A value that is the same in all lanes, in a scalar register whatever the compiler thinks (a descriptor in vector registers makes
// it wrap every load that uses it in a loop)
GX_DEVINL unsigned uniform(unsigned x) { return __builtin_amdgcn_readfirstlane(x); }
GX_DEVINL const char* uniform(const char* p) {
  const unsigned long u = (unsigned long)p;
  return reinterpret_cast<const char*>((unsigned long)uniform((unsigned)u) | ((unsigned long)uniform((unsigned)(u >> 32)) << 32));
}

// ------------------------------------------------------------------------------- keys
// Tiles of ROWS keys of K or V.  A tile has a buffer descriptor of its own (64-bit base, so that a cache may be of any
// length) that ends with the keys there are: rows beyond read as zeros.  Keys whose mask bit is clear are not read either: their
// lanes' offsets are put out of range.
template <int ROWS, int NW>
struct KeyTiles {
  static constexpr int RPI = 64 / CPR, PER = ROWS / RPI / NW;
  static_assert(PER >= 1, "tile too small for the workgroup");
  const char* base;
  long tile_bytes;
  unsigned row_bytes;
  int len;
  unsigned voff[PER];
  GX_DEVINL void init(const bf16* p, long ld, int n, int wave, int lane) {
    base = reinterpret_cast<const char*>(p);
    row_bytes = (unsigned)ld * 2u;
    tile_bytes = (long)ROWS * ld * 2;
    len = n;
#pragma unroll
    for (int i = 0; i < PER; i++) {
      const int r = row_of(i, wave, lane), c = (lane % CPR) ^ swz(r);
      voff[i] = (unsigned)r * row_bytes + (unsigned)(c * 16);
    }
  }
  GX_DEVINL static int row_of(int i, int wave, int lane) { return RPI * (wave * PER + i) + lane / CPR; }
  // where tile t is and how much of it there is; a tile beyond the last one has no row
  struct Tile { const char* p; unsigned bytes; };
  GX_DEVINL Tile tile(int t) const {
    const int left = len - t * ROWS, n = left < 0 ? 0 : left < ROWS ? left : ROWS;
    return Tile{uniform(n > 0 ? base + (long)t * tile_bytes : base), uniform((unsigned)n * row_bytes)};
  }
  GX_DEVINL void issue(const Tile& x, char* dst, int wave, int i, bool on) const {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(x.p), 0, x.bytes, 0x00020000);
    // (a variable of its own: with the expression as an argument the compiler's host pass drops the kernels that come here)
    const unsigned off = on ? voff[i] : OOB;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_ptr)(dst + (wave * PER + i) * 1024), 16, off, 0, 0, 0);
  }
};

// Which of a workgroup's keys count, as bits, key j in bit j % 32 of word j / 32: the sample's mask for the workgroup's own keys is
// turned into words in LDS first (MASK), or only the length says so.
template <bool MASK>
struct KeyBits {
  const unsigned* words;           // MASK: in LDS
  int len;
  // bits of N (32 or 64) keys from key j0 on, j0 a multiple of N
  template <int N>
  GX_DEVINL unsigned long long of(int j0) const {
    if (j0 >= len) return 0ull;
    if (MASK) return N == 64 ? (unsigned long long)words[j0 >> 5] | ((unsigned long long)words[(j0 >> 5) + 1] << 32) : words[j0 >> 5];
    const int left = len - j0;
    if (left >= N) return N == 64 ? ~0ull : 0xFFFFFFFFull;
    return (1ull << left) - 1ull;
  }
  GX_DEVINL bool on(int j) const { return !MASK || (j < len && ((words[j >> 5] >> (j & 31)) & 1u)); }
};
// A workgroup of NT threads; `n` keys from `mask` on, words up to the next multiple of 64 keys and one tile more
template <int NT>
GX_DEVINL void mask_to_words(const unsigned char* mask, int n, unsigned* words, int nwords) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int w = wave * 2; w < nwords; w += NT / 32) {
    const int j = w * 32 + lane;
    const unsigned long long bits = __builtin_amdgcn_ballot_w64(j < n && mask[j < n ? j : 0] != 0);
    if (lane < 2) words[w + lane] = (unsigned)(bits >> (32 * lane));
  }
}
constexpr int MASK_KEYS = 131072;                // keys of one workgroup, at most (16 KB of mask bits)
constexpr int mask_words(int keys, int rows) { return 2 * ((keys + rows + 63) / 64 + 1); }

// zero (or -inf) for the accumulator values whose key does not count: register v of sub-tile jt is key 32 jt + 8 (v / 4) + 4 g + v % 4
template <int NJT>
GX_DEVINL void put_where_off(f32x16 (&a)[NJT], unsigned long long bits, int g, float value) {
#pragma unroll
  for (int jt = 0; jt < NJT; jt++) {
    const unsigned w = (unsigned)(bits >> (32 * jt)) >> (4 * g);
#pragma unroll
    for (int v = 0; v < 16; v++)
      if (!((w >> (8 * (v >> 2) + (v & 3))) & 1u)) a[jt][v] = value;
  }
}

// The reference exponent of a row that has seen no key: below every score that counts, and finite, so that differences are
// numbers.  (A score that counts but is -inf thus weighs 0.)
constexpr float NO_KEY = -3.0e38f;

// What a workgroup of the forward or dQ kernel works on
struct RowBlock {
  int b, kh, pair, split, i0, key0, len;         // len: keys from key0 on
  bool one;                                      // the sample has one step of keys at most, and the last split gets it
  template <int BQ, int ROWS>
  GX_DEVINL static RowBlock of(const CrossArgs& a, int blk) {
    RowBlock w;
    const Share x = share_of(a, blk, (a.rows + BQ - 1) / BQ);
    w.b = x.b;
    w.kh = x.kh;
    w.pair = x.pair;
    w.i0 = x.block * BQ;
    w.split = x.split;
    const int n = keys_of(a, w.b), nt = (n + ROWS - 1) / ROWS;
    const int t0 = (int)((long)nt * w.split / a.splits), t1 = (int)((long)nt * (w.split + 1) / a.splits);
    w.one = nt <= 1;
    w.key0 = t0 * ROWS;
    w.len = (t1 * ROWS < n ? t1 * ROWS : n) - w.key0;
    if (w.len < 0) w.len = 0;
    return w;
  }
};

// this lane's 8 steps of a 32-row operand read straight from global memory
GX_DEVINL void load_row(const bf16* row, int g, bf16x8 (&out)[DH / 16]) {
#pragma unroll
  for (int s = 0; s < DH / 16; s++) out[s] = *reinterpret_cast<const bf16x8*>(row + 8 * g + 16 * s);
}

// ------------------------------------------------------------------------------- forward
constexpr int FWD_REGION = (4 + DH / 2) * 64;    // a wavefront's parked state, in floats
// LDS: two buffers for K and two for V, or what the merge parks
constexpr int fwd_smem(int nq, int split, int bkv) {
  const int tiles = 4 * bkv * split * ROWB, parked = split > 1 ? nq * split * FWD_REGION * 4 : 0;
  return tiles > parked ? tiles : parked;
}

// End of a forward workgroup: the SPLIT partial states of each row block are merged through LDS (the tiles are no longer
// needed), every part finishing its share of the head-dim blocks; then o and lse, or this split's sums, are stored.
template <int NQ, int SPLIT>
GX_DEVINL void fwd_finish(const CrossArgs& a, const RowBlock& w, char* smem, f32x16 (&o)[DH / 32], float m, float lsum, int part,
                          int qs, int lane) {
  constexpr int NDT = DH / 32, OWN = NDT / SPLIT > 0 ? NDT / SPLIT : 1, OWNERS = NDT / OWN;
  const int g = lane >> 5, l32 = lane & 31;
  lsum += __shfl_xor(lsum, 32, 64);
  if constexpr (SPLIT > 1) {
    constexpr int REGION = FWD_REGION;
    float* mine = reinterpret_cast<float*>(smem) + (qs * SPLIT + part) * REGION;
    *reinterpret_cast<f32x2*>(mine + lane * 4) = f32x2{m, lsum};
#pragma unroll
    for (int dt = 0; dt < NDT; dt++)
#pragma unroll
      for (int q = 0; q < 4; q++)
        if (dt / OWN != part)
          *reinterpret_cast<f32x4*>(mine + 256 + ((dt * 4 + q) * 64 + lane) * 4) =
              f32x4{o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]};
    __syncthreads();
    if (part >= OWNERS) return;
    const float* all = reinterpret_cast<const float*>(smem) + qs * SPLIT * REGION;
    float mp[SPLIT], lp[SPLIT], mm = NO_KEY;
#pragma unroll
    for (int p = 0; p < SPLIT; p++) {
      const f32x2 v = *reinterpret_cast<const f32x2*>(all + p * REGION + lane * 4);
      mp[p] = v[0];
      lp[p] = v[1];
      mm = fmaxf(mm, mp[p]);
    }
    lsum = 0.f;
#pragma unroll
    for (int p = 0; p < SPLIT; p++) {
      mp[p] = __builtin_amdgcn_exp2f(mp[p] - mm);
      lsum += lp[p] * mp[p];
    }
    m = mm;
    f32x16 t[OWN];
#pragma unroll
    for (int k = 0; k < OWN; k++) {
      t[k] = zero16();
#pragma unroll
      for (int p = 0; p < SPLIT; p++) {
        f32x16 x;                                // this part's own share comes from its registers
        if (p == part) {
#pragma unroll
          for (int dt = 0; dt < NDT; dt++)
            if (dt == part * OWN + k) x = o[dt];
        } else {
#pragma unroll
          for (int q = 0; q < 4; q++) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(all + p * REGION + 256 +
                                                            (((part * OWN + k) * 4 + q) * 64 + lane) * 4);
#pragma unroll
            for (int e = 0; e < 4; e++) x[4 * q + e] = v[e];
          }
        }
#pragma unroll
        for (int v = 0; v < 16; v++) t[k][v] += x[v] * mp[p];
      }
    }
#pragma unroll
    for (int k = 0; k < OWN; k++) o[k] = t[k];
  }
  const int r = w.i0 + qs * 32 + l32;
  if (r >= a.rows) return;
  constexpr int NB = SPLIT > 1 ? OWN : NDT;      // head-dim blocks this wavefront stores, from block `first` on
  const int first = SPLIT > 1 ? part * OWN : 0;
  if (a.splits > 1) {
    const long npair = (long)a.B * a.hk, at = (w.split * npair + w.pair) * a.rows + r;
    float* row = a.part + at * DH + 32 * first;
#pragma unroll
    for (int dt = 0; dt < NB; dt++)
#pragma unroll
      for (int q4 = 0; q4 < 4; q4++)
        *reinterpret_cast<f32x4*>(row + 32 * dt + 8 * q4 + 4 * g) =
            f32x4{o[dt][4 * q4], o[dt][4 * q4 + 1], o[dt][4 * q4 + 2], o[dt][4 * q4 + 3]};
    if (g == 0 && first == 0)
      *reinterpret_cast<f32x2*>(a.part + a.splits * npair * a.rows * DH + at * 2) = f32x2{m, lsum};
    return;
  }
  const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
  bf16* row = static_cast<bf16*>(a.out) + pair_offset(a.so, w.b, w.kh * a.group) + row_offset(a.so, a.group, r) + 32 * first;
#pragma unroll
  for (int dt = 0; dt < NB; dt++)
#pragma unroll
    for (int q4 = 0; q4 < 4; q4++) {
      bf16x4 pk;
#pragma unroll
      for (int e = 0; e < 4; e++) pk[e] = (bf16)(o[dt][4 * q4 + e] * inv);
      *reinterpret_cast<bf16x4*>(row + 32 * dt + 8 * q4 + 4 * g) = pk;
    }
  if (a.lse && g == 0 && first == 0) {
    const int s = (int)((unsigned)r / (unsigned)a.group), h = w.kh * a.group + (r - s * a.group);
    a.lse[((long)w.b * a.hk * a.group + h) * a.Sq + s] = lsum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(lsum)) * LN2;
  }
}

// A workgroup owns 32 NQ rows; its NQ * SPLIT wavefronts are NQ blocks of 32 rows times SPLIT shares of the keys of a step, each
// a tile of BKV keys; their partial softmax states are merged through LDS at the end.  With a.splits > 1 workgroups also share
// a row block's keys.
// The step is the one of the causal forward kernel: in step t the products of the step before (O += V P, t - 1) and the scores
// of the next one (S, t + 1) are issued one by one, behind each its share of the softmax of step t; K(t + 2) and V(t) are
// requested in its first slots into two buffers each.  The reference exponent follows a row's maximum only when that exceeds it by
// more than 2^8, so that O is rescaled rarely (following every rise, 128 pairs of 2048 x 2048 took 338 us instead of 301).
// Arithmetic: base-2 exponentials of fp32 scores, sums of them in fp32 before P is rounded to bf16 for the product with V (an
// error of the size that V's own type has), O in fp32 until it is stored.
// Bound by the issue of matrix and vector instructions where there are rows: a product takes 32 ns of a SIMD with its share of the
// softmax, 15 alone (2 x 4096 x 4096, 32 / 8 heads of 128: 521 us, 1.06 PFLOP/s, a library product 1.53); by memory where there are
// few (one query of 40 heads, 16 x 8192 keys of 8 heads: 105 us, 5.1 TB/s).
template <int NQ, int SPLIT, int BKV, bool MASK>
__global__ void __launch_bounds__(64 * NQ * SPLIT, 2) cross_fwd_kernel(CrossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int NW = NQ * SPLIT, BQ = 32 * NQ, ROWS = BKV * SPLIT, TILE = ROWS * ROWB, NS = DH / 16;
  constexpr int NJT = BKV / 32, NG = 2 * NJT, NDT = DH / 32;
  static_assert((NQ & (NQ - 1)) == 0 && (BKV == 32 || BKV == 64), "shape of the step");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qs = wave % NQ, part = wave / NQ;
  const int g = lane >> 5, l32 = lane & 31;
  const RowBlock w = RowBlock::of<BQ, ROWS>(a, blockIdx.x);
  const int nt = (w.len + ROWS - 1) / ROWS;
  unsigned* const words = reinterpret_cast<unsigned*>(smem + fwd_smem(NQ, SPLIT, BKV));
  if (MASK) {
    mask_to_words<64 * NW>(a.key_mask + (long)w.b * a.Sk + w.key0, w.len, words, mask_words(w.len, ROWS));
    __syncthreads();
  }
  const KeyBits<MASK> bits{words, w.len};
  bf16x8 qf[NS];
  const int r = w.i0 + qs * 32 + l32;
  load_row(static_cast<const bf16*>(a.q) + pair_offset(a.sq, w.b, w.kh * a.group) +
               row_offset(a.sq, a.group, r < a.rows ? r : a.rows - 1), g, qf);
  f32x16 o[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; dt++) o[dt] = zero16();
  float m = NO_KEY, lsum = 0.f;
  const float c2 = a.scale * LOG2E;
  unsigned coff[2][NDT];
  cols_lane_offsets(lane, coff);

  char* const kst = smem;                             // K(t) at kst + (t & 1) * TILE
  char* const vst = smem + 2 * TILE;                  // V(t) at vst + (t & 1) * TILE
  typedef KeyTiles<ROWS, NW> Tiles;
  constexpr int PER = Tiles::PER;
  Tiles kt, vt;
  kt.init(static_cast<const bf16*>(a.k) + pair_offset(a.sk, w.b, w.kh) + w.key0 * a.sk.t, a.sk.t, w.len, wave, lane);
  vt.init(static_cast<const bf16*>(a.v) + pair_offset(a.sv, w.b, w.kh) + w.key0 * a.sv.t, a.sv.t, w.len, wave, lane);
  auto on = [&](int t, int i) __attribute__((always_inline)) { return bits.on(t * ROWS + Tiles::row_of(i, wave, lane)); };
  auto load_k = [&](int t) {
    const auto tile = kt.tile(t);
#pragma unroll
    for (int i = 0; i < PER; i++) kt.issue(tile, kst + (t & 1) * TILE, wave, i, on(t, i));
  };
  load_k(0);
  {
    const auto tile = vt.tile(0);
#pragma unroll
    for (int i = 0; i < PER; i++) vt.issue(tile, vst, wave, i, on(0, i));
  }
  load_k(1);
  WAIT_VM0();
  __syncthreads();
  f32x16 s_even[NJT], s_odd[NJT];                     // scores of an even and an odd step
#pragma unroll
  for (int jt = 0; jt < NJT; jt++) s_even[jt] = zero16();
  if (nt > 0) {
    const char* k0 = kst + part * BKV * ROWB;
    streamed<NJT * NS, 4>([&](int q) { return frag_rows(k0, 32 * (q / NS) + l32, q % NS, g); },
                          [&](int q, bf16x8 f) { s_even[q / NS] = MFMA(f, qf[q % NS], s_even[q / NS]); });
  }
  __syncthreads();                                    // K(2) goes into the buffer of K(0)
  bf16x8 pf[NG];                                      // P of the step before, 16 keys per entry
  struct VFrag { bf16x4 lo, hi; };
  auto v_request = [&](unsigned tile, auto P, VFrag& f) __attribute__((always_inline)) {
    constexpr int p = decltype(P)::value, dt = p / NG, u = p % NG;
    f.lo = lds_read_tr_issue<u * 16 * ROWB>(tile + coff[0][dt]);
    f.hi = lds_read_tr_issue<u * 16 * ROWB>(tile + coff[1][dt]);
  };
  auto v_get = [&](VFrag& f) __attribute__((always_inline)) {
    lds_pin(f.lo);
    lds_pin(f.hi);
    return __builtin_shufflevector(f.lo, f.hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  constexpr int NPV = NG * NDT, NSC = NJT * NS, VD = 4 < NPV ? 4 : NPV, KD = 4 < NSC ? 4 : NSC;
  auto flush = [&](unsigned tile) __attribute__((always_inline)) {     // O^T += V^T P^T of the step before, on its own
    VFrag vf[VD];
    unroll<VD>([&](auto P) __attribute__((always_inline)) { v_request(tile, P, vf[P]); });
    unroll<NPV>([&](auto P) __attribute__((always_inline)) {
      constexpr int p = decltype(P)::value, newer = 2 * ((p + VD < NPV ? p + VD : NPV) - p - 1);
      lds_wait_le<newer>();
      o[p / NG] = MFMA(v_get(vf[p % VD]), pf[p % NG], o[p / NG]);
      if constexpr (p + VD < NPV) v_request(tile, std::integral_constant<int, p + VD>(), vf[p % VD]);
    });
  };
  auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  auto step = [&](int t, f32x16 (&sacc)[NJT], f32x16 (&snxt)[NJT], auto first_tag) __attribute__((always_inline)) {
    constexpr bool FIRST = decltype(first_tag)::value;
    const int j0 = t * ROWS + part * BKV;              // this wave's keys of the step
    const unsigned vp = lds_addr(vst + ((t - 1) & 1) * TILE + part * BKV * ROWB);
    const char* kn = kst + ((t + 1) & 1) * TILE + part * BKV * ROWB;
    constexpr int NP = FIRST ? 0 : NPV, NM = NP + NSC, RS = NM / 4;
    constexpr int NREQ = FIRST ? PER : 2 * PER;        // V(0) came with K(0)
    const auto rk = kt.tile(t + 2), rv = vt.tile(t);
    // request i of the step: first this wavefront's share of K(t + 2), then of V(t)
    auto request = [&](int i) __attribute__((always_inline)) {
      if (i < PER) kt.issue(rk, kst + (t & 1) * TILE, wave, i, on(t + 2, i));
      else vt.issue(rv, vst + (t & 1) * TILE, wave, i - PER, on(t, i - PER));
    };
    VFrag vf[VD];
    bf16x8 kf[KD];
    if constexpr (!FIRST) unroll<VD>([&](auto P) __attribute__((always_inline)) { v_request(vp, P, vf[P]); });
    if constexpr (FIRST) {
#pragma unroll
      for (int q = 0; q < KD; q++) kf[q] = frag_rows(kn, 32 * (q / NS) + l32, q % NS, g);
    }
#pragma unroll
    for (int jt = 0; jt < NJT; jt++) snxt[jt] = zero16();
    float psum = 0.f, alpha = 1.f;
    bool moved = false;
    // the softmax of step t (base-2 exponentials, scale folded into the exponent's multiply-add) in pieces: 0 mask, 1
    // reference, then EPP scores each, O to rescale, 16 keys to round each
    constexpr int EPP = 2;
    constexpr int NE = 16 * NJT / EPP, P_E = 2, P_R = P_E + NE, P_P = P_R + 1, NPIECE = P_P + NG;
    auto piece = [&](auto K) __attribute__((always_inline)) {
      constexpr int k = decltype(K)::value;
      if constexpr (k == 0) {
        if (MASK || j0 + BKV > w.len) put_where_off<NJT>(sacc, bits.template of<BKV>(j0), g, -INFINITY);
      } else if constexpr (k == 1) {
        float mloc = sacc[0][0];
#pragma unroll
        for (int jt = 0; jt < NJT; jt++)
#pragma unroll
          for (int v = 0; v < 16; v++) mloc = fmaxf(mloc, sacc[jt][v]);
        mloc = max_across_halves(mloc) * c2;
        moved = __builtin_amdgcn_ballot_w64(mloc > m + 8.f) != 0;
        const float mnew = moved ? fmaxf(m, mloc) : m;
        alpha = __builtin_amdgcn_exp2f(m - mnew);
        m = mnew;
        lsum *= alpha;
        asm volatile("" : "+v"(m), "+v"(alpha));
      } else if constexpr (k < P_R) {
        constexpr int e = EPP * (k - P_E), jt = e / 16, v0 = e % 16;
#pragma unroll
        for (int v = v0; v < v0 + EPP; v++) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[jt][v], c2, -m));
          sacc[jt][v] = p;
          psum += p;
        }
        asm volatile("" : "+v"(psum));
      } else if constexpr (k < P_P) {
        if constexpr (!FIRST) {
          if (moved) {
#pragma unroll
            for (int d = 0; d < NDT; d++)
#pragma unroll
              for (int v = 0; v < 16; v++) o[d][v] *= alpha;
          }
        }
      } else {
        constexpr int u = k - P_P;
        pf[u] = pack_half(sacc[u >> 1], u & 1);
      }
    };
    // cost of the pieces in issue slots, for spreading them over the matrix instructions
    constexpr auto cost = [](int k) constexpr {
      return k == 0 ? 4 : k == 1 ? 12 + 8 * NJT : k < P_R ? 6 * EPP : 4;
    };
    constexpr auto upto = [cost](int k) constexpr { int c = 0; for (int x = 0; x < k; x++) c += cost(x); return c; };
    constexpr int TOTAL = upto(NPIECE);
    // piece k goes behind matrix instruction slot_of(k); rescaling behind the last product into O
    constexpr auto slot_of = [upto, cost](int k) constexpr {
      int sl = (upto(k) + cost(k) / 2) * NM / TOTAL;
      if (k >= P_R && sl < NP) sl = NP;
      return sl < NM ? sl : NM - 1;
    };
    __builtin_amdgcn_sched_barrier(0);
    piece(std::integral_constant<int, 0>());
    unroll<NM>([&](auto I) __attribute__((always_inline)) {
      constexpr int x = decltype(I)::value;
      if constexpr (x < NP) {
        // untracked reads younger than this product's, and the K fragments requested so far
        constexpr int newer = 2 * ((x + VD < NPV ? x + VD : NPV) - x - 1) + (x > NPV - KD ? x - (NPV - KD) : 0);
        lds_wait_le<newer>();
        o[x / NG] = MFMA(v_get(vf[x % VD]), pf[x % NG], o[x / NG]);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (x + VD < NPV) v_request(vp, std::integral_constant<int, x + VD>(), vf[x % VD]);
        if constexpr (x >= NPV - KD) {
          constexpr int q = x - (NPV - KD);
          kf[q] = frag_rows(kn, 32 * (q / NS) + l32, q % NS, g);
        }
      } else {
        constexpr int q = x - NP;
        snxt[q / NS] = MFMA(kf[q % KD], qf[q % NS], snxt[q / NS]);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (q + KD < NSC) kf[q % KD] = frag_rows(kn, 32 * ((q + KD) / NS) + l32, (q + KD) % NS, g);
      }
#pragma unroll
      for (int i = x * NREQ / RS; i < (x + 1) * NREQ / RS && i < NREQ; i++) request(i);
      unroll<NPIECE>([&](auto K) __attribute__((always_inline)) {
        if constexpr (decltype(K)::value > 0 && slot_of(decltype(K)::value) == x) piece(K);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    lsum += psum;
    // also where no step follows: the waits above count the reads of these products
#pragma unroll
    for (int jt = 0; jt < NJT; jt++) asm volatile("" : "+v"(snxt[jt]));
    meet();
  };
  if (nt > 0) {
    step(0, s_even, s_odd, std::true_type());
    int t = 1;
    for (; t + 1 < nt; t += 2) {
      step(t, s_odd, s_even, std::false_type());
      step(t + 1, s_even, s_odd, std::false_type());
    }
    if (t < nt) {
      step(t, s_odd, s_even, std::false_type());
      t++;
    }
    flush(lds_addr(vst + ((t - 1) & 1) * TILE + part * BKV * ROWB));
  }
  if (SPLIT > 1) __syncthreads();                     // the merge reuses the tile buffers
  fwd_finish<NQ, SPLIT>(a, w, smem, o, m, lsum, part, qs, lane);
}

// ------------------------------------------------------------------------------- backward: dQ
// Rows as in the forward kernel.  dS = P (dP - D) is rounded to bf16 once, as an operand.  D is taken from o as it was stored: the
// rounding of o, 2^-8 of |dO| |o| at most, stays in dS, beside dS's own rounding the smaller the more keys share a row, and no further
// pass over the keys is needed.  Where one step holds all the keys D is made exact first: a row's dS add up to what it lacks
// (two keys: dQ and dK off by 0.0024 of their norm, 0.0039 without; 8 x 2000 x 30, 16 / 4 heads of 64: 2 us of 59).
// 2 x 4096 x 4096, 32 / 8 heads of 128: 735 us, 1.12 PFLOP/s; a product takes 30 ns of a SIMD.
// Also forms D = rowsum(dO * O) and leaves D and lse * log2(e) in row order for the other
// kernel (the first split does); a row without a key, or with scores of -inf only, gets +inf there, so that its probabilities
// are 0, and zeros for its dQ (with such scores the sum holds 0 times a key's infinity).
template <int NQ, int SPLIT, int BKV, bool MASK>
__global__ void __launch_bounds__(64 * NQ * SPLIT, NQ * SPLIT == 4 ? 2 : 1) cross_dq_kernel(CrossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int NW = NQ * SPLIT, BQ = 32 * NQ, ROWS = BKV * SPLIT, STAGE = 2 * ROWS * ROWB;
  constexpr int NJT = BKV / 32;
  static_assert((SPLIT - 1) * NQ * (DH / 2) * 256 <= 2 * STAGE, "merge area fits the tile buffers");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qs = wave % NQ, part = wave / NQ;
  const int g = lane >> 5, l32 = lane & 31;
  const RowBlock w = RowBlock::of<BQ, ROWS>(a, blockIdx.x);
  const int nt = (w.len + ROWS - 1) / ROWS;
  unsigned* const words = reinterpret_cast<unsigned*>(smem + 2 * STAGE);
  if (MASK) {
    mask_to_words<64 * NW>(a.key_mask + (long)w.b * a.Sk + w.key0, w.len, words, mask_words(w.len, ROWS));
    __syncthreads();
  }
  const KeyBits<MASK> bits{words, w.len};
  const int r = w.i0 + qs * 32 + l32, rc = r < a.rows ? r : a.rows - 1;
  const int head0 = w.kh * a.group;
  bf16x8 qf[DH / 16], dof[DH / 16], of[DH / 16];
  load_row(static_cast<const bf16*>(a.q) + pair_offset(a.sq, w.b, head0) + row_offset(a.sq, a.group, rc), g, qf);
  load_row(static_cast<const bf16*>(a.d_o) + pair_offset(a.sdo, w.b, head0) + row_offset(a.sdo, a.group, rc), g, dof);
  load_row(static_cast<const bf16*>(a.o) + pair_offset(a.so, w.b, head0) + row_offset(a.so, a.group, rc), g, of);
  const int s = (int)((unsigned)rc / (unsigned)a.group), h = head0 + (rc - s * a.group);
  const float lse = a.lse[((long)w.b * a.hk * a.group + h) * a.Sq + s];
  const float lse2 = lse == -INFINITY ? INFINITY : lse * LOG2E;
  const float c2 = a.scale * LOG2E;
  unsigned coff[2][DH / 32];
  cols_lane_offsets(lane, coff);
  f32x16 dq[DH / 32];
#pragma unroll
  for (int dt = 0; dt < DH / 32; dt++) dq[dt] = zero16();
  typedef KeyTiles<ROWS, NW> Tiles;
  Tiles kt, vt;
  kt.init(static_cast<const bf16*>(a.k) + pair_offset(a.sk, w.b, w.kh) + w.key0 * a.sk.t, a.sk.t, w.len, wave, lane);
  vt.init(static_cast<const bf16*>(a.v) + pair_offset(a.sv, w.b, w.kh) + w.key0 * a.sv.t, a.sv.t, w.len, wave, lane);
  auto load = [&](int t) {
    char* dst = smem + (t & 1) * STAGE;
    const auto rk = kt.tile(t), rv = vt.tile(t);
#pragma unroll
    for (int i = 0; i < Tiles::PER; i++) {
      const bool on = bits.on(t * ROWS + Tiles::row_of(i, wave, lane));
      kt.issue(rk, dst, wave, i, on);
      vt.issue(rv, dst + ROWS * ROWB, wave, i, on);
    }
  };
  load(0);
  // D on the matrix pipe, in dP's own order of summation: a row with one key has o = v to the bit, and its dS is exactly zero
  float dd = 0.f;
  {
    f32x16 all = zero16();
#pragma unroll
    for (int x = 0; x < DH / 16; x++) all = MFMA(of[x], dof[x], all);
#pragma unroll
    for (int v = 0; v < 16; v++) dd = 8 * (v >> 2) + 4 * g + (v & 3) == l32 ? all[v] : dd;      // the diagonal, in one half
    dd += __shfl_xor(dd, 32, 64);
  }
  auto leave = [&]() __attribute__((always_inline)) {
    if (part == 0 && g == 0 && r < a.rows) {
      a.drow[(long)w.pair * a.rows + r] = dd;
      a.lrow[(long)w.pair * a.rows + r] = lse2;
    }
  };
  if (w.split == (w.one ? a.splits - 1 : 0) && !(w.one && nt == 1)) leave();
  WAIT_VM0();
  __syncthreads();
  if (w.one && nt == 1) {                               // all of a row's keys are here: what the first dS add up to goes to D
    const char* kp = smem + part * BKV * ROWB;
    const unsigned long long on = bits.template of<BKV>(part * BKV) >> (4 * g);
    float rest = 0.f;
#pragma unroll 1
    for (int jt = 0; jt < NJT; jt++) {
      f32x16 sc = zero16(), dp = zero16();
#pragma unroll
      for (int x = 0; x < DH / 16; x++) {
        sc = MFMA(frag_rows(kp, 32 * jt + l32, x, g), qf[x], sc);
        dp = MFMA(frag_rows(kp + ROWS * ROWB, 32 * jt + l32, x, g), dof[x], dp);
      }
#pragma unroll
      for (int v = 0; v < 16; v++) {
        const float ds = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[v], c2, -lse2)) * (dp[v] - dd);
        rest += (on >> (32 * jt + 8 * (v >> 2) + (v & 3))) & 1u ? ds : 0.f;
      }
    }
    rest += __shfl_xor(rest, 32, 64);
    if (SPLIT > 1) {
      float* const shares = reinterpret_cast<float*>(smem + STAGE);     // the second stage: no tile follows
      if (g == 0) shares[(part * NQ + qs) * 32 + l32] = rest;
      __syncthreads();
      rest = 0.f;
#pragma unroll
      for (int pp = 0; pp < SPLIT; pp++) rest += shares[(pp * NQ + qs) * 32 + l32];
    }
    dd += rest;
    leave();
  }
  for (int t = 0; t < nt; t++) {
    if (t + 1 < nt) load(t + 1);
    const int j0 = t * ROWS + part * BKV;
    const char* kp = smem + (t & 1) * STAGE + part * BKV * ROWB;
    const char* vp = kp + ROWS * ROWB;
    f32x16 sacc[NJT], pacc[NJT];
#pragma unroll
    for (int jt = 0; jt < NJT; jt++) {
      sacc[jt] = zero16();
      pacc[jt] = zero16();
#pragma unroll
      for (int x = 0; x < DH / 16; x++) {
        sacc[jt] = MFMA(frag_rows(kp, 32 * jt + l32, x, g), qf[x], sacc[jt]);    // S^T[j][i]
        pacc[jt] = MFMA(frag_rows(vp, 32 * jt + l32, x, g), dof[x], pacc[jt]);   // dP^T[j][i]
      }
    }
#pragma unroll
    for (int jt = 0; jt < NJT; jt++)
#pragma unroll
      for (int v = 0; v < 16; v++) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[jt][v], c2, -lse2));
        pacc[jt][v] = p * (pacc[jt][v] - dd);                                    // dS^T
      }
    // the scores are dead: their registers take the first transposed K fragments
    const unsigned ct = lds_addr(kp);
    ColFrags cf[2];
    cols_issue<0>(ct, coff, cf[0]);
    cols_issue<1>(ct, coff, cf[1]);
    if (MASK || j0 + BKV > w.len) put_where_off<NJT>(pacc, bits.template of<BKV>(j0), g, 0.f);
    bf16x8 dsf[2 * NJT];
#pragma unroll
    for (int u = 0; u < 2 * NJT; u++) dsf[u] = pack_half(pacc[u >> 1], u & 1);
    tr_product<2 * NJT>(dq, ct, coff, cf, dsf);       // dQ^T[d][i] += K^T dS^T
    WAIT_VM0();
    __syncthreads();
  }
  if (SPLIT > 1) {
    constexpr int REGION = (DH / 2) * 64;
    if (part > 0) {
      float* park = reinterpret_cast<float*>(smem) + ((part - 1) * NQ + qs) * REGION + lane;
#pragma unroll
      for (int dt = 0; dt < DH / 32; dt++)
#pragma unroll
        for (int v = 0; v < 16; v++) park[(16 * dt + v) * 64] = dq[dt][v];
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int pp = 1; pp < SPLIT; pp++) {
      const float* park = reinterpret_cast<const float*>(smem) + ((pp - 1) * NQ + qs) * REGION + lane;
#pragma unroll
      for (int dt = 0; dt < DH / 32; dt++)
#pragma unroll
        for (int v = 0; v < 16; v++) dq[dt][v] += park[(16 * dt + v) * 64];
    }
  }
  if (r >= a.rows) return;
  if (lse == -INFINITY) {
#pragma unroll
    for (int dt = 0; dt < DH / 32; dt++) dq[dt] = zero16();
  }
  if (a.splits > 1) {
    float* row = a.part + (((long)w.split * a.B * a.hk + w.pair) * a.rows + r) * DH;
#pragma unroll
    for (int dt = 0; dt < DH / 32; dt++)
#pragma unroll
      for (int q4 = 0; q4 < 4; q4++)
        *reinterpret_cast<f32x4*>(row + 32 * dt + 8 * q4 + 4 * g) =
            f32x4{dq[dt][4 * q4], dq[dt][4 * q4 + 1], dq[dt][4 * q4 + 2], dq[dt][4 * q4 + 3]};
    return;
  }
  bf16* row = static_cast<bf16*>(a.dq) + pair_offset(a.sdq, w.b, head0) + row_offset(a.sdq, a.group, r);
#pragma unroll
  for (int dt = 0; dt < DH / 32; dt++)
#pragma unroll
    for (int q4 = 0; q4 < 4; q4++) {
      bf16x4 pk;
#pragma unroll
      for (int e = 0; e < 4; e++) pk[e] = (bf16)(dq[dt][4 * q4 + e] * a.scale);
      *reinterpret_cast<bf16x4*>(row + 32 * dt + 8 * q4 + 4 * g) = pk;
    }
}

// ------------------------------------------------------------------------------- backward: dK, dV
// A workgroup owns 128 keys as 4 blocks of 32 and goes over the pair's rows (or, with a.splits > 1, a part of them) in tiles of
// 64, two sub-tiles of 32; each block belongs to a pair of wavefronts that split the work by output, as in the causal kernel: role V
// forms S = Q K^T, the probabilities P and dV += P^T dO, role K dP = dO V^T, dS = P (dP - D) and dK += dS^T Q, a tile behind.
// A wavefront's stream mixes the first products of its next sub-tile with the vector work of the present one.  One
// workgroup of 8 wavefronts fills a compute unit; wavefronts w and w + 4 share a SIMD, one of either role.
// 2 x 4096 x 4096, 32 / 8 heads of 128: 1100 us, 1.0 PFLOP/s; 4 x 2048 x 1501 .. 938, 16 heads: 240 us, of which the last of three
// rounds fills 128 of 256 compute units.
// P crosses through LDS in 16 bits: 0 <= P < 2, so an fp32 P has two leading zero bits, and the next 16 (7 of the exponent, 9 of
// the mantissa, rounded) say P to 2^-10 over the whole range: dS is then rounded to bf16 once, not twice.  (P is 1 at most but for the
// rounding of lse: 2 takes an lse of millions, which puts P off by its own size, and then reads as nearly 0.  A NaN reads as a number,
// but its row's o and so D are NaN.)
// Keys that do not count are columns of their own in S and dP and rows of their own in dK and dV: whatever
// their lanes compute stays there, and zeros are stored.
constexpr int KV_PAIRS = 4, KV_NW = 2 * KV_PAIRS, KV_BJ = 32 * KV_PAIRS, KV_SUB = 2, KV_BI = 32 * KV_SUB;
constexpr int KV_NQ = 4, KV_NDO = 3;                         // Q tiles n-1 .. n+2, dO tiles n-1 .. n+1
constexpr int KV_TILE = KV_BI * ROWB + KV_BI * 4;            // rows of Q or dO | their D or lse
constexpr int KV_PX = KV_PAIRS * KV_SUB * 2 * 1024;          // P exchange: [pair][sub-tile][half][lane] x 16 B
constexpr int KV_OFF_DO = KV_NQ * KV_TILE, KV_OFF_PX = KV_OFF_DO + KV_NDO * KV_TILE;
constexpr int KV_OFF_SINK = KV_OFF_PX + 2 * KV_PX, KV_SMEM = KV_OFF_SINK + 256;
static_assert(KV_BI == 64 && KV_SMEM <= 160 * 1024, "a lane to a row's D or lse; one workgroup per compute unit");
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
// two probabilities in a word, the first in its low half; and back
GX_DEVINL unsigned pack_p(float a, float b) {
  const unsigned x = (__builtin_bit_cast(unsigned, a) + 0x2000u) << 2, y = (__builtin_bit_cast(unsigned, b) + 0x2000u) << 2;
  return __builtin_amdgcn_perm(y, x, 0x07060302u);
}
GX_DEVINL float unpack_p(unsigned w, int second) {
  return __builtin_bit_cast(float, second ? (w & 0xFFFF0000u) >> 2 : (w & 0xFFFFu) << 14);
}

// Tiles of 32 rows of a group of heads, one after the other: a tile's descriptor starts at its first query, a lane's offset follows
// from the head at which the tile starts (always the first one where the group divides 32).  What moves from tile to tile is
// kept in scalars.
template <int NW>
struct RowTiles {
  static constexpr int RPI = 64 / CPR, PER = KV_BI / RPI / NW;
  static_assert(PER >= 1, "tile too small for the workgroup");
  const char* at;                  // first query of the next tile
  long step, token_bytes;          // to the first query of the tile after it; of one query
  unsigned head_bytes;
  int group, h0, dh, left;         // head at which the next tile starts, and by how much that moves; rows from there on
  unsigned off[PER], off_wrapped[PER];   // modulo 2^32, without the tile's first head; wrapped: past the query's last head
  int head[PER], row0;
  GX_DEVINL void init(const bf16* p, const HeadStrides& s, int g, int rows, int t, int wave, int lane) {
    token_bytes = s.t * 2;
    head_bytes = uniform((unsigned)(s.h * 2));
    group = g;
    const unsigned q0 = uniform((unsigned)(t * KV_BI) / (unsigned)g), dq = uniform((unsigned)KV_BI / (unsigned)g);
    h0 = t * KV_BI - (int)q0 * g;
    dh = KV_BI - (int)dq * g;
    step = (long)dq * token_bytes;
    at = uniform(reinterpret_cast<const char*>(p) + (long)q0 * token_bytes);
    left = rows - t * KV_BI;
    row0 = RPI * wave * PER + lane / CPR;
#pragma unroll
    for (int i = 0; i < PER; i++) {
      const int r = row0 + RPI * i, c = (lane % CPR) ^ swz(r);
      const unsigned q = (unsigned)r / (unsigned)g;
      head[i] = r - (int)q * g;
      off[i] = q * (unsigned)token_bytes + head[i] * head_bytes + (unsigned)(c * 16);
      off_wrapped[i] = off[i] + (unsigned)token_bytes - (unsigned)g * head_bytes;
    }
  }
  // instruction i of the next tile
  GX_DEVINL void issue(char* dst, int wave, int i) const {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, 0x7FFFFFFFu, 0x00020000);
    unsigned o = (head[i] + h0 >= group ? off_wrapped[i] : off[i]) + (unsigned)h0 * head_bytes;
    asm volatile("" : "+v"(o));    // selected, not branched around
    o = row0 + RPI * i < left ? o : OOB;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_ptr)(dst + (wave * PER + i) * 1024), 16, o, 0, 0, 0);
  }
  GX_DEVINL void next() {
    left -= KV_BI;
    at += step;
    h0 += dh;
    if (h0 >= group) {
      h0 -= group;
      at += token_bytes;
    }
  }
};

__global__ void __launch_bounds__(64 * KV_NW, 2) cross_dkv_kernel(CrossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int NS = DH / 16, NDT = DH / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool role_v = wave < KV_PAIRS;
  const int pair = wave & (KV_PAIRS - 1);
  const int g = lane >> 5, l32 = lane & 31;
  const int npair = a.B * a.hk, nkb = (a.Sk + KV_BJ - 1) / KV_BJ;
  const int kp = blockIdx.x % npair, rest = blockIdx.x / npair, kb = rest % nkb, split = rest / nkb;
  const int kh = kp % a.hk, b = kp / a.hk;
  const int j0 = kb * KV_BJ, jw = j0 + pair * 32, j = jw + l32;
  const int len = keys_of(a, b);
  // a block without a key that counts has only zeros to store (none where a later launch joins the splits and does that)
  if (j0 >= len) {
    if (a.splits == 1) {
      const int key = j0 + (threadIdx.x >> 2);         // 4 lanes to a key
      if (key < a.Sk) {
        bf16* const dk = static_cast<bf16*>(a.dk) + pair_offset(a.sdk, b, kh) + key * a.sdk.t;
        bf16* const dv = static_cast<bf16*>(a.dv) + pair_offset(a.sdv, b, kh) + key * a.sdv.t;
        for (int c = threadIdx.x & 3; c < CPR; c += 4) {
          *reinterpret_cast<bf16x8*>(dk + c * 8) = bf16x8{};
          *reinterpret_cast<bf16x8*>(dv + c * 8) = bf16x8{};
        }
      }
    }
    return;
  }
  bf16x8 kvf[NS];                           // role V: this block's K rows; role K: its V rows
  {
    const int jc = j < a.Sk ? j : a.Sk - 1;
    const bf16* p = role_v ? static_cast<const bf16*>(a.k) + pair_offset(a.sk, b, kh) + jc * a.sk.t
                           : static_cast<const bf16*>(a.v) + pair_offset(a.sv, b, kh) + jc * a.sv.t;
    load_row(p, g, kvf);
  }
  f32x16 acc[NDT];                          // role V: dV; role K: dK
#pragma unroll
  for (int dt = 0; dt < NDT; dt++) acc[dt] = zero16();
  const float c2 = a.scale * LOG2E;
  char* const px = smem + KV_OFF_PX + pair * (KV_PX / KV_PAIRS) + lane * 16;
  unsigned coff[2][NDT];
  cols_lane_offsets(lane, coff);

  const int tiles = (a.rows + KV_BI - 1) / KV_BI;
  const int t0 = (int)((long)tiles * split / a.splits), nt = (int)((long)tiles * (split + 1) / a.splits);
  // lse and D of a tile's rows go to LDS by the same direct path, 4 B per lane (wavefront 0: lse, wavefront 1: D; the others
  // send an out-of-range load to a sink).  Rows beyond the last read as 0 everywhere (Q, dO, lse, D): with their S and dP set to
  // 0 (LAST) their P is 1 and their contributions are exactly 0; whole tiles beyond may be requested harmlessly.
  const float* const aux = (wave == 0 ? a.lrow : a.drow) + (long)kp * a.rows;
  RowTiles<KV_NW> srcq, srcdo;
  constexpr int PER = RowTiles<KV_NW>::PER, NREQ = 2 * PER + 1;
  srcq.init(static_cast<const bf16*>(a.q) + pair_offset(a.sq, b, kh * a.group), a.sq, a.group, a.rows, t0, wave, lane);
  srcdo.init(static_cast<const bf16*>(a.d_o) + pair_offset(a.sdo, b, kh * a.group), a.sdo, a.group, a.rows, t0, wave, lane);
  auto q_slot = [&](int slot) { return smem + slot * KV_TILE; };
  auto do_slot = [&](int slot) { return smem + KV_OFF_DO + slot * KV_TILE; };
  auto load_tile = [&](RowTiles<KV_NW>& src, char* dst) {
#pragma unroll
    for (int i = 0; i < PER; i++) src.issue(dst, wave, i);
    src.next();
  };
  auto aux_load = [&](int t, char* dst, bool on) {
    const int i = t * KV_BI + lane;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(aux), 0, (unsigned)a.rows * 4u, 0x00020000);
    const unsigned o = on && i < a.rows ? (unsigned)i * 4u : 0xFFFFFFFCu;     // rows < 2^30: beyond all of them (OOB is 2^29 rows)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_ptr)(on ? dst : smem + KV_OFF_SINK), 4, o, 0, 0, 0);
  };
  const bool lse_or_d = wave < 2, d_too = wave == 1;
  load_tile(srcq, q_slot(0));
  load_tile(srcdo, do_slot(0));
  load_tile(srcq, q_slot(1));
  aux_load(t0, wave == 0 ? do_slot(0) + KV_BI * ROWB : q_slot(0) + KV_BI * ROWB, lse_or_d);
  aux_load(t0 + 1, q_slot(1) + KV_BI * ROWB, d_too);
  // all that was requested has landed, and this wavefront is done with its reads
  auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  meet();

  int qs = 0, ds = 0;                       // ring positions of tile n
  auto q_of = [&](int d) { return q_slot((qs + d) & (KV_NQ - 1)); };                         // tile n + d, d in -1 .. 2
  auto do_of = [&](int d) {                                                                  // tile n + d, d in -1 .. 1
    const int x = ds + d;
    return do_slot(x < 0 ? x + KV_NDO : x < KV_NDO ? x : x - KV_NDO);
  };
  // request i of phase n: this wavefront's share of Q(n + 2), of dO(n + 1), then D(n + 2) or lse(n + 1)
  auto request = [&](int n, int i) __attribute__((always_inline)) {
    if (i < PER) srcq.issue(q_of(2), wave, i);
    else if (i < 2 * PER) srcdo.issue(do_of(1), wave, i - PER);
    else aux_load(wave == 0 ? n + 1 : n + 2, (wave == 0 ? do_of(1) : q_of(2)) + KV_BI * ROWB, lse_or_d);
  };
  auto advance = [&]() __attribute__((always_inline)) {
    qs = (qs + 1) & (KV_NQ - 1);
    ds = ds == KV_NDO - 1 ? 0 : ds + 1;
    srcq.next();
    srcdo.next();
  };
  auto request_all = [&](int n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NREQ; i++) request(n, i);
  };
  struct CFrag { bf16x4 lo, hi; };
  constexpr int NPC = 2 * NDT, VD = 4, KD = 4;       // products with a transposed tile; fragments requested ahead
  static_assert(NPC >= VD && NS >= KD && NREQ <= NS, "slots of a phase");
  // product p takes head-dim block p % NDT and rows 16 (p / NDT) .. + 15 of the sub-tile
  auto c_request = [&](unsigned ct, auto P, CFrag& f) __attribute__((always_inline)) {
    constexpr int p = decltype(P)::value, dt = p % NDT, u = p / NDT;
    f.lo = lds_read_tr_issue<u * 16 * ROWB>(ct + coff[0][dt]);
    f.hi = lds_read_tr_issue<u * 16 * ROWB>(ct + coff[1][dt]);
  };
  auto c_get = [&](CFrag& f) __attribute__((always_inline)) {
    lds_pin(f.lo);
    lds_pin(f.hi);
    return __builtin_shufflevector(f.lo, f.hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // S or dP of a tile's first 32 rows on their own
  auto first_product = [&](const char* rows, f32x16& out) __attribute__((always_inline)) {
    out = zero16();
    streamed<NS, KD>([&](int s) { return frag_rows(rows, l32, s, g); },
                     [&](int s, bf16x8 f) { out = MFMA(f, kvf[s], out); });
  };
  // 32 rows of a phase.  Role V, tile n: cur holds their S; P and dV from it, and S of the next 32 rows into nxt.  Role K, tile
  // n - 1: cur holds dP; dS and dK from it, dP of the next 32 rows into nxt.
  // LAST: the tile may end with rows that are not there.  It has code of its own: forward and backward of 4 x 2048 x 1501 .. 938, 16
  // heads, 433 us rather than 431 without the question, asked in every phase 434.
  auto half_phase = [&](int n, f32x16& cur, f32x16& nxt, auto role_tag, auto sub_tag, auto last_tag) __attribute__((always_inline)) {
    constexpr bool ROLE_V = decltype(role_tag)::value, LAST = decltype(last_tag)::value;
    constexpr int SUB = decltype(sub_tag)::value, NEXT = (1 - SUB) * 32 * ROWB;
    const char* rows = (ROLE_V ? q_of(SUB) : do_of(SUB - 1)) + NEXT;
    const char* tile = ROLE_V ? do_of(0) : q_of(-1);                  // dO(n) and lse(n), or Q(n - 1) and D(n - 1)
    const unsigned ct = lds_addr(tile + SUB * 32 * ROWB);
    const float* stat = reinterpret_cast<const float*>(tile + KV_BI * ROWB) + SUB * 32;
    char* const pxn = px + ((ROLE_V ? n : n - 1) & 1) * KV_PX + SUB * 2048;
    if constexpr (LAST) {                   // S and dP of rows beyond the last: 0 times a key or a value, not 0 where that is infinite
      const int left = a.rows - (ROLE_V ? n : n - 1) * KV_BI - 32 * SUB;
#pragma unroll
      for (int v = 0; v < 16; v++) cur[v] = 8 * (v >> 2) + 4 * g + (v & 3) < left ? cur[v] : 0.f;
    }
    f32x4 row_value[4];
#pragma unroll
    for (int q4 = 0; q4 < 4; q4++) row_value[q4] = *reinterpret_cast<const f32x4*>(stat + 8 * q4 + 4 * g);
    u32x4 pb[2];
    if (!ROLE_V) {
#pragma unroll
      for (int u = 0; u < 2; u++) pb[u] = *reinterpret_cast<const u32x4*>(pxn + u * 1024);
    }
    CFrag cf[VD];
    bf16x8 rf[KD], xf[2];                   // xf: P or dS, 16 rows per entry
#pragma unroll
    for (int q = 0; q < KD; q++) rf[q] = frag_rows(rows, l32, q, g);
    nxt = zero16();
    // the vector work in pieces: two values each, then 16 rows to round each
    constexpr int EPP = 2, NE = 16 / EPP, NPIECE = NE + 2;
    auto piece = [&](auto K) __attribute__((always_inline)) {
      constexpr int k = decltype(K)::value;
      if constexpr (k < NE) {
        constexpr int v0 = EPP * k;
        if constexpr (ROLE_V) {
#pragma unroll
          for (int v = v0; v < v0 + EPP; v++)
            cur[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[v], c2, -row_value[v >> 2][v & 3]));
        } else {
#pragma unroll
          for (int v = v0; v < v0 + EPP; v++)
            cur[v] = unpack_p(pb[v >> 3][(v & 7) >> 1], v & 1) * (cur[v] - row_value[v >> 2][v & 3]);
        }
      } else {
        constexpr int u = k - NE;
        xf[u] = pack_half(cur, u);
        if constexpr (ROLE_V) {
          u32x4 x;
#pragma unroll
          for (int e = 0; e < 4; e++) x[e] = pack_p(cur[8 * u + 2 * e], cur[8 * u + 2 * e + 1]);
          *reinterpret_cast<u32x4*>(pxn + u * 1024) = x;
        }
      }
    };
    constexpr auto cost = [](int k) constexpr { return k < NE ? (ROLE_V ? 6 : 4) * EPP : ROLE_V ? 18 : 6; };
    constexpr auto upto = [cost](int k) constexpr { int c = 0; for (int x = 0; x < k; x++) c += cost(x); return c; };
    constexpr int TOTAL = upto(NPIECE);
    // piece k goes behind first product slot_of(k)
    constexpr auto slot_of = [upto, cost](int k) constexpr { return (upto(k) + cost(k) / 2) * NS / TOTAL; };
    __builtin_amdgcn_sched_barrier(0);
    unroll<NS>([&](auto I) __attribute__((always_inline)) {
      constexpr int x = decltype(I)::value;
      nxt = MFMA(rf[x % KD], kvf[x], nxt);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (x + KD < NS) rf[x % KD] = frag_rows(rows, l32, x + KD, g);
      if constexpr (x >= NS - VD) c_request(ct, std::integral_constant<int, x - (NS - VD)>(), cf[x - (NS - VD)]);
      if constexpr (SUB == 0) {             // as early as can be: the phase's end waits for them
        if constexpr (x < NREQ) request(n, x);
      }
      unroll<NPIECE>([&](auto K) __attribute__((always_inline)) {
        if constexpr (slot_of(decltype(K)::value) == x) piece(K);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    unroll<NPC>([&](auto P) __attribute__((always_inline)) {
      constexpr int p = decltype(P)::value, newer = 2 * ((p + VD < NPC ? p + VD : NPC) - p - 1);   // untracked, younger
      lds_wait_le<newer>();
      acc[p % NDT] = MFMA(xf[p / NDT], c_get(cf[p % VD]), acc[p % NDT]);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (p + VD < NPC) c_request(ct, std::integral_constant<int, p + VD>(), cf[p % VD]);
    });
    asm volatile("" : "+v"(nxt));           // also where no tile follows
  };
  // One loop per role (the branch is wavefront-uniform; all pass a barrier after each of the phases t0 .. nt - 1).
  f32x16 sa, sb;
  int n = t0;
  auto phase = [&](auto role_tag, auto last_tag) __attribute__((always_inline)) {
    half_phase(n, sa, sb, role_tag, std::integral_constant<int, 0>(), last_tag);
    half_phase(n, sb, sa, role_tag, std::integral_constant<int, 1>(), last_tag);
  };
  if (jw >= len) {                          // a pair without a key that counts only brings its share of the tiles
    for (; n < nt; n++) {
      request_all(n);
      meet();
      advance();
    }
  } else if (nt > t0) {
    if (role_v) {
      first_product(q_of(0), sa);
      for (; n < nt - 1; n++) {
        phase(std::true_type(), std::false_type());
        meet();
        advance();
      }
      phase(std::true_type(), std::true_type());
      meet();
    } else {
      request_all(n);
      first_product(do_of(0), sa);
      meet();
      advance();
      for (n++; n < nt; n++) {
        phase(std::false_type(), std::false_type());
        meet();
        advance();
      }
      phase(std::false_type(), std::true_type());        // the last tile's dS and dK; the others are done
    }
  }
  WAIT_VM0();   // requests for tiles beyond the last one (zero fill) must not outlive the workgroup's LDS
  // accumulator register v of lane l is row 8 (v/4) + 4 g + v%4, column l%32 of its 32x32 tile
  const float oscale = role_v ? 1.0f : a.scale;
  if (a.splits > 1) {
    float* base = a.part + (((long)split * npair + kp) * a.Sk * 2 + (role_v ? 1 : 0)) * DH;
#pragma unroll
    for (int dt = 0; dt < NDT; dt++)
#pragma unroll
      for (int v = 0; v < 16; v++) {
        const int jr = jw + 8 * (v >> 2) + 4 * g + (v & 3);
        if (jr < len) base[(long)jr * 2 * DH + 32 * dt + l32] = acc[dt][v] * oscale;
      }
    return;
  }
  const HeadStrides& so = role_v ? a.sdv : a.sdk;
  bf16* obase = static_cast<bf16*>(role_v ? a.dv : a.dk) + pair_offset(so, b, kh);
  const unsigned char* const mask = a.key_mask ? a.key_mask + (long)b * a.Sk : nullptr;
#pragma unroll
  for (int v = 0; v < 16; v++) {
    const int jr = jw + 8 * (v >> 2) + 4 * g + (v & 3);
    if (jr < a.Sk) {
      const bool on = jr < len && (!mask || mask[jr] != 0);
#pragma unroll
      for (int dt = 0; dt < NDT; dt++) obase[(long)jr * so.t + 32 * dt + l32] = (bf16)(on ? acc[dt][v] * oscale : 0.f);
    }
  }
}

// ------------------------------------------------------------------------------- launches
template <typename K>
hipError_t set_smem(K kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
long pairs_of(const CrossArgs& a) { return (long)a.B * a.hk; }

// What a launch takes is estimated from its sizes, and the least estimate decides shape and splits.  A workgroup takes `fix` and
// `step` for each tile, `pair` where two share a compute unit (0: one at a time); keys that nobody else has brought near come
// at 5.3 TB/s to many workgroups, at 0.63 of that to `busy` of them; parts of a split are written, read and added by a launch of
// its own, which costs a small forward pass `join` of 5.5 rather than 3.5 (one query of 16 heads of 64, 1000 keys, whole 8.7, in parts 11.5).
// Microseconds and MB, from the runs listed below; only their proportions matter.
struct Shape { int rows, keys; double fix, step, pair, busy, join; };       // rows of a block, keys of a step
double estimate(const Shape& s, long blocks, long steps, int parts, double part_mb, double mb) {
  const long n = cdiv(blocks * parts, 256), per = cdiv(steps, parts);
  double t = s.pair > 0 ? (n / 2) * (s.fix + per * s.pair) + (n % 2) * (s.fix + per * s.step) : n * (s.fix + per * s.step);
  if (mb > 0) {
    const double us = mb / (5.3 * (1.0 - exp(-(double)(blocks * parts) / s.busy)));
    if (t < us) t = us;
  }
  return parts == 1 ? t : t + s.join + 0.04 * parts + parts * part_mb / 4.0;
}
// the best number of parts of a launch and its estimate
struct Choice { int shape, parts; double us; };
Choice best_parts(int shape, const Shape& s, long blocks, long steps, int least, double part_mb, double mb) {
  Choice c{shape, least, estimate(s, blocks, steps, least, part_mb, mb)};
  for (const int p : {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
    if (p > steps) break;
    const double t = p > least ? estimate(s, blocks, steps, p, part_mb, mb) : c.us;
    if (t < c.us) c = Choice{shape, p, t};
  }
  return c;
}

// Forward: 0 <4, 1, 64>: 128 rows, 1 <2, 2, 32>: 64 rows and two shares of a step's keys, 2 <1, 4, 32>: 32 rows and four shares.
// us, head dim 128, batch x queries x keys x heads / key heads: best of each shape (with its parts)
//   1 x 1024 x 1024 x 8 / 8:  12.8 (shape 2), 15.7 (1), 21.4 (0)     2 x 1024 x 1024 x 16 / 16: 24.5 (0), 26.2 (1)
//   1 x 512 x 512 x 8 / 8:    9.1 (2), 10.9 (1), 14.0 (0)            1 x 2048 x 2048 x 16 / 16: 41.0 (0), 43.6 (1)
//   1 x 200 x 200 x 64 / 8:   9.2 (1), 10.7 (0), 13.7 (2)            4 x 2048 x 1501 x 16 / 16: 107 (0), 129 (1)
//   1 x 1024 x 4096 x 8 / 8:  31.9 (2), 34.0 (1, 2 parts)            16 x 1 x 8192 x 40 / 8: 98.6 (1, 4 parts), 104 (2, 2 parts)
//   1 x 1 x 65536 x 32 / 8:   48.9 (2, 32 parts), 49.6 (1, 32)       8 x 5 x 3000 x 32 / 8: 22.5 (1, 8 parts), 22.6 (2, 4 parts)
//   16 x 1 x 8192 x 40 / 8 whole (128 workgroups) 173 (1), 140 (2); 8 x 64 x 8192 x 16 / 16 134 (1, 2 parts), 109 (1, 4 parts)
//   1 x 16 x 4096 x 16 / 4:   12.6 (2, 16 parts), 13.5 (2, 8)        4 x 1 x 512 x 32 / 8: 9.5 (2, whole), 11.8 (2, 4 parts)
// Head dim 64: 1 x 1024 x 1024 x 12 / 12 11.8 (2), 12.0 (1), 16.3 (0); 4 x 1024 x 1024 x 16 / 16 25.7 (0), 29.0 (1).
constexpr Shape FWD[3] = {{128, 64, 5.0, DH == 128 ? 1.0 : 0.72, DH == 128 ? 2.1 : 1.15, DH == 128 ? 146 : 290, 5.5},
                          {64, 64, 2.5, DH == 128 ? 0.62 : 0.41, DH == 128 ? 1.09 : 0.78, DH == 128 ? 146 : 290, 5.5},
                          {32, 128, 3.0, DH == 128 ? 0.85 : 0.5, DH == 128 ? 0.0 : 0.85, DH == 128 ? 100 : 146, 5.5}};
// Neither here nor below by whether there is a mask, so that one workspace serves both
Choice fwd_estimate(const CrossArgs& a) {
  const int least = cdiv(a.Sk, MASK_KEYS * 3 / 4) > 1 ? cdiv(a.Sk, MASK_KEYS * 3 / 4) : 1;   // mask bits have their room in LDS
  const double part_mb = pairs_of(a) * a.rows * (DH + 2) * 8e-6, mb = pairs_of(a) * a.Sk * DH * 4e-6;
  Choice c{};
  for (int k = 0; k < 3; k++) {
    const int blocks = cdiv(a.rows, FWD[k].rows);            // of a pair: two or more do not read the keys quite together
    const Choice x = best_parts(k, FWD[k], pairs_of(a) * blocks, cdiv(a.Sk, FWD[k].keys), least, part_mb,
                                blocks > 1 ? 1.33 * mb : mb);
    if (k == 0 || x.us < c.us) c = x;
  }
  return c;
}
// dQ: 0 <4, 1, 64>: 128 rows, 1 <2, 2, 32>: 64 rows.  Forward and backward, us, shape 0 / 1: 4 x 2048 x 1501 x 16 / 16 381 / 402, 2 x
// 4096 x 64 x 16 / 8 60.5 / 68.1, 1 x 2048 x 2048 x 16 / 16 141 / 139, 1 x 4096 x 1024 x 8 / 2 91.4 / 88.9; in parts, shape 1: 1 x 1024 x 1024
// x 8 / 8 whole 55.2, two 56.5, four 64.8; 4 x 40 x 4096 x 16 / 8 four 73.3, two 78.
constexpr Shape DQ[2] = {{128, 64, 5.0, DH == 128 ? 1.45 : 0.95, DH == 128 ? 2.6 : 1.5, 0, 3.5},
                         {64, 64, 3.5, DH == 128 ? 0.95 : 0.65, DH == 128 ? 1.5 : 0.95, 0, 3.5}};
Choice dq_estimate(const CrossArgs& a) {
  const int least = cdiv(a.Sk, MASK_KEYS * 3 / 4) > 1 ? cdiv(a.Sk, MASK_KEYS * 3 / 4) : 1;
  const double part_mb = pairs_of(a) * a.rows * DH * 8e-6;
  Choice c{};
  for (int k = 0; k < 2; k++) {
    const Choice x = best_parts(k, DQ[k], pairs_of(a) * cdiv(a.rows, DQ[k].rows), cdiv(a.Sk, DQ[k].keys), least, part_mb, 0);
    if (k == 0 || x.us < c.us) c = x;
  }
  return c;
}
// dK / dV, parts of the rows.  Forward and backward, us: 1 x 1024 x 1024 x 8 / 8 two parts 64.8, four 56.9, six 61.5; 2 x 4096 x 64 x
// 16 / 8 eight 69.4, sixteen 59.8, 24 70.7; head dim 64, 3 x 3000 x 300 x 16 / 16 whole 94.5, three 88.9, six 97.8.
constexpr Shape DKV = {KV_BI, KV_BJ, 5.0, DH == 128 ? 1.9 : 1.2, 0.0, 0, 3.5};
Choice dkv_estimate(const CrossArgs& a) {
  return best_parts(0, DKV, pairs_of(a) * cdiv(a.Sk, DKV.keys), cdiv(a.rows, DKV.rows), 1, pairs_of(a) * a.Sk * DH * 16e-6, 0);
}
// A call asks several times for the same sizes, and the next one mostly too: each host thread keeps its last plan (sizes in, shape
// and parts out)
template <Choice (*ESTIMATE)(const CrossArgs&)>
Choice kept(const CrossArgs& a) {
  static thread_local long pairs = -1;
  static thread_local int rows, keys;
  static thread_local Choice last;
  if (pairs != pairs_of(a) || rows != a.rows || keys != a.Sk) {
    last = ESTIMATE(a);
    pairs = pairs_of(a);
    rows = a.rows;
    keys = a.Sk;
  }
  return last;
}
Choice fwd_choice(const CrossArgs& a) { return kept<fwd_estimate>(a); }
Choice dq_choice(const CrossArgs& a) { return kept<dq_estimate>(a); }
Choice dkv_choice(const CrossArgs& a) { return kept<dkv_estimate>(a); }
int parts(const CrossArgs& a, int pass) { return (pass == 0 ? fwd_choice(a) : pass == 1 ? dq_choice(a) : dkv_choice(a)).parts; }
int mask_smem(const CrossArgs& a, int splits, int rows) {
  return a.key_mask ? 4 * mask_words(cdiv(cdiv(a.Sk, rows), splits) * rows + rows, rows) : 0;
}

template <int NQ, int SPLIT, int BKV, bool MASK>
hipError_t go_fwd(const CrossArgs& a, hipStream_t s) {
  constexpr int TILES = fwd_smem(NQ, SPLIT, BKV), ROWS = BKV * SPLIT;
  static bool configured = false;
  if (!configured) {
    const hipError_t e =
        set_smem(cross_fwd_kernel<NQ, SPLIT, BKV, MASK>, TILES + (MASK ? 4 * mask_words(MASK_KEYS, ROWS) : 0));
    if (e != hipSuccess) return e;
    configured = true;
  }
  const dim3 grid((unsigned)(pairs_of(a) * cdiv(a.rows, 32 * NQ) * a.splits));
  hipLaunchKernelGGL((cross_fwd_kernel<NQ, SPLIT, BKV, MASK>), grid, dim3(64 * NQ * SPLIT),
                     TILES + mask_smem(a, a.splits, ROWS), s, a);
  return hipGetLastError();
}
// With a mask the 128-row shape would spill registers (the untracked LDS reads forbid that): 64 rows then.
hipError_t fwd(CrossArgs a, hipStream_t s) {
  const Choice c = fwd_choice(a);
  a.splits = c.parts;
  const bool mask = a.key_mask != nullptr;
  hipError_t e;
  if (c.shape == 2) e = mask ? go_fwd<1, 4, 32, true>(a, s) : go_fwd<1, 4, 32, false>(a, s);
  else if (mask) e = go_fwd<2, 2, 32, true>(a, s);
  else e = c.shape == 1 ? go_fwd<2, 2, 32, false>(a, s) : go_fwd<4, 1, 64, false>(a, s);
  return e != hipSuccess || a.splits == 1 ? e : cross_join_fwd(true, a, s);
}

template <int NQ, int SPLIT, int BKV, bool MASK>
hipError_t go_dq(const CrossArgs& a, hipStream_t s) {
  constexpr int ROWS = BKV * SPLIT, TILES = 4 * ROWS * ROWB;
  static bool configured = false;
  if (!configured) {
    const hipError_t e = set_smem(cross_dq_kernel<NQ, SPLIT, BKV, MASK>, TILES + (MASK ? 4 * mask_words(MASK_KEYS, ROWS) : 0));
    if (e != hipSuccess) return e;
    configured = true;
  }
  const dim3 grid((unsigned)(pairs_of(a) * cdiv(a.rows, 32 * NQ) * a.splits));
  hipLaunchKernelGGL((cross_dq_kernel<NQ, SPLIT, BKV, MASK>), grid, dim3(64 * NQ * SPLIT),
                     TILES + mask_smem(a, a.splits, ROWS), s, a);
  return hipGetLastError();
}
// dQ with D, then dK / dV
hipError_t bwd(CrossArgs a, hipStream_t s) {
  static bool configured = false;
  if (!configured) {
    const hipError_t e = set_smem(cross_dkv_kernel, KV_SMEM);
    if (e != hipSuccess) return e;
    configured = true;
  }
  hipError_t e = hipSuccess;
  if (a.rows > 0) {
    const Choice c = dq_choice(a);
    a.splits = c.parts;
    if (a.key_mask) e = go_dq<2, 2, 32, true>(a, s);
    else e = c.shape == 0 ? go_dq<4, 1, 64, false>(a, s) : go_dq<2, 2, 32, false>(a, s);
    if (e == hipSuccess && a.splits > 1) e = cross_join_dq(true, a, s);
  }
  if (e != hipSuccess || a.Sk == 0) return e;
  a.splits = dkv_choice(a).parts;
  hipLaunchKernelGGL(cross_dkv_kernel, dim3((unsigned)(pairs_of(a) * cdiv(a.Sk, KV_BJ) * a.splits)), dim3(64 * KV_NW), KV_SMEM, s, a);
  e = hipGetLastError();
  return e != hipSuccess || a.splits == 1 ? e : cross_join_dkv(true, a, s);
}
