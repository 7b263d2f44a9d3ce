// What the kernels of cross attention are given (internal).
//
// No query sees another set of keys than its neighbours do, so the query heads that share a key head are one problem with that
// head's keys: row r = s * group + g of a (sample, key head) pair is query s of the group's head g, and every kernel works on
// pairs of `rows` rows and `Sk` keys.
#pragma once
#include "gx_kernels.h"

namespace gx {

struct HeadStrides { long b, t, h; };            // elements

struct CrossArgs {
  const void *q, *k, *v, *o, *d_o;
  void *out, *dq, *dk, *dv;                      // out: the forward pass's o
  HeadStrides sq, sk, sv, so, sdo, sdq, sdk, sdv;
  const int* key_lens;                           // per sample, or null
  const unsigned char* key_mask;                 // [B][Sk], or null
  float* lse;                                    // [B][q_heads][Sq]; forward: may be null
  float *lrow, *drow;                            // backward: per pair and row, lse * log2(e) (+inf where there is none) and D
  float* part;                                   // partial results of a launch that splits keys or rows, or null
  int B, Sq, Sk, hk, group, rows, dh;
  int splits;                                    // of the keys (forward, dQ) or of the rows (dK / dV)
  float scale;
};

GX_DEVINL int keys_of(const CrossArgs& a, int b) {
  const int n = a.key_lens ? a.key_lens[b] : a.Sk;
  return __builtin_amdgcn_readfirstlane(n < 0 ? 0 : n > a.Sk ? a.Sk : n);
}
// element offset of row r of a pair's group of heads
GX_DEVINL long row_offset(const HeadStrides& s, int group, int r) {
  const int i = (int)((unsigned)r / (unsigned)group);
  return (long)i * s.t + (long)(r - i * group) * s.h;
}
GX_DEVINL long pair_offset(const HeadStrides& s, int b, int head) { return (long)b * s.b + (long)head * s.h; }

// Into how many parts a launch cuts its keys (pass 0: forward, 1: dQ) or rows (2: dK / dV); host code, a rule on sizes alone
int cross_parts_bf16(const CrossArgs& a, int pass);
int cross_parts_f32(const CrossArgs& a, int pass);

hipError_t cross_fwd_bf16(const CrossArgs& a, hipStream_t s);
hipError_t cross_fwd_f32(const CrossArgs& a, hipStream_t s);
// `a.splits` is set by the callee; part serves dQ, then dK / dV
hipError_t cross_bwd_bf16(const CrossArgs& a, hipStream_t s);
hipError_t cross_bwd_f32(const CrossArgs& a, hipStream_t s);

// Joins the parts of a launch that was split (cross.hip).
//   forward: part = [split][pair][row][dh] unnormalised sums, behind them [split][pair][row][2] (reference exponent, sum of
//   exponentials; base 2 for bf16, e for fp32)
hipError_t cross_join_fwd(bool bf16, const CrossArgs& a, hipStream_t s);
//   dQ: part = [split][pair][row][dh];  dK, dV: part = [split][pair][key][2][dh] (dK, dV)
hipError_t cross_join_dq(bool bf16, const CrossArgs& a, hipStream_t s);
hipError_t cross_join_dkv(bool bf16, const CrossArgs& a, hipStream_t s);

}  // namespace gx
