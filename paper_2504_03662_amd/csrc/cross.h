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
// The sample that takes its turn `rank`-th when the longest go first, so that a launch of several rounds ends with short ones
// (4 samples of 1501 .. 938 keys, 2048 queries of 16 heads of 128: forward 99 and dQ 137 us, in the samples' order 106 and 151).  Every
// wavefront sorts the lengths for itself, a lane to a sample.
GX_DEVINL int sample_by_length(const CrossArgs& a, int rank) {
  const int lane = threadIdx.x & 63;
  const int n = lane < a.B ? a.key_lens[lane] : 0;
  int before = 0;
  for (int m = 0; m < a.B; m++) {
    const int other = __builtin_amdgcn_readlane(n, m);
    before += other > n || (other == n && m < lane) ? 1 : 0;
  }
  return __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < a.B && before == rank));
}
// Pair, row block and split of a workgroup of a launch over `blocks` row blocks of every pair.  Pairs go round the chip, so that a pair's
// workgroups share an L2 where the pairs (key heads, with lengths) are a multiple of 8.
struct Share { int b, kh, pair, block, split; };
GX_DEVINL Share share_of(const CrossArgs& a, int blk, int blocks) {
  Share x;
  if (a.key_lens && a.B <= 64) {
    x.kh = blk % a.hk;
    int rest = blk / a.hk;
    x.block = rest % blocks;
    rest /= blocks;
    x.split = rest % a.splits;
    x.b = a.B == 1 ? 0 : __builtin_amdgcn_readfirstlane(sample_by_length(a, rest / a.splits));
    x.pair = x.b * a.hk + x.kh;
  } else {
    const int npair = a.B * a.hk, rest = blk / npair;
    x.pair = blk % npair;
    x.block = rest % blocks;
    x.split = rest / blocks;
    x.kh = x.pair % a.hk;
    x.b = x.pair / a.hk;
  }
  return x;
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
