// Cross attention for gfx950, bf16 in / fp32 accumulate, head dim 128 or 64 (the kernels live in cross_bf16_impl.h, compiled
// once per head dimension).
//
// The products are taken as in the causal kernels: a wavefront keeps 32 query rows and forms S^T = K Q^T, so that a lane owns
// one query and the probabilities, rounded to bf16, are the operand of O^T = V^T P^T as they stand.  What differs is what
// decides the work: every row of a pair sees the same keys, so rows of all heads of a group are one problem (K and V are read
// once for the group), no block is shorter than another of its sample, and few rows against many keys (decoding) are
// served by cutting the keys over workgroups too.
#include "cross.h"
#include <math.h>
#include <type_traits>

namespace gx {
namespace {

constexpr unsigned OOB = 0x80000000u;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
#define MFMA(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16((a), (b), (c), 0, 0, 0)
#define WAIT_VM0() __builtin_amdgcn_s_waitcnt(0x0F70)

namespace dh128 {
#define GX_ATTN_DH 128
#include "cross_bf16_impl.h"
#undef GX_ATTN_DH
}  // namespace dh128
namespace dh64 {
#define GX_ATTN_DH 64
#include "cross_bf16_impl.h"
#undef GX_ATTN_DH
}  // namespace dh64

}  // namespace

int cross_parts_bf16(const CrossArgs& a, int pass) { return a.dh == 128 ? dh128::parts(a, pass) : dh64::parts(a, pass); }
hipError_t cross_fwd_bf16(const CrossArgs& a, hipStream_t s) { return a.dh == 128 ? dh128::fwd(a, s) : dh64::fwd(a, s); }
hipError_t cross_bwd_bf16(const CrossArgs& a, hipStream_t s) { return a.dh == 128 ? dh128::bwd(a, s) : dh64::bwd(a, s); }

}  // namespace gx
