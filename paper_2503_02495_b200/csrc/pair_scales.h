// Rule of the hand-over of scale words inside a pair of CTAs (fp8_gemm_tcgen05.cu).  The second CTA's scale warps write their words into their
// own shared memory, and a copy that the first CTA's MMA warp issues reads them there.  What orders the two is a release at cluster scope, and a
// warp that makes one per block cannot keep pace with the products: an SM gets through one in some 550 cycles, where a block of the
// contraction takes 500 (32768 x 4096 x 1024: 117 us without, 135 with one per block by the scale warps or by three others, 123 so).  So the scale
// warps arrive on barriers of their own SM, and three other warps wait there, a pair of neighbouring stages each, and pass both on behind one
// fence.  At the end of the line a pair may be half full: its warp passes on what there is.
// Why no warp waits in vain or looks a turn too late: the words of block b need the products of block b - 6 and nothing later, so they come
// whether or not the block beside them has been passed on; and a stage is written again only after its block has been passed on
// and multiplied, so a waiting warp can be no whole turn behind its barrier.
#pragma once

#if defined(__CUDACC__)
#define UOE_PAIR_FN __host__ __device__ constexpr
#else
#define UOE_PAIR_FN constexpr
#endif

namespace uoe {
constexpr int kPairStages = 6, kPassGroup = 2, kPassWarps = kPairStages / kPassGroup;
static_assert(kPassGroup * kPassWarps == kPairStages, "every stage has a warp, and no group wraps around the ring");
UOE_PAIR_FN int pass_warp(int stage) { return stage / kPassGroup; }                          // which of the warps passes this stage's block on
UOE_PAIR_FN bool pass_now(int stage, bool last) { return stage % kPassGroup == kPassGroup - 1 || last; }      // with it, its group so far
UOE_PAIR_FN int pass_first(int stage) { return stage - stage % kPassGroup; }                 // first stage of the group
}  // namespace uoe
