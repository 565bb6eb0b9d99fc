// uoe_mlp_tokens: router, experts and combine of a UoME layer for a few tokens (every row of x is a sample of one token: Eq. 21-22
// choose its experts, Eq. 38-40 follow) in two kernels.  bfloat16 and 8-bit weights here, float32 in tokens_f32.cu.
//
// Bound by the weights of the chosen experts, each read once.  They are the 128-row operand of the tensor cores (a tile is 128 of their
// columns), the tokens the narrow one: weights go from memory to shared memory by TMA and from there into the MMA, no thread touches
// them, and a CTA keeps its whole ring of stages in flight.  (Weights through registers into mma.sync fragments: eight tokens of a 16-expert
// layer, d = 4096, d_e = 1024, 8-bit, 46 us; 32 tokens 187 us, where the activations' way to every fragment costs more than the weights.)
//   first_layer_kernel   routes, then a = phi(x W1 + b1) for every (chosen expert, 128 hidden columns)
//   second_layer_kernel  y = x + sum over experts gate (a W2 + b2) for every 128 columns of y, the contraction running over all chosen
//                        experts' hidden columns in one line
// The CTAs of a cluster share the router's work, a part of d each; every cluster routes for itself (a few KB from L2, instead of a third
// kernel).  S of them share a tile's contraction; their sums meet in distributed shared memory in a fixed order.
//
// Stages: 128 columns x 64 of the contraction of bfloat16 weights (as they lie, columns contiguous), or x 128 of 8-bit weights (the
// contraction contiguous).  bfloat16: the tokens' values come by TMA as well, and one TMEM accumulator takes all of an expert.  8-bit: the
// tensor cores want both operands in 8 bits, so a token's 128 values of a stage become two e4m3 terms, x = s (hi + lo / 16), s a power of two:
// eight significant bits as bfloat16 has them, from 2^-6 s on; smaller values are off by 2^-14 s at most, 2^-21 of the largest of the 128.  hi and lo are neighbouring
// columns of one MMA.  A stage is one block of the weights' scales, so its product, times one number per token, is added to float32
// registers by the write-out warps; the weights' scales may be any numbers.
//   warp 0       TMA producer         warp 1       MMA issuer         warps 2, 3  the router's outputs
//   warps 4..7   sums: one column per thread, all tokens            warps 8..     8-bit, first kernel: the tokens' values of the stages to come
#include "tmap.cuh"
#include "tokens.cuh"

namespace uoe {
namespace tokens {
namespace {

constexpr int kCols = 128;
constexpr int kScaleSlots = 16;         // >= stages + 3: a block's factors outlive its stage by the accumulators in flight
constexpr int kMaxSmem = 226 * 1024;

template <int WT, int NT /* tokens, rounded up */> struct Cfg {
    static constexpr int N = WT == kFp8 ? 2 * NT : NT;                    // columns of an MMA
    static_assert(N % 16 == 0 && N <= 128, "shape of an MMA");
    static constexpr int K = WT == kFp8 ? 128 : 64;                       // of the contraction per stage
    static constexpr int A_BYTES = 16384, B_BYTES = N * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr int CTAS = NT <= 32 ? 2 : 1;                         // per SM
    static constexpr int CLUSTER = CTAS == 2 ? 8 : 4;                     // (eight CTAs of an SM each: some clusters wait for a second turn)
    static constexpr int STAGES = CTAS == 1 ? 6 : NT <= 16 ? 4 : 3;
    static constexpr int TMEM_COLS = 2 * N < 32 ? 32 : 2 * N;
    static constexpr int TEAM = NT / 8, TEAMS = NT == 8 ? 4 : NT == 16 ? 2 : 1;       // 8-bit: a team of warps fills a stage, 8 tokens each
    // (A team looks for its next stage's last use by parity: it must not be two uses behind, and the team's own last stage vouches for no more
    // than the uses before that.)
    static_assert(WT != kFp8 || TEAMS <= STAGES, "teams");
    static_assert(kScaleSlots >= STAGES + 3, "factors");
    static constexpr int WARPS1 = WT == kFp8 ? 8 + TEAM * TEAMS : 8, WARPS2 = 8;      // of the two kernels
    static constexpr int PITCH = kCols + 4;                               // floats of a token's sums in shared memory
    static constexpr int RING = STAGES * STAGE;
};

template <int NT> struct Ctl {
    uint64_t full[8], empty[8], tfull[2], tempty[2];
    uint32_t tmem_base;
    int abort_flag;
    alignas(16) float f[kScaleSlots * NT];      // 8-bit: scales of the tokens' values, by stage
    Routed R;
};

template <int WT, int NT> struct Smem {                                   // dynamic shared memory (aligned to 1024)
    uint8_t* ring;                      // also: the router's partial sums before, the tile's sums after the stages
    Ctl<NT>* ctl;
    float* part;                        // [Tn][n]
    __device__ Smem(uint8_t* raw) {
        ring = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
        ctl = (Ctl<NT>*)(ring + Cfg<WT, NT>::RING);
        part = (float*)(ctl + 1);
    }
    static size_t bytes(int Tn, int n) { return 1024 + Cfg<WT, NT>::RING + sizeof(Ctl<NT>) + sizeof(float) * Tn * n; }
};
// (the router's partial sums, 8 * tokens * 32 experts, and the tile's sums lie in the ring)
static_assert(Cfg<kBf16, 64>::RING >= 8 * 64 * 32 * 4 && Cfg<kBf16, 16>::RING >= 8 * 16 * 32 * 4 && Cfg<kFp8, 8>::RING >= 8 * 8 * 32 * 4, "ring");

// What one CTA multiplies: stages [lo, hi) of a line of `per` stages per expert.
struct Line { int lo, hi, per, slot0; };

// 128 values, four per lane, as s (hi + lo / 16): returns s.
__device__ __forceinline__ float two_terms(float a, float b, float c, float d, uint32_t& hi, uint32_t& lo) {
    const uint32_t m = __reduce_max_sync(0xffffffffu, max(max(abs_bits(a), abs_bits(b)), max(abs_bits(c), abs_bits(d))));
    const BlockScale k = block_scale(m);
    hi = e4m3x4(a, b, c, d, k.inv);
    uint32_t h01, h23;                                 // hi as half pairs
    halves_of_e4m3(hi, h01, h23);
    const float2 g0 = __half22float2(*reinterpret_cast<const __half2*>(&h01)), g1 = __half22float2(*reinterpret_cast<const __half2*>(&h23));
    lo = e4m3x4(fmaf(a, k.inv, -g0.x), fmaf(b, k.inv, -g0.y), fmaf(c, k.inv, -g1.x), fmaf(d, k.inv, -g1.y), k.inv == 0.f ? 0.f : 16.f);
    return k.s;
}

// The tile's sums: on return every thread of warps 4..7 holds column 32 (warp % 4) + lane of NT tokens in sum[].
//   tmW, tmX   the weights [n, ..] (tile column c0); bfloat16: the tokens' values, one matrix [rows, K] per slot (x: one for all)
//              8-bit, SECOND: their two terms, [2 n, rows, Kp], and the terms' scales f [n, K / 128, rows]
//   x, ld      8-bit, first kernel: the tokens' values
//   weight(tok, e): factor of a token's product with expert e (SECOND: only for the tokens that chose it)
template <int WT, int NT, bool SECOND, typename Weight>
__device__ __forceinline__ void run_line(const Smem<WT, NT>& sm, const CUtensorMap* tmW, const CUtensorMap* tmX, const __nv_bfloat16* x, int ld, const float* f,
                                         const float* scale /* 8-bit: [n][N / 128][K / 128] of this column block */, size_t scale_stride, int c0, int K, int Tn,
                                         const Line& line, int* status, float* sum, Weight weight) {
    using Cf = Cfg<WT, NT>;
    Ctl<NT>* ctl = sm.ctl;
    volatile int* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem_base = ctl->tmem_base;
    const Routed& R = ctl->R;
    // position in the line -> slot, stage of its expert; a group of stages goes to one accumulator
    auto slot_of = [&](int u, int& kb) { const int s = u / line.per; kb = u - s * line.per; return line.slot0 + s; };
    auto begins = [&](int u, int kb) { return WT == kFp8 || u == line.lo || kb == 0; };
    auto ends = [&](int u, int kb) { return WT == kFp8 || u == line.hi - 1 || kb == line.per - 1; };
    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0, issued = 0, issued_parity = 0;
        for (int u = line.lo; u < line.hi; ++u) {
            int kb;
            const int slot = slot_of(u, kb), e = R.list[slot];
            if (!mbar_wait_warp_quick(&ctl->empty[stage], phase ^ 1, abort_flag, status)) break;
            if (lane == 0) {
                uint8_t* st = sm.ring + stage * Cf::STAGE;
                mbar_arrive_expect_tx(&ctl->full[stage], Cf::A_BYTES + (WT == kBf16 || SECOND ? Cf::B_BYTES : 0) + (WT == kFp8 && SECOND ? NT * 4 : 0));
                if constexpr (WT == kFp8) {
                    tma_load_3d(st, tmW, kb * 128, c0, e, &ctl->full[stage]);
                    if constexpr (SECOND) {
                        tma_load_3d(st + Cf::A_BYTES, tmX, kb * 128, 0, 2 * slot, &ctl->full[stage]);
                        tma_load_3d(st + Cf::A_BYTES + NT * 128, tmX, kb * 128, 0, 2 * slot + 1, &ctl->full[stage]);
                        bulk_load(ctl->f + (u - line.lo) % kScaleSlots * NT, f + ((size_t)slot * line.per + kb) * kMaxTokens, NT * 4, &ctl->full[stage]);
                    }
                } else {
                    tma_load_3d(st, tmW, c0, kb * 64, e, &ctl->full[stage]);
                    tma_load_3d(st + 8192, tmW, c0 + 64, kb * 64, e, &ctl->full[stage]);
                    tma_load_3d(st + Cf::A_BYTES, tmX, kb * 64, 0, SECOND ? slot : 0, &ctl->full[stage]);
                }
            }
            __syncwarp();
            issued |= 1u << stage;
            issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
            if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
        }
        if (lane == 0 && *abort_flag)                  // copies in flight land before the CTA exits
            for (int s = 0; s < Cf::STAGES; ++s)
                if (issued & (1u << s)) mbar_wait(&ctl->full[s], (issued_parity >> s) & 1, abort_flag, status);
    } else if (warp == 1) {
        const uint32_t el = elect_one();
        constexpr uint32_t idesc = WT == kFp8 ? instr_desc_e4m3(128, Cf::N) : instr_desc_bf16(128, Cf::N, true, false);
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        for (int u = line.lo; u < line.hi; ++u) {
            int kb;
            slot_of(u, kb);
            const bool first = begins(u, kb);
            if (first && !mbar_wait_warp_quick(&ctl->tempty[acc], acc_phase ^ 1, abort_flag, status)) break;
            if (!mbar_wait_warp_quick(&ctl->full[stage], phase, abort_flag, status)) break;
            tc_fence_after();
            const uint32_t sa = smem_u32(sm.ring + stage * Cf::STAGE), sb = sa + Cf::A_BYTES;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const uint64_t bd = smem_desc(sb + ks * 32, 16, 1024);
                if constexpr (WT == kFp8) mma_f8(el, tmem_base + acc * Cf::N, smem_desc(sa + ks * 32, 16, 1024), bd, idesc, ks != 0);
                else mma_bf16(el, tmem_base + acc * Cf::N, smem_desc(sa + ks * 2048, 8192, 1024), bd, idesc, !(first && ks == 0));
            }
            mma_commit(el, &ctl->empty[stage]);
            if (ends(u, kb)) {
                mma_commit(el, &ctl->tfull[acc]);
                if (++acc == 2) { acc = 0; acc_phase ^= 1; }
            }
            if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
        }
    } else if (warp >= 8) {
        // teams take the stages in turn; a warp has eight tokens, a lane four of their 128 values
        const int team = (warp - 8) / Cf::TEAM, tok0 = (warp - 8) % Cf::TEAM * 8;
        uint2 v[8];
        auto ask = [&](int u) {
            const int k = (u % line.per) * 128 + 4 * lane;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = make_uint2(0, 0);
                if (k < K && tok0 + i < Tn) v[i] = *(const uint2*)(x + (size_t)(tok0 + i) * ld + k);
            }
        };
        if (line.lo + team < line.hi) ask(line.lo + team);
        for (int u = line.lo + team; u < line.hi; u += Cf::TEAMS) {
            const int i_u = u - line.lo, stage = i_u % Cf::STAGES, at = i_u % kScaleSlots;
            const uint32_t phase = (i_u / Cf::STAGES) & 1;
            if (!mbar_wait_warp_quick(&ctl->empty[stage], phase ^ 1, abort_flag, status)) break;
            uint8_t* st = sm.ring + stage * Cf::STAGE + Cf::A_BYTES;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int tok = tok0 + i;
                uint32_t hi, lo;
                const float sc = two_terms(__uint_as_float(v[i].x << 16), __uint_as_float(v[i].x & 0xffff0000u), __uint_as_float(v[i].y << 16),
                                           __uint_as_float(v[i].y & 0xffff0000u), hi, lo);
                uint8_t* o = st + tok * 128 + ((16 * (lane >> 2)) ^ (i << 4)) + 4 * (lane & 3);      // (128-byte swizzle: tok % 8 = i)
                *(uint32_t*)o = hi;
                *(uint32_t*)(o + NT * 128) = lo;
                if (lane == 0) ctl->f[at * NT + tok] = sc;
            }
            if (u + Cf::TEAMS < line.hi) ask(u + Cf::TEAMS);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl->full[stage]);
        }
    } else if (warp >= 4) {
        int acc = 0, at = 0;
        uint32_t acc_phase = 0;
        for (int u = line.lo; u < line.hi; ++u) {
            int kb;
            const int slot = slot_of(u, kb);
            if (!ends(u, kb)) continue;
            const int e = R.list[slot];
            const unsigned long long of = SECOND ? R.of[slot] : ~0ull;
            float w[(NT + 31) / 32];                   // factors of tokens lane, lane + 32
#pragma unroll
            for (int i = 0; i < (NT + 31) / 32; ++i) w[i] = lane + 32 * i < Tn ? weight(lane + 32 * i, e) : 0.f;
            float s = 1.f;
            if constexpr (WT == kFp8) s = __ldg(scale + (size_t)e * scale_stride + kb);
            if (!mbar_wait_warp_quick(&ctl->tfull[acc], acc_phase, abort_flag, status)) break;
            tc_fence_after();
            if constexpr (WT == kFp8) {
#pragma unroll
                for (int i = 0; i < (NT + 31) / 32; ++i) w[i] *= s * ctl->f[at * NT + (lane + 32 * i) % NT];
            }
            const uint32_t taddr = tmem_base + acc * Cf::N + ((uint32_t)((warp & 3) * 32) << 16);
            constexpr int STEP = Cf::N < 32 ? 16 : 32;                    // columns at a time: 8-bit: 16 hi columns, then their 16 lo columns
            if constexpr (WT == kFp8) {
                constexpr int H = NT < 16 ? 8 : 16;                       // tokens at a time
#pragma unroll
                for (int t = 0; t < NT; t += H) {
                    uint32_t vh[H], vl[H];
                    if constexpr (H == 8) { tmem_ld8(taddr + t, vh); tmem_ld8(taddr + NT + t, vl); }
                    else { tmem_ld16(taddr + t, vh); tmem_ld16(taddr + NT + t, vl); }
                    tmem_ld_wait();
                    if (t + H >= NT) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&ctl->tempty[acc]);
                    }
#pragma unroll
                    for (int i = 0; i < H; ++i) {
                        const int tok = t + i;
                        const float f = __shfl_sync(0xffffffffu, w[tok / 32], tok % 32);
                        if ((of >> tok) & 1) sum[tok] = fmaf(f, fmaf(0.0625f, __uint_as_float(vl[i]), __uint_as_float(vh[i])), sum[tok]);
                    }
                }
            } else {
#pragma unroll
                for (int t = 0; t < NT; t += STEP) {
                    uint32_t v[STEP];
                    if constexpr (STEP == 16) tmem_ld16(taddr + t, v);
                    else tmem_ld32(taddr + t, v);
                    tmem_ld_wait();
                    if (t + STEP >= NT) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&ctl->tempty[acc]);
                    }
#pragma unroll
                    for (int i = 0; i < STEP; ++i) {
                        const float f = __shfl_sync(0xffffffffu, w[(t + i) / 32], (t + i) % 32);
                        if ((of >> (t + i)) & 1) sum[t + i] = fmaf(f, __uint_as_float(v[i]), sum[t + i]);
                    }
                }
            }
            if (++acc == 2) { acc = 0; acc_phase ^= 1; }
            if (++at == kScaleSlots) at = 0;
        }
    }
}

// Barriers and TMEM of a CTA.  TMEM is taken when the grids before this one are complete, and the grid behind it let in when it is taken: no CTA
// holds TMEM while it waits for an earlier grid that still needs some.  It is taken before the router, whose cluster barriers wait for CTAs that
// may still be at theirs: the SMs start a second CTA only when the first has its TMEM (behind the router: 27 -> 34 us for a token, d = 4096), and
// nothing else that waits for its cluster with TMEM in hand (tiles by pairs of CTAs, projections and attention by clusters) fits beside
// one of these CTAs (more than 190 KB of shared memory each), so that what holds it back there always comes to an end.
template <int WT, int NT, bool SECOND>
__device__ __forceinline__ void set_up(const Smem<WT, NT>& sm) {
    using Cf = Cfg<WT, NT>;
    static_assert(Cf::RING >= 40 * 1024, "room that such a kernel would need");
    if (threadIdx.x == 0) {
        for (int s = 0; s < Cf::STAGES; ++s) { mbar_init(&sm.ctl->full[s], WT == kFp8 && !SECOND ? 1 + Cf::TEAM : 1); mbar_init(&sm.ctl->empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sm.ctl->tfull[i], 1); mbar_init(&sm.ctl->tempty[i], 4); }
        sm.ctl->abort_flag = 0;
        fence_barrier_init();
    }
    pdl_wait();
    if (threadIdx.x >> 5 == 1) tmem_alloc(&sm.ctl->tmem_base, Cf::TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
}

// The tile's sums from the registers of warps 4..7 to [token][128] floats where the ring was, visible to the CTAs that share the tile.
template <int WT, int NT>
__device__ __forceinline__ float* meet(const Smem<WT, NT>& sm, const float* sum, int Tn, int S) {
    using Cf = Cfg<WT, NT>;
    float* cta = (float*)sm.ring;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    tc_fence_before();
    __syncthreads();                                   // every stage has been read (the last accumulator is complete), every role is done
    if (warp == 1) tmem_dealloc(sm.ctl->tmem_base, Cf::TMEM_COLS);
    if (warp >= 4 && warp < 8) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (t < Tn) cta[t * Cf::PITCH + 32 * (warp & 3) + lane] = sum[t];
    }
    if (S > 1) cluster_sync_all();
    else __syncthreads();
    return cta;
}

template <int WT, int NT>
__global__ void __launch_bounds__(32 * Cfg<WT, NT>::WARPS1, Cfg<WT, NT>::CTAS)
first_layer_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ TokArgs a, int S, int* status) {
    using Cf = Cfg<WT, NT>;
    using bf16 = __nv_bfloat16;
    extern __shared__ uint8_t smem_raw[];
    const int rank = (int)cluster_ctarank(), Tn = a.T;
    const Smem<WT, NT> sm(smem_raw);
    if (threadIdx.x == 0) { prefetch_tmap(&tmW); if (WT == kBf16) prefetch_tmap(&tmX); }
    set_up<WT, NT, false>(sm);
    route_tokens<WT, (NT + 15) / 16, Cf::CLUSTER>(a, 0, Tn, rank, (float*)sm.ring, sm.part, sm.ctl->R);
    fence_async_smem();                                // the ring is the copies' from here on
    __syncthreads();
    const Routed& R = sm.ctl->R;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (blockIdx.x == 0 && (warp & ~1) == 2) write_routing(a, R, 0, Tn, warp - 2, 2);      // (warps without a part in what follows)
    const int tiles_n = (a.d_e + kCols - 1) / kCols, tile = blockIdx.x / S, kr = rank % S, first = rank - kr;
    const bool live = tile < R.experts * tiles_n;
    const int slot = live ? tile / tiles_n : 0, c0 = (tile - slot * tiles_n) * kCols, e = R.list[slot], Kb = (a.d + Cf::K - 1) / Cf::K;
    float sum[NT] = {};
    if (live) {
        Line line{0, 0, Kb, slot};
        cut(Kb, S, kr, line.lo, line.hi);
        const size_t blocks = (a.d + kQ - 1) / kQ;     // of the scales, along d
        run_line<WT, NT, false>(sm, &tmW, &tmX, (const bf16*)a.x, a.d, nullptr, WT == kFp8 ? a.s1 + c0 / kQ * blocks : nullptr,
                                (size_t)((a.d_e + kQ - 1) / kQ) * blocks, c0, a.d, Tn, line, status, sum, [](int, int) { return 1.f; });
    }
    cluster_wait();
    const float* cta = meet(sm, sum, Tn, S);
    if (live) {
        // (token, 32 columns) per warp, or the token's 128 columns, a lane four of them, where they become two terms
        constexpr int W = 4, WARPS = Cf::WARPS1;
        for (int tok = kr * WARPS + warp; tok < Tn; tok += S * WARPS) {
            if (!((R.of[slot] >> tok) & 1)) continue;
            float h[W];
#pragma unroll
            for (int v = 0; v < W; ++v) {
                const int col = c0 + W * lane + v;
                h[v] = 0.f;
                for (int s = 0; s < S; ++s) h[v] += ld_cluster_f32(cta + tok * Cf::PITCH + W * lane + v, first + s);
                if (a.b1 && col < a.d_e) h[v] += to_f32(((const bf16*)a.b1)[(size_t)e * a.d_e + col]);
                // (half a step, 2^-8 of the value, like the hidden rows of uoe_mlp_forward)
                h[v] = col < a.d_e ? to_f32(__float2bfloat16_rn(act_fast(h[v], a.act))) : 0.f;
            }
            if constexpr (WT == kFp8) {
                uint32_t hi, lo;
                const float sc = two_terms(h[0], h[1], h[2], h[3], hi, lo);
                const size_t dp = (size_t)tiles_n * kCols;
                uint8_t* o = (uint8_t*)a.a + ((size_t)2 * slot * a.group + tok) * dp + c0 + W * lane;
                *(uint32_t*)o = hi;
                *(uint32_t*)(o + a.group * dp) = lo;
                if (lane == 0) a.af[((size_t)slot * tiles_n + c0 / kCols) * kMaxTokens + tok] = sc;
            } else if (c0 + W * lane < a.d_e) {        // (d_e is a multiple of 8)
                *(uint2*)((bf16*)a.a + ((size_t)slot * a.group + tok) * a.d_e + c0 + W * lane) = make_uint2(pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3]));
            }
        }
    }
    if (S > 1) cluster_sync_all();      // nobody's shared memory goes while another CTA may read it
}

template <int WT, int NT>
__global__ void __launch_bounds__(32 * Cfg<WT, NT>::WARPS2, Cfg<WT, NT>::CTAS)
second_layer_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ TokArgs a, int S, int* status) {
    using Cf = Cfg<WT, NT>;
    using bf16 = __nv_bfloat16;
    extern __shared__ uint8_t smem_raw[];
    const int rank = (int)cluster_ctarank(), Tn = a.T;
    const Smem<WT, NT> sm(smem_raw);
    if (threadIdx.x == 0) { prefetch_tmap(&tmW); if (WT == kBf16) prefetch_tmap(&tmX); }
    set_up<WT, NT, true>(sm);
    read_routing(a, sm.ctl->R, Tn);
    const Routed& R = sm.ctl->R;
    if (blockIdx.x == 0 && threadIdx.x >> 5 == 2 && a.r.expert_offsets) write_offsets(a);
    const int c0 = blockIdx.x / S * kCols, kr = rank % S, first = rank - kr;
    auto weight = [&](int tok, int e) { const float p = R.p[tok][e]; return a.use_gate ? p * p : 1.f; };
    Line line{0, 0, (a.d_e + Cf::K - 1) / Cf::K, 0};
    cut(c0 < a.d ? R.experts * line.per : 0, S, kr, line.lo, line.hi);      // (the grid is whole clusters)
    float sum[NT] = {};
    const size_t blocks = (a.d_e + kQ - 1) / kQ;
    run_line<WT, NT, true>(sm, &tmW, &tmX, nullptr, 0, a.af, WT == kFp8 ? a.s2 + c0 / kQ * blocks : nullptr,
                           (size_t)((a.d + kQ - 1) / kQ) * blocks, c0, a.d_e, Tn, line, status, sum, weight);
    const float* cta = meet(sm, sum, Tn, S);
    for (int q = kr * blockDim.x + threadIdx.x; q < Tn * kCols; q += S * blockDim.x) {
        const int tok = q / kCols, col = c0 + q % kCols;
        if (col >= a.d) continue;
        float s = 0.f;
        for (int r = 0; r < S; ++r) s += ld_cluster_f32(cta + tok * Cf::PITCH + q % kCols, first + r);
        if (a.b2)
            for (uint32_t m = R.mask[tok]; m; m &= m - 1) {
                const int e = __ffs(m) - 1;
                s = fmaf(weight(tok, e), to_f32(((const bf16*)a.b2)[(size_t)e * a.d + col]), s);
            }
        const size_t at = (size_t)tok * a.d + col;
        if (a.residual) s += to_f32(((const bf16*)a.x)[at]);
        ((bf16*)a.y)[at] = __float2bfloat16_rn(s);
    }
    if (S > 1) cluster_sync_all();
}

// weights of a layer, K x N per expert
template <int WT>
bool weight_map(CUtensorMap* tm, const void* W, int n, int K, int N) {
    if (WT == kFp8) {                   // [n, N, Kp]
        const uint64_t Kp = q_pad(K);
        const uint64_t dims[3] = {Kp, (uint64_t)N, (uint64_t)n}, str[2] = {Kp, Kp * N};
        const uint32_t box[3] = {128, kCols, 1};
        return make_tmap(tm, W, 3, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8);
    }
    const uint64_t dims[3] = {(uint64_t)N, (uint64_t)K, (uint64_t)n}, str[2] = {(uint64_t)N * 2, (uint64_t)N * K * 2};
    const uint32_t box[3] = {64, 64, 1};
    return make_tmap(tm, W, 3, dims, str, box);
}
// tokens' values: `slots` matrices [rows, K], read NT rows at a time
bool value_map(CUtensorMap* tm, const void* x, int rows, int K, int slots, size_t slot_stride, int NT) {
    const uint64_t dims[3] = {(uint64_t)K, (uint64_t)rows, (uint64_t)slots}, str[2] = {(uint64_t)K * 2, (uint64_t)slot_stride * 2};
    const uint32_t box[3] = {64, (uint32_t)NT, 1};
    return make_tmap(tm, x, 3, dims, str, box);
}

// the hidden rows' two terms, [2 n, group, d_e padded]
bool term_map(CUtensorMap* tm, const void* a, int group, int d_e, int n, int NT) {
    const uint64_t dp = q_pad(d_e), dims[3] = {dp, (uint64_t)group, 2 * (uint64_t)n}, str[2] = {dp, dp * group};
    const uint32_t box[3] = {128, (uint32_t)NT, 1};
    return make_tmap(tm, a, 3, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8);
}

template <int WT, int NT>
uoe_status launch_layers(const TokArgs& a, int* status, cudaStream_t s) {
    using Cf = Cfg<WT, NT>;
    static DeviceOnce once1, once2;
    uoe_status st = smem_opt_in(once1, first_layer_kernel<WT, NT>, kMaxSmem);
    if (st == UOE_OK) st = smem_opt_in(once2, second_layer_kernel<WT, NT>, kMaxSmem);
    if (st != UOE_OK) return st;
    CUtensorMap tmW, tmX;
    const size_t smem = Smem<WT, NT>::bytes(a.T, a.n);
    auto grid = [&](long long tiles, int S) { return dim3((unsigned)((tiles * S + Cf::CLUSTER - 1) / Cf::CLUSTER * Cf::CLUSTER)); };
    const long long chosen = a.n < (long long)a.T * a.k ? a.n : (long long)a.T * a.k;      // experts at most
    {
        const long long tiles = chosen * ((a.d_e + kCols - 1) / kCols);
        const int S = split_of((a.d + Cf::K - 1) / Cf::K, tiles, Cf::CLUSTER, Cf::CTAS);
        if (!weight_map<WT>(&tmW, a.W1, a.n, a.d, a.d_e)) return UOE_ERR_CUDA;
        if (WT != kBf16) tmX = tmW;
        else if (!value_map(&tmX, a.x, a.T, a.d, 1, (size_t)a.T * a.d, NT)) return UOE_ERR_CUDA;
        ProfScope ps("tokens_first", s);
        launch_k_cluster(first_layer_kernel<WT, NT>, grid(tiles, S), dim3(32 * Cf::WARPS1), Cf::CLUSTER, smem, s, tmW, tmX, a, S, status);
        UOE_LAUNCHED();
    }
    {
        const long long tiles = (a.d + kCols - 1) / kCols;
        const int S = split_of(a.k * ((a.d_e + Cf::K - 1) / Cf::K), tiles, Cf::CLUSTER, Cf::CTAS);
        if (!weight_map<WT>(&tmW, a.W2, a.n, a.d_e, a.d)) return UOE_ERR_CUDA;
        if (WT != kBf16) tmX = tmW;
        else if (!value_map(&tmX, a.a, a.group, a.d_e, a.n, (size_t)a.group * a.d_e, NT)) return UOE_ERR_CUDA;
        if (WT == kFp8 && !term_map(&tmX, a.a, a.group, a.d_e, a.n, NT)) return UOE_ERR_CUDA;
        ProfScope ps("tokens_second", s);
        launch_k_cluster(second_layer_kernel<WT, NT>, grid(tiles, S), dim3(32 * Cf::WARPS2), Cf::CLUSTER, smem, s, tmW, tmX, a, S, status);
        UOE_LAUNCHED();
    }
    return UOE_OK;
}

template <int WT>
uoe_status launch_tensor(const TokArgs& a, int* status, cudaStream_t s) {
    if (a.T <= 8 && WT == kFp8) return launch_layers<WT, WT == kFp8 ? 8 : 16>(a, status, s);
    if (a.T <= 16) return launch_layers<WT, 16>(a, status, s);
    return a.T <= 32 ? launch_layers<WT, 32>(a, status, s) : launch_layers<WT, 64>(a, status, s);
}

int group_of(bool bf16) { return bf16 ? kMaxTokens : group_f32(); }

}  // namespace
}  // namespace tokens

// Workspace: status, the router's word, the hidden rows (bfloat16, or two e4m3 terms and a scale per 128), float32 groups behind one another.
static size_t tokens_ws(const Dims& D, size_t* routed, size_t* a, size_t* af) {
    using namespace tokens;
    const int group = group_of(D.bf16), groups = (D.B + group - 1) / group;
    const size_t width = D.bf16 ? (size_t)q_pad(D.d_e) * 2 : (size_t)D.d_e * 4;
    WsCarver w;
    w.take(kStatusBytes);
    const size_t r = w.take(groups * sizeof(Routed)), h = w.take((size_t)groups * D.n * group * width), f = w.take((size_t)D.n * q_blocks(D.d_e) * kMaxTokens * 4);
    if (routed) { *routed = r; *a = h; *af = f; }
    return w.off;
}

size_t mlp_tokens_workspace_bytes(const Dims& D) {
    using namespace tokens;
    if (D.L != 1 || D.B > kMaxTokens) return 0;
    return tokens_ws(D, nullptr, nullptr, nullptr);
}

}  // namespace uoe

using namespace uoe;

extern "C" uoe_status uoe_mlp_tokens(const uoe_problem* prob, const void* x, const void* W_r, const void* W1, const float* w1_scale,
                                     const void* W2, const float* w2_scale, const void* b1, const void* b2, const uoe_routing* r, void* y,
                                     void* ws, size_t ws_bytes, void* cuda_stream) {
    using namespace uoe::tokens;
    Dims D;
    const uoe_status st = make_dims(prob, D);
    if (st != UOE_OK) return st;
    if (D.d_e < 1 || !x || !W_r || !W1 || !W2 || !y || !ws || (w1_scale == nullptr) != (w2_scale == nullptr)) return UOE_ERR_INVALID_ARG;
    for (const void* p : {x, W_r, W1, W2, (const void*)w1_scale, (const void*)w2_scale, b1, b2, (const void*)y, (const void*)ws})
        if (p && !aligned16(p)) return UOE_ERR_INVALID_ARG;
    if (x == y) return UOE_ERR_INVALID_ARG;
    if (r && (!r->expert_idx || !r->patch_idx || !r->gate || !r->p_samp || !r->p_patch || !r->expert_offsets)) return UOE_ERR_INVALID_ARG;
    if (D.L != 1 || D.B > kMaxTokens || (w1_scale && !D.bf16)) return UOE_ERR_UNSUPPORTED;
    if (!w1_scale && (D.d_e * D.esize) % 16 != 0) return UOE_ERR_UNSUPPORTED;      // rows of W1 and of the hidden values move in 16-byte pieces
    if (ws_bytes < mlp_tokens_workspace_bytes(D)) return UOE_ERR_WORKSPACE;
    TokArgs a = {};
    a.x = x; a.Wr = W_r; a.W1 = W1; a.W2 = W2; a.b1 = b1; a.b2 = b2; a.s1 = w1_scale; a.s2 = w2_scale;
    a.group = group_of(D.bf16);
    size_t o_r, o_a, o_f;
    tokens_ws(D, &o_r, &o_a, &o_f);
    a.routed = (Routed*)((char*)ws + o_r);
    a.a = (char*)ws + o_a;
    a.af = (float*)((char*)ws + o_f);
    a.y = y;
    if (r) a.r = RoutingPtrs{r->expert_idx, r->patch_idx, r->gate, r->p_samp, r->p_patch, r->expert_offsets};
    a.T = D.B; a.d = D.d; a.d_e = D.d_e; a.n = D.n; a.k = D.k; a.act = prob->act;
    a.use_gate = (prob->flags & UOE_FLAG_GATE) != 0; a.residual = (prob->flags & UOE_FLAG_RESIDUAL) != 0;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (!D.bf16) return launch_f32(a, s);
    return w1_scale ? launch_tensor<kFp8>(a, (int*)ws, s) : launch_tensor<kBf16>(a, (int*)ws, s);
}
