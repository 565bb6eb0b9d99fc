// Products of 8-bit operands with a scale per block of 128 (fp8.cuh) on the tcgen05 tensor cores, grouped by expert:
//
//   rows    C[r, j]    = sum_kb sa[kb, r] sb[e(r), j / 128, kb]  sum_{k in block kb} A[r, k] B[e(r), j, k]
//   wgrad   C[e, i, j] = sum_kb sa[kb, i] sb[kb, j]              sum_{r in block kb} A[i, r] B[j, r],   kb over expert e's region
//
// The tensor cores form one block's product at a time (K = 128: four instructions) in TMEM, and eight warps add it, times its
// scales, to accumulators in registers: the scales are any float32 numbers, and the sum over blocks is float32 arithmetic.
// A persistent CTA per SM walks the 128 x BN tiles:
//   warp 0      TMA producer: a stage is one block, 128 x 128 bytes of A and BN x 128 of B (128-byte rows, swizzled)
//   warp 1      MMA issuer: a block's product into one of two TMEM accumulators, which the other warps empty in turn
//   warp 2      the scales of the blocks to come, by 4-byte asynchronous copies (their rows start anywhere) into a ring of their own
//   warps 4..11 a warp has 32 rows (its TMEM lane quarter) and half of the columns: one row's BN / 2 sums per thread.  The
//               columns are one block of B's scales, so a thread's factor is one number per block.
// Regions of experts are whole 128-row tiles, so no tile straddles two experts, and in wgrad no block does.
#include "fp8_tile.cuh"
#include "tc.cuh"
#include "tmap.cuh"

namespace uoe {
namespace {

using namespace tc;

constexpr int BM = 128;
constexpr int kScaleSlots = 8;
template <int BN> struct Cfg {
    static constexpr int A_BYTES = BM * kQ, B_BYTES = BN * kQ, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = BN == 256 ? 4 : 6;
    static constexpr int CW = BN / 2;                 // columns of an accumulating warp
    static constexpr int EPI_WARPS = 8, THREADS = 128 + 32 * EPI_WARPS;
    static constexpr int TMEM_COLS = 2 * BN;
    static constexpr int SCALES = BM + BN;            // floats of a block's scales: the rows', then the columns' (or column blocks')
    static constexpr int CTL_BYTES = 1024;
    static constexpr int SMEM = STAGES * STAGE + 1024 /* alignment */ + CTL_BYTES + kScaleSlots * SCALES * 4 + EPI_WARPS * kTurnBytes;
};

struct Ctl {
    uint64_t full[8], empty[8], tfull[2], tempty[2], sfull[kScaleSlots], sempty[kScaleSlots];
    uint32_t tmem_base;
    int abort_flag;
    Regions reg;
};
static_assert(sizeof(Ctl) <= 1024, "control block");

template <int BN, bool WGRAD, int EPI>
__global__ void __launch_bounds__(Cfg<BN>::THREADS, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmC,
                const __grid_constant__ Fp8Args a) {
    using Cf = Cfg<BN>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Ctl* ctl = (Ctl*)(smem + Cf::STAGES * Cf::STAGE);
    volatile int* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = a.n;
    if (threadIdx.x == 0) {
        for (int s = 0; s < Cf::STAGES; ++s) { mbar_init(&ctl->full[s], 1); mbar_init(&ctl->empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&ctl->tfull[i], 1); mbar_init(&ctl->tempty[i], Cf::EPI_WARPS); }
        for (int i = 0; i < kScaleSlots; ++i) { mbar_init(&ctl->sfull[i], 32); mbar_init(&ctl->sempty[i], Cf::EPI_WARPS); }
        ctl->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
    }
    pdl_wait();
    // (TMEM only when the grids before this one are complete, and the grid behind it only when it is taken: no CTA holds TMEM while it waits
    // for one that still needs some)
    if (warp == 1) tmem_alloc(&ctl->tmem_base, Cf::TMEM_COLS);
    // tiles of the rows: per expert its 128-row blocks; without offsets all rows are one expert's; wgrad: every expert has all of C
    const int m_tiles = (int)((a.M + BM - 1) / BM);
    if (warp == 2) {
        load_regions<WGRAD, BM>(ctl->reg, a, m_tiles, lane);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem_base = ctl->tmem_base;
    float* s_scales = (float*)((uint8_t*)ctl + Cf::CTL_BYTES);
    const int n_tiles = (a.N + BN - 1) / BN;
    const int total = ctl->reg.tstart[n] * n_tiles;

    // tile -> expert, first row of A and C, first block of the contraction and their number
    auto locate = [&](int tile, int& e, int& row0, int& col0, int& kb0, int& kbs) {
        const int rt = tile / n_tiles;
        while (e + 1 < n && rt >= ctl->reg.tstart[e + 1]) ++e;
        row0 = (rt - ctl->reg.tstart[e]) * BM + (WGRAD ? 0 : ctl->reg.offs[e]);
        col0 = (tile - rt * n_tiles) * BN;
        kb0 = WGRAD ? ctl->reg.offs[e] / kQ : 0;
        kbs = WGRAD ? (ctl->reg.offs[e + 1] - ctl->reg.offs[e]) / kQ : a.Kb;
    };

    // Registers: 384 threads start with 168 each; the first warpgroup gives 128 of its up, the accumulating ones take 64 more
    // (128 * 40 + 256 * 232 = 384 * 168).
    if (warp >= 4) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        constexpr int CW = Cf::CW;
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        float* turn = s_scales + kScaleSlots * Cf::SCALES + (warp - 4) * (kTurnBytes / 4);
        int acc = 0, e = 0, slot = 0;
        uint32_t acc_phase = 0, slot_phase = 0;
        bool stop = false;
        for (int tile = blockIdx.x; tile < total && !stop; tile += gridDim.x) {
            int row0, col0, kb0, kbs;
            locate(tile, e, row0, col0, kb0, kbs);
            const int col = col0 + half * CW;
            float sum[CW];
#pragma unroll
            for (int q = 0; q < CW; ++q) sum[q] = 0.f;
            for (int kb = 0; kb < kbs; ++kb) {
                if (!mbar_wait_warp_quick(&ctl->sfull[slot], slot_phase, abort_flag, a.status)) { stop = true; break; }
                const float* sc = s_scales + slot * Cf::SCALES;
                const float f = WGRAD ? sc[quarter * 32 + lane] : sc[quarter * 32 + lane] * sc[BM + half];
                const float* s_sb = sc + BM + half * CW;
                if (!mbar_wait_warp_quick(&ctl->tfull[acc], acc_phase, abort_flag, a.status)) { stop = true; break; }
                tc_fence_after();
                const uint32_t taddr = tmem_base + acc * BN + half * CW + ((uint32_t)(quarter * 32) << 16);
                // 32 columns at a time, two pieces on their way while two are added: a thread waits twice per block (one piece of
                // 16 at a time, eight waits: 1390 cycles per block of 128 x 256 x 128 where the tensor cores take 540)
                uint32_t v[2][32];
                tmem_ld32(taddr, v[0]);
                tmem_ld32(taddr + 32, v[1]);
                auto add = [&](const uint32_t* w, int g) {
#pragma unroll
                    for (int q = 0; q < 32; q += 4) {
                        if constexpr (WGRAD) {
                            const float4 c = *(const float4*)(s_sb + g * 32 + q);
                            sum[g * 32 + q] = fmaf(__uint_as_float(w[q]), f * c.x, sum[g * 32 + q]);
                            sum[g * 32 + q + 1] = fmaf(__uint_as_float(w[q + 1]), f * c.y, sum[g * 32 + q + 1]);
                            sum[g * 32 + q + 2] = fmaf(__uint_as_float(w[q + 2]), f * c.z, sum[g * 32 + q + 2]);
                            sum[g * 32 + q + 3] = fmaf(__uint_as_float(w[q + 3]), f * c.w, sum[g * 32 + q + 3]);
                        } else {
#pragma unroll
                            for (int u = 0; u < 4; ++u) sum[g * 32 + q + u] = fmaf(__uint_as_float(w[q + u]), f, sum[g * 32 + q + u]);
                        }
                    }
                };
                auto release = [&]() {                           // all of it is in registers: the accumulator is free
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl->tempty[acc]);
                };
                tmem_ld_wait();
                if constexpr (CW == 64) {
                    release();
                    add(v[0], 0);
                    add(v[1], 1);
                } else {
                    add(v[0], 0);
                    tmem_ld32(taddr + 64, v[0]);
                    add(v[1], 1);
                    tmem_ld32(taddr + 96, v[1]);
                    tmem_ld_wait();
                    release();
                    add(v[0], 2);
                    add(v[1], 3);
                }
                if constexpr (WGRAD) __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->sempty[slot]);
                if (++acc == 2) { acc = 0; acc_phase ^= 1; }
                if (++slot == kScaleSlots) { slot = 0; slot_phase ^= 1; }
            }
            if (stop) break;
            store_tile<CW, WGRAD, EPI>(a, &tmC, sum, e, row0 + quarter * 32, a.M, col, turn);
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 0) {
            int stage = 0, e = 0;
            uint32_t phase = 0, issued = 0, issued_parity = 0;
            bool stop = false;
            for (int tile = blockIdx.x; tile < total && !stop; tile += gridDim.x) {
                int row0, col0, kb0, kbs;
                locate(tile, e, row0, col0, kb0, kbs);
                for (int kb = 0; kb < kbs; ++kb) {
                    if (!mbar_wait_warp_quick(&ctl->empty[stage], phase ^ 1, abort_flag, a.status)) { stop = true; break; }
                    if (lane == 0) {
                        uint8_t* st = smem + stage * Cf::STAGE;
                        mbar_arrive_expect_tx(&ctl->full[stage], Cf::STAGE);
                        tma_load_2d(st, &tmA, (kb0 + kb) * kQ, row0, &ctl->full[stage]);
                        tma_load_3d(st + Cf::A_BYTES, &tmB, (kb0 + kb) * kQ, col0, WGRAD ? 0 : e, &ctl->full[stage]);
                    }
                    __syncwarp();
                    issued |= 1u << stage;
                    issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
                    if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
                }
            }
            if (lane == 0 && *abort_flag)                 // copies in flight land before the CTA exits
                for (int s = 0; s < Cf::STAGES; ++s)
                    if (issued & (1u << s)) mbar_wait(&ctl->full[s], (issued_parity >> s) & 1, abort_flag, a.status);
        } else if (warp == 1) {
            const uint32_t el = elect_one();
            constexpr uint32_t idesc = instr_desc_e4m3(BM, BN);
            int stage = 0, acc = 0, e = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool stop = false;
            for (int tile = blockIdx.x; tile < total && !stop; tile += gridDim.x) {
                int row0, col0, kb0, kbs;
                locate(tile, e, row0, col0, kb0, kbs);
                for (int kb = 0; kb < kbs; ++kb) {
                    if (!mbar_wait_warp_quick(&ctl->tempty[acc], acc_phase ^ 1, abort_flag, a.status) ||
                        !mbar_wait_warp_quick(&ctl->full[stage], phase, abort_flag, a.status)) { stop = true; break; }
                    tc_fence_after();
                    const uint32_t st = smem_u32(smem + stage * Cf::STAGE);
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        mma_f8(el, tmem_base + acc * BN, smem_desc(st + ks * 32, 16, 1024), smem_desc(st + Cf::A_BYTES + ks * 32, 16, 1024), idesc, ks != 0);
                    mma_commit(el, &ctl->empty[stage]);
                    mma_commit(el, &ctl->tfull[acc]);
                    if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
                    if (++acc == 2) { acc = 0; acc_phase ^= 1; }
                }
            }
        } else if (warp == 2) {
            int slot = 0, e = 0;
            uint32_t phase = 0;
            bool stop = false;
            for (int tile = blockIdx.x; tile < total && !stop; tile += gridDim.x) {
                int row0, col0, kb0, kbs;
                locate(tile, e, row0, col0, kb0, kbs);
                const float* sa = a.sa + (size_t)kb0 * a.M + row0;
                const int rows = (int)(a.M - row0 < BM ? a.M - row0 : BM);
                const float* sb = WGRAD ? a.sb + (size_t)kb0 * a.N + col0 : a.sb + ((size_t)e * a.Nb + col0 / kQ) * a.Kb;
                const int cols = WGRAD ? min(a.N - col0, BN) : 0, nb = min(a.Nb - col0 / kQ, 2);
                for (int kb = 0; kb < kbs; ++kb, sa += a.M) {
                    if (!mbar_wait_warp_quick(&ctl->sempty[slot], phase ^ 1, abort_flag, a.status)) { stop = true; break; }
                    const uint32_t dst = smem_u32(s_scales + slot * Cf::SCALES);
#pragma unroll
                    for (int r = lane; r < BM; r += 32)
                        if (r < rows) cp_async4(dst + 4 * r, sa + r);
                    if constexpr (WGRAD) {
                        for (int c = lane; c < BN; c += 32)
                            if (c < cols) cp_async4(dst + 4 * (BM + c), sb + c);
                        sb += a.N;
                    } else {      // a warp of either column half reads its own: with 128 columns they are the same block
                        const int b = BN == 256 ? lane : 0;
                        if (lane < 2 && b < nb) cp_async4(dst + 4 * (BM + lane), sb + (size_t)b * a.Kb + kb);
                    }
                    cp_async_arrive(&ctl->sfull[slot]);
                    if (++slot == kScaleSlots) { slot = 0; phase ^= 1; }
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");      // none in flight when the CTA exits
        }
    }
    if (warp >= 4 && lane == 0) bulk_wait_all();        // this warp's tensor stores are complete
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tmem_dealloc(tmem_base, Cf::TMEM_COLS);
    }
}

template <int BN, bool WGRAD, int EPI>
uoe_status launch_one(const Fp8Gemm& g, int* status, cudaStream_t s) {
    using Cf = Cfg<BN>;
    static DeviceOnce once;
    auto kern = fp8_gemm_kernel<BN, WGRAD, EPI>;
    const uoe_status st = smem_opt_in(once, kern, Cf::SMEM);
    if (st != UOE_OK) return st;
    const uint64_t Kp = (uint64_t)((g.K + kQ - 1) / kQ * kQ);
    CUtensorMap tmA, tmB;
    {
        const uint64_t dims[2] = {Kp, (uint64_t)g.M};
        const uint64_t str[1] = {Kp};
        const uint32_t box[2] = {kQ, BM};
        if (!make_tmap(&tmA, g.A, 2, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    }
    {
        const uint64_t dims[3] = {Kp, (uint64_t)g.N, (uint64_t)(g.wgrad ? 1 : g.n)};
        const uint64_t str[2] = {Kp, Kp * (uint64_t)g.N};
        const uint32_t box[3] = {kQ, BN, 1};
        if (!make_tmap(&tmB, g.B, 3, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    }
    const Fp8Args a = fp8_args(g, status);
    CUtensorMap tmC = tmA;
    if (g.epi == kFp8Store && a.vec && !result_map(&tmC, g)) return UOE_ERR_CUDA;
    const long long m_tiles = (g.M + BM - 1) / BM, n_tiles = (g.N + BN - 1) / BN;
    const long long tiles = m_tiles * n_tiles * (g.wgrad ? g.n : 1);
    if (tiles > 0x3fffffffll) return UOE_ERR_UNSUPPORTED;
    const int grid = (int)(tiles < sm_count() ? tiles : sm_count());
    ProfScope ps(g.label, s);
    launch_k(kern, dim3(grid), dim3(Cf::THREADS), (size_t)Cf::SMEM, s, tmA, tmB, tmC, a);
    UOE_LAUNCHED();
    return UOE_OK;
}

}  // namespace

uoe_status launch_fp8_gemm_any(const Fp8Gemm& g, int* status, cudaStream_t s) {
    if (g.epi == kFp8ActQuant) return launch_one<256, false, kFp8ActQuant>(g, status, s);
    const long long tiles256 = (g.M + BM - 1) / BM * ((g.N + 255) / 256) * (g.wgrad ? g.n : 1);
    const bool wide = g.N > 128 && tiles256 >= sm_count();
    if (g.wgrad) return wide ? launch_one<256, true, kFp8Store>(g, status, s) : launch_one<128, true, kFp8Store>(g, status, s);
    return wide ? launch_one<256, false, kFp8Store>(g, status, s) : launch_one<128, false, kFp8Store>(g, status, s);
}

}  // namespace uoe
