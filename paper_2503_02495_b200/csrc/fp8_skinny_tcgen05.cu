// uoe_fp8_gemm for up to 64 rows of one weight matrix (the form for single tokens):
//   C[r, j] = sum_kb sa[kb, r] sb[j / 128, kb]  sum_{k in block kb} A[r, k] B[j, k]
//
// Bound by the weights, which are read once.  They are the 128-row operand of the tensor cores, the rows of A the narrow one: a 128-row tile of
// A would be mostly padding, and 128 columns of C at a time leave enough tiles to divide.  A cluster's CTAs share a tile's contraction (S of
// them, the largest split that leaves no more than two CTAs per SM) and add up in distributed shared memory, in a fixed order.  A stage is one block
// of the contraction; its product, times the block's two scales, is added to float32 registers, so the scales may be any numbers.
// (One row, N = K = 4096: 11.5 us in 32 CTAs of the tile kernel, which walk all of K one after the other.)
//   warp 0  TMA producer      warp 1  MMA issuer      warps 4..7  sums: one column of C per thread, all rows
#include "fp8_tile.cuh"
#include "tc.cuh"
#include "tmap.cuh"

namespace uoe {
namespace {

using namespace tc;

constexpr int kCols = 128, kCluster = 8, kThreads = 256;

template <int NT /* rows of A, rounded up */> struct Cfg {
    static constexpr int A_BYTES = kCols * kQ, B_BYTES = NT * kQ, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = NT == 16 ? 5 : 4, RING = STAGES * STAGE;
    static constexpr int TMEM_COLS = 2 * NT;
    static constexpr int PITCH = kCols + 4;           // floats of a row's sums in shared memory (where the ring was)
};
struct Ctl {
    uint64_t full[8], empty[8], tfull[2], tempty[2];
    uint32_t tmem_base;
    int abort_flag;
};

template <int NT>
__global__ void __launch_bounds__(kThreads, 2)
fp8_skinny_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA, const __grid_constant__ Fp8Args a, int S) {
    using Cf = Cfg<NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Ctl* ctl = (Ctl*)(ring + Cf::RING);
    volatile int* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < Cf::STAGES; ++s) { mbar_init(&ctl->full[s], 1); mbar_init(&ctl->empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&ctl->tfull[i], 1); mbar_init(&ctl->tempty[i], 4); }
        ctl->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tmW);
        prefetch_tmap(&tmA);
    }
    pdl_wait();
    // (TMEM only when the grids before this one are complete, and the grid behind it only when it is taken: no CTA holds TMEM while it waits
    // for one that still needs some)
    if (warp == 1) tmem_alloc(&ctl->tmem_base, Cf::TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem_base = ctl->tmem_base;
    const int c0 = blockIdx.x / S * kCols, rank = (int)cluster_ctarank(), kr = rank % S, first = rank - kr, M = (int)a.M;
    const int units = c0 < a.N ? a.Kb : 0;            // (the grid is whole clusters)
    const int lo = (int)((long long)units * kr / S), hi = (int)((long long)units * (kr + 1) / S);
    float sum[NT] = {};
    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0, issued = 0, issued_parity = 0;
        for (int kb = lo; kb < hi; ++kb) {
            if (!mbar_wait_warp_quick(&ctl->empty[stage], phase ^ 1, abort_flag, a.status)) break;
            if (lane == 0) {
                uint8_t* st = ring + stage * Cf::STAGE;
                mbar_arrive_expect_tx(&ctl->full[stage], Cf::STAGE);
                tma_load_2d(st, &tmW, kb * kQ, c0, &ctl->full[stage]);
                tma_load_2d(st + Cf::A_BYTES, &tmA, kb * kQ, 0, &ctl->full[stage]);
            }
            __syncwarp();
            issued |= 1u << stage;
            issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
            if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
        }
        if (lane == 0 && *abort_flag)                  // copies in flight land before the CTA exits
            for (int s = 0; s < Cf::STAGES; ++s)
                if (issued & (1u << s)) mbar_wait(&ctl->full[s], (issued_parity >> s) & 1, abort_flag, a.status);
    } else if (warp == 1) {
        const uint32_t el = elect_one();
        constexpr uint32_t idesc = instr_desc_e4m3(128, NT);
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        for (int kb = lo; kb < hi; ++kb) {
            if (!mbar_wait_warp_quick(&ctl->tempty[acc], acc_phase ^ 1, abort_flag, a.status) ||
                !mbar_wait_warp_quick(&ctl->full[stage], phase, abort_flag, a.status)) break;
            tc_fence_after();
            const uint32_t st = smem_u32(ring + stage * Cf::STAGE);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                mma_f8(el, tmem_base + acc * NT, smem_desc(st + ks * 32, 16, 1024), smem_desc(st + Cf::A_BYTES + ks * 32, 16, 1024), idesc, ks != 0);
            mma_commit(el, &ctl->empty[stage]);
            mma_commit(el, &ctl->tfull[acc]);
            if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
            if (++acc == 2) { acc = 0; acc_phase ^= 1; }
        }
    } else if (warp >= 4) {
        constexpr int L = (NT + 31) / 32;              // rows per lane: their factors, asked for a block ahead
        float next[L];
        const float* sb = a.sb + (size_t)(min(c0, a.N - 1) / kQ) * a.Kb;
        auto ask = [&](int kb) {
            const float s = __ldg(sb + kb);
#pragma unroll
            for (int i = 0; i < L; ++i) next[i] = s * (lane + 32 * i < M ? __ldg(a.sa + (size_t)kb * M + lane + 32 * i) : 0.f);
        };
        if (lo < hi) ask(lo);
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int kb = lo; kb < hi; ++kb) {
            float w[L];
#pragma unroll
            for (int i = 0; i < L; ++i) w[i] = next[i];
            if (kb + 1 < hi) ask(kb + 1);
            if (!mbar_wait_warp_quick(&ctl->tfull[acc], acc_phase, abort_flag, a.status)) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + acc * NT + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll
            for (int t = 0; t < NT; t += 16) {
                uint32_t v[16];
                tmem_ld16(taddr + t, v);
                tmem_ld_wait();
                if (t + 16 >= NT) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl->tempty[acc]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)           // (rows past M: zeros times zero)
                    sum[t + i] = fmaf(__shfl_sync(0xffffffffu, w[(t + i) / 32], (t + i) % 32), __uint_as_float(v[i]), sum[t + i]);
            }
            if (++acc == 2) { acc = 0; acc_phase ^= 1; }
        }
    }
    tc_fence_before();
    __syncthreads();                                   // every stage has been read
    if (warp == 1) tmem_dealloc(tmem_base, Cf::TMEM_COLS);
    float* cta = (float*)ring;
    if (warp >= 4) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (t < M) cta[t * Cf::PITCH + 32 * (warp & 3) + lane] = sum[t];
    }
    if (S > 1) cluster_sync_all();
    else __syncthreads();
    for (int q = kr * kThreads + threadIdx.x; q < M * kCols; q += S * kThreads) {
        const int r = q / kCols, c = q % kCols;
        if (c0 + c >= a.N) continue;
        float s = 0.f;
        for (int i = 0; i < S; ++i) s += ld_cluster_f32(cta + r * Cf::PITCH + c, first + i);
        const size_t at = (size_t)r * a.N + c0 + c;
        if (a.out_bf16) ((__nv_bfloat16*)a.C)[at] = __float2bfloat16_rn(s);
        else ((float*)a.C)[at] = s;
    }
    if (S > 1) cluster_sync_all();                     // nobody's shared memory goes while another CTA may read it
}

template <int NT>
uoe_status launch_one(const Fp8Gemm& g, int* status, cudaStream_t s) {
    using Cf = Cfg<NT>;
    static DeviceOnce once;
    auto kern = fp8_skinny_kernel<NT>;
    const size_t smem = 1024 + Cf::RING + sizeof(Ctl);
    const uoe_status st = smem_opt_in(once, kern, (int)smem);
    if (st != UOE_OK) return st;
    const uint64_t Kp = (uint64_t)((g.K + kQ - 1) / kQ * kQ), str[1] = {Kp};
    CUtensorMap tmW, tmA;
    {
        const uint64_t dims[2] = {Kp, (uint64_t)g.N};
        const uint32_t box[2] = {kQ, kCols};
        if (!make_tmap(&tmW, g.B, 2, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    }
    {
        const uint64_t dims[2] = {Kp, (uint64_t)g.M};
        const uint32_t box[2] = {kQ, NT};
        if (!make_tmap(&tmA, g.A, 2, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    }
    const Fp8Args a = fp8_args(g, status);
    const long long tiles = (g.N + kCols - 1) / kCols;
    int S = kCluster;
    while (S > 1 && (a.Kb < S || tiles * S > 2ll * sm_count())) S >>= 1;
    const long long ctas = (tiles * S + kCluster - 1) / kCluster * kCluster;
    if (ctas > 0x7fffffffll) return UOE_ERR_UNSUPPORTED;
    ProfScope ps(g.label, s);
    launch_k_cluster(kern, dim3((unsigned)ctas), dim3(kThreads), kCluster, smem, s, tmW, tmA, a, S);
    UOE_LAUNCHED();
    return UOE_OK;
}

}  // namespace

bool fp8_is_skinny(const Fp8Gemm& g) { return !g.wgrad && g.epi == kFp8Store && !g.bias && !g.offsets && g.n == 1 && g.M <= 64; }

uoe_status launch_fp8_skinny(const Fp8Gemm& g, int* status, cudaStream_t s) {
    return g.M <= 16 ? launch_one<16>(g, status, s) : g.M <= 32 ? launch_one<32>(g, status, s) : launch_one<64>(g, status, s);
}

}  // namespace uoe
