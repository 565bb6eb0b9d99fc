// Second expert layer and combine on 8-bit operands in one kernel, walked by output patch (Eq. 39-40), for patches of 128 tokens:
//
//   y[b, 128 j + r, :] = x[b, 128 j + r, :] + sum over the slots s that selected patch j  gate_s ( a[row_s + r, :] W2[e_s] + b2[e_s] )
//
// A 128-row tile is one patch, so the CTA that owns (patch, 256 columns) multiplies for every expert that selected it and adds the products,
// times their float32 weights, in registers, in ascending slot order: the experts' outputs never reach memory.  (Apart, for 4 x 4096 tokens of
// 4096 and 16 experts of 1024: product 113 us, combine 84 us; together 175 us.  The 256 x 256 tile of two CTAs, which the product has
// when it is apart, needs a third fewer operand bytes, but two patches do not share their experts.)
// What bounds it: a block takes 0.36 us of the 0.33 that the tensor cores need at that clock; between products the accumulator is read (1 us), and a
// tile's x and y (some 3 us more than the next tile's first product hides).
// The block-scaled products are those of fp8_gemm_tcgen05.cu.  A tile costs as many products as its patch has experts, so tiles are handed out
// as the CTAs get to them (which CTA computes a tile varies, its value does not):
//   warp 0       TMA producer: a stage is one block of the contraction
//   warp 1       MMA issuer
//   warp 2       scheduler: takes the next tile from a counter in the workspace's control block, looks up who selected the patch, a few tiles ahead
//   warps 4..7   the stages' scales in turn
//   warps 8..15  sums: 32 rows (the warp's TMEM lane quarter) x 128 columns, a row per lane
#include "fp8_tile.cuh"
#include "tc.cuh"
#include "tmap.cuh"

namespace uoe {
namespace {

using namespace tc;

constexpr int BM = 128, BN = 256, CW = BN / 2;
constexpr int A_BYTES = BM * kQ, STAGE = A_BYTES + BN * kQ, STAGES = 4;
static_assert(STAGES >= 4, "four warps in turn: none looks for a stage's last use by parity two uses ahead");
constexpr int SF_COL = 256, SF_STRIDE = 16, SFB = 8, SF_BYTES = 512 + 4 * BN, TMEM_COLS = 512;
constexpr int THREADS = 512, EPI_WARPS = 8, CONSUMERS = 2 + 4 + EPI_WARPS;
constexpr int kSlots = 4;          // tiles the scheduler may run ahead of the slowest consumer
constexpr int kSchedWord = 64;     // words [64, 66) of the workspace's control block: next tile, CTAs finished (zero between launches)
constexpr int kMaxK = 32;

struct Work { int tile, count, row[kMaxK], expert[kMaxK]; float gate[kMaxK]; };
struct Ctl {
    uint64_t full[STAGES], empty[STAGES], tfull, tempty, sfull[kSlots], sempty[kSlots];
    uint32_t tmem_base;
    int abort_flag;
    int offs[kMaxExperts + 1];
    Work work[kSlots];
};
constexpr int CTL_BYTES = 2048;
static_assert(sizeof(Ctl) <= CTL_BYTES, "control block");
constexpr int SMEM = STAGES * (STAGE + SF_BYTES) + 1024 /* alignment */ + CTL_BYTES + EPI_WARPS * kTurnBytes;

struct PatchArgs {
    const float *sa, *sb;
    const int *inv_row, *offsets;      // [patches, k], [n+1]
    const float* inv_gate;             // [patches, k]
    const __nv_bfloat16 *x, *b2;
    long long rows;                    // routed
    int patches, m, k, n, N, Nb, Kb, Lv, use_gate, residual;
    int* status;
    int* sched;                        // [2], zero between launches
};

__global__ void __launch_bounds__(THREADS, 1)
fp8_patch_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmY,
                 const __grid_constant__ PatchArgs p, const __grid_constant__ Fp8Args out) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Ctl* ctl = (Ctl*)(smem + STAGES * STAGE);
    uint8_t* s_sf = (uint8_t*)ctl + CTL_BYTES;
    volatile int* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&ctl->full[s], 2); mbar_init(&ctl->empty[s], 1); }
        for (int s = 0; s < kSlots; ++s) { mbar_init(&ctl->sfull[s], 1); mbar_init(&ctl->sempty[s], CONSUMERS); }
        mbar_init(&ctl->tfull, 1);
        mbar_init(&ctl->tempty, EPI_WARPS);
        ctl->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
        prefetch_tmap(&tmY);
    }
    pdl_wait();
    if (warp == 1) tmem_alloc(&ctl->tmem_base, TMEM_COLS);      // (order of TMEM and the grids around this one: fp8_gemm_tcgen05.cu)
    if (warp == 2)
        for (int i = lane; i <= p.n; i += 32) ctl->offs[i] = p.offsets[i];
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem_base = ctl->tmem_base;
    const int n_tiles = (p.N + BN - 1) / BN, total = p.patches * n_tiles;      // (column tiles of a patch are neighbours: its rows stay in L2)

    // A consumer warp's next tile: its place among the slots, or -1 at the end.  done() gives the place back.
    int slot = 0;
    uint32_t sphase = 0;
    auto next = [&]() -> const Work* {
        if (!mbar_wait_warp_quick(&ctl->sfull[slot], sphase, abort_flag, p.status)) return nullptr;
        const Work* w = &ctl->work[slot];
        return w->tile < total ? w : nullptr;
    };
    auto done = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl->sempty[slot]);
        if (++slot == kSlots) { slot = 0; sphase ^= 1; }
    };

    // Registers: 512 threads start with 128 each (256 * 80 + 256 * 176 = 512 * 128).
    if (warp >= 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
        const int quarter = warp & 3, half = (warp - 8) >> 2;
        float* turn = (float*)(s_sf + STAGES * SF_BYTES + (warp - 8) * kTurnBytes);
        uint32_t phase = 0;
        bool stop = false;
        while (const Work* w = next()) {
            const int patch = w->tile / n_tiles, col = (w->tile - patch * n_tiles) * BN + half * CW;
            const long long row0 = (long long)patch * BM + quarter * 32;
            const bool real = (patch % p.m) * BM + quarter * 32 + lane < p.Lv;       // (pad tokens: y = x)
            float sum[CW];                       // from x on, which is on its way while the first product is computed (asked for by L2 prefetches: no gain)
            if (p.residual) {
                // whole sectors, eight rows of 64 bytes per load, turned to a row per lane in shared memory (a row per lane from memory, 16 bytes
                // of 32 lines per load: 185 us in place of 177)
                uint4 in[CW / 8];
#pragma unroll
                for (int i = 0; i < CW / 8; ++i) {
                    const int c = col + i / 4 * 32 + (lane & 3) * 8;                 // (N is a multiple of 8)
                    in[i] = c < p.N ? *(const uint4*)(p.x + (row0 + (i & 3) * 8 + (lane >> 2)) * p.N + c) : make_uint4(0, 0, 0, 0);
                }
                if (lane == 0) bulk_wait_read();                                     // the last store has read `turn`
#pragma unroll
                for (int g = 0; g < CW / 32; ++g) {
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 8 + (lane >> 2);
                        *(uint4*)((uint8_t*)turn + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4)) = in[g * 4 + i];
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        unpack16<__nv_bfloat16>(*(const uint4*)((uint8_t*)turn + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)), sum + g * 32 + i * 8);
                }
            } else {
#pragma unroll
                for (int q = 0; q < CW; ++q) sum[q] = 0.f;
            }
            for (int i = 0; i < w->count && !stop; ++i) {
                const float gate = real ? w->gate[i] : 0.f;          // (on a pad token 0 times 0 is added, whatever the patch's gate is)
                if (!mbar_wait_warp_quick(&ctl->tfull, phase, abort_flag, p.status)) { stop = true; break; }
                phase ^= 1;
                tc_fence_after();
                const uint32_t from = tmem_base + half * CW + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
                for (int g = 0; g < CW / 32; ++g) {
                    float v[32];
                    tmem_ld32(from + g * 32, (uint32_t*)v);
                    tmem_ld_wait();
                    if (g + 1 == CW / 32) {                  // everything is in registers
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&ctl->tempty);
                    }
#pragma unroll
                    for (int q = 0; q < 32; ++q) sum[g * 32 + q] = fmaf(gate, real ? v[q] : 0.f, sum[g * 32 + q]);
                }
                if (p.b2 && real) {
                    const __nv_bfloat16* b = p.b2 + (size_t)w->expert[i] * p.N + col;
#pragma unroll
                    for (int q = 0; q < CW; ++q)
                        if (col + q < p.N) sum[q] = fmaf(gate, to_f32(b[q]), sum[q]);
                }
            }
            if (stop) break;
            done();
            store_tile<CW, false, kFp8Store>(out, &tmY, sum, 0, row0, out.M, col, turn);
        }
    } else if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        int stage = 0, turn = 0;
        uint32_t phase = 0;
        bool stop = false, bad = false;
        while (const Work* w = next()) {
            const int patch = w->tile / n_tiles, col0 = (w->tile - patch * n_tiles) * BN, cols = p.N - col0, blocks = w->count * p.Kb;
            const int first = ((warp & 3) - turn) & 3;               // this warp's first block of the tile
            float ra[4], rb[2] = {1.f, 1.f};
            int i_next = 0, kb_next = first;                         // slot and block of the contraction that it asks for next
            auto ask = [&]() {
                while (kb_next >= p.Kb) { kb_next -= p.Kb; ++i_next; }
                if (i_next >= w->count) return;
                const float* sa = p.sa + (size_t)kb_next * p.rows + w->row[i_next] + lane;
                const float* sb = p.sb + ((size_t)w->expert[i_next] * p.Nb + col0 / kQ) * p.Kb + kb_next;
#pragma unroll
                for (int q = 0; q < 4; ++q) ra[q] = __ldg(sa + q * 32);
                rb[0] = __ldg(sb);
                if (cols > kQ) rb[1] = __ldg(sb + p.Kb);
                kb_next += 4;
            };
            if (first < blocks) ask();
            for (int t = 0; t < blocks; ++t) {
                if (((t - first) & 3) == 0) {
                    uint32_t wa[4], wb[2];
#pragma unroll
                    for (int q = 0; q < 4; ++q) wa[q] = exponent_word(ra[q], true, bad);
#pragma unroll
                    for (int q = 0; q < 2; ++q) wb[q] = exponent_word(rb[q], cols > q * kQ, bad);
                    if (t + 4 < blocks) ask();
                    if (!mbar_wait_warp_quick(&ctl->empty[stage], phase ^ 1, abort_flag, p.status)) { stop = true; break; }
                    uint8_t* sf = s_sf + stage * SF_BYTES + lane * 16;
                    *(uint4*)sf = make_uint4(wa[0], wa[1], wa[2], wa[3]);
                    *(uint4*)(sf + 512) = make_uint4(wb[0], wb[0], wb[0], wb[0]);
                    *(uint4*)(sf + 1024) = make_uint4(wb[1], wb[1], wb[1], wb[1]);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl->full[stage]);
                }
                if (++stage == STAGES) { stage = 0; phase ^= 1; }
            }
            if (stop) break;
            turn += blocks;
            done();
        }
        if (bad) set_status(p.status, UOE_ERR_FP8_SCALE);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (warp == 0) {
            int stage = 0;
            uint32_t phase = 0, issued = 0, issued_parity = 0;
            bool stop = false;
            while (const Work* w = next()) {
                const int patch = w->tile / n_tiles, col0 = (w->tile - patch * n_tiles) * BN;
                for (int i = 0; i < w->count && !stop; ++i) {
                    const int row = w->row[i], e = w->expert[i];
                    for (int kb = 0; kb < p.Kb; ++kb) {
                        if (!mbar_wait_warp_quick(&ctl->empty[stage], phase ^ 1, abort_flag, p.status)) { stop = true; break; }
                        if (lane == 0) {
                            uint8_t* st = smem + stage * STAGE;
                            mbar_arrive_expect_tx(&ctl->full[stage], STAGE);
                            tma_load_2d(st, &tmA, kb * kQ, row, &ctl->full[stage]);
                            tma_load_3d(st + A_BYTES, &tmB, kb * kQ, col0, e, &ctl->full[stage]);
                        }
                        __syncwarp();
                        issued |= 1u << stage;
                        issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
                        if (++stage == STAGES) { stage = 0; phase ^= 1; }
                    }
                }
                if (stop) break;
                done();
            }
            if (lane == 0 && *abort_flag)                     // copies counted by this CTA's barriers land before it exits
                for (int s = 0; s < STAGES; ++s)
                    if (issued & (1u << s)) mbar_wait(&ctl->full[s], (issued_parity >> s) & 1, abort_flag, p.status);
        } else if (warp == 1) {
            const uint32_t el = elect_one();
            constexpr uint32_t idesc = instr_desc_mxe4m3(BM, BN);
            int stage = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool stop = false;
            while (const Work* w = next()) {
                const int count = w->count;
                done();
                for (int i = 0; i < count && !stop; ++i) {
                    if (!mbar_wait_warp_quick(&ctl->tempty, acc_phase ^ 1, abort_flag, p.status)) { stop = true; break; }
                    acc_phase ^= 1;
                    tc_fence_after();
                    for (int kb = 0; kb < p.Kb; ++kb) {
                        if (!mbar_wait_warp_quick(&ctl->full[stage], phase, abort_flag, p.status)) { stop = true; break; }
                        tc_fence_after();
                        const uint32_t st = smem_u32(smem + stage * STAGE), sf = tmem_base + SF_COL + stage * SF_STRIDE;
                        const uint32_t ss = smem_u32(s_sf + stage * SF_BYTES);
#pragma unroll
                        for (int q = 0; q < 3; ++q) scales_to_tmem(el, q == 0 ? sf : sf + SFB + 4 * (q - 1), smem_desc_rows16(ss + 512 * q));
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            mma_mxf8(el, tmem_base, smem_desc(st + ks * 32, 16, 1024), smem_desc(st + A_BYTES + ks * 32, 16, 1024), idesc, sf, sf + SFB,
                                     (kb | ks) != 0);
                        mma_commit(el, &ctl->empty[stage]);
                        if (++stage == STAGES) { stage = 0; phase ^= 1; }
                    }
                    if (!stop) mma_commit(el, &ctl->tfull);
                }
                if (stop) break;
            }
        } else if (warp == 2) {
            int tile = blockIdx.x;
            for (;;) {
                if (!mbar_wait_warp_quick(&ctl->sempty[slot], sphase ^ 1, abort_flag, p.status)) break;
                Work* w = &ctl->work[slot];
                int count = 0;
                if (tile < total) {
                    // a lane per slot: its first routed row, if it selected the patch, and the expert whose region holds it
                    const int at = tile / n_tiles * p.k + lane;
                    int r = lane < p.k ? p.inv_row[at] : -1;
                    if (r > p.rows - BM) r = -1;
                    int e = 0;
                    while (e + 1 < p.n && r >= ctl->offs[e + 1]) ++e;
                    const uint32_t who = __ballot_sync(0xffffffffu, r >= 0);
                    count = __popc(who);
                    if (r >= 0) {
                        const int i = __popc(who & ((1u << lane) - 1));
                        w->row[i] = r;
                        w->expert[i] = e;
                        w->gate[i] = p.use_gate ? p.inv_gate[at] : 1.f;
                    }
                }
                if (lane == 0) { w->tile = tile; w->count = count; }
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->sfull[slot]);
                if (tile >= total) break;
                if (++slot == kSlots) { slot = 0; sphase ^= 1; }
                if (lane == 0) {
                    tile = (int)gridDim.x + atomicAdd(p.sched, 1);
                    if (tile > total) tile = total;
                }
                tile = __shfl_sync(0xffffffffu, tile, 0);
            }
        }
    }
    if (warp >= 8 && lane == 0) bulk_wait_all();        // this warp's tensor stores are complete
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
    if (threadIdx.x == 0) {         // this CTA's last fetch lies before the barrier above: the last CTA to get here resets
        __threadfence();
        if (atomicAdd(p.sched + 1, 1) == (int)gridDim.x - 1) {
            p.sched[0] = 0;
            p.sched[1] = 0;
            __threadfence();
        }
    }
}

}  // namespace

// As many tiles as SMs, or more: with fewer, smaller tiles by expert and a combine keep more SMs busy (whole layer, us by patch / apart: d = 1024,
// d_e = 256, 32 tiles 31 / 26, 128 tiles 34.6 / 35.5, 256 tiles 45.4 / 45.9; d = d_e = 1024, 128 tiles 48 / 46, 256 tiles 76 / 75; d = 4096, d_e = 1024,
// 256 tiles 66 / 71, 2048 tiles 340 / 371).
bool fp8_patch_can(const Dims& D) {
    const long long tiles = (long long)D.B * D.m * ((D.d + BN - 1) / BN);
    return D.l_p == BM && D.k <= kMaxK && D.n <= kMaxExperts && tiles >= sm_count() && tiles < (1ll << 30) && (long long)D.B * D.L < (1ll << 31);
}

uoe_status launch_fp8_patch(const Dims& D, const void* a, const float* as, const void* W2, const float* w2_scale, const void* b2, const void* x, void* y,
                            const int* offsets, const PlanPtrs& P, bool use_gate, bool residual, int* status, cudaStream_t s) {
    static DeviceOnce once;
    const uoe_status st = smem_opt_in(once, fp8_patch_kernel, SMEM);
    if (st != UOE_OK) return st;
    const uint64_t Kp = (uint64_t)q_pad(D.d_e);
    CUtensorMap tmA, tmB, tmY;
    {
        const uint64_t dims[2] = {Kp, (uint64_t)D.Rmax}, str[1] = {Kp};
        const uint32_t box[2] = {kQ, BM};
        if (!make_tmap(&tmA, a, 2, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    }
    {
        const uint64_t dims[3] = {Kp, (uint64_t)D.d, (uint64_t)D.n}, str[2] = {Kp, Kp * D.d};
        const uint32_t box[3] = {kQ, BN, 1};
        if (!make_tmap(&tmB, W2, 3, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    }
    Fp8Gemm g{a, as, W2, w2_scale, nullptr, 1, (long long)D.B * D.L, D.d, D.d_e, false, y, true};
    const Fp8Args out = fp8_args(g, status);             // y's rows are multiples of 16 bytes
    if (!out.vec || !result_map(&tmY, g)) return UOE_ERR_CUDA;
    PatchArgs p = {};
    p.sa = as; p.sb = w2_scale; p.inv_row = P.inv_row; p.offsets = offsets; p.inv_gate = P.inv_gate;
    p.x = (const __nv_bfloat16*)x; p.b2 = (const __nv_bfloat16*)b2;
    p.rows = D.Rmax; p.patches = D.B * D.m; p.m = D.m; p.k = D.k; p.n = D.n; p.N = D.d; p.Nb = q_blocks(D.d); p.Kb = q_blocks(D.d_e); p.Lv = D.Lv;
    p.use_gate = use_gate; p.residual = residual; p.status = status; p.sched = status + kSchedWord;
    ProfScope ps("fp8_gemm2_combine", s);
    launch_k(fp8_patch_kernel, dim3((unsigned)sm_count()), dim3(THREADS), (size_t)SMEM, s, tmA, tmB, tmY, p, out);
    UOE_LAUNCHED();
    return UOE_OK;
}

}  // namespace uoe
