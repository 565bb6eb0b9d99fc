// Products of 8-bit operands whose scales are powers of two (fp8.cuh) on the tcgen05 tensor cores, grouped by expert:
//
//   rows    C[r, j]    = sum_kb sa[kb, r] sb[e(r), j / 128, kb]  sum_{k in block kb} A[r, k] B[e(r), j, k]
//   wgrad   C[e, i, j] = sum_kb sa[kb, i] sb[kb, j]              sum_{r in block kb} A[i, r] B[j, r],   kb over expert e's region
//
// The block-scaled MMA takes an exponent byte per row of A and of B, so the sum over all blocks stays in one float32 TMEM
// accumulator and nothing has to be added outside (any other scale: fp8_gemm_any_tcgen05.cu, where that addition is what bounds the
// kernel).  A persistent CTA (pair) per SM (two) walks the tiles, 128 x BN or, by a pair of CTAs (cta_group::2), 256 x 256:
//   warp 0       TMA producer: a stage is one block of the contraction, 128 bytes of every row of A and of B (128-byte swizzle)
//   warp 1       MMA issuer: four steps of 32 per stage
//   warps 4..7   the stages' scales in turn: float32 -> exponent byte -> shared memory, in the order in which the issuer's copies put
//                them into TMEM.  A scale holds for the whole stage, so its byte fills the word and the four steps need no index.
//   warps 8..15  write-out: a warp has 32 rows (its TMEM lane quarter) and half of the columns, all of them in registers before it
//                gives the accumulator back (256 columns and the scales leave room for one accumulator: the next tile's products
//                wait for these loads, not for the arithmetic and the stores)
// The routed rows of A may be gathered (Eq. 18 inside the loads): A holds every token once, quantised, and a tile's rows come in one copy per
// source patch, their scales by their source rows.
// Regions of experts are whole 128-row blocks; the second half of a pair's last tile may be rows of nobody, which are not stored.
#include "fp8_tile.cuh"
#include "tc.cuh"
#include "tmap.cuh"

#include <type_traits>

namespace uoe {
namespace {

using namespace tc;

constexpr int BM = 128;
constexpr int kSplitPitch = 132;          // floats of a row of a split tile's sums (where the stages were)

template <int BN, bool PAIR> struct Cfg {
    static_assert(!PAIR || BN == 256, "a pair works 256 x 256");
    static constexpr int BN_CTA = PAIR ? BN / 2 : BN;                 // rows of B this CTA loads
    static constexpr int TILE = PAIR ? 2 * BM : BM;
    static constexpr int A_BYTES = BM * kQ, B_BYTES = BN_CTA * kQ, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = BN_CTA == 256 ? 4 : 6;
    static_assert(STAGES >= 4, "four warps in turn: none looks for a stage's last use by parity two uses ahead");
    static constexpr int NACC = BN == 256 ? 1 : 2;
    static constexpr int CW = BN / 2;
    static constexpr int EPI_WARPS = 8, THREADS = 128 + 128 + 32 * EPI_WARPS;
    static constexpr int TMEM_COLS = 512, SF_COL = 256, SF_STRIDE = 16, SFB = 8;      // scales of stage s: A at SF_COL + 16 s, B 8 behind
    static constexpr int SF_BYTES = 512 + 4 * BN;                     // a stage's scale words: A's 128 rows, then B's BN
    static constexpr int SMEM = STAGES * (STAGE + SF_BYTES) + 1024 /* alignment */ + 1024 /* control */ + EPI_WARPS * kTurnBytes;
};

struct Ctl {
    uint64_t full[8], empty[8], tfull[2], tempty[2];
    uint32_t tmem_base;
    int abort_flag;
    Regions reg;
};
static_assert(sizeof(Ctl) <= 1024, "control block");

struct NoMap {};                          // what a kernel without gathered rows takes in the map's place

template <int BN, bool WGRAD, int EPI, bool PAIR, bool SPLIT, bool GATHER>
__global__ void __launch_bounds__(Cfg<BN, PAIR>::THREADS, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmC,
                const __grid_constant__ Fp8Args a, const typename std::conditional<GATHER, SrcMap, NoMap>::type map) {
    using Cf = Cfg<BN, PAIR>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Ctl* ctl = (Ctl*)(smem + Cf::STAGES * Cf::STAGE);
    volatile int* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    static_assert(!SPLIT || (BN == 128 && !PAIR && EPI == kFp8Store), "a split tile is 128 x 128");
    const int rank = PAIR ? (int)cluster_ctarank() : 0;
    const int share = SPLIT ? (int)cluster_ctarank() : 0, shares = SPLIT ? a.split : 1;      // of a tile's contraction
    const int worker = PAIR ? blockIdx.x >> 1 : SPLIT ? blockIdx.x / shares : blockIdx.x;
    const int workers = PAIR ? gridDim.x >> 1 : SPLIT ? gridDim.x / shares : gridDim.x;
    const int n = a.n;
    constexpr int CTAS = PAIR ? 2 : 1;
    if (threadIdx.x == 0) {
        // (a pair's products are issued by rank 0, on whose barriers both CTAs' copies, scales and write-outs arrive)
        for (int s = 0; s < Cf::STAGES; ++s) { mbar_init(&ctl->full[s], 1 + CTAS); mbar_init(&ctl->empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&ctl->tfull[i], 1); mbar_init(&ctl->tempty[i], CTAS * Cf::EPI_WARPS); }
        ctl->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
    }
    pdl_wait();
    // (TMEM only when the grids before this one are complete, and the grid behind it only when it is taken: no CTA holds TMEM while it waits
    // for one that still needs some)
    if (warp == 1) {
        if constexpr (PAIR) tmem_alloc_pair(&ctl->tmem_base, Cf::TMEM_COLS);
        else tmem_alloc(&ctl->tmem_base, Cf::TMEM_COLS);
    }
    const int m_tiles = (int)((a.M + Cf::TILE - 1) / Cf::TILE);
    if (warp == 2) load_regions<WGRAD, Cf::TILE>(ctl->reg, a, m_tiles, lane);
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();           // the other CTA's barriers exist before anything arrives on them
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem_base = ctl->tmem_base;
    uint8_t* s_sf = (uint8_t*)ctl + 1024;
    const int n_tiles = (a.N + BN - 1) / BN;
    const int total = ctl->reg.tstart[n] * n_tiles;

    // tile -> expert, first row of A and C in this CTA and where the expert's rows end, first block of the contraction and their number
    struct Tile { int row0, row_end, col0, kb0, kbs; };
    auto locate = [&](int tile, int& e) {
        Tile t;
        const int rt = tile / n_tiles;
        while (e + 1 < n && rt >= ctl->reg.tstart[e + 1]) ++e;
        t.row0 = (rt - ctl->reg.tstart[e]) * Cf::TILE + rank * BM + (WGRAD ? 0 : ctl->reg.offs[e]);
        t.row_end = (int)(WGRAD || ctl->reg.offs[e + 1] > a.M ? a.M : ctl->reg.offs[e + 1]);
        t.col0 = (tile - rt * n_tiles) * BN;
        t.kb0 = WGRAD ? ctl->reg.offs[e] / kQ : 0;
        t.kbs = WGRAD ? (ctl->reg.offs[e + 1] - ctl->reg.offs[e]) / kQ : a.Kb;
        if constexpr (SPLIT) {
            const int lo = (int)((long long)t.kbs * share / shares), hi = (int)((long long)t.kbs * (share + 1) / shares);
            t.kb0 += lo;
            t.kbs = hi - lo;
        }
        return t;
    };

    // Registers: 512 threads start with 128 each (128 * 56 + 128 * 56 + 256 * 200 = 512 * 128).
    if (warp >= 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        constexpr int CW = Cf::CW;
        const int quarter = warp & 3, half = (warp - 8) >> 2;
        [[maybe_unused]] float* turn = (float*)(s_sf + Cf::STAGES * Cf::SF_BYTES + (warp - 8) * kTurnBytes);
        int acc = 0, e = 0;
        uint32_t acc_phase = 0;
        for (int tile = worker; tile < total; tile += workers) {
            const Tile t = locate(tile, e);
            float sum[CW];
            if (t.kbs > 0) {
                if (!mbar_wait_warp_quick(&ctl->tfull[acc], acc_phase, abort_flag, a.status)) break;
                tc_fence_after();
                const uint32_t taddr = tmem_base + acc * BN + half * CW + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
                for (int g = 0; g < CW / 32; ++g) tmem_ld32(taddr + g * 32, (uint32_t*)sum + g * 32);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) mbar_arrive_cluster_relaxed(map_to_cta(&ctl->tempty[acc], 0));
                    else mbar_arrive(&ctl->tempty[acc]);
                }
                if (++acc == Cf::NACC) { acc = 0; acc_phase ^= 1; }
            } else {
#pragma unroll
                for (int q = 0; q < CW; ++q) sum[q] = 0.f;
            }
            if constexpr (SPLIT) {                    // (its only tile: the stages have all been read)
                float* o = (float*)smem + (quarter * 32 + lane) * kSplitPitch + half * CW;
#pragma unroll
                for (int q = 0; q < CW; q += 4) *(float4*)(o + q) = make_float4(sum[q], sum[q + 1], sum[q + 2], sum[q + 3]);
            } else {
                store_tile<CW, WGRAD, EPI>(a, &tmC, sum, e, t.row0 + quarter * 32, t.row_end, t.col0 + half * CW, turn);
            }
            __syncwarp();
        }
    } else if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        constexpr int NB = WGRAD ? BN / 32 : (BN + kQ - 1) / kQ;      // scales of B per lane: its columns', or the column blocks'
        // The blocks of all this CTA's tiles are one sequence, and the four warps take turns: what a block costs is a chain (loads,
        // a wait for the stage, the release), four of which run at a time.
        int stage = 0, e = 0, turn = 0;
        uint32_t phase = 0;
        bool stop = false, bad = false;
        for (int tile = worker; tile < total && !stop; tile += workers) {
            const Tile t = locate(tile, e);
            const int rows = t.row_end - t.row0, cols = a.N - t.col0;
            const float* sa = GATHER ? a.sa : a.sa + (size_t)t.kb0 * a.M + t.row0;
            [[maybe_unused]] int from[4] = {0, 0, 0, 0};              // source row of this lane's rows, -1: none
            if constexpr (GATHER) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int r = t.row0 + q * 32 + lane, p = r < t.row_end ? src_of(map, r, e, ctl->reg.offs[e], -1) : -1;
                    from[q] = p >= 0 && p < map.B * map.m ? p * map.l_p + r % map.l_p : -1;       // (a table that a bad index left unwritten: no row)
                }
            }
            auto has = [&](int q) { return GATHER ? from[q] >= 0 : lane < rows - q * 32; };
            const float* sb = WGRAD ? a.sb + (size_t)t.kb0 * a.N + t.col0 : a.sb + ((size_t)e * a.Nb + t.col0 / kQ) * a.Kb + t.kb0;
            float ra[4], rb[NB];                                      // (whatever is there where there are no rows of this expert, or no columns)
            auto ask = [&](int kb) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (has(q)) ra[q] = __ldg(GATHER ? sa + (size_t)kb * a.x_rows + from[q] : sa + (size_t)kb * a.M + q * 32 + lane);
#pragma unroll
                for (int q = 0; q < NB; ++q) {
                    if constexpr (WGRAD) { if (lane < cols - q * 32) rb[q] = __ldg(sb + (size_t)kb * a.N + q * 32 + lane); }
                    else if (cols > q * kQ) rb[q] = __ldg(sb + (size_t)q * a.Kb + kb);
                }
            };
            const int first = ((warp & 3) - turn) & 3;                // this warp's first block of the tile
            if (first < t.kbs) ask(first);
            for (int kb = 0; kb < t.kbs; ++kb) {
                if (((kb - first) & 3) == 0) {
                    uint32_t wa[4], wn[NB], wb[8];
#pragma unroll
                    for (int q = 0; q < 4; ++q) wa[q] = exponent_word(ra[q], has(q), bad);
#pragma unroll
                    for (int q = 0; q < NB; ++q) wn[q] = exponent_word(rb[q], WGRAD ? lane < cols - q * 32 : cols > q * kQ, bad);
#pragma unroll
                    for (int q = 0; q < 8; ++q) wb[q] = wn[WGRAD ? q % NB : (q / 4) % NB];
                    if (kb + 4 < t.kbs) ask(kb + 4);
                    if (!mbar_wait_warp_quick(&ctl->empty[stage], phase ^ 1, abort_flag, a.status)) { stop = true; break; }
                    uint8_t* sf = s_sf + stage * Cf::SF_BYTES + lane * 16;
                    *(uint4*)sf = make_uint4(wa[0], wa[1], wa[2], wa[3]);
                    *(uint4*)(sf + 512) = make_uint4(wb[0], wb[1], wb[2], wb[3]);
                    if constexpr (BN == 256) *(uint4*)(sf + 1024) = make_uint4(wb[4], wb[5], wb[6], wb[7]);
                    // (every lane's words are in place for the copy, which reads this SM's shared memory, once its fence is behind it)
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if (PAIR && rank) {                  // to the other CTA's issuer
                            fence_release_smem();
                            mbar_arrive_cluster_relaxed(map_to_cta(&ctl->full[stage], 0));
                        } else {
                            mbar_arrive(&ctl->full[stage]);
                        }
                    }
                }
                if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
            }
            turn += t.kbs;
        }
        if (bad) set_status(a.status, UOE_ERR_FP8_SCALE);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 0) {
            int stage = 0, e = 0;
            uint32_t phase = 0, issued = 0, issued_parity = 0;
            bool stop = false;
            for (int tile = worker; tile < total && !stop; tile += workers) {
                const Tile t = locate(tile, e);
                [[maybe_unused]] int boxes = 0, src = 0;      // source patches of the CTA's 128 rows; this lane's one
                if constexpr (GATHER) {
                    boxes = BM / map.l_p;
                    const int r = t.row0 + lane * map.l_p;
                    src = lane < boxes && r < t.row_end ? src_of(map, r, e, ctl->reg.offs[e], map.B * map.m) : map.B * map.m;    // (past the last patch: zeros)
                }
                for (int kb = 0; kb < t.kbs; ++kb) {
                    if (!mbar_wait_warp_quick(&ctl->empty[stage], phase ^ 1, abort_flag, a.status)) { stop = true; break; }
                    if constexpr (GATHER) {                   // a copy per source patch, each by a lane of its own
                        uint8_t* st = smem + stage * Cf::STAGE;
                        const int k = (t.kb0 + kb) * kQ;
                        if (lane == 0 && rank == 0) mbar_arrive_expect_tx(&ctl->full[stage], CTAS * Cf::STAGE);
                        __syncwarp();
                        if constexpr (PAIR) {
                            const uint32_t full0 = map_to_cta(&ctl->full[stage], 0);
                            if (lane < boxes) tma_load_3d_pair(st + lane * map.l_p * kQ, &tmA, k, 0, src, full0);
                            if (lane == 0) tma_load_3d_pair(st + Cf::A_BYTES, &tmB, k, t.col0 + rank * Cf::BN_CTA, e, full0);
                        } else {
                            if (lane < boxes) tma_load_3d(st + lane * map.l_p * kQ, &tmA, k, 0, src, &ctl->full[stage]);
                            if (lane == 0) tma_load_3d(st + Cf::A_BYTES, &tmB, k, t.col0, e, &ctl->full[stage]);
                        }
                    } else if (lane == 0) {
                        uint8_t* st = smem + stage * Cf::STAGE;
                        const int k = (t.kb0 + kb) * kQ, row = min(t.row0, (int)a.M);        // (a block behind the rows: all zeros)
                        if (rank == 0) mbar_arrive_expect_tx(&ctl->full[stage], CTAS * Cf::STAGE);
                        if constexpr (PAIR) {
                            const uint32_t full0 = map_to_cta(&ctl->full[stage], 0);
                            tma_load_2d_pair(st, &tmA, k, row, full0);
                            tma_load_3d_pair(st + Cf::A_BYTES, &tmB, k, t.col0 + rank * Cf::BN_CTA, WGRAD ? 0 : e, full0);
                        } else {
                            tma_load_2d(st, &tmA, k, row, &ctl->full[stage]);
                            tma_load_3d(st + Cf::A_BYTES, &tmB, k, t.col0, WGRAD ? 0 : e, &ctl->full[stage]);
                        }
                    }
                    __syncwarp();
                    issued |= 1u << stage;
                    issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
                    if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
                }
            }
            if (lane == 0 && rank == 0 && *abort_flag)        // copies counted by this CTA's barriers land before it exits
                for (int s = 0; s < Cf::STAGES; ++s)
                    if (issued & (1u << s)) mbar_wait(&ctl->full[s], (issued_parity >> s) & 1, abort_flag, a.status);
        } else if (warp == 1 && rank == 0) {
            const uint32_t el = elect_one();
            constexpr uint32_t idesc = instr_desc_mxe4m3(PAIR ? 2 * BM : BM, BN);
            int stage = 0, acc = 0, e = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool stop = false;
            for (int tile = worker; tile < total && !stop; tile += workers) {
                const Tile t = locate(tile, e);
                if (t.kbs == 0) continue;
                if (!mbar_wait_warp_quick(&ctl->tempty[acc], acc_phase ^ 1, abort_flag, a.status)) break;
                tc_fence_after();
                for (int kb = 0; kb < t.kbs; ++kb) {
                    if (!(PAIR ? mbar_wait_warp_cluster(&ctl->full[stage], phase, abort_flag, a.status)
                               : mbar_wait_warp_quick(&ctl->full[stage], phase, abort_flag, a.status))) { stop = true; break; }
                    tc_fence_after();
                    const uint32_t st = smem_u32(smem + stage * Cf::STAGE), sf = tmem_base + Cf::SF_COL + stage * Cf::SF_STRIDE;
                    const uint32_t ss = smem_u32(s_sf + stage * Cf::SF_BYTES);
#pragma unroll
                    for (int q = 0; q < 1 + BN / 128; ++q) {
                        const uint32_t to = q == 0 ? sf : sf + Cf::SFB + 4 * (q - 1);
                        if constexpr (PAIR) scales_to_tmem_pair(el, to, smem_desc_rows16(ss + 512 * q));
                        else scales_to_tmem(el, to, smem_desc_rows16(ss + 512 * q));
                    }
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {
                        const uint64_t ad = smem_desc(st + ks * 32, 16, 1024), bd = smem_desc(st + Cf::A_BYTES + ks * 32, 16, 1024);
                        if constexpr (PAIR) mma_mxf8_pair(el, tmem_base + acc * BN, ad, bd, idesc, sf, sf + Cf::SFB, (kb | ks) != 0);
                        else mma_mxf8(el, tmem_base + acc * BN, ad, bd, idesc, sf, sf + Cf::SFB, (kb | ks) != 0);
                    }
                    if constexpr (PAIR) mma_commit_pair(el, &ctl->empty[stage]);
                    else mma_commit(el, &ctl->empty[stage]);
                    if (++stage == Cf::STAGES) { stage = 0; phase ^= 1; }
                }
                if (stop) break;
                if constexpr (PAIR) mma_commit_pair(el, &ctl->tfull[acc]);
                else mma_commit(el, &ctl->tfull[acc]);
                if (++acc == Cf::NACC) { acc = 0; acc_phase ^= 1; }
            }
        }
    }
    if (warp >= 8 && lane == 0) bulk_wait_all();        // this warp's tensor stores are complete
    tc_fence_before();
    __syncthreads();
    if constexpr (SPLIT) {                            // the shares' sums, in order; a CTA stores its part of the rows
        cluster_sync_all();
        if (worker < total) {
            int e = 0;
            const Tile t = locate(worker, e);
            for (int r = BM * share / shares + warp; r < BM * (share + 1) / shares; r += Cf::THREADS / 32) {
                const long long row = t.row0 + r;
                if (row >= t.row_end) break;
#pragma unroll
                for (int c = lane; c < BN; c += 32) {
                    if (t.col0 + c >= a.N) break;
                    float v = a.bias ? to_f32(a.bias[(size_t)e * a.N + t.col0 + c]) : 0.f;
                    for (int q = 0; q < shares; ++q) v += ld_cluster_f32((const float*)smem + r * kSplitPitch + c, q);
                    const size_t at = ((WGRAD ? (size_t)e * a.M : 0) + row) * a.N + t.col0 + c;
                    if (!WGRAD && a.out_bf16) ((__nv_bfloat16*)a.C)[at] = __float2bfloat16_rn(v);
                    else ((float*)a.C)[at] = v;
                }
            }
        }
        cluster_sync_all();                           // nobody's shared memory goes while another CTA may read it
    }
    if constexpr (PAIR) cluster_sync_all();           // neither CTA leaves while the other may still arrive on its barriers or read its tiles
    if (warp == 1) {
        __syncwarp();
        if constexpr (PAIR) tmem_dealloc_pair(tmem_base, Cf::TMEM_COLS);
        else tmem_dealloc(tmem_base, Cf::TMEM_COLS);
    }
}

template <int BN, bool WGRAD, int EPI, bool PAIR, bool SPLIT = false, bool GATHER = false>
uoe_status launch_one(const Fp8Gemm& g, int* status, cudaStream_t s, int split = 1) {
    using Cf = Cfg<BN, PAIR>;
    static DeviceOnce once;
    static DeviceValue pairs_cache;
    auto kern = fp8_gemm_kernel<BN, WGRAD, EPI, PAIR, SPLIT, GATHER>;
    const uoe_status st = smem_opt_in(once, kern, Cf::SMEM);
    if (st != UOE_OK) return st;
    const uint64_t Kp = (uint64_t)((g.K + kQ - 1) / kQ * kQ);
    CUtensorMap tmA, tmB;
    if constexpr (GATHER) {       // the source rows as [patches][l_p][Kp]
        const uint64_t dims[3] = {Kp, (uint64_t)g.map.l_p, (uint64_t)g.map.B * g.map.m}, str[2] = {Kp, Kp * g.map.l_p};
        const uint32_t box[3] = {kQ, (uint32_t)g.map.l_p, 1};
        if (!make_tmap(&tmA, g.A, 3, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    } else {
        const uint64_t dims[2] = {Kp, (uint64_t)g.M};
        const uint64_t str[1] = {Kp};
        const uint32_t box[2] = {kQ, BM};
        if (!make_tmap(&tmA, g.A, 2, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    }
    {
        const uint64_t dims[3] = {Kp, (uint64_t)g.N, (uint64_t)(g.wgrad ? 1 : g.n)};
        const uint64_t str[2] = {Kp, Kp * (uint64_t)g.N};
        const uint32_t box[3] = {kQ, Cf::BN_CTA, 1};
        if (!make_tmap(&tmB, g.B, 3, dims, str, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return UOE_ERR_CUDA;
    }
    Fp8Args a = fp8_args(g, status);
    a.split = split;
    a.x_rows = (long long)g.map.B * g.map.m * g.map.l_p;
    typename std::conditional<GATHER, SrcMap, NoMap>::type map;
    if constexpr (GATHER) map = g.map;
    CUtensorMap tmC = tmA;
    if (g.epi == kFp8Store && a.vec && !result_map(&tmC, g)) return UOE_ERR_CUDA;
    const long long tiles = ((g.M + Cf::TILE - 1) / Cf::TILE + (PAIR && !g.wgrad ? g.n : 0)) * ((g.N + BN - 1) / BN) * (g.wgrad ? g.n : 1);
    if (tiles > 0x3fffffffll) return UOE_ERR_UNSUPPORTED;
    ProfScope ps(g.label, s);
    if constexpr (PAIR) {
        const int dev = current_device();
        if (dev < 0) return UOE_ERR_CUDA;
        if (!pairs_cache.has(dev)) {
            int v = 0;
            UOE_CUDA_OK(max_resident_pairs(kern, Cf::THREADS, Cf::SMEM, &v));
            if (v < 1) return UOE_ERR_CUDA;
            pairs_cache.set(dev, v);
        }
        const long long pairs = pairs_cache.get(dev);
        launch_k_pairs(kern, dim3(2 * (unsigned)(tiles < pairs ? tiles : pairs)), dim3(Cf::THREADS), (size_t)Cf::SMEM, s, tmA, tmB, tmC, a, map);
    } else if constexpr (SPLIT) {
        launch_k_cluster(kern, dim3((unsigned)tiles * split), dim3(Cf::THREADS), split, (size_t)Cf::SMEM, s, tmA, tmB, tmC, a, map);
    } else {
        launch_k(kern, dim3((unsigned)(tiles < sm_count() ? tiles : sm_count())), dim3(Cf::THREADS), (size_t)Cf::SMEM, s, tmA, tmB, tmC, a, map);
    }
    UOE_LAUNCHED();
    return UOE_OK;
}

template <bool WGRAD, int EPI>
uoe_status dispatch(const Fp8Gemm& g, int* status, cudaStream_t s) {
    const long long cols256 = (g.N + 255) / 256, mats = g.wgrad ? g.n : 1;
    const bool pairs = g.N > 128 && (g.M + 255) / 256 * cols256 * mats >= sm_count();
    if constexpr (EPI == kFp8ActQuant) {
        if (g.map.on()) return pairs ? launch_one<256, WGRAD, EPI, true, false, true>(g, status, s) : launch_one<256, WGRAD, EPI, false, false, true>(g, status, s);
    }
    if (pairs) return launch_one<256, WGRAD, EPI, true>(g, status, s);
    if (EPI == kFp8ActQuant || (g.N > 128 && (g.M + 127) / 128 * cols256 * mats >= sm_count())) return launch_one<256, WGRAD, EPI, false>(g, status, s);
    if constexpr (EPI != kFp8ActQuant) {
        // Tiles that leave SMs idle and have far to go: the contraction of a tile in up to eight parts, a CTA of a cluster each, from 24 blocks on
        // (a block is 0.3 us, the sums' meeting some 4; wgrad: an expert's rows are an even share, as far as the host knows).  wgrad 128 x 128 x
        // 30000 55.7 -> 13.5 us, 128 x 100 x 4096 15.1 -> 8.1, 300 x 1000 x 4096 12.8 -> 10.3; of 16 blocks, in two, 1000 x 500 x 2000 9.1 -> 11.4.
        const long long tiles = (g.M + 127) / 128 * ((g.N + 127) / 128) * mats, blocks = (g.K + kQ - 1) / kQ / mats;
        // (clusters of eight CTAs, one per SM, find room for two thirds of the SMs at once, of four for seven eighths)
        const int sms = sm_count();
        int split = 8;
        while (split > 1 && (tiles * split > (split == 8 ? sms * 2 / 3 : split == 4 ? sms * 7 / 8 : sms) || blocks < 24 || blocks < 4 * split)) split >>= 1;
        if (split > 1) return launch_one<128, WGRAD, EPI, false, true>(g, status, s, split);
        return launch_one<128, WGRAD, EPI, false>(g, status, s);
    }
    return UOE_ERR_UNSUPPORTED;
}

}  // namespace

uoe_status launch_fp8_gemm(const Fp8Gemm& g, int* status, cudaStream_t s) {
    if (g.n > kMaxExperts) return UOE_ERR_UNSUPPORTED;
    if (fp8_is_skinny(g)) return launch_fp8_skinny(g, status, s);
    if (g.map.on() && (g.any_scale || g.epi != kFp8ActQuant || !fp8_can_gather(g.map.l_p))) return UOE_ERR_UNSUPPORTED;
    if (g.any_scale) return launch_fp8_gemm_any(g, status, s);
    if (g.wgrad) return dispatch<true, kFp8Store>(g, status, s);
    return g.epi == kFp8ActQuant ? dispatch<false, kFp8ActQuant>(g, status, s) : dispatch<false, kFp8Store>(g, status, s);
}

}  // namespace uoe

using namespace uoe;

namespace {
uoe_status fp8_check(const uoe_fp8_problem* p, const void* A, const float* sa, const void* B, const float* sb, const int32_t* offsets, const void* C,
                     const void* ws, size_t ws_bytes) {
    if (!p || p->n < 1 || p->M < 1 || p->N < 1 || p->K < 1) return UOE_ERR_INVALID_ARG;
    if ((p->dtype != UOE_F32 && p->dtype != UOE_BF16) || (p->flags & ~UOE_FP8_ANY_SCALE)) return UOE_ERR_INVALID_ARG;
    if (!A || !sa || !B || !sb || !C || !ws) return UOE_ERR_INVALID_ARG;
    if (!aligned16(A) || !aligned16(sa) || !aligned16(B) || !aligned16(sb) || !aligned16(C) || !aligned16(ws)) return UOE_ERR_INVALID_ARG;
    if (!offsets && p->n > 1) return UOE_ERR_INVALID_ARG;
    if (p->n > kMaxExperts || p->M > (1 << 30) || p->N > (1 << 30) || p->K > (1 << 30)) return UOE_ERR_UNSUPPORTED;
    if (ws_bytes < uoe_fp8_workspace_bytes(p)) return UOE_ERR_WORKSPACE;
    return UOE_OK;
}
}  // namespace

extern "C" size_t uoe_fp8_workspace_bytes(const uoe_fp8_problem* p) {
    if (!p || p->n < 1 || p->M < 1 || p->N < 1 || p->K < 1) return 0;
    return kStatusBytes;
}

extern "C" uoe_status uoe_fp8_gemm(const uoe_fp8_problem* p, const void* A, const float* a_scale, const void* W, const float* w_scale,
                                   const int32_t* expert_offsets, void* C, void* ws, size_t ws_bytes, void* cuda_stream) {
    const uoe_status st = fp8_check(p, A, a_scale, W, w_scale, expert_offsets, C, ws, ws_bytes);
    if (st != UOE_OK) return st;
    Fp8Gemm g{A, a_scale, W, w_scale, expert_offsets, p->n, p->M, p->N, p->K, false, C, p->dtype == UOE_BF16};
    g.any_scale = p->flags & UOE_FP8_ANY_SCALE;
    return launch_fp8_gemm(g, (int*)ws, (cudaStream_t)cuda_stream);
}

extern "C" uoe_status uoe_fp8_wgrad(const uoe_fp8_problem* p, const void* A, const float* a_scale, const void* B, const float* b_scale,
                                    const int32_t* expert_offsets, float* dW, void* ws, size_t ws_bytes, void* cuda_stream) {
    const uoe_status st = fp8_check(p, A, a_scale, B, b_scale, expert_offsets, dW, ws, ws_bytes);
    if (st != UOE_OK) return st;
    if (p->dtype != UOE_F32) return UOE_ERR_UNSUPPORTED;
    Fp8Gemm g{A, a_scale, B, b_scale, expert_offsets, p->n, p->M, p->N, p->K, true, dW, false};
    g.any_scale = p->flags & UOE_FP8_ANY_SCALE;
    g.label = "fp8_wgrad";
    return launch_fp8_gemm(g, (int*)ws, (cudaStream_t)cuda_stream);
}
