// What the kernels for products of 8-bit operands share: arguments, the experts' regions, what becomes of a tile's sums.
#pragma once
#include "fp8.cuh"
#include "tc.cuh"
#include "tmap.cuh"

namespace uoe {

constexpr int kMaxExperts = 32;

struct Fp8Args {
    const float *sa, *sb;
    const int* offsets;
    int n, N, Nb;                     // columns of C, blocks of 128 of them
    long long M;                      // rows of C (rows of the A operand)
    int Kb;                           // blocks of the contraction (wgrad: in all regions together)
    void* C;
    int out_bf16, vec;                // vec: rows of C may be stored in 32-byte pieces
    const __nv_bfloat16* bias;
    int act;
    uint8_t* q;
    float* qs;
    long long ldq;
    int split;                        // CTAs that share a tile's contraction
    long long x_rows;                 // gathered: rows of A
    int* status;
};

// First row (wgrad: position in the contraction) of every expert, and its first row tile.
struct Regions {
    int offs[kMaxExperts + 1];
    int tstart[kMaxExperts + 1];
};
// By one warp.  Without offsets all rows are one expert's; wgrad: every expert has all row tiles of C.  Offsets that are no regions
// (not ascending multiples of 128 within the operand) are reported, and there are no tiles.
template <bool WGRAD, int TILE>
__device__ __forceinline__ void load_regions(Regions& g, const Fp8Args& a, int m_tiles, int lane) {
    const int n = a.n;
    const long long limit = WGRAD ? (long long)a.Kb * kQ : a.M;
    int o = 0, o1 = 0;
    if (a.offsets) {
        o = lane < n ? a.offsets[lane] : 0;
        o1 = lane < n ? a.offsets[lane + 1] : 0;
    } else if (lane == 0) {
        o1 = WGRAD ? a.Kb * kQ : (int)((a.M + kQ - 1) / kQ * kQ);
    }
    const bool ok = lane >= n || !a.offsets || (o >= 0 && o1 >= o && o1 <= limit && ((o | o1) & (kQ - 1)) == 0);
    const bool bad = !__all_sync(0xffffffffu, ok);
    const int tiles = lane < n && !bad ? (WGRAD ? m_tiles : (o1 - o + TILE - 1) / TILE) : 0;
    int incl = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += v;
    }
    if (lane < n) {
        g.offs[lane] = o;
        g.offs[lane + 1] = o1;                 // (the neighbour writes the same number)
        g.tstart[lane] = incl - tiles;
        if (lane == n - 1) g.tstart[n] = incl;
    }
    if (lane == 0 && bad) set_status(a.status, UOE_ERR_DEVICE_INDEX);
}

// The scale's exponent byte in all four bytes of a word; 0xff, which stands for NaN, where it is no power of two (a scale that is NaN
// itself is no news).  Without a branch: a look at the status word per scale cost 1000 cycles per block.
__device__ __forceinline__ uint32_t exponent_word(float s, bool there, bool& bad) {
    const uint32_t b = there ? __float_as_uint(s) : 0x3f800000u, e = b >> 23;
    const bool pow2 = (b & 0x7fffffu) == 0 && e - 1 < 254u;
    bad |= !pow2 && (b & 0x7fffffffu) <= 0x7f800000u;           // an infinity is no power of two; NaN of either sign
    return __byte_perm(pow2 ? e : 255u, 0, 0);
}

// Shared memory of a write-out warp: 32 rows of 64 bytes (swizzled, for a tensor store), or of 16 columns and a gap.
constexpr int kTurnPitch = 17, kTurnBytes = 2560;
static_assert(kTurnBytes >= 32 * kTurnPitch * 4 && kTurnBytes % 512 == 0, "");
// C as [n][rows][N] in pieces of 32 rows x 64 bytes (rows of C are multiples of 16 bytes: Fp8Args::vec)
inline bool result_map(CUtensorMap* tm, const Fp8Gemm& g) {
    const uint64_t size = g.out_bf16 ? 2 : 4;
    const uint64_t dims[3] = {(uint64_t)g.N, (uint64_t)g.M, (uint64_t)(g.wgrad ? g.n : 1)}, str[2] = {(uint64_t)g.N * size, (uint64_t)g.N * g.M * size};
    const uint32_t box[3] = {(uint32_t)(64 / size), 32, 1};
    return make_tmap(tm, g.C, 3, dims, str, box, g.out_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, CU_TENSOR_MAP_SWIZZLE_64B);
}

// A warp's sums: CW of row `row0` + lane in every lane, columns col .. col + CW.  Rows from row_end and columns from N on are not stored.
template <int CW, bool WGRAD, int EPI>
__device__ __forceinline__ void store_tile(const Fp8Args& a, const CUtensorMap* tmC, float* sum, int e, long long row0, long long row_end, int col, float* turn) {
    const int lane = threadIdx.x & 31;
    const long long row = row0 + lane;
    if (col >= a.N) return;
    if (!WGRAD && a.bias) {
#pragma unroll
        for (int q = 0; q < CW; ++q)
            if (col + q < a.N) sum[q] += to_f32(a.bias[(size_t)e * a.N + col + q]);
    }
    if constexpr (EPI == kFp8ActQuant) {
        static_assert(EPI != kFp8ActQuant || (!WGRAD && CW == kQ), "a thread holds one block of the result");
        if (row >= row_end) return;
        uint32_t m = 0;
        act_fast_n<CW>(sum, a.act);
#pragma unroll
        for (int q = 0; q < CW; ++q) m = max(m, abs_bits(sum[q]));
        const BlockScale b = block_scale(m);
        a.qs[(size_t)(col / kQ) * a.M + row] = b.s;
        uint8_t* o = a.q + (size_t)row * a.ldq + col;
        const bool whole = sector_aligned(o);
#pragma unroll
        for (int q = 0; q < CW; q += 32) {
            uint32_t w[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) w[u] = e4m3x4(sum[q + 4 * u], sum[q + 4 * u + 1], sum[q + 4 * u + 2], sum[q + 4 * u + 3], b.inv);
            st_sector(o + q, make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7]), whole);
        }
    } else {
        if (a.vec) {
            // tensor stores of 32 rows x 64 bytes, which leave behind the arithmetic on the next piece (rows and columns past C are clipped;
            // a region is whole blocks of 32 rows).  A row per lane and 32 bytes of it per store: 32768 x 4096 x 1024 127 us
            if (row0 >= row_end) return;
            auto put = [&](const uint4* v, int c) {
                if (lane == 0) tc::bulk_wait_read();
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) *(uint4*)((uint8_t*)turn + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) = v[i];
                tc::fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    tc::tma_store_3d(tmC, turn, col + c, (int)row0, WGRAD ? e : 0);
                    tc::bulk_commit();
                }
            };
            if (!WGRAD && a.out_bf16) {
#pragma unroll
                for (int c = 0; c < CW; c += 32) {
                    if (col + c >= a.N) break;
                    const uint4 v[4] = {pack16<__nv_bfloat16>(sum + c), pack16<__nv_bfloat16>(sum + c + 8), pack16<__nv_bfloat16>(sum + c + 16),
                                        pack16<__nv_bfloat16>(sum + c + 24)};
                    put(v, c);
                }
            } else {
#pragma unroll
                for (int c = 0; c < CW; c += 16) {
                    if (col + c >= a.N) break;
                    const uint4 v[4] = {pack16<float>(sum + c), pack16<float>(sum + c + 4), pack16<float>(sum + c + 8), pack16<float>(sum + c + 12)};
                    put(v, c);
                }
            }
        } else {
            // rows that start anywhere: 16 columns of two rows per store (a row per lane, 4 bytes of 32 rows each: 1334 x 333 x 1000,
            // float32, 15 us)
#pragma unroll
            for (int c = 0; c < CW; c += 16) {
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 16; ++q) turn[lane * kTurnPitch + q] = sum[c + q];
                __syncwarp();
                const int cc = col + c + (lane & 15);
                if (cc >= a.N) continue;
#pragma unroll 4
                for (int i = 0; i < 16; ++i) {
                    const int r = 2 * i + (lane >> 4);
                    if (row0 + r >= row_end) break;
                    const float v = turn[r * kTurnPitch + (lane & 15)];
                    const size_t to = ((WGRAD ? (size_t)e * a.M : 0) + row0 + r) * a.N + cc;
                    if (!WGRAD && a.out_bf16) ((__nv_bfloat16*)a.C)[to] = __float2bfloat16_rn(v);
                    else ((float*)a.C)[to] = v;
                }
            }
            __syncwarp();
        }
    }
}

inline Fp8Args fp8_args(const Fp8Gemm& g, int* status) {
    const uint64_t Kp = (uint64_t)((g.K + kQ - 1) / kQ * kQ);
    Fp8Args a = {};
    a.sa = g.sa; a.sb = g.sb; a.offsets = g.offsets;
    a.n = g.n; a.N = g.N; a.Nb = q_blocks(g.N); a.M = g.M; a.Kb = (int)(Kp / kQ);
    a.C = g.C; a.out_bf16 = g.out_bf16;
    a.vec = ((size_t)g.N * (g.out_bf16 ? 2 : 4)) % 16 == 0 && aligned16(g.C);
    a.bias = (const __nv_bfloat16*)g.bias; a.act = g.act;
    a.q = (uint8_t*)g.q; a.qs = g.qs; a.ldq = q_pad(g.N);
    a.status = status;
    return a;
}

// Factors of any size: blocks' products added outside the tensor cores (fp8_gemm_any_tcgen05.cu).
uoe_status launch_fp8_gemm_any(const Fp8Gemm& g, int* status, cudaStream_t s);

// Up to 64 rows of one matrix, scales of any size: split along the contraction (fp8_skinny_tcgen05.cu).
bool fp8_is_skinny(const Fp8Gemm& g);
uoe_status launch_fp8_skinny(const Fp8Gemm& g, int* status, cudaStream_t s);

}  // namespace uoe
