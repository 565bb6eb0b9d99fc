// uoe_fp8_quantize: float matrices to e4m3 with a scale per block (fp8.cuh), in the four layouts the products read, and the
// quantising gather of the routed rows (Eq. 18) in front of the 8-bit expert products.
//
// Bound by memory: every element is read once (16-byte loads, eight in flight per thread) and written once as a byte.
//   quantize_rows_kernel   a scale per row and 128 columns, storage as it is read.  A CTA takes 32 rows x 4 blocks of columns, so
//                          that the scales [block, row] leave in whole lines; a block is 16 lanes (bfloat16) or 32 (float32), its
//                          maximum a few shuffles.
//   quantize_tile_kernel   a CTA per 128 x 128 tile held in registers (a thread: 8 rows x 8 columns): a scale per tile, stored as
//                          it is or transposed, or a scale per column and 128 rows, transposed.  Transposed bytes pass through
//                          shared memory, eight rows of a column in one 8-byte store, swizzled so that neither side meets a bank
//                          twice.
//   transpose_kernel       uoe_fp8_transpose: bytes of a quantised operand whose contraction is not contiguous, a CTA per 128 x 128 tile, a
//                          thread 4 rows x 16 columns: 4 x 4 bytes turned in registers, words swizzled through shared memory (33920 x 4096 bytes: 50 us, 5.6 TB/s read and
//                          written).
#include "fp8.cuh"

namespace uoe {
namespace {

constexpr int kRowsPerCta = 32, kBlocksPerCta = 4;

// 16 bytes of a row from element c on, zeros behind C (whole: the row is a multiple of 16 bytes and so starts on a boundary)
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* row, int c, int C, bool whole) {
    constexpr int V = Vec16<T>::N;
    if (whole) return c < C ? ld_stream16(row + c) : make_uint4(0, 0, 0, 0);
    T t[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (c + i < C) t[i] = row[c + i];
        else memset(&t[i], 0, sizeof(T));
    }
    uint4 v;
    memcpy(&v, t, 16);
    return v;
}

template <typename T>
__global__ void __launch_bounds__(256)
quantize_rows_kernel(const T* __restrict__ x, uint8_t* __restrict__ q, float* __restrict__ scale, long long rows, int C, int Cb, int groups /* of kBlocksPerCta blocks */,
                     int splits, int whole, const SrcMap map, const int* __restrict__ offsets, int n, int beside_plan) {
    pdl_trigger();
    constexpr int V = Vec16<T>::N;                    // elements per 16 bytes
    constexpr int LPB = kQ / V;                       // lanes per block: 16 or 32
    constexpr int BPW = 32 / LPB;                     // blocks a warp loads at a time
    constexpr int ROUNDS = kBlocksPerCta / BPW;
    constexpr int RPW = kRowsPerCta / 8;              // rows per warp
    __shared__ float s_scale[2][kBlocksPerCta][kRowsPerCta];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long per_mat = ((rows + kRowsPerCta - 1) / kRowsPerCta) * splits;
    const long long mat = blockIdx.x / per_mat;
    const long long rest = blockIdx.x - mat * per_mat;
    const long long row0 = rest / splits * kRowsPerCta;
    if (!beside_plan) pdl_wait();
    // where the warp's rows come from: looked up once for all columns, a lane per row
    long long mine = row0 + warp * RPW + (lane % RPW) < rows ? mat * rows + row0 + warp * RPW + (lane % RPW) : -1;
    if (map.on()) {
        if (row0 >= offsets[n]) return;               // (regions are multiples of 128 rows: the CTA's rows are one expert's)
        int e = 0;
        while (e + 1 < n && row0 >= offsets[e + 1]) ++e;
        mine = source_row(map, (int)row0 + warp * RPW + (lane % RPW), e, offsets[e]);
    }
    long long src[RPW];
#pragma unroll
    for (int i = 0; i < RPW; ++i) src[i] = __shfl_sync(0xffffffffu, mine, i);
    const long long Cp = (long long)Cb * kQ;
    uint4 v[RPW][ROUNDS];
    auto load = [&](int group) {
#pragma unroll
        for (int i = 0; i < RPW; ++i)
#pragma unroll
            for (int u = 0; u < ROUNDS; ++u) {
                const int c = (group * kBlocksPerCta + u * BPW + lane / LPB) * kQ + (lane % LPB) * V;
                v[i][u] = src[i] >= 0 ? load_piece(x + src[i] * C, c, C, whole) : make_uint4(0, 0, 0, 0);
            }
    };
    int group = (int)(rest % splits), b = 0;
    load(group);
    for (; group < groups; group += splits, b ^= 1) {
        const int cb0 = group * kBlocksPerCta;
#pragma unroll
        for (int i = 0; i < RPW; ++i) {
            const long long r = row0 + warp * RPW + i;
#pragma unroll
            for (int u = 0; u < ROUNDS; ++u) {
                float f[V];
                unpack16<T>(v[i][u], f);
                uint32_t m = 0;
#pragma unroll
                for (int j = 0; j < V; ++j) m = max(m, abs_bits(f[j]));
#pragma unroll
                for (int o = LPB / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                const BlockScale k = block_scale(m);
                const int cb = cb0 + u * BPW + lane / LPB;
                if (lane % LPB == 0) s_scale[b][u * BPW + lane / LPB][warp * RPW + i] = k.s;
                if (r < rows && cb < Cb) {
                    uint8_t* o = q + (mat * rows + r) * Cp + cb * kQ + (lane % LPB) * V;
                    if constexpr (V == 8) *(uint2*)o = make_uint2(e4m3x4(f[0], f[1], f[2], f[3], k.inv), e4m3x4(f[4], f[5], f[6], f[7], k.inv));
                    else *(uint32_t*)o = e4m3x4(f[0], f[1], f[2], f[3], k.inv);
                }
            }
        }
        if (group + splits < groups) load(group + splits);
        __syncthreads();                              // (two buffers: the next group's scales wait for nobody)
        if (threadIdx.x < kBlocksPerCta * kRowsPerCta) {
            const int cb = cb0 + threadIdx.x / kRowsPerCta;
            const long long r = row0 + threadIdx.x % kRowsPerCta;
            if (cb < Cb && r < rows) scale[(mat * Cb + cb) * rows + r] = s_scale[b][threadIdx.x / kRowsPerCta][threadIdx.x % kRowsPerCta];
        }
    }
    if (beside_plan) pdl_wait();                      // this kernel is complete only when the plan is: the next one reads both
}

template <typename T, int LAYOUT>
__global__ void __launch_bounds__(256)
quantize_tile_kernel(const T* __restrict__ x, uint8_t* __restrict__ q, float* __restrict__ scale, int R, int C, int Rb, int Cb, int whole) {
    pdl_trigger();
    constexpr int V = Vec16<T>::N, PIECES = 8 / V;    // 16-byte loads for a thread's eight columns: 1 or 2
    __shared__ __align__(16) uint8_t s_t[LAYOUT == UOE_FP8_BLOCKS ? 16 : kQ * kQ];
    __shared__ uint32_t s_max[LAYOUT == UOE_FP8_COLS ? 16 * kQ : 8];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cg = tid & 15, rg = tid >> 4;           // this thread's 8 columns and 8 rows of the tile
    const long long per_mat = (long long)Rb * Cb;
    const long long mat = blockIdx.x / per_mat;
    const int rb = (int)((blockIdx.x - mat * per_mat) / Cb), cb = (int)((blockIdx.x - mat * per_mat) % Cb);
    const int r0 = rb * kQ + rg * 8, c0 = cb * kQ + cg * 8;
    x += mat * R * C;
    pdl_wait();
    uint4 v[8][PIECES];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int u = 0; u < PIECES; ++u)
            v[i][u] = r0 + i < R ? load_piece(x + (long long)(r0 + i) * C, c0 + u * V, C, whole) : make_uint4(0, 0, 0, 0);
    float f[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int u = 0; u < PIECES; ++u) unpack16<T>(v[i][u], f[i] + u * V);
    float inv[8];                                     // per column (LAYOUT_COLS) or all the same
    if constexpr (LAYOUT == UOE_FP8_COLS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, abs_bits(f[i][j]));
            s_max[rg * kQ + cg + 16 * j] = m;       // column cg * 8 + j kept at 16 j + cg: lanes side by side
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) m = max(m, s_max[i * kQ + cg + 16 * j]);
            const BlockScale b = block_scale(m);
            inv[j] = b.inv;
            if (rg == 0 && c0 + j < C) scale[(mat * Rb + rb) * C + c0 + j] = b.s;
        }
    } else {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, abs_bits(f[i][j]));
        m = __reduce_max_sync(0xffffffffu, m);
        if (lane == 0) s_max[warp] = m;
        __syncthreads();
        m = s_max[lane & 7];
        m = __reduce_max_sync(0xffffffffu, m);
        const BlockScale b = block_scale(m);
#pragma unroll
        for (int j = 0; j < 8; ++j) inv[j] = b.inv;
        if (tid == 0) scale[LAYOUT == UOE_FP8_BLOCKS ? (mat * Rb + rb) * Cb + cb : (mat * Cb + cb) * Rb + rb] = b.s;
    }
    if constexpr (LAYOUT == UOE_FP8_BLOCKS) {
        const long long Cp = (long long)Cb * kQ;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r0 + i < R)
                *(uint2*)(q + (mat * R + r0 + i) * Cp + c0) = make_uint2(e4m3x4(f[i][0], f[i][1], f[i][2], f[i][3], inv[0]),
                                                                        e4m3x4(f[i][4], f[i][5], f[i][6], f[i][7], inv[0]));
    } else {
        // row `col` of the transposed tile: 16 groups of 8 bytes, group rg at place rg ^ (col / 8)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            *(uint2*)(s_t + (cg * 8 + j) * kQ + ((rg ^ cg) << 3)) =
                make_uint2(e4m3x4(f[0][j], f[1][j], f[2][j], f[3][j], inv[j]), e4m3x4(f[4][j], f[5][j], f[6][j], f[7][j], inv[j]));
        __syncthreads();
        const long long Rp = (long long)Rb * kQ;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int col = p * 32 + (tid >> 3), t = tid & 7, c8 = col >> 3;      // 16 bytes: groups 2 t and 2 t + 1
            uint4 w = *(const uint4*)(s_t + col * kQ + ((((2 * t) ^ c8) & ~1) << 3));
            if (c8 & 1) w = make_uint4(w.z, w.w, w.x, w.y);
            if (cb * kQ + col < C) *(uint4*)(q + (mat * C + cb * kQ + col) * Rp + rb * kQ + t * 16) = w;
        }
    }
}

// q [C, R] = x [R, C] transposed, R a multiple of 128: the rows of q are whole 16-byte pieces, those of x where whole16 says so.
__global__ void __launch_bounds__(256)
transpose_kernel(const uint8_t* __restrict__ x, uint8_t* __restrict__ q, int R, int C, int Cb, int whole16) {
    pdl_trigger();
    __shared__ __align__(16) uint32_t s_t[kQ * 32];   // word (column, four rows g) at column * 32 + (g ^ 4 (column / 16)): no bank twice on either side
    const int tid = threadIdx.x, cg = tid & 7, rg = tid >> 3;
    const long long per_mat = (long long)(R / kQ) * Cb;
    const long long mat = blockIdx.x / per_mat;
    const int rb = (int)((blockIdx.x - mat * per_mat) / Cb), cb = (int)((blockIdx.x - mat * per_mat) % Cb);
    const int c0 = cb * kQ + cg * 16;
    x += (mat * R + rb * kQ + rg * 4) * C;
    pdl_wait();
    uint32_t v[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint8_t* row = x + (long long)i * C;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (whole16) {
            if (c0 < C) w = ld_stream16(row + c0);
        } else {
            uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c0 + j < C) b[j / 4] |= (uint32_t)row[c0 + j] << (8 * (j % 4));
            w = make_uint4(b[0], b[1], b[2], b[3]);
        }
        v[i][0] = w.x; v[i][1] = w.y; v[i][2] = w.z; v[i][3] = w.w;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {                      // columns 4 j .. 4 j + 3 of the thread's sixteen
        const uint32_t a = __byte_perm(v[0][j], v[1][j], 0x5140), b = __byte_perm(v[2][j], v[3][j], 0x5140);      // columns 0, 1 of rows 0, 1 / 2, 3
        const uint32_t c = __byte_perm(v[0][j], v[1][j], 0x7362), d = __byte_perm(v[2][j], v[3][j], 0x7362);      // columns 2, 3
        const uint32_t o[4] = {__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632), __byte_perm(c, d, 0x5410), __byte_perm(c, d, 0x7632)};
#pragma unroll
        for (int i = 0; i < 4; ++i) s_t[(cg * 16 + 4 * j + i) * 32 + (rg ^ (4 * cg))] = o[i];
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int col = p * 32 + (tid >> 3), t = tid & 7;
        const uint4 w = *(const uint4*)(s_t + col * 32 + 4 * (t ^ (col >> 4)));
        if (cb * kQ + col < C) *(uint4*)(q + (mat * C + cb * kQ + col) * R + rb * kQ + t * 16) = w;
    }
}

template <typename T>
uoe_status launch_tile(int layout, int G, int R, int C, const void* x, void* q, float* scale, cudaStream_t s) {
    const int Rb = q_blocks(R), Cb = q_blocks(C), whole = ((size_t)C * sizeof(T)) % 16 == 0;
    // (three factors, past 64 bits together: the first two are looked at alone)
    const long long tile_rows = (long long)G * Rb, tiles = tile_rows * Cb;
    if (tile_rows > 0x7fffffffll || tiles > 0x7fffffffll) return UOE_ERR_UNSUPPORTED;
    ProfScope ps("fp8_quantize", s);
    const dim3 grid((unsigned)tiles), block(256);
    if (layout == UOE_FP8_COLS) launch_k(quantize_tile_kernel<T, UOE_FP8_COLS>, grid, block, 0, s, (const T*)x, (uint8_t*)q, scale, R, C, Rb, Cb, whole);
    else if (layout == UOE_FP8_BLOCKS) launch_k(quantize_tile_kernel<T, UOE_FP8_BLOCKS>, grid, block, 0, s, (const T*)x, (uint8_t*)q, scale, R, C, Rb, Cb, whole);
    else launch_k(quantize_tile_kernel<T, UOE_FP8_BLOCKS_T>, grid, block, 0, s, (const T*)x, (uint8_t*)q, scale, R, C, Rb, Cb, whole);
    UOE_LAUNCHED();
    return UOE_OK;
}

}  // namespace

uoe_status launch_quantize_rows(const void* x, bool bf16, int G, long long rows, int C, void* q, float* scale, const SrcMap& map,
                                const int* offsets, int n, const char* label, cudaStream_t s, bool beside_plan) {
    const int Cb = q_blocks(C), groups = (Cb + kBlocksPerCta - 1) / kBlocksPerCta, whole = ((size_t)C * (bf16 ? 2 : 4)) % 16 == 0;
    // CTAs of a row block: as many as keep some eight per SM; a row's columns are a loop otherwise
    const long long row_ctas = (long long)G * ((rows + kRowsPerCta - 1) / kRowsPerCta);
    if (row_ctas > 0x7fffffffll) return UOE_ERR_UNSUPPORTED;
    int splits = groups;
    while (splits > 1 && row_ctas * (splits / 2) >= 8ll * sm_count()) splits = (splits + 1) / 2;
    const long long ctas = row_ctas * splits;
    if (ctas > 0x7fffffffll) return UOE_ERR_UNSUPPORTED;
    ProfScope ps(label, s);
    if (bf16) launch_k(quantize_rows_kernel<__nv_bfloat16>, dim3((unsigned)ctas), dim3(256), 0, s, (const __nv_bfloat16*)x, (uint8_t*)q, scale, rows, C, Cb, groups, splits, whole, map, offsets, n, beside_plan ? 1 : 0);
    else launch_k(quantize_rows_kernel<float>, dim3((unsigned)ctas), dim3(256), 0, s, (const float*)x, (uint8_t*)q, scale, rows, C, Cb, groups, splits, whole, map, offsets, n, beside_plan ? 1 : 0);
    UOE_LAUNCHED();
    return UOE_OK;
}

}  // namespace uoe

using namespace uoe;

extern "C" uoe_status uoe_fp8_quantize(int32_t G, int32_t R, int32_t C, int32_t dtype, int32_t layout, const void* x, void* q, float* scale,
                                       void* cuda_stream) {
    if (G < 1 || R < 1 || C < 1 || (dtype != UOE_F32 && dtype != UOE_BF16)) return UOE_ERR_INVALID_ARG;
    if (layout < UOE_FP8_ROWS || layout > UOE_FP8_BLOCKS_T) return UOE_ERR_INVALID_ARG;
    if (!x || !q || !scale || !aligned16(x) || !aligned16(q) || !aligned16(scale)) return UOE_ERR_INVALID_ARG;
    if (R > 0x7fffffff - kQ || C > 0x7fffffff - kQ) return UOE_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (layout == UOE_FP8_ROWS) return launch_quantize_rows(x, dtype == UOE_BF16, G, R, C, q, scale, SrcMap(), nullptr, 0, "fp8_quantize", s);
    return dtype == UOE_BF16 ? launch_tile<__nv_bfloat16>(layout, G, R, C, x, q, scale, s) : launch_tile<float>(layout, G, R, C, x, q, scale, s);
}

extern "C" uoe_status uoe_fp8_transpose(int32_t G, int32_t R, int32_t C, const void* x, void* q, void* cuda_stream) {
    if (G < 1 || R < 1 || C < 1 || R % kQ != 0) return UOE_ERR_INVALID_ARG;
    if (!x || !q || x == q || !aligned16(x) || !aligned16(q)) return UOE_ERR_INVALID_ARG;
    if (C > 0x7fffffff - kQ) return UOE_ERR_UNSUPPORTED;
    const int Cb = q_blocks(C);
    const long long rows = (long long)G * (R / kQ);
    if (rows > 0x7fffffffll || rows * Cb > 0x7fffffffll) return UOE_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    ProfScope ps("fp8_transpose", s);
    launch_k(transpose_kernel, dim3((unsigned)(rows * Cb)), dim3(256), 0, s, (const uint8_t*)x, (uint8_t*)q, R, C, Cb, C % 16 == 0 ? 1 : 0);
    UOE_LAUNCHED();
    return UOE_OK;
}
