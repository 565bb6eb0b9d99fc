// 8-bit operands: e4m3 values with a power-of-two scale for each block of 128 (one row) or 128 x 128 of a matrix.
//
// A quantised operand of `rows` rows and a contraction axis of K elements is stored as bytes [rows, Kp], Kp = K rounded up to 128,
// zeros behind K: the contraction axis is contiguous and whole blocks long, so every copy of it is aligned whatever K is, and a
// block is one 128-byte row of a swizzled shared-memory tile.  Scales: [Kp / 128, rows] where every row has its own (a warp
// whose lanes hold 32 rows reads one line), [rows / 128, Kp / 128] for square blocks.
#pragma once
#include <cuda_fp8.h>

#include "kernels.cuh"

namespace uoe {

constexpr int kQ = 128;                       // block length
inline __host__ __device__ int q_blocks(int v) { return (v + kQ - 1) / kQ; }
inline __host__ __device__ int q_pad(int v) { return q_blocks(v) * kQ; }

// Scale of a block from its largest magnitude (float bits without the sign: as integers NaN > infinity > finite, so a maximum
// taken on the bits keeps them): the smallest power of two s with amax <= 448 s, amax taken as at least 2^-100.  448 = 1.75 * 2^8, so
// with amax = f 2^E, 1 <= f < 2, the exponent of s is E - 8 where f <= 1.75 and E - 7 beyond.  x / s is then exact, and the one
// rounding of a value is that to e4m3 (half a step: 2^-4 of the value); a scale of 448 / amax itself, rounded, would break ties
// between e4m3 values at random, and bfloat16 inputs are full of ties.  A block that holds an infinity or NaN gets the scale NaN
// (every product with it is NaN) and zeros as values.
struct BlockScale { float s, inv; };
__device__ __forceinline__ BlockScale block_scale(uint32_t amax_bits) {
    const uint32_t b = max(amax_bits, 0x0d800000u);                     // 2^-100
    const uint32_t e = (b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    BlockScale r;
    r.s = __uint_as_float(e << 23);
    r.inv = __uint_as_float((254u - e) << 23);
    if (b >= 0x7f800000u) { r.s = __uint_as_float(0x7fc00000u); r.inv = 0.f; }
    return r;
}
__device__ __forceinline__ uint32_t abs_bits(float f) { return __float_as_uint(f) & 0x7fffffffu; }

// four values times `inv` as e4m3 bytes, the first in the lowest byte; zeros where the block holds no finite scale
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d, float inv) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a * inv, b * inv), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c * inv, d * inv), __NV_SATFINITE, __NV_E4M3);
    return inv == 0.f ? 0u : lo | (hi << 16);
}

// phi by the fast exponential and division, for results that are rounded to 8 or 16 bits: __expf is off by 2 + 1.17 |x| steps of float32, so
// SiLU is off by 1.2e-6 of its value up to |h| = 5, 3.3e-6 of it at -20 and 1.3e-5 at -88 (half a step of e4m3 is 2^-4, of bfloat16 2^-8: only values next to
// a border between two of them can fall on its other side).  With expf and a division: language-model layer 39-42 -> 47-50 us, scale
// layer 313-320 -> 325.
__device__ __forceinline__ float act_fast(float h, int act) {
    switch (act) {
        case UOE_ACT_SILU: return __fdividef(h, 1.0f + __expf(-h));
        case UOE_ACT_GELU_TANH: {
            const float u = 0.79788456080286536f * (h + 0.044715f * h * h * h);
            return __fdividef(h, 1.0f + __expf(-2.0f * u));             // h/2 (1 + tanh u)
        }
        default: return act_apply(h, act);
    }
}

// phi in float32
__device__ __forceinline__ float act_f32(float h, int act) {
    switch (act) {
        case UOE_ACT_SILU: return h / (1.0f + expf(-h));
        case UOE_ACT_GELU_TANH: {
            const float u = 0.79788456080286536f * (h + 0.044715f * h * h * h);
            return h / (1.0f + expf(-2.0f * u));                        // h/2 (1 + tanh u), without its cancellation
        }
        default: return act_apply(h, act);
    }
}

// act_fast for N values, chosen once.
template <int N>
__device__ __forceinline__ void act_fast_n(float* f, int act) {
    if (act == UOE_ACT_SILU) {
#pragma unroll
        for (int q = 0; q < N; ++q) f[q] = act_fast(f[q], UOE_ACT_SILU);
    } else if (act == UOE_ACT_GELU_TANH) {
#pragma unroll
        for (int q = 0; q < N; ++q) f[q] = act_fast(f[q], UOE_ACT_GELU_TANH);
    } else if (act == UOE_ACT_GELU_ERF) {
#pragma unroll
        for (int q = 0; q < N; ++q) f[q] = act_fast(f[q], UOE_ACT_GELU_ERF);
    }
}

// x [rows of C elements] -> q [rows, Cp], scale [Cp / 128, rows]: every row by itself.  With map.on() row r of the output is the
// token that routed row r holds (zeros on padding rows and unused slots), and only rows below offsets[n] are written.
uoe_status launch_quantize_rows(const void* x, bool bf16, int G, long long rows, int C, void* q, float* scale, const SrcMap& map,
                                const int* offsets, int n, const char* label, cudaStream_t s, bool beside_plan = false);

// What a tile of the product becomes.
enum Fp8Epilogue {
    kFp8Store = 0,       // rounded to bfloat16 or float32
    kFp8ActQuant = 1     // bias, activation, and quantised again (a scale per row and 128 columns): the operand of the next product
};
struct Fp8Gemm {
    const void* A; const float* sa;        // [M, Kp], [Kp / 128, M]
    const void* B; const float* sb;        // [n, N, Kp], [n, N / 128, Kp / 128]; wgrad: [N, Kp], [Kp / 128, N]
    const int* offsets;                    // [n+1] rows (wgrad: K positions) of every expert, or null (n = 1: all of them)
    int n; long long M; int N; long long K;
    bool wgrad;                            // contraction over the rows of an expert's region: C [n, M, N] float32
    void* C; bool out_bf16;                // [M, N]
    const void* bias = nullptr;            // [n, N] bfloat16 or null
    int act = UOE_ACT_IDENTITY;
    Fp8Epilogue epi = kFp8Store;
    void* q = nullptr; float* qs = nullptr;      // kFp8ActQuant: [M, Np], [Np / 128, M]
    bool any_scale = false;                // scales need not be powers of two
    SrcMap map;                            // kFp8ActQuant: if on, A and sa are those of the source rows [B m l_p]; row r of a region is gathered
    const char* label = "fp8_gemm";
};
// Patches that a tile's rows can be copied by: whole ones in 128 rows, whole 8-row groups of the swizzle.
inline bool fp8_can_gather(int l_p) { return l_p % 8 == 0 && 128 % l_p == 0; }
uoe_status launch_fp8_gemm(const Fp8Gemm& g, int* status, cudaStream_t s);

// Second layer and combine in one kernel, walked by output patch (fp8_patch_tcgen05.cu; scales are powers of two).
//   a [Rmax, d_e padded], as: the hidden rows, quantised by row; W2, w2_scale and b2 as for uoe_mlp_forward_fp8
bool fp8_patch_can(const Dims& D);
uoe_status launch_fp8_patch(const Dims& D, const void* a, const float* as, const void* W2, const float* w2_scale, const void* b2, const void* x, void* y,
                            const int* offsets, const PlanPtrs& P, bool use_gate, bool residual, int* status, cudaStream_t s);

}  // namespace uoe
