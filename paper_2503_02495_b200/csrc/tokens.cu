// uoe_mlp_tokens: router, experts and combine of a UoME layer for a few tokens (every row of x is a sample of one token: Eq. 21-22
// choose its experts, Eq. 38-40 follow) in two kernels.
//
// Bound by the weights of the chosen experts, each read once: one token per row tile of 128 would leave the tensor cores waiting for
// memory all the same, so the products run on mma.sync fragments that come straight from global memory, without a pass through
// shared memory.  Up to 32 tokens (one or two 16-row fragments) share a weight fragment.
//   first_layer_kernel   routes, then a = phi(x W1 + b1) for every (chosen expert, 64 hidden columns)
//   second_layer_kernel  y = x + sum over experts gate (a W2 + b2) for every 64 columns of y, the contraction running over all chosen
//                        experts' hidden columns in one line
// Both run in clusters of eight CTAs.  The first kernel's share the router's work, an eighth of d each, and every cluster routes for itself
// (a few KB from L2, instead of a third kernel).  S CTAs of a cluster share a tile's contraction, and their sums meet in distributed shared
// memory; S is the largest split that leaves no more than two CTAs per SM.
// Sums are added in an order that depends on sizes alone.
//
// Fragments (m16n8k16): the weights are the 16-row operand (two fragments of 8 columns), the tokens the 8-column one, so up to eight tokens cost
// one instruction per 16 columns and step.  A lane g * 4 + t holds k = 2t, 2t+1, 2t+8, 2t+9 of rows g and g + 8 of the one and of column g of
// the other; the order of k inside a step is free as long as both have the same one: those slots hold k = 4t .. 4t+3.
//   bfloat16 weights [K, N]   a lane loads 16 bytes, columns 8g .. 8g+7, of rows 4t .. 4t+3 (a warp: 16 whole 128-byte lines) and pairs the
//                             rows' halves: fragment j holds columns 8g + j
//   8-bit weights [N, Kp]     a lane loads 16 bytes of k, 16t .. 16t+15, of row 8j + g: four steps of fragment j.  As half they are
//                             exact (one instruction a pair; to bfloat16 it takes four); the activations become half by a power of two per
//                             token and 64 of the contraction, which with the block's scale multiplies the float32 sums of those 64
//   float32 weights [K, N]    float32 multiply-adds, eight tokens at a time
#include "fp8.cuh"
#include "tc.cuh"

namespace uoe {
namespace {

using namespace tc;

constexpr int kTok = 32;            // tokens of a group (a z slice of the grid)
constexpr int kMaxTokens = 64;
constexpr int kCols = 64;           // columns of a tile
constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kCluster = 8;         // CTAs; the router's sums have as many pieces
enum { kBf16 = 0, kFp8 = 1, kF32 = 2 };

struct TokArgs {
    const void *x, *Wr, *W1, *W2, *b1, *b2;
    const float *s1, *s2;
    struct Routed* routed;          // [groups]: what the first kernel's router says, for the second
    void *a, *y;                    // a [groups, n, kTok, d_e]: hidden rows by place in the group's list of chosen experts
    RoutingPtrs r;                  // all null, or all to be written
    int T, d, d_e, n, k, act, use_gate, residual;
};

template <int WT> struct Elem { using T = __nv_bfloat16; };
template <> struct Elem<kF32> { using T = float; };

struct Routed {                     // what the router says about a group's tokens
    uint32_t mask[kTok];            // chosen experts
    float p[kTok][32];              // sample gate (Eq. 21)
    uint32_t any;                   // experts that some token chose
};

__device__ __forceinline__ float ld_cluster(const float* p, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(map_to_cta(p, rank)) : "memory");
    return v;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

__device__ __forceinline__ void mma16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma16_half(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// four e4m3 bytes -> two half pairs, exact
__device__ __forceinline__ void halves_of_e4m3(uint32_t v, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(v));
}

// Sums over this CTA's piece of d: part[token * n + expert].
template <int WT, int MT>
__device__ void router_piece(const TokArgs& a, int t0, int Tn, int rank, float* red /* [8][Tn * n] */, float* part) {
    using T = typename Elem<WT>::T;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int d = a.d, n = a.n, len = ((d + kCluster - 1) / kCluster + 15) / 16 * 16;
    const T* x = (const T*)a.x + (size_t)t0 * d;
    const T* Wr = (const T*)a.Wr;
    const int k0 = rank * len, k1 = min(d, k0 + len);
    {
        if constexpr (WT == kF32) {
            // a warp per (token, expert)
            for (int q = warp; q < Tn * n; q += kWarps) {
                const int tok = q / n, i = q - tok * n;
                float s = 0.f;
                for (int kk = k0 + lane; kk < k1; kk += 32) s = fmaf(x[(size_t)tok * d + kk], Wr[(size_t)kk * n + i], s);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                if (lane == 0) part[q] = s;
            }
        } else {
            const int J = (n + 7) / 8;                 // fragment j: experts g * J + j
            float c[MT][4][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int u = 0; u < 4; ++u) c[m][j][u] = 0.f;
#pragma unroll 4
            for (int kk = k0 + warp * 16; kk < k1; kk += kWarps * 16) {
                const int kt = kk + 4 * t;
                uint32_t af[MT][4];
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint2 v = make_uint2(0, 0);
                        const int row = m * 16 + h * 8 + g;
                        if (row < Tn && kt < k1) v = *(const uint2*)(x + (size_t)row * d + kt);
                        af[m][h] = v.x; af[m][2 + h] = v.y;
                    }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j >= J) break;
                    const int i = g * J + j;
                    uint32_t w[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) w[r] = i < n && kt < k1 ? *(const uint16_t*)(Wr + (size_t)(kt + r) * n + i) : 0u;
#pragma unroll
                    for (int m = 0; m < MT; ++m) mma16(c[m][j], af[m], w[0] | (w[1] << 16), w[2] | (w[3] << 16));
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int row = m * 16 + (u >> 1) * 8 + g, i = (2 * t + (u & 1)) * J + j;
                        if (j < J && row < Tn && i < n) red[warp * Tn * n + row * n + i] = c[m][j][u];
                    }
            __syncthreads();
            for (int q = threadIdx.x; q < Tn * n; q += kThreads) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) s += red[w * Tn * n + q];
                part[q] = s;
            }
        }
    }
}

// Eq. 21-22 for the group's tokens, the same in every CTA.
template <int WT, int MT>
__device__ void route_tokens(const TokArgs& a, int t0, int Tn, int rank, float* red, float* part, Routed& R) {
    router_piece<WT, MT>(a, t0, Tn, rank, red, part);
    if (threadIdx.x == 0) R.any = 0;
    cluster_sync_all();                                // every CTA's piece is there
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = a.n;
    uint32_t any = 0;
    for (int tok = warp; tok < Tn; tok += kWarps) {
        float v = -INFINITY;
        if (lane < n) {
            v = 0.f;
#pragma unroll
            for (int p = 0; p < kCluster; ++p) v += ld_cluster(part + tok * n + lane, p);
        }
        float mx = v;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float e = lane < n ? expf(v - mx) : 0.f;
        float sum = e;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float ps = (lane < n ? e : 1.f) / sum;
        // (a token that holds a NaN has no order: it gets the first k experts, as many as every other)
        const float key = ps == ps ? ps : -1.f;
        int rank_i = 0;
        for (int i = 0; i < n; ++i) {
            const float w = __shfl_sync(0xffffffffu, key, i);
            rank_i += (w > key) || (w == key && i < lane);
        }
        const uint32_t m = __ballot_sync(0xffffffffu, lane < n && rank_i < a.k);
        R.p[tok][lane] = lane < n ? ps : 0.f;
        if (lane == 0) R.mask[tok] = m;
        any |= m;
    }
    if (lane == 0 && any) atomicOr(&R.any, any);
    cluster_arrive();                                  // done with the others' pieces (cluster_wait follows before the next meeting)
    __syncthreads();
}

__device__ __forceinline__ int nth_bit(uint32_t m, int i) {
    for (; i > 0; --i) m &= m - 1;
    return __ffs(m) - 1;
}

// How the CTA's eight warps divide a tile.  Up to eight tokens: 64 columns, every warp by itself on an eighth of the contraction, its
// activations straight from L2.  More tokens: 256 columns, four warps side by side times two halves of every 128 of the contraction,
// which the CTA first brings into shared memory (as half, or as they are): that work is shared by four warps.  float32: 64 columns, 16
// of every 128 of the contraction per warp, activations in shared memory as well.
template <int WT, int G> struct Shape {
    static constexpr bool STAGED = WT == kF32 || G > 1;
    static constexpr int COLS = STAGED && WT != kF32 ? 256 : 64;
    static constexpr int PARTS = kWarps * kCols / COLS;        // of the contraction, whose sums are added at the end
    static constexpr int UNIT = STAGED ? 128 : WT == kFp8 ? 64 : 16;                      // of the contraction, in which it is cut
    static constexpr int PITCH = WT == kFp8 ? 272 : WT == kBf16 ? 288 : 32 * G;           // bytes of a staged token (float32: of one k of all)
    static constexpr int STAGE = WT == kF32 ? 128 * PITCH : 8 * G * PITCH;
    static constexpr int BACK = WT == kFp8 ? 2 * 8 * G * 4 : 0;                           // factors of the two halves behind it
    static constexpr int CTAS = G == 1 && WT != kF32 ? 2 : 1;                             // per SM
};

// A token's values as half: times a power of two that brings the largest of a 64 to [2^14, 2^15), exact but for what lies 2^-29 below it (an
// error of 2^-40 of the largest, where the float32 sums have 2^-24); the power goes back in with the block's scale.  v: 16 values of
// bfloat16 in each of the four neighbouring lanes that hold the 64; returns the power.
__device__ __forceinline__ float to_half64(uint32_t* v) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = __vmaxu2(top, v[i] & 0x7fff7fffu);
    top = max(top >> 16, top & 0xffffu) << 16;                  // float bits of the largest magnitude
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // (a token with an infinity or NaN keeps it: half has both.  Factors within the floats' normal range.)
    const uint32_t e = min(max(top >> 23, 16u), 254u);
    const float f = __uint_as_float((268u - e) << 23);          // 2^(14 - (e - 127))
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const __half2 p = __floats2half2_rn(__uint_as_float(v[i] << 16) * f, __uint_as_float(v[i] & 0xffff0000u) * f);
        v[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return __uint_as_float((e - 14u) << 23);
}

// 64 of the contraction of 64 columns of 8-bit weights: w[j] holds k = 16 t .. 16 t + 15 of column 8 j + g.  x(q, v): this lane's 16 values of
// token 8 q + g as half; back[q]: factors of the sums of tokens 8 q + 2 t and the next.
template <int G, typename X>
__device__ __forceinline__ void multiply_fp8(float (*c)[4][4], const uint4* w, X x, const float (*back)[2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t* wa = (const uint32_t*)&w[2 * i];
        const uint32_t* wb = (const uint32_t*)&w[2 * i + 1];
        float p[G][4] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) {                          // k = 16 t + 4 k .. + 3
            uint32_t f[4];
            halves_of_e4m3(wa[k], f[0], f[2]);
            halves_of_e4m3(wb[k], f[1], f[3]);
#pragma unroll
            for (int q = 0; q < G; ++q) {
                const uint2 v = x(q, k);
                mma16_half(p[q], f, v.x, v.y);
            }
        }
#pragma unroll
        for (int q = 0; q < G; ++q)
#pragma unroll
            for (int v = 0; v < 4; ++v) c[q][i][v] = fmaf(back[q][v & 1], p[q][v], c[q][i][v]);
    }
}
// A step of 16 of the contraction of 64 columns of bfloat16 weights: w[r] holds columns 8 g .. 8 g + 7 of k = 4 t + r.
template <int G>
__device__ __forceinline__ void multiply_bf16(float (*c)[4][4], const uint4* w, const uint2* x) {
    const uint32_t* r0 = (const uint32_t*)&w[0];
    const uint32_t* r1 = (const uint32_t*)&w[1];
    const uint32_t* r2 = (const uint32_t*)&w[2];
    const uint32_t* r3 = (const uint32_t*)&w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t f[4] = {__byte_perm(r0[i], r1[i], 0x5410), __byte_perm(r0[i], r1[i], 0x7632),
                               __byte_perm(r2[i], r3[i], 0x5410), __byte_perm(r2[i], r3[i], 0x7632)};
#pragma unroll
        for (int q = 0; q < G; ++q) mma16(c[q][i], f, x[q].x, x[q].y);
    }
}

// 64 columns of 8-bit weights from column c0 on, 64 of the contraction from kk on.  (Columns past the matrix are its last one again, whose
// sums nobody takes; k past the matrix meets its zero padding.)
struct Fp8Columns {
    const uint8_t* p;
    uint32_t Kp;
    int last;
    __device__ Fp8Columns(const void* W, int c0, int N, int K) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        Kp = (uint32_t)((K + kQ - 1) / kQ * kQ);
        p = (const uint8_t*)W + (size_t)min(c0 + g, N - 1) * Kp + 16 * t;
        last = max(N - 1 - c0 - g, 0);
    }
    __device__ __forceinline__ void load(uint4* w, int kk) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = ld_stream16(p + kk + (size_t)(uint32_t)min(8 * j, last) * Kp);
    }
};

// Up to eight tokens, one warp by itself: c[i] += the products of A's rows with W[k0 .. k1, columns of fragments 2 i and 2 i + 1].  A [Tn rows,
// ld]; W the expert's matrix, its first column c0 of N.  scale: 8-bit weights only, [K / 128] of this column block.
template <int WT>
__device__ __forceinline__ void accumulate(float (*c)[4][4], const __nv_bfloat16* A, int ld, int Tn, const void* W, const float* scale, int c0, int N, int K,
                                           int k0, int k1) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const __nv_bfloat16* mine = A + (size_t)min(g, Tn - 1) * ld;           // (tokens past the last are the last again, whose sums nobody takes)
    if (k0 >= k1) return;
    if constexpr (WT == kBf16) {
        constexpr int U = 4;                           // steps of 16 in flight: 8 KB of weights per warp
        // (columns past the matrix are other columns again; rows of k past the cut are other rows, times zero)
        const __nv_bfloat16* w0 = (const __nv_bfloat16*)W + min(c0 + 8 * g, N - 8);
        for (int kk = k0; kk < k1; kk += 16 * U) {
            uint4 w[U][4];
            uint2 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (kk + 16 * u >= k1) break;
                const int kt = kk + 16 * u + 4 * t, kc = min(kt, k1 - 4);             // (K and the cuts are multiples of 4)
#pragma unroll
                for (int r = 0; r < 4; ++r) w[u][r] = ld_stream16(w0 + (size_t)(kc + r) * N);
                x[u] = *(const uint2*)(mine + kc);
                if (kt >= k1) x[u] = make_uint2(0, 0);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (kk + 16 * u >= k1) break;
                multiply_bf16<1>(c, w[u], &x[u]);
            }
        }
    } else {
        const Fp8Columns cols(W, c0, N, K);
        struct Unit { uint4 w[8], x[2]; float s; };
        auto load = [&](Unit& v, int kk) {
            cols.load(v.w, kk);
#pragma unroll
            for (int h = 0; h < 2; ++h) v.x[h] = *(const uint4*)(mine + min(kk + 16 * t + 8 * h, K - 8));
            v.s = __ldg(scale + kk / kQ);
        };
        auto multiply = [&](Unit& n) {
            uint32_t* v = (uint32_t*)&n.x[0];
            const float r = n.s * to_half64(v);
            const float back[1][2] = {{__shfl_sync(0xffffffffu, r, 8 * t), __shfl_sync(0xffffffffu, r, 8 * t + 4)}};
            multiply_fp8<1>(c, n.w, [&](int, int k) { return make_uint2(v[2 * k], v[2 * k + 1]); }, back);
        };
        // (cuts are multiples of 64) a unit's loads are on their way while the one before it is multiplied
        Unit u0, u1;
        load(u0, k0);
        for (int kk = k0; kk < k1; kk += 128) {
            if (kk + 64 < k1) load(u1, kk + 64);
            multiply(u0);
            if (kk + 64 >= k1) break;
            if (kk + 128 < k1) load(u0, kk + 128);
            multiply(u1);
        }
    }
}

// The staged form, by the whole CTA: 128 of the contraction at a time.  `hold` / `put`: a thread's share of the activations, first to
// registers (while the 128 before them are multiplied), then to shared memory.
template <int WT, int G> struct Staged {
    using T = typename Elem<WT>::T;
    using Sh = Shape<WT, G>;
    static constexpr int VECS = WT == kF32 ? 4 : 2;            // 16 values of one token
    uint4 v[VECS];
    __device__ __forceinline__ void hold(const T* A, int ld, int Tn, int K, int k0) {
        const int tok = threadIdx.x >> 3, kx = k0 + 16 * (threadIdx.x & 7);
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int k = kx + i * (16 / VECS);
            v[i] = make_uint4(0, 0, 0, 0);
            if (tok < Tn && k < K) v[i] = *(const uint4*)(A + (size_t)tok * ld + k);
        }
    }
    __device__ __forceinline__ void put(uint8_t* buf) {
        const int tok = threadIdx.x >> 3, part = threadIdx.x & 7;
        if constexpr (WT == kF32) {
            if (tok < 8 * G) {
                const float* f = (const float*)v;
#pragma unroll
                for (int i = 0; i < 16; ++i) *(float*)(buf + (16 * part + i) * Sh::PITCH + 4 * tok) = f[i];
            }
        } else {
            float back = 0.f;
            if constexpr (WT == kFp8) back = to_half64((uint32_t*)v);
            if (tok < 8 * G) {
                *(uint4*)(buf + tok * Sh::PITCH + 32 * part) = v[0];
                *(uint4*)(buf + tok * Sh::PITCH + 32 * part + 16) = v[1];
                if (WT == kFp8 && (part & 3) == 0) ((float*)(buf + Sh::STAGE))[(part >> 2) * 8 * G + tok] = back;
            }
        }
    }
};

// c += A[rows, k0 .. k1) W[k0 .. k1, the warp's 64 columns from c0 on] (k0 a multiple of 128; every warp takes its part of every 128).  buf: two
// stages.  All threads of the CTA call it with the same k0, k1.  float32: c is [8 G tokens][4 columns 4 (lane % 16) ..] of every other k.
template <int WT, int G, typename C>
__device__ __forceinline__ void accumulate_staged(C& c, const typename Elem<WT>::T* A, int ld, int Tn, const void* W, const float* scale, int c0, int N, int K,
                                                  int k0, int k1, uint8_t* buf) {
    using Sh = Shape<WT, G>;
    constexpr int SZ = Sh::STAGE + Sh::BACK;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int part = warp / (Sh::COLS / kCols);                // of every 128
    Staged<WT, G> st;
    if (k0 >= k1) return;
    st.hold(A, ld, Tn, K, k0);
    __syncthreads();                                           // whoever still reads the stages of an earlier call
    st.put(buf);
    __syncthreads();
    int b = 0;
    auto next = [&](int kk) {                                  // activations of the next 128, behind the work on this one
        b ^= 1;
        if (kk + 128 < k1) st.put(buf + b * SZ);
        __syncthreads();
    };
    if constexpr (WT == kFp8) {
        const Fp8Columns cols(W, c0, N, K);
        uint4 w[2][8];
        float s[2];
        cols.load(w[0], k0 + 64 * part);
        s[0] = __ldg(scale + k0 / kQ);
#pragma unroll 2
        for (int kk = k0, u = 0; kk < k1; kk += 128, u ^= 1) {
            if (kk + 128 < k1) {
                st.hold(A, ld, Tn, K, kk + 128);
                cols.load(w[u ^ 1], kk + 128 + 64 * part);
                s[u ^ 1] = __ldg(scale + (kk + 128) / kQ);
            }
            const uint8_t* x = buf + b * SZ + g * Sh::PITCH + 128 * part + 32 * t;
            const float* bk = (const float*)(buf + b * SZ + Sh::STAGE) + part * 8 * G + 2 * t;
            float back[G][2];
#pragma unroll
            for (int q = 0; q < G; ++q) { back[q][0] = s[u] * bk[8 * q]; back[q][1] = s[u] * bk[8 * q + 1]; }
            multiply_fp8<G>(c, w[u], [&](int q, int k) { return *(const uint2*)(x + q * 8 * Sh::PITCH + 8 * k); }, back);
            next(kk);
        }
    } else if constexpr (WT == kBf16) {
        const __nv_bfloat16* w0 = (const __nv_bfloat16*)W + min(c0 + 8 * g, N - 8);
        uint4 w[2][2][4];                                      // two steps of 16 at a time, the next two on their way
        auto load = [&](uint4 (*v)[4], int k) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) v[h][r] = ld_stream16(w0 + (size_t)min(k + 16 * h + 4 * t + r, K - 1) * N);
        };
        load(w[0], k0 + 64 * part);
        for (int kk = k0; kk < k1; kk += 128) {
            const bool more = kk + 128 < k1;
            if (more) st.hold(A, ld, Tn, K, kk + 128);
            const uint8_t* x = buf + b * SZ + g * Sh::PITCH + 128 * part + 8 * t;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (u == 0) load(w[1], kk + 64 * part + 32);
                else if (more) load(w[0], kk + 128 + 64 * part);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint2 v[G];
#pragma unroll
                    for (int q = 0; q < G; ++q) v[q] = *(const uint2*)(x + q * 8 * Sh::PITCH + 64 * u + 32 * h);
                    multiply_bf16<G>(c, w[u][h], v);
                }
            }
            next(kk);
        }
    } else {
        const int h = lane >> 4;
        const float* w0 = (const float*)W + min(c0 + 4 * (lane & 15), N - 4);
        uint4 w[2][8];                                         // rows h, h + 2, .. of the warp's 16
        auto load = [&](uint4* v, int kk) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = ld_stream16(w0 + (size_t)min(kk + 16 * part + 2 * i + h, K - 1) * N);
        };
        load(w[0], k0);
#pragma unroll 2
        for (int kk = k0, u = 0; kk < k1; kk += 128, u ^= 1) {
            if (kk + 128 < k1) {
                st.hold(A, ld, Tn, K, kk + 128);
                load(w[u ^ 1], kk + 128);
            }
            const uint8_t* x = buf + b * SZ + (16 * part + h) * Sh::PITCH;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float wf[4] = {__uint_as_float(w[u][i].x), __uint_as_float(w[u][i].y), __uint_as_float(w[u][i].z), __uint_as_float(w[u][i].w)};
#pragma unroll
                for (int q = 0; q < 2 * G; ++q) {
                    const float4 xv = *(const float4*)(x + 2 * i * Sh::PITCH + 16 * q);
                    const float xf[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
                    for (int m = 0; m < 4; ++m)
#pragma unroll
                        for (int v = 0; v < 4; ++v) c[4 * q + m][v] = fmaf(xf[m], wf[v], c[4 * q + m][v]);
                }
            }
            next(kk);
        }
    }
}

// Column of the tile, and token, of sum v of c[q][i].
template <int WT>
__device__ __forceinline__ int col_of(int i, int v, int g) {
    return WT == kBf16 ? 8 * g + 2 * i + (v >> 1) : 8 * (2 * i + (v >> 1)) + g;
}
__device__ __forceinline__ int token_of_sum(int q, int v, int t) { return 8 * q + 2 * t + (v & 1); }

// Cut of `units` pieces of work among `workers`: worker w's [lo, hi).
__device__ __forceinline__ void cut(int units, int workers, int w, int& lo, int& hi) {
    lo = (int)((long long)units * w / workers);
    hi = (int)((long long)units * (w + 1) / workers);
}
template <int WT, int G> struct Smem {         // dynamic shared memory
    using Sh = Shape<WT, G>;
    float *red, *cta, *part;                   // [PARTS][Tn][COLS] (the router's partial sums fit as well: n <= 32), [Tn][COLS], [Tn][n]
    Routed* R;
    uint8_t* stage;
    __device__ Smem(uint8_t* base, int Tn, int n) {
        red = (float*)base;
        cta = red + kWarps * Tn * kCols;
        stage = (uint8_t*)(cta + Tn * Sh::COLS);
        R = (Routed*)(stage + (Sh::STAGED ? 2 * (Sh::STAGE + Sh::BACK) : 0));
        part = (float*)(R + 1);
    }
    static size_t bytes(int Tn, int n) {
        return sizeof(float) * ((size_t)kWarps * Tn * kCols + Tn * Sh::COLS + (size_t)Tn * n) + (Sh::STAGED ? 2 * (Sh::STAGE + Sh::BACK) : 0) + sizeof(Routed);
    }
};

// This CTA's sums of a tile (its parts' added in order) into its buffer `cta`, visible to the CTAs that share the tile.
template <int PARTS>
__device__ __forceinline__ void meet(const float* red, float* cta, int size, int S) {
    __syncthreads();
    for (int q = threadIdx.x; q < size; q += kThreads) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < PARTS; ++w) s += red[w * size + q];
        cta[q] = s;
    }
    if (S > 1) cluster_sync_all();
    else __syncthreads();
}

// A warp's sums to its part of `red` ([Tn][COLS], this warp's 64 columns).
template <int WT, int G, typename C>
__device__ __forceinline__ void put_sums(float* red, int Tn, C& c) {
    constexpr int COLS = Shape<WT, G>::COLS;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    if constexpr (WT == kF32) {
#pragma unroll
        for (int m = 0; m < 8 * G; ++m) {
            float4 f;
            f.x = c[m][0] + __shfl_xor_sync(0xffffffffu, c[m][0], 16);
            f.y = c[m][1] + __shfl_xor_sync(0xffffffffu, c[m][1], 16);
            f.z = c[m][2] + __shfl_xor_sync(0xffffffffu, c[m][2], 16);
            f.w = c[m][3] + __shfl_xor_sync(0xffffffffu, c[m][3], 16);
            if (m < Tn && lane < 16) *(float4*)(red + m * COLS + 4 * lane) = f;
        }
    } else {
#pragma unroll
        for (int q = 0; q < G; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (token_of_sum(q, v, t) < Tn) red[token_of_sum(q, v, t) * COLS + col_of<WT>(i, v, g)] = c[q][i][v];
    }
}
template <int WT, int G> struct Sums { float c[G][4][4]; };
template <int G> struct Sums<kF32, G> { float c[8 * G][4]; };

template <int WT>
__device__ __forceinline__ size_t matrix_bytes(int K, int N) {
    return WT == kFp8 ? (size_t)N * ((K + kQ - 1) / kQ * kQ) : (size_t)K * N * sizeof(typename Elem<WT>::T);
}

template <int WT, int G>
__global__ void __launch_bounds__(kThreads, Shape<WT, G>::CTAS)
first_layer_kernel(const TokArgs a, int S) {
    using T = typename Elem<WT>::T;
    using Sh = Shape<WT, G>;
    constexpr int COLS = Sh::COLS;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    const int rank = (int)cluster_ctarank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t0 = blockIdx.z * kTok, Tn = min(kTok, a.T - t0);
    const Smem<WT, G> sm(smem_raw, Tn, a.n);
    pdl_trigger();
    pdl_wait();
    route_tokens<WT, (G + 1) / 2>(a, t0, Tn, rank, sm.red, sm.part, *sm.R);
    const Routed& R = *sm.R;
    if (blockIdx.x == 0)
        for (int q = threadIdx.x; q < (int)(sizeof(Routed) / 4); q += kThreads) ((uint32_t*)(a.routed + blockIdx.z))[q] = ((const uint32_t*)sm.R)[q];
    if (blockIdx.x == 0 && a.r.expert_idx) {
        for (int tok = warp; tok < Tn; tok += kWarps) {
            const uint32_t m = R.mask[tok];
            const size_t b = t0 + tok;
            if (lane < a.n) a.r.p_samp[b * a.n + lane] = a.r.p_patch[b * a.n + lane] = R.p[tok][lane];
            if ((m >> lane) & 1) {
                const int s = __popc(m & ((1u << lane) - 1u));
                a.r.expert_idx[b * a.k + s] = lane;
                a.r.patch_idx[b * a.k + s] = 0;
                a.r.gate[b * a.k + s] = a.use_gate ? R.p[tok][lane] * R.p[tok][lane] : 1.f;
            }
        }
    }
    const int tiles_n = (a.d_e + COLS - 1) / COLS;
    const int tile = blockIdx.x / S, kr = rank % S, first = rank - kr;        // this CTA's tile, its place among the tile's CTAs, the first of them
    const bool live = tile < __popc(R.any) * tiles_n;
    const int slot = live ? tile / tiles_n : 0, c0 = (tile - slot * tiles_n) * COLS, e = nth_bit(R.any, slot);
    const T* x = (const T*)a.x + (size_t)t0 * a.d;
    T* out = (T*)a.a + (size_t)blockIdx.z * a.n * kTok * a.d_e;
    if (live) {
        const void* W = (const uint8_t*)a.W1 + (size_t)e * matrix_bytes<WT>(a.d, a.d_e);
        const int c1 = c0 + warp * kCols % COLS;              // this warp's columns
        const float* sc = WT == kFp8 ? a.s1 + ((size_t)e * ((a.d_e + kQ - 1) / kQ) + min(c1, a.d_e - 1) / kQ) * ((a.d + kQ - 1) / kQ) : nullptr;
        Sums<WT, G> s = {};
        int lo, hi;
        const int units = (a.d + Sh::UNIT - 1) / Sh::UNIT;
        if constexpr (Sh::STAGED) {
            cut(units, S, kr, lo, hi);
            accumulate_staged<WT, G>(s.c, x, a.d, Tn, W, sc, c1, a.d_e, a.d, lo * Sh::UNIT, min(a.d, hi * Sh::UNIT), sm.stage);
        } else {
            cut(units, S * kWarps, kr * kWarps + warp, lo, hi);
            accumulate<WT>(s.c, x, a.d, Tn, W, sc, c1, a.d_e, a.d, lo * Sh::UNIT, min(a.d, hi * Sh::UNIT));
        }
        put_sums<WT, G>(sm.red + warp / (COLS / kCols) * Tn * COLS + warp * kCols % COLS, Tn, s.c);
    }
    cluster_wait();
    meet<Sh::PARTS>(sm.red, sm.cta, Tn * COLS, S);
    if (live) {
        for (int q = kr * kThreads + threadIdx.x; q < Tn * COLS; q += S * kThreads) {
            const int tok = q / COLS, col = c0 + q % COLS;
            if (col >= a.d_e || !((R.mask[tok] >> e) & 1)) continue;
            float h = 0.f;
            for (int s = 0; s < S; ++s) h += ld_cluster(sm.cta + q, first + s);
            if (a.b1) h += to_f32(((const T*)a.b1)[(size_t)e * a.d_e + col]);
            // (bfloat16: half a step, 2^-9 of the value, like the hidden rows of uoe_mlp_forward)
            out[((size_t)slot * kTok + tok) * a.d_e + col] = (T)act_precise(h, a.act);
        }
    }
    if (S > 1) cluster_sync_all();      // nobody's shared memory goes while another CTA may read it
}

template <int WT, int G>
__global__ void __launch_bounds__(kThreads, Shape<WT, G>::CTAS)
second_layer_kernel(const TokArgs a, int S) {
    using T = typename Elem<WT>::T;
    using Sh = Shape<WT, G>;
    constexpr int COLS = Sh::COLS;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    const int rank = (int)cluster_ctarank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & 3;
    const int t0 = blockIdx.z * kTok, Tn = min(kTok, a.T - t0);
    const Smem<WT, G> sm(smem_raw, Tn, a.n);
    pdl_trigger();
    pdl_wait();
    for (int q = threadIdx.x; q < (int)(sizeof(Routed) / 4); q += kThreads) ((uint32_t*)sm.R)[q] = __ldcg((const uint32_t*)(a.routed + blockIdx.z) + q);
    __syncthreads();
    const Routed& R = *sm.R;
    if (blockIdx.x == 0 && blockIdx.z == 0 && warp == 0 && a.r.expert_offsets) {      // Eq. 23, from every group's choices
        int cnt = 0;
        for (int q0 = 0; q0 < a.T * a.k; q0 += 32) {
            const int v = q0 + lane < a.T * a.k ? __ldcg(a.r.expert_idx + q0 + lane) : -1;
            for (int j = 0; j < 32; ++j) cnt += __shfl_sync(0xffffffffu, v, j) == lane;
        }
        const int rows = lane < a.n ? (cnt + UOE_ROW_ALIGN - 1) / UOE_ROW_ALIGN * UOE_ROW_ALIGN : 0;
        int incl = rows;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane < a.n) a.r.expert_offsets[lane + 1] = incl;
        if (lane == 0) a.r.expert_offsets[0] = 0;
    }
    const int c0 = blockIdx.x / S * COLS, kr = rank % S, first = rank - kr, c1 = c0 + warp * kCols % COLS;
    const bool live = c0 < a.d;                        // (the grid is whole clusters)
    const int per = (a.d_e + Sh::UNIT - 1) / Sh::UNIT; // units of one expert
    int lo, hi;
    if constexpr (Sh::STAGED) cut(live ? __popc(R.any) * per : 0, S, kr, lo, hi);
    else cut(live ? __popc(R.any) * per : 0, S * kWarps, kr * kWarps + warp, lo, hi);
    const T* hid = (const T*)a.a + (size_t)blockIdx.z * a.n * kTok * a.d_e;
    auto weight = [&](int tok, int e, float& w) {      // combine weight of (token, expert); false: not chosen
        const float p = R.p[tok][e];
        w = a.use_gate ? p * p : 1.f;
        return ((R.mask[tok] >> e) & 1) != 0;
    };
    Sums<WT, G> tot = {};
    for (int u = lo; u < hi;) {
        const int slot = u / per, k0 = (u - slot * per) * Sh::UNIT, n_u = min(hi - u, per - (u - slot * per)), k1 = min(a.d_e, k0 + n_u * Sh::UNIT);
        const int e = nth_bit(R.any, slot);
        const T* A = hid + (size_t)slot * kTok * a.d_e;
        const void* W = (const uint8_t*)a.W2 + (size_t)e * matrix_bytes<WT>(a.d_e, a.d);
        const float* sc = WT == kFp8 ? a.s2 + ((size_t)e * ((a.d + kQ - 1) / kQ) + min(c1, a.d - 1) / kQ) * ((a.d_e + kQ - 1) / kQ) : nullptr;
        Sums<WT, G> s = {};
        if constexpr (Sh::STAGED) accumulate_staged<WT, G>(s.c, A, a.d_e, Tn, W, sc, c1, a.d, a.d_e, k0, k1, sm.stage);
        else accumulate<WT>(s.c, A, a.d_e, Tn, W, sc, c1, a.d, a.d_e, k0, k1);
        // the tokens that chose this expert take its sums (the hidden rows of the others were never written)
        if constexpr (WT == kF32) {
#pragma unroll
            for (int m = 0; m < 8 * G; ++m) {
                float w = 0.f;
                if (m < Tn && weight(m, e, w)) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) tot.c[m][v] = fmaf(w, s.c[m][v], tot.c[m][v]);
                }
            }
        } else {
#pragma unroll
            for (int q = 0; q < G; ++q)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int tok = token_of_sum(q, h, t);
                    float w = 0.f;
                    if (tok < Tn && weight(tok, e, w)) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            tot.c[q][i][h] = fmaf(w, s.c[q][i][h], tot.c[q][i][h]);
                            tot.c[q][i][2 + h] = fmaf(w, s.c[q][i][2 + h], tot.c[q][i][2 + h]);
                        }
                    }
                }
        }
        u += n_u;
    }
    put_sums<WT, G>(sm.red + warp / (COLS / kCols) * Tn * COLS + warp * kCols % COLS, Tn, tot.c);
    meet<Sh::PARTS>(sm.red, sm.cta, Tn * COLS, S);
    for (int q = kr * kThreads + threadIdx.x; q < Tn * COLS; q += S * kThreads) {
        const int tok = q / COLS, col = c0 + q % COLS;
        if (col >= a.d) continue;
        float s = 0.f;
        for (int r = 0; r < S; ++r) s += ld_cluster(sm.cta + q, first + r);
        if (a.b2) {
            for (uint32_t m = R.mask[tok]; m; m &= m - 1) {
                const int e = __ffs(m) - 1;
                float w;
                weight(tok, e, w);
                s = fmaf(w, to_f32(((const T*)a.b2)[(size_t)e * a.d + col]), s);
            }
        }
        const size_t at = (size_t)(t0 + tok) * a.d + col;
        if (a.residual) s += to_f32(((const T*)a.x)[at]);
        ((T*)a.y)[at] = (T)s;
    }
    if (S > 1) cluster_sync_all();
}

template <typename... KArgs, typename... Args>
cudaError_t launch_clusters(void (*kern)(KArgs...), dim3 grid, size_t smem, cudaStream_t s, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = kCluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

constexpr int kMaxSmem = 160 * 1024;

// CTAs of a tile: the largest split that leaves every worker (a warp, or the CTA where it works together) a unit of the contraction and no
// more CTAs than the SMs hold.
int split_of(int units, int workers, long long tiles, int ctas) {
    int S = kCluster;
    while (S > 1 && (units < S * workers || tiles * S > (long long)ctas * sm_count())) S >>= 1;
    return S;
}

template <int WT, int G>
uoe_status launch_layers(const TokArgs& a, cudaStream_t s) {
    static DeviceOnce once1, once2;
    uoe_status st = smem_opt_in(once1, first_layer_kernel<WT, G>, kMaxSmem);
    if (st == UOE_OK) st = smem_opt_in(once2, second_layer_kernel<WT, G>, kMaxSmem);
    if (st != UOE_OK) return st;
    const int groups = (a.T + kTok - 1) / kTok, Tn = a.T < kTok ? a.T : kTok;
    using Sh = Shape<WT, G>;
    constexpr int workers = Sh::STAGED ? 1 : kWarps;
    const long long chosen = a.n < (long long)Tn * a.k ? a.n : (long long)Tn * a.k;      // experts at most
    auto grid = [&](long long tiles, int S) { return dim3((unsigned)((tiles * S + kCluster - 1) / kCluster * kCluster), 1, groups); };
    const size_t smem = Smem<WT, G>::bytes(Tn, a.n);
    {
        const long long tiles = chosen * ((a.d_e + Sh::COLS - 1) / Sh::COLS);
        const int S = split_of((a.d + Sh::UNIT - 1) / Sh::UNIT, workers, tiles * groups, Sh::CTAS);
        ProfScope ps("tokens_first", s);
        launch_clusters(first_layer_kernel<WT, G>, grid(tiles, S), smem, s, a, S);
        UOE_LAUNCHED();
    }
    {
        const long long tiles = (a.d + Sh::COLS - 1) / Sh::COLS;
        const int S = split_of((int)(a.k * ((a.d_e + Sh::UNIT - 1) / Sh::UNIT)), workers, tiles * groups, Sh::CTAS);
        ProfScope ps("tokens_second", s);
        launch_clusters(second_layer_kernel<WT, G>, grid(tiles, S), smem, s, a, S);
        UOE_LAUNCHED();
    }
    return UOE_OK;
}

template <int WT>
uoe_status launch_tokens(const TokArgs& a, cudaStream_t s) {
    if (a.T <= 8) return launch_layers<WT, 1>(a, s);
    return a.T <= 16 ? launch_layers<WT, 2>(a, s) : launch_layers<WT, 4>(a, s);
}

}  // namespace

size_t mlp_tokens_workspace_bytes(const Dims& D) {
    if (D.L != 1 || D.B > kMaxTokens) return 0;
    const int groups = (D.B + kTok - 1) / kTok;
    return align_up(kStatusBytes + align_up(groups * sizeof(Routed), 1024) + (size_t)groups * D.n * kTok * D.d_e * D.esize, 1024);
}

}  // namespace uoe

using namespace uoe;

extern "C" uoe_status uoe_mlp_tokens(const uoe_problem* prob, const void* x, const void* W_r, const void* W1, const float* w1_scale,
                                     const void* W2, const float* w2_scale, const void* b1, const void* b2, const uoe_routing* r, void* y,
                                     void* ws, size_t ws_bytes, void* cuda_stream) {
    Dims D;
    const uoe_status st = make_dims(prob, D);
    if (st != UOE_OK) return st;
    if (D.d_e < 1 || !x || !W_r || !W1 || !W2 || !y || !ws || (w1_scale == nullptr) != (w2_scale == nullptr)) return UOE_ERR_INVALID_ARG;
    for (const void* p : {x, W_r, W1, W2, (const void*)w1_scale, (const void*)w2_scale, b1, b2, (const void*)y, (const void*)ws})
        if (p && !aligned16(p)) return UOE_ERR_INVALID_ARG;
    if (x == y) return UOE_ERR_INVALID_ARG;
    if (r && (!r->expert_idx || !r->patch_idx || !r->gate || !r->p_samp || !r->p_patch || !r->expert_offsets)) return UOE_ERR_INVALID_ARG;
    if (D.L != 1 || D.B > kMaxTokens || (D.d_e * D.esize) % 16 != 0 || (w1_scale && !D.bf16)) return UOE_ERR_UNSUPPORTED;
    if (ws_bytes < mlp_tokens_workspace_bytes(D)) return UOE_ERR_WORKSPACE;
    TokArgs a = {};
    a.x = x; a.Wr = W_r; a.W1 = W1; a.W2 = W2; a.b1 = b1; a.b2 = b2; a.s1 = w1_scale; a.s2 = w2_scale;
    a.routed = (Routed*)((char*)ws + kStatusBytes);
    a.a = (char*)ws + kStatusBytes + align_up((D.B + kTok - 1) / kTok * sizeof(Routed), 1024);
    a.y = y;
    if (r) a.r = RoutingPtrs{r->expert_idx, r->patch_idx, r->gate, r->p_samp, r->p_patch, r->expert_offsets};
    a.T = D.B; a.d = D.d; a.d_e = D.d_e; a.n = D.n; a.k = D.k; a.act = prob->act;
    a.use_gate = (prob->flags & UOE_FLAG_GATE) != 0; a.residual = (prob->flags & UOE_FLAG_RESIDUAL) != 0;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (!D.bf16) return launch_tokens<kF32>(a, s);
    return w1_scale ? launch_tokens<kFp8>(a, s) : launch_tokens<kBf16>(a, s);
}
