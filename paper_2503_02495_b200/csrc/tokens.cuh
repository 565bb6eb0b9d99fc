// What the kernels of uoe_mlp_tokens share: arguments, the router (Eq. 13-14, 21-22 for samples of one token), clusters.
#pragma once
#include "fp8.cuh"
#include "tc.cuh"

namespace uoe {
namespace tokens {

using namespace tc;

constexpr int kMaxTokens = 64;
constexpr int kRouteWarps = 8;
enum { kBf16 = 0, kFp8 = 1, kF32 = 2 };

struct Routed {                     // what the router says about a group's tokens
    unsigned long long of[32];      // tokens that chose expert list[i]
    int experts;                    // that some token chose
    int list[32];                   // these, ascending
    uint32_t mask[kMaxTokens];      // experts that token chose
    float p[kMaxTokens][32];        // sample gate (Eq. 21)
};
// words of it that say something about Tn tokens
__device__ __forceinline__ int routed_words(int Tn) { return (int)(offsetof(Routed, p) / 4) + 32 * Tn; }

struct TokArgs {
    const void *x, *Wr, *W1, *W2, *b1, *b2;
    const float *s1, *s2;
    Routed* routed;                 // [groups]: what the first kernel's router says, for the second
    void *a, *y;                    // a [groups, n, group, d_e]: hidden rows by place in the group's list of chosen experts
    float* af;                      // 8-bit: a is [n, 2 terms, group, d_e padded] bytes, af their scales [n, d_e / 128, group]
    RoutingPtrs r;                  // all null, or all to be written
    int T, d, d_e, n, k, act, use_gate, residual;
    int group;                      // tokens of a z slice of the grid
};

template <int WT> struct Elem { using T = __nv_bfloat16; };
template <> struct Elem<kF32> { using T = float; };

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

__device__ __forceinline__ void mma16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// four e4m3 bytes -> two half pairs, exact
__device__ __forceinline__ void halves_of_e4m3(uint32_t v, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(v));
}

// Sums over this CTA's piece of d: part[token * n + expert].
template <int WT, int MT, int CL>
__device__ void router_piece(const TokArgs& a, int t0, int Tn, int rank, float* red /* [8][Tn * n] */, float* part) {
    using T = typename Elem<WT>::T;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int d = a.d, n = a.n, len = ((d + CL - 1) / CL + 15) / 16 * 16;
    const T* x = (const T*)a.x + (size_t)t0 * d;
    const T* Wr = (const T*)a.Wr;
    const int k0 = rank * len, k1 = min(d, k0 + len);
    if (warp < kRouteWarps) {
        if constexpr (WT == kF32) {
            // lanes side by side along the experts of a row of W_r (and along rows, where experts are few), sixteen tokens at a time
            int np2 = 1;
            while (np2 < n) np2 <<= 1;
            const int i = lane % np2, rows = 32 / np2;
            for (int tb = 0; tb < Tn; tb += 16) {
                float s[16] = {};
#pragma unroll 2
                for (int kk = k0 + warp * rows + lane / np2; kk < k1; kk += kRouteWarps * rows) {
                    const float w = i < n ? Wr[(size_t)kk * n + i] : 0.f;
#pragma unroll
                    for (int m = 0; m < 16; ++m) s[m] = fmaf(x[(size_t)min(tb + m, Tn - 1) * d + kk], w, s[m]);
                }
#pragma unroll
                for (int m = 0; m < 16; ++m) {
                    for (int o = np2; o < 32; o <<= 1) s[m] += __shfl_xor_sync(0xffffffffu, s[m], o);
                    if (tb + m < Tn && lane < n) red[warp * Tn * n + (tb + m) * n + lane] = s[m];
                }
            }
        } else {
            const int J = (n + 7) / 8;                 // fragment j: experts g * J + j
            const bool whole = n == 8 * J && J != 3;   // a lane's experts of a row of W_r in one load
            constexpr int U = MT == 1 ? 4 : 2;         // steps of 16 whose loads are in flight together
            float c[MT][4][4] = {};
            for (int kb = k0 + warp * 16; kb < k1; kb += kRouteWarps * 16 * U) {
                uint2 xv[U][MT][2], wv[U][4];          // a row's (up to) four experts, two per word
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int kt = kb + u * kRouteWarps * 16 + 4 * t;
                    const bool in = kt < k1;
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int row = m * 16 + h * 8 + g;
                            xv[u][m][h] = make_uint2(0, 0);
                            if (row < Tn && in) xv[u][m][h] = *(const uint2*)(x + (size_t)row * d + kt);
                        }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const T* p = Wr + (size_t)(kt + r) * n + g * J;
                        wv[u][r] = make_uint2(0, 0);
                        if (!in) continue;
                        if (whole) {
                            if (J == 1) wv[u][r].x = *(const uint16_t*)p;
                            else if (J == 2) wv[u][r].x = *(const uint32_t*)p;
                            else wv[u][r] = *(const uint2*)p;
                        } else {
                            uint32_t q[4] = {0, 0, 0, 0};
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (j < J && g * J + j < n) q[j] = *(const uint16_t*)(p + j);
                            wv[u][r] = make_uint2(q[0] | (q[1] << 16), q[2] | (q[3] << 16));
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (kb + u * kRouteWarps * 16 >= k1) break;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j >= J) break;
                        const uint32_t sel = j & 1 ? 0x7632 : 0x5410;
                        const uint32_t b0 = j < 2 ? __byte_perm(wv[u][0].x, wv[u][1].x, sel) : __byte_perm(wv[u][0].y, wv[u][1].y, sel);
                        const uint32_t b1 = j < 2 ? __byte_perm(wv[u][2].x, wv[u][3].x, sel) : __byte_perm(wv[u][2].y, wv[u][3].y, sel);
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            const uint32_t af[4] = {xv[u][m][0].x, xv[u][m][1].x, xv[u][m][0].y, xv[u][m][1].y};
                            mma16(c[m][j], af, b0, b1);
                        }
                    }
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
        }
    }
    __syncthreads();
    for (int q = threadIdx.x; q < Tn * n; q += blockDim.x) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kRouteWarps; ++w) s += red[w * Tn * n + q];
        part[q] = s;
    }
}

// Eq. 21-22 for the group's tokens, the same in every CTA.
template <int WT, int MT, int CL /* CTAs of the cluster */>
__device__ void route_tokens(const TokArgs& a, int t0, int Tn, int rank, float* red, float* part, Routed& R) {
    router_piece<WT, MT, CL>(a, t0, Tn, rank, red, part);
    if (threadIdx.x < 32) R.of[threadIdx.x] = 0;       // (by expert for now)
    cluster_sync_all();                                // every CTA's piece is there
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = a.n;
    for (int tok = warp; tok < Tn; tok += (int)(blockDim.x >> 5)) {
        float v = -INFINITY;
        if (lane < n) {
            v = 0.f;
#pragma unroll
            for (int p = 0; p < CL; ++p) v += ld_cluster_f32(part + tok * n + lane, p);
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
        if ((m >> lane) & 1) atomicOr(&R.of[lane], 1ull << tok);
    }
    cluster_arrive();                                  // done with the others' pieces (cluster_wait follows before the next meeting)
    __syncthreads();
    if (warp == 0) {                                   // the chosen experts in a row
        const unsigned long long of = R.of[lane];
        const uint32_t any = __ballot_sync(0xffffffffu, of != 0);
        __syncwarp();
        if (of) {
            const int at = __popc(any & ((1u << lane) - 1u));
            R.list[at] = lane;
            R.of[at] = of;                             // (at <= lane, and every lane holds its own)
        }
        if (lane == 0) R.experts = __popc(any);
    }
    __syncthreads();
}

// Cut of `units` pieces of work among `workers`: worker w's [lo, hi).
__device__ __forceinline__ void cut(int units, int workers, int w, int& lo, int& hi) {
    lo = (int)((long long)units * w / workers);
    hi = (int)((long long)units * (w + 1) / workers);
}
// The router's outputs for the second kernel and for the caller, by `warps` warps (this one: `warp`) of one CTA of the group.
__device__ __forceinline__ void write_routing(const TokArgs& a, const Routed& R, int t0, int Tn, int warp, int warps) {
    const int lane = threadIdx.x & 31;
    for (int q = 32 * warp + lane; q < routed_words(Tn); q += 32 * warps) ((uint32_t*)(a.routed + blockIdx.z))[q] = ((const uint32_t*)&R)[q];
    if (!a.r.expert_idx) return;
    for (int tok = warp; tok < Tn; tok += warps) {
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
// Eq. 23, from every group's choices, by one warp of the second kernel.
__device__ __forceinline__ void write_offsets(const TokArgs& a) {
    const int lane = threadIdx.x & 31;
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
// The router's word from the first kernel, into shared memory.
__device__ __forceinline__ void read_routing(const TokArgs& a, Routed& R, int Tn) {
    for (int q = threadIdx.x; q < routed_words(Tn); q += blockDim.x) ((uint32_t*)&R)[q] = __ldcg((const uint32_t*)(a.routed + blockIdx.z) + q);
    __syncthreads();
}

// CTAs of a tile: the largest split that leaves every CTA a unit of the contraction and no more CTAs than the SMs hold.
inline int split_of(int units, long long tiles, int cluster, int ctas_per_sm) {
    int S = cluster;
    while (S > 1 && (units < S || tiles * S > (long long)ctas_per_sm * sm_count())) S >>= 1;
    return S;
}

int group_f32();                    // tokens of a group
uoe_status launch_f32(const TokArgs& a, cudaStream_t s);

}  // namespace tokens
}  // namespace uoe
