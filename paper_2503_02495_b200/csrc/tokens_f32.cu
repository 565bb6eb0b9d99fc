// uoe_mlp_tokens on float32 weights: the two kernels of tokens_tcgen05.cu with float32 multiply-adds.
//
// Groups of up to 16 tokens (slices of the grid along z) x 64 columns per CTA; the CTA brings 128 of the contraction of its tokens into shared
// memory at a time, a warp multiplies 16 of these (a half warp every other row of W, a lane four columns and all tokens), its weights in
// registers 128 ahead.
#include "tokens.cuh"

namespace uoe {
namespace tokens {
namespace {

constexpr int kCols = 64, kWarps = 8, kThreads = 32 * kWarps, kGroup = 16, kStep = 128;
constexpr int kCluster = 4;

// Tokens in steps of 8: TG = 1 or 2.
template <int TG> struct Smem {
    static constexpr int PITCH = 32 * TG, STAGE = kStep * PITCH;           // bytes of one k of all tokens, of a stage
    float *red, *cta, *part;                   // [8][Tn][64], [Tn][64], [Tn][n]
    uint8_t* stage;
    Routed* R;
    __device__ Smem(uint8_t* base, int Tn, int n) {
        red = (float*)base;
        cta = red + kWarps * Tn * kCols;       // (the router's partial sums fit in red: n <= 32)
        stage = (uint8_t*)(cta + Tn * kCols);
        R = (Routed*)(stage + 2 * STAGE);
        part = (float*)(R + 1);
    }
    static size_t bytes(int Tn, int n) { return 4 * ((size_t)(kWarps + 1) * Tn * kCols + (size_t)Tn * n) + 2 * STAGE + sizeof(Routed); }
};

// c[token][v] += A[token, k0 .. k1) W[k0 .. k1, c0 + 4 (lane % 16) + v], this lane's half of the rows (k0 a multiple of 128), by the whole CTA.
template <int TG>
__device__ __forceinline__ void accumulate(float (&c)[8 * TG][4], const float* A, int ld, int Tn, const float* W, int c0, int N, int K, int k0, int k1,
                                           uint8_t* buf) {
    using Sm = Smem<TG>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = lane >> 4;
    const int tok = threadIdx.x >> 4, k8 = 8 * (threadIdx.x & 15);         // this thread's share of a stage: 8 values of one token
    if (k0 >= k1) return;
    float4 v[2];
    auto hold = [&](int k) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[i] = make_float4(0, 0, 0, 0);
            if (tok < Tn && k + k8 + 4 * i < K) v[i] = *(const float4*)(A + (size_t)tok * ld + k + k8 + 4 * i);
        }
    };
    auto put = [&](uint8_t* b) {
        if (tok >= 8 * TG) return;
        const float f[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) *(float*)(b + (k8 + i) * Sm::PITCH + 4 * tok) = f[i];
    };
    // (columns past the matrix are other columns again, whose sums nobody takes; rows past it are zeros: the last row in their place would make
    // NaN of an infinity there, times activations of zero)
    const float* w0 = W + min(c0 + 4 * (lane & 15), N - 4);
    uint4 w[2][8];
    auto load = [&](uint4* o, int kk) {
        const float* r = w0 + (size_t)(kk + 16 * warp + h) * N;
        if (kk + kStep <= K) {                                 // (looking at every row by itself: eight tokens, d = 4096, 192 -> 202 us)
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = ld_stream16(r + (size_t)(2 * i) * N);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = kk + 16 * warp + h + 2 * i < K ? ld_stream16(r + (size_t)(2 * i) * N) : make_uint4(0, 0, 0, 0);
        }
    };
    load(w[0], k0);
    hold(k0);
    __syncthreads();                                           // whoever still reads the stages of an earlier call
    put(buf);
    __syncthreads();
    int b = 0;
#pragma unroll 2
    for (int kk = k0, u = 0; kk < k1; kk += kStep, u ^= 1) {
        if (kk + kStep < k1) {
            hold(kk + kStep);
            load(w[u ^ 1], kk + kStep);
        }
        const uint8_t* x = buf + b * Sm::STAGE + (16 * warp + h) * Sm::PITCH;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float wf[4] = {__uint_as_float(w[u][i].x), __uint_as_float(w[u][i].y), __uint_as_float(w[u][i].z), __uint_as_float(w[u][i].w)};
#pragma unroll
            for (int q = 0; q < 2 * TG; ++q) {
                const float4 xv = *(const float4*)(x + 2 * i * Sm::PITCH + 16 * q);
                const float xf[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) c[4 * q + m][j] = fmaf(xf[m], wf[j], c[4 * q + m][j]);
            }
        }
        b ^= 1;
        if (kk + kStep < k1) put(buf + b * Sm::STAGE);
        __syncthreads();
    }
}

// The warps' sums, added in order, to `cta`, visible to the CTAs that share the tile.
template <int TG>
__device__ __forceinline__ void meet(const Smem<TG>& sm, float (&c)[8 * TG][4], int Tn, int S) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* red = sm.red + warp * Tn * kCols;
#pragma unroll
    for (int m = 0; m < 8 * TG; ++m) {
        float4 f;
        f.x = c[m][0] + __shfl_xor_sync(0xffffffffu, c[m][0], 16);
        f.y = c[m][1] + __shfl_xor_sync(0xffffffffu, c[m][1], 16);
        f.z = c[m][2] + __shfl_xor_sync(0xffffffffu, c[m][2], 16);
        f.w = c[m][3] + __shfl_xor_sync(0xffffffffu, c[m][3], 16);
        if (m < Tn && lane < 16) *(float4*)(red + m * kCols + 4 * lane) = f;
    }
    __syncthreads();
    for (int q = threadIdx.x; q < Tn * kCols; q += kThreads) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += sm.red[w * Tn * kCols + q];
        sm.cta[q] = s;
    }
    if (S > 1) cluster_sync_all();
    else __syncthreads();
}

template <int TG>
__global__ void __launch_bounds__(kThreads, 1)
first_layer_f32_kernel(const TokArgs a, int S) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    const int rank = (int)cluster_ctarank(), t0 = blockIdx.z * kGroup, Tn = min(kGroup, a.T - t0);
    const Smem<TG> sm(smem_raw, Tn, a.n);
    pdl_trigger();
    pdl_wait();
    route_tokens<kF32, 1, kCluster>(a, t0, Tn, rank, sm.red, sm.part, *sm.R);
    const Routed& R = *sm.R;
    if (blockIdx.x == 0) write_routing(a, R, t0, Tn, threadIdx.x >> 5, kWarps);
    const int tiles_n = (a.d_e + kCols - 1) / kCols, tile = blockIdx.x / S, kr = rank % S, first = rank - kr;
    const bool live = tile < R.experts * tiles_n;
    const int slot = live ? tile / tiles_n : 0, c0 = (tile - slot * tiles_n) * kCols, e = R.list[slot];
    float c[8 * TG][4] = {};
    if (live) {
        int lo, hi;
        cut((a.d + kStep - 1) / kStep, S, kr, lo, hi);
        accumulate<TG>(c, (const float*)a.x + (size_t)t0 * a.d, a.d, Tn, (const float*)a.W1 + (size_t)e * a.d * a.d_e, c0, a.d_e, a.d, lo * kStep,
                       min(a.d, hi * kStep), sm.stage);
    }
    cluster_wait();
    meet(sm, c, Tn, S);
    if (live) {
        float* out = (float*)a.a + ((size_t)blockIdx.z * a.n + slot) * kGroup * a.d_e;
        for (int q = kr * kThreads + threadIdx.x; q < Tn * kCols; q += S * kThreads) {
            const int tok = q / kCols, col = c0 + q % kCols;
            if (col >= a.d_e || !((R.of[slot] >> tok) & 1)) continue;
            float h = a.b1 ? ((const float*)a.b1)[(size_t)e * a.d_e + col] : 0.f;
            for (int s = 0; s < S; ++s) h += ld_cluster_f32(sm.cta + q, first + s);
            out[(size_t)tok * a.d_e + col] = act_f32(h, a.act);
        }
    }
    if (S > 1) cluster_sync_all();      // nobody's shared memory goes while another CTA may read it
}

template <int TG>
__global__ void __launch_bounds__(kThreads, 1)
second_layer_f32_kernel(const TokArgs a, int S) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    const int rank = (int)cluster_ctarank(), t0 = blockIdx.z * kGroup, Tn = min(kGroup, a.T - t0);
    const Smem<TG> sm(smem_raw, Tn, a.n);
    pdl_trigger();
    pdl_wait();
    read_routing(a, *sm.R, Tn);
    const Routed& R = *sm.R;
    if (blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x < 32 && a.r.expert_offsets) write_offsets(a);
    const int c0 = blockIdx.x / S * kCols, kr = rank % S, first = rank - kr, per = (a.d_e + kStep - 1) / kStep;
    int lo, hi;
    cut(c0 < a.d ? R.experts * per : 0, S, kr, lo, hi);        // (the grid is whole clusters)
    auto weight = [&](int tok, int e) { return a.use_gate ? R.p[tok][e] * R.p[tok][e] : 1.f; };
    float tot[8 * TG][4] = {};
    for (int u = lo; u < hi;) {
        const int slot = u / per, n_u = min(hi - u, per - (u - slot * per)), k0 = (u - slot * per) * kStep, e = R.list[slot];
        float c[8 * TG][4] = {};
        accumulate<TG>(c, (const float*)a.a + ((size_t)blockIdx.z * a.n + slot) * kGroup * a.d_e, a.d_e, Tn, (const float*)a.W2 + (size_t)e * a.d_e * a.d, c0,
                       a.d, a.d_e, k0, min(a.d_e, k0 + n_u * kStep), sm.stage);
        // the tokens that chose this expert take its sums (the hidden rows of the others were never written)
#pragma unroll
        for (int m = 0; m < 8 * TG; ++m)
            if (m < Tn && ((R.of[slot] >> m) & 1)) {
                const float w = weight(m, e);
#pragma unroll
                for (int v = 0; v < 4; ++v) tot[m][v] = fmaf(w, c[m][v], tot[m][v]);
            }
        u += n_u;
    }
    meet(sm, tot, Tn, S);
    for (int q = kr * kThreads + threadIdx.x; q < Tn * kCols; q += S * kThreads) {
        const int tok = q / kCols, col = c0 + q % kCols;
        if (col >= a.d) continue;
        float s = 0.f;
        for (int r = 0; r < S; ++r) s += ld_cluster_f32(sm.cta + q, first + r);
        if (a.b2)
            for (uint32_t m = R.mask[tok]; m; m &= m - 1) {
                const int e = __ffs(m) - 1;
                s = fmaf(weight(tok, e), ((const float*)a.b2)[(size_t)e * a.d + col], s);
            }
        const size_t at = (size_t)(t0 + tok) * a.d + col;
        ((float*)a.y)[at] = s + (a.residual ? ((const float*)a.x)[at] : 0.f);
    }
    if (S > 1) cluster_sync_all();
}

template <int TG>
uoe_status launch_layers(const TokArgs& a, cudaStream_t s) {
    static DeviceOnce once1, once2;
    const int groups = (a.T + kGroup - 1) / kGroup, Tn = a.T < kGroup ? a.T : kGroup;
    constexpr int kMaxSmem = 160 * 1024;
    uoe_status st = smem_opt_in(once1, first_layer_f32_kernel<TG>, kMaxSmem);
    if (st == UOE_OK) st = smem_opt_in(once2, second_layer_f32_kernel<TG>, kMaxSmem);
    if (st != UOE_OK) return st;
    const size_t smem = Smem<TG>::bytes(Tn, a.n);
    auto grid = [&](long long tiles, int S) { return dim3((unsigned)((tiles * S + kCluster - 1) / kCluster * kCluster), 1, groups); };
    const long long chosen = a.n < (long long)Tn * a.k ? a.n : (long long)Tn * a.k;      // experts at most
    {
        const long long tiles = chosen * ((a.d_e + kCols - 1) / kCols);
        const int S = split_of((a.d + kStep - 1) / kStep, tiles * groups, kCluster, 1);
        ProfScope ps("tokens_first", s);
        launch_k_cluster(first_layer_f32_kernel<TG>, grid(tiles, S), dim3(kThreads), kCluster, smem, s, a, S);
        UOE_LAUNCHED();
    }
    {
        const long long tiles = (a.d + kCols - 1) / kCols;
        const int S = split_of(a.k * ((a.d_e + kStep - 1) / kStep), tiles * groups, kCluster, 1);
        ProfScope ps("tokens_second", s);
        launch_k_cluster(second_layer_f32_kernel<TG>, grid(tiles, S), dim3(kThreads), kCluster, smem, s, a, S);
        UOE_LAUNCHED();
    }
    return UOE_OK;
}

}  // namespace

int group_f32() { return kGroup; }
uoe_status launch_f32(const TokArgs& a, cudaStream_t s) { return a.T <= 8 ? launch_layers<1>(a, s) : launch_layers<2>(a, s); }

}  // namespace tokens
}  // namespace uoe
