// uoe_mlp_forward_fp8: the UoME forward (Eq. 37-40) on 8-bit expert weights:
//   plan, quantisation of x -> gather (Eq. 18) inside the product's loads, bias, phi and quantisation again (Eq. 38) -> product and bias
//   (Eq. 39) -> weighted combine (Eq. 20 / 40), these two in one kernel for patches of 128 tokens (fp8_patch_tcgen05.cu).
// The rows exist as bytes only: every token is quantised once, the first product's write-out finds the largest of a row's 128 hidden columns
// in one thread's registers, and only the experts' outputs are bfloat16, if they reach memory at all.  Where patches do not tile 128 rows, where fewer rows are routed than
// there are tokens, or where the weights' scales are not powers of two, the routed rows are quantised into a buffer of their own (scale layer,
// 4 x 4096 tokens of 4096, each routed twice: 79 us for that, 44 us for the tokens once, and 3 us more in the product).
#include "fp8.cuh"

namespace uoe {
namespace {

struct MlpFp8Ws { size_t plan, xq, xs, aq, as, z, total; };

MlpFp8Ws mlp_fp8_ws(const Dims& D) {
    WsCarver w;
    w.take(kStatusBytes);
    MlpFp8Ws r;
    r.plan = w.take(plan_bytes(D));
    r.xq = w.take((size_t)D.Rmax * q_pad(D.d));       // routed rows, or no more tokens than them
    r.xs = w.take((size_t)D.Rmax * q_blocks(D.d) * 4);
    r.aq = w.take((size_t)D.Rmax * q_pad(D.d_e));
    r.as = w.take((size_t)D.Rmax * q_blocks(D.d_e) * 4);
    r.z = w.take((size_t)D.Rmax * D.d * 2);
    r.total = w.off;
    return r;
}

}  // namespace

size_t mlp_fp8_workspace_bytes(const Dims& D) { return mlp_fp8_ws(D).total; }

}  // namespace uoe

using namespace uoe;

extern "C" uoe_status uoe_mlp_forward_fp8(const uoe_problem* prob, const void* x, const void* W1, const float* w1_scale, const void* W2,
                                          const float* w2_scale, const void* b1, const void* b2, const int32_t* expert_idx,
                                          const int32_t* patch_idx, const float* gate, const int32_t* expert_offsets, void* y, void* ws,
                                          size_t ws_bytes, void* cuda_stream) {
    Dims D;
    uoe_status st = make_dims(prob, D);
    if (st != UOE_OK) return st;
    if (D.d_e < 1 || !x || !W1 || !w1_scale || !W2 || !w2_scale || !expert_idx || !patch_idx || !gate || !expert_offsets || !y || !ws) return UOE_ERR_INVALID_ARG;
    for (const void* p : {x, W1, (const void*)w1_scale, W2, (const void*)w2_scale, b1, b2, (const void*)y, (const void*)ws})
        if (p && !aligned16(p)) return UOE_ERR_INVALID_ARG;
    if (!D.bf16) return UOE_ERR_UNSUPPORTED;
    const MlpFp8Ws W = mlp_fp8_ws(D);
    if (ws_bytes < W.total) return UOE_ERR_WORKSPACE;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    char* base = (char*)ws;
    int* status = (int*)base;
    const PlanPtrs P = plan_ptrs(D, base + W.plan);
    const bool any_scale = (prob->flags & UOE_FLAG_FP8_ANY_SCALE) != 0;
    const long long tokens = (long long)D.B * D.L;
    const bool gather = !any_scale && fp8_can_gather(D.l_p) && D.R >= tokens && tokens < (1ll << 31);
    st = launch_plan(D, expert_idx, patch_idx, gate, expert_offsets, P, status, s, true, PlanTails(), gather);
    if (st != UOE_OK) return st;
    if (gather) st = launch_quantize_rows(x, true, 1, tokens, D.d, base + W.xq, (float*)(base + W.xs), SrcMap(), nullptr, 0, "fp8_quantize_x", s, true);
    else st = launch_quantize_rows(x, true, 1, D.Rmax, D.d, base + W.xq, (float*)(base + W.xs), row_map_of(D, P, patch_idx), expert_offsets, D.n, "fp8_gather", s);
    if (st != UOE_OK) return st;
    Fp8Gemm g1{base + W.xq, (float*)(base + W.xs), W1, w1_scale, expert_offsets, D.n, D.Rmax, D.d_e, D.d, false, nullptr, true};
    if (gather) g1.map = src_map_of(D, P, patch_idx);
    g1.bias = b1;
    g1.act = prob->act;
    g1.epi = kFp8ActQuant;
    g1.q = base + W.aq;
    g1.qs = (float*)(base + W.as);
    g1.any_scale = any_scale;
    g1.label = "fp8_gemm1_act";
    st = launch_fp8_gemm(g1, status, s);
    if (st != UOE_OK) return st;
    if (!any_scale && fp8_patch_can(D))
        return launch_fp8_patch(D, base + W.aq, (float*)(base + W.as), W2, w2_scale, b2, x, y, expert_offsets, P, (prob->flags & UOE_FLAG_GATE) != 0,
                                (prob->flags & UOE_FLAG_RESIDUAL) != 0, status, s);
    // z in bfloat16 (off by half a step, 2^-8 of the value, as between uoe_mlp_forward's product and combine): in float32 the combine, which these
    // bytes bound, would read twice as many
    Fp8Gemm g2{base + W.aq, (float*)(base + W.as), W2, w2_scale, expert_offsets, D.n, D.Rmax, D.d, D.d_e, false, base + W.z, true};
    g2.bias = b2;
    g2.any_scale = any_scale;
    g2.label = "fp8_gemm2";
    st = launch_fp8_gemm(g2, status, s);
    if (st != UOE_OK) return st;
    return launch_combine(D, x, base + W.z, P, (prob->flags & UOE_FLAG_RESIDUAL) != 0, (prob->flags & UOE_FLAG_GATE) != 0, y, s);
}
