// Residual addition between two norms, backward: the entry points, the reduction of what the blocks leave, and the kernel for rows of bf16
// with checkpoints.
#include "norm_bwd.cuh"

namespace mx {

template cudaError_t launch_norm_bwd<__nv_bfloat16, true>(const NormBwd &, const RowPlan &, bool, bool, bool, cudaStream_t);
extern template cudaError_t launch_norm_bwd<__nv_bfloat16, false>(const NormBwd &, const RowPlan &, bool, bool, bool, cudaStream_t);
extern template cudaError_t launch_norm_bwd<float, true>(const NormBwd &, const RowPlan &, bool, bool, bool, cudaStream_t);
extern template cudaError_t launch_norm_bwd<float, false>(const NormBwd &, const RowPlan &, bool, bool, bool, cudaStream_t);

struct NormBwdFinish {
    const float *part, *slots;
    NormSide post;
    const void *gate;
    int64_t ldg, gates;
    int gate_fp32, several;
    float s;
    int blocks, pre, use_f, has_post, bias;
    int64_t rows, rows_per_gate, rows_per_team;
    int cols, split;          // split: lanes of rows that share a gate, a power of two
    float *dw_pre, *db_pre, *dw_post, *db_post, *dgate;
};

// Adds up what the blocks and teams have left, in a fixed order.  A block has 16 columns, 4 lanes of 4 columns by 64 lanes of rows.
__global__ void __launch_bounds__(256) k_norm_bwd_finish(const __grid_constant__ NormBwdFinish p)
{
    __shared__ float4 s_a[64][4], s_b[64][4];
    pdl_launch_dependents();
    pdl_wait();
    const int q = threadIdx.x & 3, r = threadIdx.x >> 2;
    const int c = blockIdx.x * 16 + q * 4;
    const auto add = [](float4 &a, const float4 &b) { a.x += b.x, a.y += b.y, a.z += b.z, a.w += b.w; };
    // sums over the 64 lanes of rows, in every lane
    const auto all_rows = [&](float4 &a, float4 &b) {
        for (int o = 32; o; o >>= 1) {
            __syncthreads();
            s_a[r][q] = a, s_b[r][q] = b;
            __syncthreads();
            add(a, s_a[r ^ o][q]), add(b, s_b[r ^ o][q]);
        }
    };
    const float4 zero = make_float4(0, 0, 0, 0);
    if (p.pre && (p.dw_pre || p.db_pre)) {
        float4 a = zero, b = zero;
        for (int k = r; k < p.blocks; k += 64) {
            const float *s = p.part + (int64_t)k * 4 * p.cols + c;
            add(a, *reinterpret_cast<const float4 *>(s));
            if (p.bias) add(b, *reinterpret_cast<const float4 *>(s + p.cols));
        }
        all_rows(a, b);
        if (r == 0) {
            if (p.dw_pre) *reinterpret_cast<float4 *>(p.dw_pre + c) = a;
            if (p.db_pre) *reinterpret_cast<float4 *>(p.db_pre + c) = b;
        }
    }
    if (!p.use_f || !(p.dw_post || p.db_post || p.dgate)) return;
    float4 w = make_float4(1, 1, 1, 1), bias = zero;
    const auto param = [&](const void *v, int fp32, int64_t at) {
        if (fp32) return *reinterpret_cast<const float4 *>(static_cast<const float *>(v) + at);
        const uint2 u = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(v) + at);
        return make_float4(bf16lo(u.x), bf16hi(u.x), bf16lo(u.y), bf16hi(u.y));
    };
    if (p.has_post && p.post.w) w = param(p.post.w, p.post.fp32, c);
    if (p.has_post && p.post.b) bias = param(p.post.b, p.post.fp32, c);
    const int in_turn = 64 / p.split;         // gates at a time
    const int sub = r & (p.split - 1);
    float4 cw = zero, cb = zero;              // sums over this lane's gates of g B and g A
    for (int64_t g0 = 0; g0 < p.gates; g0 += in_turn) {
        const int64_t g = g0 + r / p.split;
        float4 B = zero, A = zero;
        if (g < p.gates) {
            if (p.several) {
                const int64_t t0 = g * p.rows_per_gate / p.rows_per_team, t1 = ((g + 1) * p.rows_per_gate - 1) / p.rows_per_team;
                for (int64_t k = t0 + sub; k <= t1; k += p.split) {
                    const float *s = p.slots + (k + g) * 2 * (int64_t)p.cols + c;
                    add(B, *reinterpret_cast<const float4 *>(s));
                    if (p.bias) add(A, *reinterpret_cast<const float4 *>(s + p.cols));
                }
            } else {
                for (int k = sub; k < p.blocks; k += p.split) {
                    const float *s = p.part + (int64_t)k * 4 * p.cols + 2 * p.cols + c;
                    add(B, *reinterpret_cast<const float4 *>(s));
                    if (p.bias) add(A, *reinterpret_cast<const float4 *>(s + p.cols));
                }
            }
        }
        for (int o = p.split >> 1; o; o >>= 1) {
            __syncthreads();
            s_a[r][q] = B, s_b[r][q] = A;
            __syncthreads();
            add(B, s_a[r ^ o][q]), add(A, s_b[r ^ o][q]);
        }
        if (g < p.gates && sub == 0) {
            if (p.dgate)
                *reinterpret_cast<float4 *>(p.dgate + g * p.cols + c) = make_float4(p.s * fmaf(w.x, B.x, bias.x * A.x), p.s * fmaf(w.y, B.y, bias.y * A.y),
                                                                                    p.s * fmaf(w.z, B.z, bias.z * A.z), p.s * fmaf(w.w, B.w, bias.w * A.w));
            const float4 gg = p.gate ? param(p.gate, p.gate_fp32, g * p.ldg + c) : make_float4(1, 1, 1, 1);
            cw.x = fmaf(gg.x, B.x, cw.x), cw.y = fmaf(gg.y, B.y, cw.y), cw.z = fmaf(gg.z, B.z, cw.z), cw.w = fmaf(gg.w, B.w, cw.w);
            cb.x = fmaf(gg.x, A.x, cb.x), cb.y = fmaf(gg.y, A.y, cb.y), cb.z = fmaf(gg.z, A.z, cb.z), cb.w = fmaf(gg.w, A.w, cb.w);
        }
    }
    if (!p.has_post) return;
    all_rows(cw, cb);
    if (r == 0) {
        if (p.dw_post) *reinterpret_cast<float4 *>(p.dw_post + c) = make_float4(p.s * cw.x, p.s * cw.y, p.s * cw.z, p.s * cw.w);
        if (p.db_post) *reinterpret_cast<float4 *>(p.db_post + c) = make_float4(p.s * cb.x, p.s * cb.y, p.s * cb.z, p.s * cb.w);
    }
}

}  // namespace mx

using namespace mx;

extern "C" {

size_t mxfp4_residual_norm_workspace_bytes(int64_t rows, int64_t cols, int64_t gates)
{
    if (rows <= 0 || cols <= 0 || cols > kNormMaxCols || gates < 0) return 0;
    const RowPlan b = row_plan(rows, cols, kBwdThreads);
    return (size_t)(part_floats(b, cols) + slot_floats(b, cols, gates)) * 4;
}

mxfp4_status_t mxfp4_residual_norm_bwd(const mxfp4_residual_norm_t *n, const mxfp4_residual_norm_bwd_t *b, void *workspace, size_t workspace_bytes, void *stream)
{
    mxfp4_status_t s;
    if ((s = check_plan(n))) return s;
    if (!b) return MXFP4_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t rows = n->rows, cols = n->cols;
    const bool pre = n->pre.kind != MXFP4_NORM_NONE, post = n->post.kind != MXFP4_NORM_NONE, need_f = post || n->gate;
    if (pre != (b->dh_bf16 != nullptr) && rows > 0) return MXFP4_INVALID_ARG;
    if ((!pre && (b->dw_pre || b->db_pre)) || (!post && (b->dw_post || b->db_post)) || (!n->gate && b->dgate)) return MXFP4_INVALID_ARG;
    for (const float *g : {b->dw_pre, b->db_pre, b->dw_post, b->db_post, b->dgate})
        if (!aligned16(g)) return MXFP4_MISALIGNED;
    if (rows == 0) {
        for (float *g : {b->dw_pre, b->db_pre, b->dw_post, b->db_post})
            if (g) MX_CHECK_CUDA(cudaMemsetAsync(g, 0, (size_t)cols * 4, st));
        if (b->dgate) MX_CHECK_CUDA(cudaMemsetAsync(b->dgate, 0, (size_t)(n->gates * cols) * 4, st));
        return MXFP4_OK;
    }
    const int64_t xb = dtype_bytes(n->x_dtype);
    if (pre && (s = check_rows(b->dh_bf16, b->lddh, cols, MXFP4_OUT_BF16))) return s;
    if (b->dx_out && (s = check_rows(b->dx_out, b->lddxo, cols, n->x_dtype))) return s;
    if ((s = check_rows(b->dx, b->lddx, cols, n->x_dtype))) return s;
    if (b->df_bf16 && (s = check_rows(b->df_bf16, b->lddf, cols, MXFP4_OUT_BF16))) return s;
    if (!pre && !b->dx_out) return MXFP4_INVALID_ARG;       // no gradient at all
    if ((pre || post) && !b->stats) return MXFP4_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(b->stats) & 3u) return MXFP4_MISALIGNED;
    const bool eight = pre ? b->x_ckpt.codes != nullptr : need_f && b->f_ckpt.codes != nullptr;
    if (pre && eight && (s = check_ckpt(b->x_ckpt, rows, cols))) return s;
    if (need_f && eight && (s = check_ckpt(b->f_ckpt, rows, cols))) return s;
    if (pre && !eight && (s = check_rows(b->x_out, b->ldxo, cols, n->x_dtype))) return s;
    if (need_f && !eight && (s = check_rows(b->f_bf16, b->ldf, cols, MXFP4_OUT_BF16))) return s;
    if (!workspace) return MXFP4_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return MXFP4_MISALIGNED;
    const RowPlan plan = row_plan(rows, cols, kBwdThreads);
    if (workspace_bytes < (size_t)(part_floats(plan, cols) + slot_floats(plan, cols, n->gates)) * 4) return MXFP4_WORKSPACE_TOO_SMALL;
    {
        // dx and df are written row by row while later rows are still to be read
        const Span dx = span_of_rows(b->dx, b->lddx, rows, cols, xb), df = span_of_rows(b->df_bf16, b->lddf, rows, cols, 2);
        const Span dxo = span_of_rows(b->dx_out, b->lddxo, rows, cols, xb), dh = span_of_rows(b->dh_bf16, b->lddh, rows, cols, 2);
        if (meet(dx, df) || !rows_over_or_apart(dx, b->lddx, xb, dxo, b->lddxo, xb) || !rows_over_or_apart(dx, b->lddx, xb, dh, b->lddh, 2) ||
            !rows_over_or_apart(df, b->lddf, 2, dxo, b->lddxo, xb) || !rows_over_or_apart(df, b->lddf, 2, dh, b->lddh, 2))
            return MXFP4_INVALID_ARG;
        const Span kept[4] = {pre && eight ? span_of(b->x_ckpt.codes, rows * cols) : Span{0, 0}, need_f && eight ? span_of(b->f_ckpt.codes, rows * cols) : Span{0, 0},
                              pre && !eight ? span_of_rows(b->x_out, b->ldxo, rows, cols, xb) : Span{0, 0},
                              need_f && !eight ? span_of_rows(b->f_bf16, b->ldf, rows, cols, 2) : Span{0, 0}};
        for (const Span &k : kept)
            if (k.hi && (meet(dx, k) || meet(df, k))) return MXFP4_INVALID_ARG;
    }
    NormBwd p = {};
    p.dh = static_cast<const __nv_bfloat16 *>(b->dh_bf16), p.dxo = b->dx_out, p.lddh = b->lddh, p.lddxo = b->lddxo, p.stats = b->stats;
    p.xcodes = b->x_ckpt.codes, p.xscales = b->x_ckpt.scales, p.fcodes = b->f_ckpt.codes, p.fscales = b->f_ckpt.scales;
    p.xo = b->x_out, p.f = static_cast<const __nv_bfloat16 *>(b->f_bf16), p.ldxo = b->ldxo, p.ldf = b->ldf;
    p.dx = b->dx, p.df = static_cast<__nv_bfloat16 *>(b->df_bf16), p.lddx = b->lddx, p.lddf = b->lddf;
    p.pre = side_of(n->pre), p.post = side_of(n->post);
    p.gate = n->gate, p.ldg = n->ld_gate, p.gate_fp32 = n->gate_dtype == MXFP4_OUT_FP32;
    p.several = n->gates > 1, p.rows_per_gate = (uint32_t)(n->gates > 1 ? rows / n->gates : rows);
    p.a = n->residual_scale, p.s = n->branch_scale;
    p.part = static_cast<float *>(workspace), p.slots = p.part + part_floats(plan, cols);
    p.rows = rows, p.rows_per_team = plan.rows_per_team, p.cols = (int)cols, p.nvec = (int)(cols / 8), p.warps = plan.warps(), p.teams = plan.teams;
    const bool bias = b->db_pre || b->db_post || (n->gate && n->post.bias && post);
    const auto go = n->x_dtype == MXFP4_OUT_FP32 ? (eight ? launch_norm_bwd<float, true> : launch_norm_bwd<float, false>)
                                                 : (eight ? launch_norm_bwd<__nv_bfloat16, true> : launch_norm_bwd<__nv_bfloat16, false>);
    MX_CHECK_CUDA(go(p, plan, need_f, post, pre, st));
    if (!b->dw_pre && !b->db_pre && !b->dw_post && !b->db_post && !b->dgate) return MXFP4_OK;
    NormBwdFinish e = {};
    e.part = p.part, e.slots = p.slots, e.post = p.post, e.gate = p.gate, e.ldg = p.ldg, e.gate_fp32 = p.gate_fp32;
    e.gates = n->gates > 1 ? n->gates : 1, e.several = p.several, e.s = p.s, e.blocks = plan.blocks, e.pre = pre, e.use_f = need_f, e.has_post = post, e.bias = bias;
    e.rows = rows, e.rows_per_gate = p.rows_per_gate, e.rows_per_team = plan.rows_per_team, e.cols = (int)cols;
    e.split = 64;
    while (e.split > 1 && 64 / e.split < e.gates) e.split >>= 1;
    e.dw_pre = b->dw_pre, e.db_pre = b->db_pre, e.dw_post = b->dw_post, e.db_post = b->db_post, e.dgate = b->dgate;
    MX_CHECK_CUDA(launch_pdl(k_norm_bwd_finish, (unsigned)(cols / 16), 1, 256, 0, st, e));
    return MXFP4_OK;
}

}  // extern "C"
