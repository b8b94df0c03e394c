// Residual addition between two norms, forward: the entry point, and the kernel for rows of bf16.
#include "norm_fwd.cuh"

namespace mx {

extern template cudaError_t launch_norm_fwd<float>(NormFwd &, const RowPlan &, bool, bool, bool, cudaStream_t);
template cudaError_t launch_norm_fwd<__nv_bfloat16>(NormFwd &, const RowPlan &, bool, bool, bool, cudaStream_t);

}  // namespace mx

using namespace mx;

extern "C" {

mxfp4_status_t mxfp4_residual_norm_fwd(const mxfp4_residual_norm_t *n, const void *x, int64_t ldx, const void *f_bf16, int64_t ldf, void *x_out, int64_t ldxo,
                                       void *h_bf16, int64_t ldh, const mxfp4_mat_t *hq, float *stats, mxfp4_ckpt_t x_ckpt, mxfp4_ckpt_t f_ckpt,
                                       int32_t scale_mode, uint32_t *dev_status, void *stream)
{
    mxfp4_status_t s;
    if ((s = check_plan(n))) return s;
    if (scale_mode != MXFP4_SCALE_TRUNCATION_FREE && scale_mode != MXFP4_SCALE_FLOOR) return MXFP4_INVALID_ARG;
    const int64_t rows = n->rows, cols = n->cols;
    if (rows == 0) return MXFP4_OK;        // (of empty tensors the addresses may be missing)
    const bool pre = n->pre.kind != MXFP4_NORM_NONE, post = n->post.kind != MXFP4_NORM_NONE, has_f = f_bf16 != nullptr;
    if (!has_f && (post || n->gate || x_out || f_ckpt.codes || n->residual_scale != 1.0f || n->branch_scale != 1.0f)) return MXFP4_INVALID_ARG;
    if (!pre && (h_bf16 || hq || x_ckpt.codes)) return MXFP4_INVALID_ARG;
    if (!x_out && !h_bf16 && !hq) return MXFP4_INVALID_ARG;
    const int64_t xb = dtype_bytes(n->x_dtype);
    if ((s = check_rows(x, ldx, cols, n->x_dtype))) return s;
    if (has_f && (s = check_rows(f_bf16, ldf, cols, MXFP4_OUT_BF16))) return s;
    if (x_out && (s = check_rows(x_out, ldxo, cols, n->x_dtype))) return s;
    if (h_bf16 && (s = check_rows(h_bf16, ldh, cols, MXFP4_OUT_BF16))) return s;
    if (x_ckpt.codes && (s = check_ckpt(x_ckpt, rows, cols))) return s;
    if (f_ckpt.codes && (s = check_ckpt(f_ckpt, rows, cols))) return s;
    if (reinterpret_cast<uintptr_t>(stats) & 3u) return MXFP4_MISALIGNED;
    if (hq) {
        if (!hq->data || !hq->scales) return MXFP4_INVALID_ARG;
        if (hq->rows != rows || hq->cols != cols) return MXFP4_BAD_SHAPE;
        if (!aligned16(hq->data) || !aligned16(hq->scales)) return MXFP4_MISALIGNED;
    }
    const Span sx = span_of_rows(x, ldx, rows, cols, xb), sf = span_of_rows(f_bf16, ldf, rows, cols, 2);
    const Span so = span_of_rows(x_out, ldxo, rows, cols, xb), sh = span_of_rows(h_bf16, ldh, rows, cols, 2);
    if (!rows_over_or_apart(so, ldxo, xb, sx, ldx, xb) || !rows_over_or_apart(so, ldxo, xb, sf, ldf, 2) || !rows_over_or_apart(sh, ldh, 2, sx, ldx, xb) ||
        !rows_over_or_apart(sh, ldh, 2, sf, ldf, 2))
        return MXFP4_INVALID_ARG;
    Memory m;
    m.written(so), m.written(sh), m.read(sx), m.read(sf);
    const int over = m.writes, under = m.reads;
    for (const mxfp4_ckpt_t *c : {&x_ckpt, &f_ckpt})
        if (c->codes) m.written(c->codes, rows * cols), m.written(c->scales, rows * cols / 32);
    if (hq) m.written(hq->data, rows * cols / 2), m.written(hq->scales, (int64_t)mxfp4_scale_bytes(rows, cols));
    if (pre || post) m.written(stats, 16 * rows);
    read_plan(m, *n);
    if (!m.apart(over, under)) return MXFP4_INVALID_ARG;
    NormFwd p = {};
    const RowPlan plan = row_plan(cols, 0);
    p.warps = plan.warps(), p.teams = plan.teams;
    p.x = x, p.f = static_cast<const __nv_bfloat16 *>(f_bf16), p.xo = x_out, p.h = static_cast<__nv_bfloat16 *>(h_bf16);
    p.ldx = ldx, p.ldf = ldf, p.ldxo = ldxo, p.ldh = ldh;
    p.pre = side_of(n->pre), p.post = side_of(n->post);
    p.gate = n->gate, p.ldg = n->ld_gate, p.gate_fp32 = n->gate_dtype == MXFP4_OUT_FP32, p.several = n->gates > 1, p.wide = rows_on_32(x_out, ldxo);
    p.has_cw = n->gate || (post && n->post.weight) || (post && n->post.bias), p.has_cb = post && n->post.bias;
    p.rows_per_gate = (uint32_t)(n->gates > 1 ? rows / n->gates : rows);
    p.a = n->residual_scale, p.s = n->branch_scale, p.stats = stats;
    p.xc = {x_ckpt.codes, x_ckpt.scales, ckpt_tf_add(scale_mode)};
    p.fc = {f_ckpt.codes, f_ckpt.scales, ckpt_tf_add(scale_mode)};
    p.nblk4 = (int)ceil_div(cols / 32, 4);
    if (hq) p.hq = static_cast<uint8_t *>(hq->data), p.hq_scales = hq->scales, p.hq_tf_add = scale_mode == MXFP4_SCALE_FLOOR ? 0u : 63u;
    p.rows = rows, p.cols = (int)cols, p.nvec = (int)(cols / 8), p.dev_status = dev_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    MX_CHECK_CUDA(n->x_dtype == MXFP4_OUT_FP32 ? launch_norm_fwd<float>(p, plan, has_f, post, pre, st) : launch_norm_fwd<__nv_bfloat16>(p, plan, has_f, post, pre, st));
    return MXFP4_OK;
}

}  // extern "C"
