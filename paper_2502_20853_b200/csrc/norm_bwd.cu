// Residual addition between two norms, backward: the entry points, the reduction of what the blocks leave, and the kernel for rows of bf16
// with checkpoints.
#include <algorithm>

#include "norm_bwd.cuh"

namespace mx {

template cudaError_t launch_norm_bwd<__nv_bfloat16, true>(const NormBwd &, const RowPlan &, bool, bool, bool, bool, bool, cudaStream_t);
extern template cudaError_t launch_norm_bwd<__nv_bfloat16, false>(const NormBwd &, const RowPlan &, bool, bool, bool, bool, bool, cudaStream_t);
extern template cudaError_t launch_norm_bwd<float, true>(const NormBwd &, const RowPlan &, bool, bool, bool, bool, bool, cudaStream_t);
extern template cudaError_t launch_norm_bwd<float, false>(const NormBwd &, const RowPlan &, bool, bool, bool, bool, bool, cudaStream_t);

struct NormBwdFinish {
    const float *part, *slots;
    NormSide post;
    const void *gate;
    int64_t ldg, gates;
    int gate_fp32, several;
    float s;
    int blocks, pre, use_f, has_post, sb, sa;
    int64_t rows, rows_per_gate, rows_per_block;
    int cols, slices;         // slices of 128 columns
    int warp_gates;           // a gate's slice is one warp's
    float *dw_pre, *db_pre, *dw_post, *db_post, *dgate;
};

__device__ __forceinline__ void add4(float4 &a, const float4 &b) { a.x += b.x, a.y += b.y, a.z += b.z, a.w += b.w; }
__device__ __forceinline__ float4 mul4(const float4 &a, const float4 &b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
__device__ __forceinline__ float4 all4(float v) { return make_float4(v, v, v, v); }
__device__ __forceinline__ float4 param4(const void *v, int fp32, int64_t at)
{
    if (fp32) return *reinterpret_cast<const float4 *>(static_cast<const float *>(v) + at);
    const uint2 u = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(v) + at);
    return make_float4(bf16lo(u.x), bf16hi(u.x), bf16lo(u.y), bf16hi(u.y));
}
__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }

// dg = s (w1 B + b1 A)
__device__ __forceinline__ float4 gate_gradient(const NormBwdFinish &p, int c, const float4 &B, const float4 &A)
{
    float4 o = B;
    if (p.has_post && p.post.w) o = mul4(o, param4(p.post.w, p.post.fp32, c));
    if (p.has_post && p.post.b) add4(o, mul4(A, param4(p.post.b, p.post.fp32, c)));
    return mul4(o, all4(p.s));
}

// Adds up what the blocks and teams have left, in a fixed order.  Two kinds of blocks: the first cols / 8 take 8 columns each, 2 lanes of
// 4 columns by 128 lanes of rows, for the sums over all rows; then, where there are several gates, one (or a warp of one) for each gate and 128 columns.
// 3 to 5 us with the launch, of which 1.5 pass before the other kernel's results are visible.
__global__ void __launch_bounds__(256) k_norm_bwd_finish(const __grid_constant__ NormBwdFinish p)
{
    __shared__ float4 s_v[8][4][2], s_g[8][2][32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if ((int)blockIdx.x < p.cols / 8) {
        const int q = threadIdx.x & 1, r = threadIdx.x >> 1, c = blockIdx.x * 8 + q * 4;
        float4 v[4] = {all4(0), all4(0), all4(0), all4(0)};     // of dh x^, dh, t f^ (with several gates times g), t (the same)
        const bool f = p.use_f && !p.several;
        // (a lane's few blocks all at once: one after the other each would take a trip to the L2)
        constexpr int kMost = (2 * kSms + 127) / 128;
        const bool slots = p.use_f && p.several && (p.dw_post || p.db_post);
        float4 part[kMost][4], w[kMost];
        uint32_t now[kMost], last[kMost];
#pragma unroll
        for (int i = 0; i < kMost; i++) {
            const int k = r + i * 128;
            const float *at = p.part + (int64_t)k * 4 * p.cols + c;
            const bool on = k < p.blocks;
#pragma unroll
            for (int j = 0; j < 4; j++) part[i][j] = all4(0);
            w[i] = all4(1), now[i] = 1, last[i] = 0;
            if (on && p.pre) part[i][0] = load4(at);
            if (on && p.sb) part[i][1] = load4(at + p.cols);
            if (on && f) part[i][2] = load4(at + 2 * p.cols);
            if (on && f && p.sa) part[i][3] = load4(at + 3 * p.cols);
            if (on && slots) {
                const int64_t first = k * p.rows_per_block, end = first + p.rows_per_block < p.rows ? first + p.rows_per_block : p.rows;
                now[i] = (uint32_t)first / (uint32_t)p.rows_per_gate, last[i] = (uint32_t)(end - 1) / (uint32_t)p.rows_per_gate;
                const float *s = p.slots + (int64_t)(k + now[i]) * 2 * p.cols + c;
                part[i][2] = load4(s);
                if (p.sa) part[i][3] = load4(s + p.cols);
                w[i] = param4(p.gate, p.gate_fp32, now[i] * p.ldg + c);
            }
        }
#pragma unroll
        for (int i = 0; i < kMost; i++) add4(v[0], part[i][0]), add4(v[1], part[i][1]), add4(v[2], mul4(part[i][2], w[i])), add4(v[3], mul4(part[i][3], w[i]));
        if (slots)
            for (bool more = true; more;) {      // the next gate of each of them
                more = false;
#pragma unroll
                for (int i = 0; i < kMost; i++) {
                    part[i][2] = part[i][3] = all4(0);
                    if (now[i]++ < last[i]) {
                        const float *s = p.slots + (int64_t)(r + i * 128 + now[i]) * 2 * p.cols + c;
                        part[i][2] = load4(s);
                        if (p.sa) part[i][3] = load4(s + p.cols);
                        w[i] = param4(p.gate, p.gate_fp32, now[i] * p.ldg + c);
                        more = true;
                    }
                }
#pragma unroll
                for (int i = 0; i < kMost; i++) add4(v[2], mul4(part[i][2], w[i])), add4(v[3], mul4(part[i][3], w[i]));
            }
#pragma unroll
        for (int i = 0; i < 4; i++) {
#pragma unroll
            for (int o = 2; o < 32; o <<= 1)
                add4(v[i], make_float4(__shfl_xor_sync(0xFFFFFFFFu, v[i].x, o), __shfl_xor_sync(0xFFFFFFFFu, v[i].y, o), __shfl_xor_sync(0xFFFFFFFFu, v[i].z, o),
                                       __shfl_xor_sync(0xFFFFFFFFu, v[i].w, o)));
            if (lane < 2) s_v[warp][i][lane] = v[i];
        }
        __syncthreads();
        if (threadIdx.x >= 2) return;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            v[i] = s_v[0][i][q];
#pragma unroll
            for (int k = 1; k < 8; k++) add4(v[i], s_v[k][i][q]);
        }
        const auto put = [&](float *out, const float4 &x) { if (out) *reinterpret_cast<float4 *>(out + c) = x; };
        put(p.dw_pre, v[0]), put(p.db_pre, v[1]);
        if (f) put(p.dgate, gate_gradient(p, c, v[2], v[3]));
        const float4 g = f && p.gate ? mul4(param4(p.gate, p.gate_fp32, c), all4(p.s)) : all4(p.s);
        put(p.dw_post, mul4(v[2], g)), put(p.db_post, mul4(v[3], g));
        return;
    }
    const int64_t job = p.warp_gates ? (int64_t)(blockIdx.x - p.cols / 8) * 8 + warp : blockIdx.x - p.cols / 8, g = job / p.slices;
    const int c = (int)(job - g * p.slices) * 128 + lane * 4;
    const bool on = g < p.gates && c < p.cols;
    const int64_t t0 = g * p.rows_per_gate / p.rows_per_block, t1 = ((g + 1) * p.rows_per_gate - 1) / p.rows_per_block;     // blocks
    const float *at = p.slots + (t0 + g) * 2 * (int64_t)p.cols + c;
    float4 B = all4(0), A = all4(0);
    if (p.warp_gates) {
        float4 part[2][4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            part[0][k] = on && t0 + k <= t1 ? load4(at + k * 2 * p.cols) : all4(0);
            part[1][k] = on && p.sa && t0 + k <= t1 ? load4(at + k * 2 * p.cols + p.cols) : all4(0);
        }
#pragma unroll
        for (int k = 0; k < 4; k++) add4(B, part[0][k]), add4(A, part[1][k]);
        if (!on) return;
    } else {
        if (on)
            for (int64_t k = warp; k <= t1 - t0; k += 8) {
                add4(B, load4(at + k * 2 * p.cols));
                if (p.sa) add4(A, load4(at + k * 2 * p.cols + p.cols));
            }
        s_g[warp][0][lane] = B, s_g[warp][1][lane] = A;
        __syncthreads();
        if (warp > 0 || !on) return;
#pragma unroll
        for (int k = 1; k < 8; k++) add4(B, s_g[k][0][lane]), add4(A, s_g[k][1][lane]);
    }
    *reinterpret_cast<float4 *>(p.dgate + g * p.cols + c) = gate_gradient(p, c, B, A);
}

}  // namespace mx

using namespace mx;

extern "C" {

size_t mxfp4_residual_norm_workspace_bytes(int64_t rows, int64_t cols, int64_t gates)
{
    if (rows <= 0 || cols <= 0 || cols > kNormMaxCols || gates < 0) return 0;
    int64_t most = 0;      // whichever gradients are asked for
    for (int sums = 2; sums <= 4; sums++) {
        const RowPlan b = bwd_plan(rows, cols, sums);
        most = std::max(most, part_floats(b, cols) + slot_floats(b, cols, gates));
    }
    return (size_t)most * 4;
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
    const bool sb = b->db_pre, sa = post && (b->db_post || (b->dgate && n->post.bias));
    const RowPlan plan = bwd_plan(rows, cols, 2 + sb + sa);
    const size_t needed = mxfp4_residual_norm_workspace_bytes(rows, cols, n->gates);
    if (workspace_bytes < needed) return MXFP4_WORKSPACE_TOO_SMALL;
    {
        // dx and df are written row by row while later rows are still to be read
        const Span dx = span_of_rows(b->dx, b->lddx, rows, cols, xb), df = span_of_rows(b->df_bf16, b->lddf, rows, cols, 2);
        const Span dxo = span_of_rows(b->dx_out, b->lddxo, rows, cols, xb), dh = span_of_rows(b->dh_bf16, b->lddh, rows, cols, 2);
        if (!rows_over_or_apart(dx, b->lddx, xb, dxo, b->lddxo, xb) || !rows_over_or_apart(dx, b->lddx, xb, dh, b->lddh, 2) ||
            !rows_over_or_apart(df, b->lddf, 2, dxo, b->lddxo, xb) || !rows_over_or_apart(df, b->lddf, 2, dh, b->lddh, 2))
            return MXFP4_INVALID_ARG;
        Memory m;
        m.written(dx), m.written(df), m.read(dxo), m.read(dh);
        const int over = m.writes, under = m.reads;
        for (const float *g : {b->dw_pre, b->db_pre, b->dw_post, b->db_post}) m.written(g, cols * 4);
        m.written(b->dgate, n->gates * cols * 4), m.written(workspace, (int64_t)needed);
        if (pre && eight) m.read(b->x_ckpt.codes, rows * cols), m.read(b->x_ckpt.scales, rows * cols / 32);
        if (need_f && eight) m.read(b->f_ckpt.codes, rows * cols), m.read(b->f_ckpt.scales, rows * cols / 32);
        if (pre && !eight) m.read(span_of_rows(b->x_out, b->ldxo, rows, cols, xb));
        if (need_f && !eight) m.read(span_of_rows(b->f_bf16, b->ldf, rows, cols, 2));
        if (pre || post) m.read(b->stats, 16 * rows);
        read_plan(m, *n);
        if (!m.apart(over, under)) return MXFP4_INVALID_ARG;
    }
    NormBwd p = {};
    p.dh = static_cast<const __nv_bfloat16 *>(b->dh_bf16), p.dxo = b->dx_out, p.lddh = b->lddh, p.lddxo = b->lddxo, p.stats = b->stats;
    p.xcodes = b->x_ckpt.codes, p.xscales = b->x_ckpt.scales, p.fcodes = b->f_ckpt.codes, p.fscales = b->f_ckpt.scales;
    p.xo = b->x_out, p.f = static_cast<const __nv_bfloat16 *>(b->f_bf16), p.ldxo = b->ldxo, p.ldf = b->ldf;
    p.dx = b->dx, p.df = static_cast<__nv_bfloat16 *>(b->df_bf16), p.lddx = b->lddx, p.lddf = b->lddf;
    p.pre = side_of(n->pre), p.post = side_of(n->post);
    p.gate = n->gate, p.ldg = n->ld_gate, p.gate_fp32 = n->gate_dtype == MXFP4_OUT_FP32;
    p.several = n->gates > 1, p.wide = rows_on_32(b->dx, b->lddx), p.rows_per_gate = (uint32_t)(n->gates > 1 ? rows / n->gates : rows);
    p.a = n->residual_scale, p.s = n->branch_scale;
    p.part = static_cast<float *>(workspace), p.slots = p.part + part_floats(plan, cols), p.heads = p.slots + ((int64_t)plan.blocks + n->gates) * 2 * cols;
    p.rows = rows, p.rows_per_team = plan.rows_per_team, p.cols = (int)cols, p.nvec = (int)(cols / 8), p.warps = plan.warps(), p.teams = plan.teams;
    const auto go = n->x_dtype == MXFP4_OUT_FP32 ? (eight ? launch_norm_bwd<float, true> : launch_norm_bwd<float, false>)
                                                 : (eight ? launch_norm_bwd<__nv_bfloat16, true> : launch_norm_bwd<__nv_bfloat16, false>);
    MX_CHECK_CUDA(go(p, plan, need_f, post, pre, sb, sa, st));
    if (!b->dw_pre && !b->db_pre && !b->dw_post && !b->db_post && !b->dgate) return MXFP4_OK;
    NormBwdFinish e = {};
    e.part = p.part, e.slots = p.slots, e.post = p.post, e.gate = p.gate, e.ldg = p.ldg, e.gate_fp32 = p.gate_fp32;
    e.gates = n->gates > 1 ? n->gates : 1, e.several = p.several, e.s = p.s, e.blocks = plan.blocks, e.pre = pre, e.use_f = need_f, e.has_post = post, e.sb = sb, e.sa = sa;
    e.rows = rows, e.rows_per_gate = p.rows_per_gate, e.rows_per_block = plan.rows_per_team * plan.teams, e.cols = (int)cols;
    e.slices = (int)ceil_div(cols, 128);
    e.dw_pre = b->dw_pre, e.db_pre = b->db_pre, e.dw_post = b->dw_post, e.db_post = b->db_post, e.dgate = b->dgate;
    // a warp takes a gate that at most four blocks have rows of, and eight warps one of more (47039 x 1024 with 2767 gates 158 us with eight for each, 99 so)
    e.warp_gates = e.rows_per_gate <= 3 * e.rows_per_block;
    const int64_t jobs = e.several && b->dgate ? e.gates * e.slices : 0, blocks = cols / 8 + (e.warp_gates ? ceil_div(jobs, 8) : jobs);
    MX_CHECK_CUDA(launch_pdl(k_norm_bwd_finish, (unsigned)blocks, 1, 256, 0, st, e));
    return MXFP4_OK;
}

}  // extern "C"
