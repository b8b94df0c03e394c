// Residual addition between two norms, forward.
#include "norm.cuh"

namespace mx {

struct NormFwd {
    const void *x;
    const __nv_bfloat16 *f;
    void *xo;
    __nv_bfloat16 *h;
    int64_t ldx, ldf, ldxo, ldh;
    NormSide pre, post;
    const void *gate;
    int64_t ldg;
    uint32_t rows_per_gate;
    int gate_fp32;
    float a, s;
    float *stats;
    CkptOut xc, fc;
    uint8_t *hq, *hq_scales;
    uint32_t hq_tf_add;
    int nblk4;
    int64_t rows, rows_per_team;
    int cols, nvec, log2_lanes;
    uint32_t *dev_status;
};

// mean and 1 / sqrt(var + eps) of the row that the lanes hold (zeros behind its end), by two passes; then the row is normalized.
// `have`: vectors that this lane holds of the row (all, where it is FULL).
template <int V, bool FULL>
__device__ __forceinline__ void normalize(Team &t, const NormSide &n, float inv, int have, f2 (&v)[V][4], float &mean, float &rstd)
{
    float s[1];
    mean = 0.0f;
    if (!n.rms) {
        f2 acc[V];
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] = f2_add(f2_add(v[i][0], v[i][1]), f2_add(v[i][2], v[i][3]));
#pragma unroll
        for (int i = 1; i < V; i++) acc[0] = f2_add(acc[0], acc[i]);
        s[0] = f2_sum(acc[0]);
        team_sum(t, s);
        mean = s[0] * inv;
        const f2 m2 = f2_of(-mean, -mean);
#pragma unroll
        for (int i = 0; i < V; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) v[i][j] = FULL || i < have ? f2_add(v[i][j], m2) : 0ull;     // zeros behind the row's end stay zeros
    }
    f2 acc[V];
#pragma unroll
    for (int i = 0; i < V; i++) {
        acc[i] = f2_mul(v[i][0], v[i][0]);
#pragma unroll
        for (int j = 1; j < 4; j++) acc[i] = f2_fma(v[i][j], v[i][j], acc[i]);
    }
#pragma unroll
    for (int i = 1; i < V; i++) acc[0] = f2_add(acc[0], acc[i]);
    s[0] = f2_sum(acc[0]);
    team_sum(t, s);
    rstd = 1.0f / sqrtf(s[0] * inv + n.eps);
    const f2 r2 = f2_of(rstd, rstd);
#pragma unroll
    for (int i = 0; i < V; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) v[i][j] = f2_mul(v[i][j], r2);
}

// The checkpoint of the row.  `n`: vectors of this lane that are written.
template <int V>
__device__ __forceinline__ bool row_ckpt(const CkptOut &o, const Team &t, int n, const f2 (&v)[V][4], int64_t row, int nvec)
{
    uint32_t m[V];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < V; i++) m[i] = amax8(v[i]);
#pragma unroll
    for (int i = 0; i < V; i++) m[i] = group_max4(m[i]);
#pragma unroll
    for (int i = 0; i < V; i++)
        if (i < n) bad |= ckpt_write(o, m[i], v[i], row * nvec + i * t.lanes + t.lane);
    return bad;
}

template <class XT, int V, bool HAS_F> struct FwdRing {
    static constexpr int kF = kSlots<XT> * V * kThreads * 16;                        // where f starts in a stage
    static constexpr int kStage = kF + (HAS_F ? V * kThreads * 16 : 0);
    static constexpr int kDepth = ring_depth(kStage, 0);
};

// x' = a x + f^ cw + cb with cw = s g w1 and cb = s g b1, h = x^ pw + pb: cw, cb, pw, pb stay in registers (cw and cb until the gate changes).
template <class XT, int V, bool FULL, bool HAS_F, bool POST, bool PRE>
__global__ void __launch_bounds__(kThreads, 1) k_norm_fwd(const __grid_constant__ NormFwd p)
{
    using Ring = FwdRing<XT, V, HAS_F>;
    constexpr int S = Ring::kDepth;
    __shared__ float4 s_sum[2 * 8];
    extern __shared__ __align__(128) uint8_t s_ring[];
    pdl_launch_dependents();
    Team t = make_team(p.log2_lanes, s_sum);
    const int64_t team = (int64_t)blockIdx.x * (kThreads >> p.log2_lanes) + t.id;
    const int64_t first = min(team * p.rows_per_team, p.rows), end = min(first + p.rows_per_team, p.rows);
    const int have = FULL ? V : max(0, min(V, (p.nvec - t.lane + t.lanes - 1) >> p.log2_lanes));   // vectors of this lane
    const float inv = 1.0f / (float)p.cols;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + threadIdx.x * 16;
    pdl_wait();

    const auto fetch = [&](int64_t row, uint32_t stage) {
        if (row < end) {
            const XT *x = static_cast<const XT *>(p.x) + row * p.ldx;
#pragma unroll
            for (int i = 0; i < V; i++)
                if (i < have) async_row8(stage + i * kSlots<XT> * kThreads * 16, x + (i * t.lanes + t.lane) * 8);
            if (HAS_F) {
                const __nv_bfloat16 *f = p.f + row * p.ldf;
#pragma unroll
                for (int i = 0; i < V; i++)
                    if (i < have) async_row8(stage + Ring::kF + i * kThreads * 16, f + (i * t.lanes + t.lane) * 8);
            }
        }
        async_commit();
    };
#pragma unroll
    for (int k = 0; k < S - 1; k++) fetch(first + k, ring + k * Ring::kStage);

    f2 pw[V][4], pb[V][4], cw[V][4], cb[V][4];
#pragma unroll
    for (int i = 0; i < V; i++) {
        zero8(pw[i]), zero8(pb[i]);
        if (PRE && i < have) load_side8(p.pre, i * t.lanes + t.lane, pw[i], pb[i]);
    }
    const auto new_gate = [&](int64_t gate) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            zero8(cw[i]), zero8(cb[i]);
            if (i < have) {
                const int vec = i * t.lanes + t.lane;
                f2 g[4];
#pragma unroll
                for (int j = 0; j < 4; j++) g[j] = f2_of(1.0f, 1.0f), cw[i][j] = g[j];
                if (POST) load_side8(p.post, vec, cw[i], cb[i]);
                if (p.gate) load_param8(p.gate, p.gate_fp32, gate * p.ldg + vec * 8, g);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    g[j] = f2_mul(g[j], f2_of(p.s, p.s));
                    cw[i][j] = f2_mul(cw[i][j], g[j]);
                    cb[i][j] = f2_mul(cb[i][j], g[j]);
                }
            }
        }
    };
    uint32_t gate = (uint32_t)first / p.rows_per_gate, left = p.rows_per_gate - ((uint32_t)first - gate * p.rows_per_gate);   // rows of this gate still to come
    if (HAS_F && first < end) new_gate(gate);

    bool bad = false;
    uint32_t slot = 0;
    const int64_t turns = turns_of(t, p.rows_per_team, first, end);
    for (int64_t k = 0; k < turns; k++) {
        const int64_t row = first + k;
        const bool live = row < end;
        fetch(row + S - 1, ring + (slot == 0 ? S - 1 : slot - 1) * Ring::kStage);
        const uint32_t stage = ring + slot * Ring::kStage;
        slot = slot == S - 1 ? 0 : slot + 1;
        if (HAS_F && live) {
            if (left == 0) new_gate(++gate), left = p.rows_per_gate;
            left--;
        }
        const int n = live ? have : 0;
        async_wait<S - 1>();
        f2 v[V][4];
        if (HAS_F) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (FULL || i < n) ring_row8<__nv_bfloat16>(stage + Ring::kF + i * kThreads * 16, v[i]);
                else zero8(v[i]);
            }
            if (POST) {
                float mean, rstd;
                normalize<V, FULL>(t, p.post, inv, n, v, mean, rstd);
                if (p.stats && live && t.lane == 0) p.stats[2 * p.rows + row] = mean, p.stats[3 * p.rows + row] = rstd;
            }
            if (p.fc.codes) bad |= row_ckpt(p.fc, t, n, v, row, p.nvec);
            const f2 a2 = f2_of(p.a, p.a);
#pragma unroll
            for (int i = 0; i < V; i++) {
                f2 xx[4];
                if (FULL || i < n) ring_row8<XT>(stage + i * kSlots<XT> * kThreads * 16, xx);
                else zero8(xx);
#pragma unroll
                for (int j = 0; j < 4; j++) v[i][j] = f2_fma(v[i][j], cw[i][j], f2_fma(xx[j], a2, cb[i][j]));
            }
            if (p.xo && live) {
                XT *o = static_cast<XT *>(p.xo) + row * p.ldxo;
#pragma unroll
                for (int i = 0; i < V; i++)
                    if (FULL || i < n) store8(o + (i * t.lanes + t.lane) * 8, v[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (FULL || i < n) ring_row8<XT>(stage + i * kSlots<XT> * kThreads * 16, v[i]);
                else zero8(v[i]);
            }
        }
        if (PRE) {
            float mean, rstd;
            normalize<V, FULL>(t, p.pre, inv, n, v, mean, rstd);
            if (p.stats && live && t.lane == 0) p.stats[row] = mean, p.stats[p.rows + row] = rstd;
            if (p.xc.codes) bad |= row_ckpt(p.xc, t, n, v, row, p.nvec);
            uint4 q[V];
#pragma unroll
            for (int i = 0; i < V; i++) {
#pragma unroll
                for (int j = 0; j < 4; j++) v[i][j] = f2_fma(v[i][j], pw[i][j], pb[i][j]);
                q[i] = pack8(v[i]);
            }
            if (p.h && live) {
                __nv_bfloat16 *o = p.h + row * p.ldh;
#pragma unroll
                for (int i = 0; i < V; i++)
                    if (FULL || i < n) *reinterpret_cast<uint4 *>(o + (i * t.lanes + t.lane) * 8) = q[i];
            }
            if (p.hq) {      // Q1 of the bf16 result, as the row-wise quantizer makes it
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const int vec = i * t.lanes + t.lane;
                    uint32_t am = absmax_fold(absmax_fold(absmax_fold(absmax_fold(0u, q[i].x), q[i].y), q[i].z), q[i].w);
                    am = group_max4(hmax_halves(absmax_fold_end(am)));
                    const bool odd = am >= 0x7F80u;
                    const uint32_t byte = odd ? 0xFFu : scale_byte_from_amax(am, p.hq_tf_add);
                    const uint32_t c = odd ? 0u : rne8(q[i], inv_scale_bf16x2(byte));
                    if (i < n) {
                        bad |= odd;
                        *reinterpret_cast<uint32_t *>(p.hq + row * (p.cols >> 1) + vec * 4) = c;
                        if ((vec & 3) == 0) p.hq_scales[scale_offset(row, vec >> 2, p.nblk4)] = (uint8_t)byte;
                    }
                }
            }
            if (p.hq && live) {          // the scales' padding: blocks to a multiple of 4, rows to one of 128
                const int nblk = p.cols >> 5;
                if (nblk + t.lane < p.nblk4 * 4) p.hq_scales[scale_offset(row, nblk + t.lane, p.nblk4)] = 0x7F;
                if (row == p.rows - 1)
                    for (int64_t r = p.rows; r & 127; r++)
                        for (int b = t.lane; b < p.nblk4 * 4; b += t.lanes) p.hq_scales[scale_offset(r, b, p.nblk4)] = 0x7F;
            }
        }
    }
    if (bad && p.dev_status) atomicOr(p.dev_status, MXFP4_DEV_NONFINITE);
}

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
        !rows_over_or_apart(sh, ldh, 2, sf, ldf, 2) || meet(so, sh))
        return MXFP4_INVALID_ARG;
    NormFwd p = {};
    const RowPlan plan = row_plan(rows, cols);
    p.log2_lanes = plan.log2_lanes, p.rows_per_team = plan.rows_per_team;
    p.x = x, p.f = static_cast<const __nv_bfloat16 *>(f_bf16), p.xo = x_out, p.h = static_cast<__nv_bfloat16 *>(h_bf16);
    p.ldx = ldx, p.ldf = ldf, p.ldxo = ldxo, p.ldh = ldh;
    p.pre = side_of(n->pre), p.post = side_of(n->post);
    p.gate = n->gate, p.ldg = n->ld_gate, p.gate_fp32 = n->gate_dtype == MXFP4_OUT_FP32;
    p.rows_per_gate = (uint32_t)(n->gates > 1 ? rows / n->gates : rows);
    p.a = n->residual_scale, p.s = n->branch_scale, p.stats = stats;
    p.xc = {x_ckpt.codes, x_ckpt.scales, ckpt_tf_add(scale_mode)};
    p.fc = {f_ckpt.codes, f_ckpt.scales, ckpt_tf_add(scale_mode)};
    p.nblk4 = (int)ceil_div(cols / 32, 4);
    if (hq) p.hq = static_cast<uint8_t *>(hq->data), p.hq_scales = hq->scales, p.hq_tf_add = scale_mode == MXFP4_SCALE_FLOOR ? 0u : 63u;
    p.rows = rows, p.cols = (int)cols, p.nvec = (int)(cols / 8), p.dev_status = dev_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    MX_CHECK_CUDA(with_row(n->x_dtype == MXFP4_OUT_FP32, plan, [&](auto xt, auto vv, auto full) {
        using XT = decltype(xt);
        constexpr int V = decltype(vv)::value;
        return with_bools(has_f, post, pre, [&](auto f, auto q, auto r) -> cudaError_t {
            constexpr bool F = decltype(f)::value, Q = decltype(q)::value, R = decltype(r)::value;
            if constexpr (!F && (Q || !R)) return cudaErrorInvalidValue;     // refused above
            else return launch_ring<k_norm_fwd<XT, V, decltype(full)::value, F, Q, R>, FwdRing<XT, V, F>::kDepth * FwdRing<XT, V, F>::kStage>(plan.blocks, st, p);
        });
    }));
    return MXFP4_OK;
}

}  // extern "C"
