// 8-bit checkpoints of activations, and the activation between two linear layers with the checkpoint that its backward pass reads.
// Single passes over memory: a thread takes eight columns at a time (16 bytes of bf16), four neighbouring lanes a group of 32; its two or four
// loads are under way together.  Bytes are the bound, with few issue slots to spare (77 % of them used): GELU with its checkpoint 50432 x 4096
// 179.5 us (one vector a thread 197, four 176), its gradient 25216 x 1536 34.5 (40, 36.5), SwiGLU's gradient 6311 x 2336 20.7, a
// checkpoint of 50432 x 768 20.3 (two 20.4, eight 22.4): 0.86 to 0.88 of the copy rate each.
#include "ckpt.cuh"
#include "quant_tile.cuh"

namespace mx {

constexpr int kEw = 256;    // threads per block of the element-wise passes

// Where the i-th eight columns of a [rows, nvec * 8] matrix with leading dimension ld start.
__device__ __forceinline__ int64_t row_of(int64_t i, int64_t nvec) { return (i | nvec) >> 32 ? i / nvec : (int64_t)((uint32_t)i / (uint32_t)nvec); }
__device__ __forceinline__ int64_t place(int64_t i, int64_t nvec, int64_t ld)
{
    if (ld == nvec * 8) return i * 8;
    const int64_t r = row_of(i, nvec);
    return r * ld + (i - r * nvec) * 8;
}

template <class T, int U>
__global__ void __launch_bounds__(kEw) k_ckpt_store(const T *src, int64_t ld, int64_t total, int64_t nvec, bool wide, const CkptOut out, uint32_t *dev_status)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t i0 = blockIdx.x * (int64_t)(kEw * U) + threadIdx.x;
    Raw8<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t i = i0 + u * kEw;
        raw[u].zero();
        if (i < total) raw[u].load(src + place(i, nvec, ld), wide);
    }
    bool bad = false;
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t i = i0 + u * kEw;
        f2 v[4];
        raw[u].get(v);
        const uint32_t m = group_max4(amax8(v));
        if (i < total) bad |= ckpt_write(out, m, v, i);
    }
    if (bad && dev_status) atomicOr(dev_status, MXFP4_DEV_NONFINITE);
}

template <class T, int U>
__global__ void __launch_bounds__(kEw) k_ckpt_load(const uint8_t *codes, const uint8_t *scales, int64_t total, int64_t nvec, T *dst, int64_t ld, bool wide)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t i0 = blockIdx.x * (int64_t)(kEw * U) + threadIdx.x;
    RawCkpt raw[U];
#pragma unroll
    for (int u = 0; u < U; u++)
        if (i0 + u * kEw < total) raw[u].load(codes, scales, i0 + u * kEw);
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t i = i0 + u * kEw;
        if (i >= total) continue;
        f2 v[4];
        raw[u].get(v);
        store8(dst + place(i, nvec, ld), v, wide);
    }
}

// ---- activations, on pairs in FP32 ----------------------------------------------------------------
__device__ __forceinline__ f2 f2_abs(f2 v) { return v & 0x7FFFFFFF7FFFFFFFull; }
__device__ __forceinline__ f2 f2_ex2(f2 v)
{
    float a, b;
    f2_to(v, a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    return f2_of(a, b);
}
__device__ __forceinline__ f2 f2_all(float c) { return f2_of(c, c); }

// e = erfc(|y| / sqrt 2) / 2, the standard normal's tail beyond |y|, times 8 (see gelu_bf16x2)
__device__ __forceinline__ f2 tail8(f2 y) { return f2_ex2(gelu_tail_log2(f2_mul(f2_abs(y), f2_all(0.125f)))); }
// 1 / (1 + e^-y)
__device__ __forceinline__ f2 logistic(f2 y)
{
    float a, b;
    f2_to(f2_add(f2_ex2(f2_mul(y, f2_all(-1.44269504f))), f2_all(1.0f)), a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return f2_of(a, b);
}

__host__ __device__ constexpr bool act_is_gelu(int act) { return act == MXFP4_ACT_GELU || act == MXFP4_ACT_GEGLU; }
__host__ __device__ constexpr bool act_is_gated(int act) { return act == MXFP4_ACT_GEGLU || act == MXFP4_ACT_SWIGLU; }

// act(y) of a pair (VALUE) and act'(y) (SLOPE), from one logistic or one tail:
//   GELU  max(y, 0) - |y| e (no cancellation) and Phi(y) + y phi(y) with Phi = e or 1 - e by the sign
//   SiLU  y p and p (1 + y (1 - p))
// +Inf gives the value +Inf, NaN NaN.
template <int ACT, bool VALUE, bool SLOPE>
__device__ __forceinline__ void act_pair(f2 y, f2 &value, f2 &slope)
{
    if (!act_is_gelu(ACT)) {
        const f2 p = logistic(y);
        if (VALUE) value = f2_mul(y, p);
        if (SLOPE) slope = f2_mul(p, f2_fma(y, f2_fma(p, f2_all(-1.0f), f2_all(1.0f)), f2_all(1.0f)));
        return;
    }
    float a, b;
    f2_to(y, a, b);
    const f2 c = f2_of(fminf(fabsf(a), 3e38f), fminf(fabsf(b), 3e38f)), e8 = tail8(c);
    if (VALUE) value = f2_fma(f2_mul(c, f2_all(-0.125f)), e8, f2_of(a < 0.0f ? 0.0f : a, b < 0.0f ? 0.0f : b));     // a NaN stays
    if (SLOPE) {
        float e0, e1;
        f2_to(f2_mul(e8, f2_all(0.125f)), e0, e1);
        e0 = a > 0.0f ? 1.0f - e0 : e0, e1 = b > 0.0f ? 1.0f - e1 : e1;
        // phi(y) = 2^(-y^2 log2(e) / 2 - log2(2 pi) / 2)
        slope = f2_fma(y, f2_ex2(f2_fma(f2_mul(y, y), f2_all(-0.72134752f), f2_all(-1.32574806f))), f2_of(e0, e1));
    }
}

template <int ACT, int U>
__global__ void __launch_bounds__(kEw) k_act_fwd(const __nv_bfloat16 *y, int64_t ldy, int64_t total, int64_t nvec, __nv_bfloat16 *z, int64_t ldz, const CkptOut out,
                                                 uint32_t *dev_status)
{
    constexpr int H = act_is_gated(ACT) ? 2 : 1;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t i0 = blockIdx.x * (int64_t)(kEw * U) + threadIdx.x;
    uint4 raw[U][H];
    int64_t at[U][H];   // of the checkpoint
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t i = i0 + u * kEw;
        raw[u][0] = raw[u][H - 1] = make_uint4(0, 0, 0, 0);
        if (i < total) {
            if (H == 1) {
                at[u][0] = i;
                raw[u][0] = ld_stream_16(y + place(i, nvec, ldy));
            } else {
                const int64_t r = row_of(i, nvec), c = i - r * nvec;
                at[u][0] = i + r * nvec, at[u][H - 1] = at[u][0] + nvec;
                raw[u][0] = ld_stream_16(y + r * ldy + c * 8);
                raw[u][H - 1] = ld_stream_16(y + r * ldy + (c + nvec) * 8);
            }
        }
    }
    bool bad = false;
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t i = i0 + u * kEw;
        f2 v[H][4];
#pragma unroll
        for (int k = 0; k < H; k++) {
            unpack8(raw[u][k], v[k]);
            if (out.codes) {
                const uint32_t m = group_max4(amax8(v[k]));
                if (i < total) bad |= ckpt_write(out, m, v[k], at[u][k]);
            }
        }
        if (i < total && z) {
            uint4 q;
            if (ACT == MXFP4_ACT_GELU) {
                const uint4 w = raw[u][0];
                q = make_uint4(gelu_bf16x2(w.x), gelu_bf16x2(w.y), gelu_bf16x2(w.z), gelu_bf16x2(w.w));
            } else {
                f2 o[4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    f2 none;
                    act_pair<ACT, true, false>(v[0][j], o[j], none);
                    if (H == 2) o[j] = f2_mul(o[j], v[H - 1][j]);
                }
                q = pack8(o);
            }
            *reinterpret_cast<uint4 *>(z + place(i, nvec, ldz)) = q;
        }
    }
    if (bad && dev_status) atomicOr(dev_status, MXFP4_DEV_NONFINITE);
}

template <int ACT, int U>
__global__ void __launch_bounds__(kEw) k_act_bwd(const __nv_bfloat16 *dz, int64_t lddz, int64_t total, int64_t nvec, const uint8_t *codes, const uint8_t *scales,
                                                 __nv_bfloat16 *dy, int64_t lddy)
{
    constexpr int H = act_is_gated(ACT) ? 2 : 1;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t i0 = blockIdx.x * (int64_t)(kEw * U) + threadIdx.x;
    uint4 raw[U];
    RawCkpt ck[U][H];
    int64_t row[U];      // of a gated activation
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t i = i0 + u * kEw;
        row[u] = H == 2 ? row_of(i, nvec) : 0;
        if (i < total) {
            raw[u] = ld_stream_16(dz + (H == 2 ? row[u] * lddz + (i - row[u] * nvec) * 8 : place(i, nvec, lddz)));
            const int64_t at = H == 1 ? i : i + row[u] * nvec;
            ck[u][0].load(codes, scales, at);
            if (H == 2) ck[u][H - 1].load(codes, scales, at + nvec);
        }
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t i = i0 + u * kEw;
        if (i >= total) continue;
        f2 d[4], a[4], b[4], o[4], q[4];
        unpack8(raw[u], d);
        ck[u][0].get(a);
        if (H == 2) ck[u][H - 1].get(b);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            f2 value, slope;
            act_pair<ACT, H == 2, true>(a[j], value, slope);
            o[j] = f2_mul(H == 2 ? f2_mul(d[j], b[j]) : d[j], slope);
            if (H == 2) q[j] = f2_mul(d[j], value);
        }
        __nv_bfloat16 *p = dy + (H == 2 ? row[u] * lddy + (i - row[u] * nvec) * 8 : place(i, nvec, lddy));
        store8(p, o);
        if (H == 2) store8(p + nvec * 8, q);
    }
}

// An output may lie over an input exactly (a thread writes where it has read), or not at all.
static bool over_or_apart(const void *out, int64_t ldo, int64_t out_cols, const void *in, int64_t ldi, int64_t in_cols, int64_t rows)
{
    return !meet(span_of_rows(out, ldo, rows, out_cols, 2), span_of_rows(in, ldi, rows, in_cols, 2)) || (out_cols == in_cols && out == in && ldo == ldi);
}
static mxfp4_status_t blocks_of(int64_t total, int per_thread, unsigned *blocks)
{
    const int64_t n = ceil_div(total, (int64_t)kEw * per_thread);
    if (n > 0x7FFFFFFF) return MXFP4_BAD_SHAPE;
    *blocks = (unsigned)n;
    return MXFP4_OK;
}

}  // namespace mx

using namespace mx;

extern "C" {

mxfp4_status_t mxfp4_checkpoint_store(const void *src, int32_t dtype, int64_t ld, mxfp4_ckpt_t dst, int32_t scale_mode, uint32_t *dev_status, void *stream)
{
    if (dst.rows < 0 || dst.cols < 0 || (dtype != MXFP4_OUT_BF16 && dtype != MXFP4_OUT_FP32)) return MXFP4_INVALID_ARG;
    if (scale_mode != MXFP4_SCALE_TRUNCATION_FREE && scale_mode != MXFP4_SCALE_FLOOR) return MXFP4_INVALID_ARG;
    if (dst.cols % 32 != 0) return MXFP4_BAD_SHAPE;
    if (dst.rows == 0 || dst.cols == 0) return MXFP4_OK;
    mxfp4_status_t s;
    if ((s = check_rows(src, ld, dst.cols, dtype)) || (s = check_ckpt(dst, dst.rows, dst.cols))) return s;
    Memory m;
    m.written(dst.codes, dst.rows * dst.cols), m.written(dst.scales, dst.rows * dst.cols / 32), m.read(span_of_rows(src, ld, dst.rows, dst.cols, dtype_bytes(dtype)));
    if (!m.apart()) return MXFP4_INVALID_ARG;
    const int64_t nvec = dst.cols / 8, total = dst.rows * nvec;
    const CkptOut out = {dst.codes, dst.scales, ckpt_tf_add(scale_mode)};
    unsigned blocks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == MXFP4_OUT_FP32) {
        if ((s = blocks_of(total, 2, &blocks))) return s;
        MX_CHECK_CUDA(launch_pdl(k_ckpt_store<float, 2>, blocks, 1, kEw, 0, st, static_cast<const float *>(src), ld, total, nvec, rows_on_32(src, ld), out, dev_status));
    } else {
        if ((s = blocks_of(total, 4, &blocks))) return s;
        MX_CHECK_CUDA(launch_pdl(k_ckpt_store<__nv_bfloat16, 4>, blocks, 1, kEw, 0, st, static_cast<const __nv_bfloat16 *>(src), ld, total, nvec, false, out, dev_status));
    }
    return MXFP4_OK;
}

mxfp4_status_t mxfp4_checkpoint_load(mxfp4_ckpt_t src, void *dst, int32_t dtype, int64_t ld, void *stream)
{
    if (src.rows < 0 || src.cols < 0 || (dtype != MXFP4_OUT_BF16 && dtype != MXFP4_OUT_FP32)) return MXFP4_INVALID_ARG;
    if (src.cols % 32 != 0) return MXFP4_BAD_SHAPE;
    if (src.rows == 0 || src.cols == 0) return MXFP4_OK;
    mxfp4_status_t s;
    if ((s = check_rows(dst, ld, src.cols, dtype)) || (s = check_ckpt(src, src.rows, src.cols))) return s;
    Memory m;
    m.written(span_of_rows(dst, ld, src.rows, src.cols, dtype_bytes(dtype))), m.read(src.codes, src.rows * src.cols), m.read(src.scales, src.rows * src.cols / 32);
    if (!m.apart()) return MXFP4_INVALID_ARG;
    const int64_t nvec = src.cols / 8, total = src.rows * nvec;
    unsigned blocks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const uint8_t *codes = src.codes, *scales = src.scales;
    if ((s = blocks_of(total, 4, &blocks))) return s;
    if (dtype == MXFP4_OUT_FP32) MX_CHECK_CUDA(launch_pdl(k_ckpt_load<float, 4>, blocks, 1, kEw, 0, st, codes, scales, total, nvec, static_cast<float *>(dst), ld, rows_on_32(dst, ld)));
    else MX_CHECK_CUDA(launch_pdl(k_ckpt_load<__nv_bfloat16, 4>, blocks, 1, kEw, 0, st, codes, scales, total, nvec, static_cast<__nv_bfloat16 *>(dst), ld, false));
    return MXFP4_OK;
}

mxfp4_status_t mxfp4_act_fwd(const void *y_bf16, int64_t ldy, int64_t rows, int64_t cols, int32_t act, void *z_bf16, int64_t ldz, mxfp4_ckpt_t ckpt,
                             int32_t scale_mode, uint32_t *dev_status, void *stream)
{
    if (rows < 0 || cols < 0 || act < MXFP4_ACT_GELU || act > MXFP4_ACT_SWIGLU) return MXFP4_INVALID_ARG;
    if (scale_mode != MXFP4_SCALE_TRUNCATION_FREE && scale_mode != MXFP4_SCALE_FLOOR) return MXFP4_INVALID_ARG;
    if (cols % 32 != 0) return MXFP4_BAD_SHAPE;
    if (rows == 0 || cols == 0) return MXFP4_OK;        // (of empty tensors the addresses may be missing)
    if (!z_bf16 && !ckpt.codes) return MXFP4_INVALID_ARG;
    const bool gated = act_is_gated(act);
    const int64_t ycols = gated ? 2 * cols : cols;
    mxfp4_status_t s;
    if ((s = check_rows(y_bf16, ldy, ycols, MXFP4_OUT_BF16))) return s;
    if (z_bf16 && (s = check_rows(z_bf16, ldz, cols, MXFP4_OUT_BF16))) return s;
    if (ckpt.codes && (s = check_ckpt(ckpt, rows, ycols))) return s;
    Memory m;
    m.written(span_of_rows(z_bf16, ldz, rows, cols, 2)), m.read(span_of_rows(y_bf16, ldy, rows, ycols, 2));
    if (ckpt.codes) m.written(ckpt.codes, rows * ycols), m.written(ckpt.scales, rows * ycols / 32);
    if ((z_bf16 && !over_or_apart(z_bf16, ldz, cols, y_bf16, ldy, ycols, rows)) || !m.apart(z_bf16 != nullptr, 1)) return MXFP4_INVALID_ARG;
    const int64_t nvec = cols / 8, total = rows * nvec;
    const CkptOut out = {ckpt.codes, ckpt.scales, ckpt_tf_add(scale_mode)};
    unsigned blocks;
    if ((s = blocks_of(total, 2, &blocks))) return s;
    const auto go = [&](auto kernel) {
        return launch_pdl(kernel, blocks, 1, kEw, 0, static_cast<cudaStream_t>(stream), static_cast<const __nv_bfloat16 *>(y_bf16), ldy, total, nvec,
                          static_cast<__nv_bfloat16 *>(z_bf16), ldz, out, dev_status);
    };
    MX_CHECK_CUDA(act == MXFP4_ACT_GELU ? go(k_act_fwd<MXFP4_ACT_GELU, 2>) : act == MXFP4_ACT_SILU ? go(k_act_fwd<MXFP4_ACT_SILU, 2>)
                  : act == MXFP4_ACT_GEGLU ? go(k_act_fwd<MXFP4_ACT_GEGLU, 2>) : go(k_act_fwd<MXFP4_ACT_SWIGLU, 2>));
    return MXFP4_OK;
}

mxfp4_status_t mxfp4_act_bwd(const void *dz_bf16, int64_t lddz, mxfp4_ckpt_t ckpt, int32_t act, void *dy_bf16, int64_t lddy, void *stream)
{
    if (ckpt.rows < 0 || ckpt.cols < 0 || act < MXFP4_ACT_GELU || act > MXFP4_ACT_SWIGLU) return MXFP4_INVALID_ARG;
    const bool gated = act_is_gated(act);
    if (ckpt.cols % (gated ? 64 : 32) != 0) return MXFP4_BAD_SHAPE;
    const int64_t rows = ckpt.rows, cols = gated ? ckpt.cols / 2 : ckpt.cols;
    if (rows == 0 || cols == 0) return MXFP4_OK;
    mxfp4_status_t s;
    if ((s = check_rows(dz_bf16, lddz, cols, MXFP4_OUT_BF16)) || (s = check_rows(dy_bf16, lddy, ckpt.cols, MXFP4_OUT_BF16)) || (s = check_ckpt(ckpt, rows, ckpt.cols))) return s;
    Memory m;
    m.written(span_of_rows(dy_bf16, lddy, rows, ckpt.cols, 2)), m.read(ckpt.codes, rows * ckpt.cols), m.read(ckpt.scales, rows * ckpt.cols / 32);
    if (!over_or_apart(dy_bf16, lddy, ckpt.cols, dz_bf16, lddz, cols, rows) || !m.apart()) return MXFP4_INVALID_ARG;
    const int64_t nvec = cols / 8, total = rows * nvec;
    unsigned blocks;
    if ((s = blocks_of(total, 2, &blocks))) return s;
    const auto go = [&](auto kernel) {
        return launch_pdl(kernel, blocks, 1, kEw, 0, static_cast<cudaStream_t>(stream), static_cast<const __nv_bfloat16 *>(dz_bf16), lddz, total, nvec,
                          static_cast<const uint8_t *>(ckpt.codes), static_cast<const uint8_t *>(ckpt.scales), static_cast<__nv_bfloat16 *>(dy_bf16), lddy);
    };
    MX_CHECK_CUDA(act == MXFP4_ACT_GELU ? go(k_act_bwd<MXFP4_ACT_GELU, 2>) : act == MXFP4_ACT_SILU ? go(k_act_bwd<MXFP4_ACT_SILU, 2>)
                  : act == MXFP4_ACT_GEGLU ? go(k_act_bwd<MXFP4_ACT_GEGLU, 2>) : go(k_act_bwd<MXFP4_ACT_SWIGLU, 2>));
    return MXFP4_OK;
}

}  // extern "C"
