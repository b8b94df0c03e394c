// Building blocks of the 8-bit activation checkpoints (E4M3 codes, one E8M0 scale per 32 columns) and of the passes that write and
// read them.  A lane holds eight consecutive columns (16 bytes of bf16, 8 bytes of codes); four neighbouring lanes hold a group.
#pragma once
#include "common.cuh"

namespace mx {

// ---- pairs of FP32 values in one 64-bit register: an operation on a pair takes one issue slot (the passes have few to spare) ----
typedef unsigned long long f2;
__device__ __forceinline__ f2 f2_of(float a, float b)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void f2_to(f2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 f2_mul(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 f2_add(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 f2_fma(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float f2_sum(f2 v)
{
    float a, b;
    f2_to(v, a, b);
    return a + b;
}

// ---- loads and stores of eight consecutive elements as four pairs ----
__device__ __forceinline__ void unpack8(const uint4 &w, f2 (&o)[4])
{
    o[0] = f2_of(bf16lo(w.x), bf16hi(w.x));
    o[1] = f2_of(bf16lo(w.y), bf16hi(w.y));
    o[2] = f2_of(bf16lo(w.z), bf16hi(w.z));
    o[3] = f2_of(bf16lo(w.w), bf16hi(w.w));
}
__device__ __forceinline__ uint32_t pack2(f2 v)
{
    float a, b;
    f2_to(v, a, b);
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
__device__ __forceinline__ uint4 pack8(const f2 (&v)[4]) { return make_uint4(pack2(v[0]), pack2(v[1]), pack2(v[2]), pack2(v[3])); }

// What a lane has loaded of a row of type T (bf16 or float) and not converted yet.
template <class T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, bool = false) { a = ld_stream_16(p); }
    __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(f2 (&o)[4]) const { unpack8(a, o); }
};
template <> struct Raw8<float> {
    f2 v[4];
    __device__ __forceinline__ void load(const float *p, bool wide = false)       // (wide: see store8)
    {
        if (wide) {
            asm volatile("ld.global.L1::no_allocate.v4.b64 {%0, %1, %2, %3}, [%4];" : "=l"(v[0]), "=l"(v[1]), "=l"(v[2]), "=l"(v[3]) : "l"(p));
        } else {
            const uint4 a = ld_stream_16(p), b = ld_stream_16(p + 4);
            v[0] = (f2)a.y << 32 | a.x, v[1] = (f2)a.w << 32 | a.z, v[2] = (f2)b.y << 32 | b.x, v[3] = (f2)b.w << 32 | b.z;
        }
    }
    __device__ __forceinline__ void zero() { v[0] = v[1] = v[2] = v[3] = 0; }
    __device__ __forceinline__ void get(f2 (&o)[4]) const { o[0] = v[0], o[1] = v[1], o[2] = v[2], o[3] = v[3]; }
};
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const f2 (&v)[4]) { *reinterpret_cast<uint4 *>(p) = pack8(v); }
__device__ __forceinline__ void store8(float *p, const f2 (&v)[4])
{
    reinterpret_cast<ulonglong2 *>(p)[0] = make_ulonglong2(v[0], v[1]);
    reinterpret_cast<ulonglong2 *>(p)[1] = make_ulonglong2(v[2], v[3]);
}
// `wide`: the address is a multiple of 32 bytes.  Eight FP32 values then go in one access: as two, each would touch every 32-byte sector of
// the warp's kilobyte and the L2 would see all of them twice (x + f of 50432 x 1024 in FP32: 112 us that way).
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const f2 (&v)[4], bool) { store8(p, v); }
__device__ __forceinline__ void store8(float *p, const f2 (&v)[4], bool wide)
{
    if (wide) asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(v[0]), "l"(v[1]), "l"(v[2]), "l"(v[3]) : "memory");
    else store8(p, v);
}

// ---- the format ----
// E8M0 byte of a group from the bit pattern (sign cleared) of its largest magnitude, an FP32 number:
//   truncation-free: s = ceil(log2(M / 448)) = floor(log2 M) - 8 + [mantissa(M) > 1.75]
//   floor          : s = floor(log2 M) - 8
// M = 0 takes 1e-8: s = -35 in both; s >= -127.  Inf / NaN (bits >= 0x7F800000) are the caller's business.
__device__ __forceinline__ uint32_t ckpt_scale_byte(uint32_t amax_bits, uint32_t tf_add)
{
    const int b = (int)((amax_bits + tf_add) >> 23) - 8;
    return amax_bits ? (uint32_t)max(b, 0) : 92u;
}
__host__ __device__ __forceinline__ uint32_t ckpt_tf_add(int scale_mode) { return scale_mode == MXFP4_SCALE_FLOOR ? 0u : 0x1FFFFFu; }

// Eight values times `inv` -> eight E4M3 codes, to nearest even, saturating at 448.
__device__ __forceinline__ uint2 e4m3_x8(const f2 (&v)[4], float inv)
{
    const f2 i2 = f2_of(inv, inv);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        float a, b;
        f2_to(f2_mul(v[j], i2), a, b);
        uint16_t c;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(b), "f"(a));
        w[j] = c;
    }
    return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

// Eight codes times 2^s (NaN for the scale byte 0xFF).
__device__ __forceinline__ float ckpt_scale(uint32_t byte) { return byte == 0xFFu ? __uint_as_float(0x7FC00000u) : scale_from_byte(byte); }
__device__ __forceinline__ void e4m3_to8(const uint2 &c, float scale, f2 (&o)[4])
{
    const f2 s2 = f2_of(scale, scale);
    const uint32_t w[4] = {c.x & 0xFFFFu, c.x >> 16, c.y & 0xFFFFu, c.y >> 16};
#pragma unroll
    for (int j = 0; j < 4; j++) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w[j]));
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        o[j] = f2_mul(f2_of(f.x, f.y), s2);
    }
}

// Largest magnitude of a lane's eight values as a bit pattern (what is not finite compares as larger than everything finite).
__device__ __forceinline__ uint32_t amax8(const f2 (&v)[4])
{
    float a[8], m;
#pragma unroll
    for (int j = 0; j < 4; j++) f2_to(v[j], a[2 * j], a[2 * j + 1]);
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a[0]), "f"(a[1]), "f"(a[2]));       // a NaN gives 0x7FFFFFFF
    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(a[3]), "f"(a[4]));
    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(a[5]), "f"(a[6]));
    asm("max.NaN.abs.f32 %0, %0, %1, %1;" : "+f"(m) : "f"(a[7]));
    return __float_as_uint(m);
}
// ... and of its group of four lanes.  All lanes of the warp take part.
__device__ __forceinline__ uint32_t group_max4(uint32_t m)
{
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    return max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
}

// Where a checkpoint is written.  A lane passes the bit pattern of its group's largest magnitude, its eight values and its place.
struct CkptOut {
    uint8_t *codes, *scales;
    uint32_t tf_add;
};
// (`at`: which eight columns of the whole matrix, counted along its rows.)
__device__ __forceinline__ bool ckpt_write(const CkptOut &o, uint32_t amax_bits, const f2 (&v)[4], int64_t at)
{
    const bool bad = amax_bits >= 0x7F800000u;
    const uint32_t byte = bad ? 0xFFu : ckpt_scale_byte(amax_bits, o.tf_add);
    uint2 c = e4m3_x8(v, __uint_as_float((254u - byte) << 23));
    if (bad) c = make_uint2(0, 0);
    *reinterpret_cast<uint2 *>(o.codes + at * 8) = c;
    if ((at & 3) == 0) o.scales[at >> 2] = (uint8_t)byte;
    return bad;
}

// Where one is read: a lane's codes and its group's scale byte.
struct RawCkpt {
    uint2 c;
    uint32_t s;
    __device__ __forceinline__ void load(const uint8_t *codes, const uint8_t *scales, int64_t at)
    {
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(c.x), "=r"(c.y) : "l"(codes + at * 8));
        s = scales[at >> 2];
    }
    __device__ __forceinline__ void zero() { c = make_uint2(0, 0), s = 0; }
    __device__ __forceinline__ void get(f2 (&o)[4]) const { e4m3_to8(c, ckpt_scale(s), o); }
};

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// Whether every eighth element of every row of an FP32 matrix lies on 32 bytes.
inline bool rows_on_32(const void *p, int64_t ld) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * 4)) & 31u) == 0; }
inline int64_t dtype_bytes(int dtype) { return dtype == MXFP4_OUT_FP32 ? 4 : 2; }
inline Span span_of_rows(const void *p, int64_t ld, int64_t rows, int64_t cols, int64_t bytes) { return span_of(p, p && rows > 0 ? bytes * ((rows - 1) * ld + cols) : 0); }

// What a call writes and what it reads.  A thread reads and writes in an order of its own, so that written memory has to lie apart from all other.
struct Memory {
    Span w[9], r[13];
    int writes = 0, reads = 0;

    void written(const void *p, int64_t bytes) { if (p) w[writes++] = span_of(p, bytes); }
    void written(const Span &s) { if (s.hi) w[writes++] = s; }
    void read(const void *p, int64_t bytes) { if (p) r[reads++] = span_of(p, bytes); }
    void read(const Span &s) { if (s.hi) r[reads++] = s; }
    // `over`: the first so many of the written may lie over the first `under` of the read (that is the caller's to check)
    bool apart(int over = 0, int under = 0) const
    {
        for (int i = 0; i < writes; i++) {
            for (int k = 0; k < i; k++)
                if (meet(w[i], w[k])) return false;
            for (int k = i < over ? under : 0; k < reads; k++)
                if (meet(w[i], r[k])) return false;
        }
        return true;
    }
};

// A row-major matrix argument: a present pointer on 16 bytes, rows that do not overlap and start on 16 bytes.
inline mxfp4_status_t check_rows(const void *p, int64_t ld, int64_t cols, int dtype)
{
    if (!p) return MXFP4_INVALID_ARG;
    if (ld < cols) return MXFP4_BAD_SHAPE;
    return !aligned16(p) || (ld * dtype_bytes(dtype)) % 16 != 0 ? MXFP4_MISALIGNED : MXFP4_OK;
}
inline mxfp4_status_t check_ckpt(const mxfp4_ckpt_t &c, int64_t rows, int64_t cols)
{
    if (!c.codes || !c.scales) return MXFP4_INVALID_ARG;
    if (c.rows != rows || c.cols != cols) return MXFP4_BAD_SHAPE;
    return aligned16(c.codes) ? MXFP4_OK : MXFP4_MISALIGNED;
}

}  // namespace mx
