// Residual addition between two norms, forward: the kernel.
//     x' = a x + s g (w1 f^ + b1),  h = w2 x^ + b2;  f^ and x^ normalized in registers, the mean first and then the deviation around it
// One read of x and f, one write of x', h and the checkpoints; per row four reductions over its lanes.  Bytes are the bound: x + f alone runs
// at the copy rate (50432 x 1024 in FP32 78.7 us, 6.56 TB/s), with a norm and its checkpoint at 0.94 of it (bf16, 75.6 us), with norms and
// checkpoints on both sides at 0.94 (FP32, RMS, 118 us) or, with layer norms and biases, 0.84 (1024 columns, 94 us: the reductions' latency
// and the planes' reads; 768 columns in three blocks per SM 73 us, 0.82).  25216 x 384 with a layer scale: 19.5 us of 14.9 (five rows for
// each team, a start and an end of 2 us each).
#pragma once
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
    int gate_fp32, several;     // several gates
    int gate_in_ring;
    int has_cw, has_cb;         // f^ has a factor other than s, a summand
    int stages;                 // of the ring
    int wide;                   // x' in FP32 lies on 32 bytes
    float a, s;
    float *stats;
    CkptOut xc, fc;
    uint8_t *hq, *hq_scales;
    uint32_t hq_tf_add;
    int nblk4;
    int64_t rows, rows_per_team;
    int cols, nvec, warps, teams;     // of a team; of a block
    uint32_t *dev_status;
};

// s / n, by 1 / n and the remainder; NaN where s is not finite, which the header promises of such a row
__device__ __forceinline__ float over(float s, float n, float inv)
{
    const float q = s * inv;
    return fmaf(fmaf(-q, n, s), inv, q);
}

// mean and 1 / sqrt(var + eps) of the row that the lanes hold (zeros behind its end), by two passes; the row is left without its mean.
// `have`: vectors that this lane holds of the row (all, where it is FULL).
template <int V, bool FULL, int L>
__device__ __forceinline__ void normalize(Team<L> &t, const NormSide &n, float cols, float inv, int have, f2 (&v)[V][4], float &mean, float &rstd)
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
        mean = over(s[0], cols, inv);
        const f2 m2 = f2_of(-mean, -mean);
#pragma unroll
        for (int i = 0; i < V; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) v[i][j] = always<V, FULL, L>(i) || i < have ? f2_add(v[i][j], m2) : 0ull;     // zeros behind the row's end stay zeros
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
    // to an ulp: every row of checkpoints that is a little off puts some codes on the other side of a border
    const float x = over(s[0], cols, inv) + n.eps, r = rsqrtf(x);
    rstd = x > 0.0f && x < __uint_as_float(0x7F800000u) ? fmaf(0.5f * r, fmaf(-x * r, r, 1.0f), r) : r;
}

constexpr float kFinite = 3.40282347e38f;

// The checkpoint of the row v r.  `n`: vectors of this lane that are written; `at`: where the lane's first one is, in eights of the matrix.
template <int V, bool FULL, int L>
__device__ __forceinline__ bool row_ckpt(const CkptOut &o, const Team<L> &t, int n, const f2 (&v)[V][4], float r, int64_t at)
{
    uint32_t m[V], byte[V], worst = 0;
    bool low = false;
    uint2 c[V];
#pragma unroll
    for (int i = 0; i < V; i++) m[i] = amax8(v[i]);
#pragma unroll
    for (int i = 0; i < V; i++) m[i] = __float_as_uint(__uint_as_float(group_max4(m[i])) * r);     // the largest |v r|: rounding keeps the order
#pragma unroll
    for (int i = 0; i < V; i++) {
        byte[i] = ckpt_scale_byte(m[i], o.tf_add);
        const float k = __uint_as_float((254u - byte[i]) << 23) * r;
        c[i] = e4m3_x8(v[i], k);
        worst = max(worst, m[i]);
        low |= k > kFinite;
    }
    if (worst >= 0x7F800000u || low) {      // aside, they cost the others one comparison: a group that is not finite, and one so small that 2^-s r overflows
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (__uint_as_float((254u - byte[i]) << 23) * r > kFinite) {
                f2 u[4];
#pragma unroll
                for (int j = 0; j < 4; j++) u[j] = f2_mul(v[i][j], f2_of(r, r));
                c[i] = e4m3_x8(u, __uint_as_float((254u - byte[i]) << 23));
            }
            if (m[i] >= 0x7F800000u) c[i] = make_uint2(0, 0), byte[i] = 0xFFu;
        }
    }
    if (n > 0) {
        uint8_t *codes = o.codes + at * 8, *scales = o.scales + (at >> 2);
#pragma unroll
        for (int i = 0; i < V; i++)
            if (always<V, FULL, L>(i) || i < n) {
                *reinterpret_cast<uint2 *>(codes + i * L * 8) = c[i];
                if ((t.lane & 3) == 0) scales[i * (L / 4)] = (uint8_t)byte[i];
            }
    }
    return n > 0 && worst >= 0x7F800000u;
}

template <class XT, int V, bool HAS_F> struct FwdRing {
    static constexpr int N = kFwdThreads;
    static constexpr int kF = kSlots<XT> * V * N * 16;                        // where f starts in a stage
    static constexpr int kG = kF + (HAS_F ? V * N * 16 : 0);                  // and, of several gates, the row's gate where there is room for it
    static constexpr int gate_bytes(bool fp32) { return V * N * (fp32 ? 32 : 16); }
};

// x' = a x + (f^ cw + cb) [g], h = x^ pw + pb; cw = s w1 and cb = s b1, with one gate s g w1 and s g b1: the block keeps them in shared
// memory as far as there are any (in registers they would leave room for eight warps instead of sixteen).
template <class XT, int L, int V, bool FULL, bool HAS_F, bool POST, bool PRE>
__global__ void __launch_bounds__(kFwdThreads, fwd_blocks_per_sm(V, sizeof(XT), POST, FULL)) k_norm_fwd(const __grid_constant__ NormFwd p)
{
    using Ring = FwdRing<XT, V, HAS_F>;
    constexpr int N = kFwdThreads;
    __shared__ float4 s_sum[2 * (N / 32)];
    extern __shared__ __align__(128) uint8_t s_ring[];
    pdl_launch_dependents();
    Team<L> t(p.warps, p.nvec, s_sum);
    const int64_t team = (int64_t)blockIdx.x * p.teams + t.id;
    // rows first, first + step, ...: what is read at a time lies side by side (401408 x 96: 73 us, with a run of rows for each team 98); where
    // gates come by way of L1 the block has a run of rows, for its teams to share them
    const bool runs = HAS_F && p.several && !p.gate_in_ring;
    const int64_t run = runs ? (int64_t)blockIdx.x * p.teams * p.rows_per_team : 0, end = runs ? min(run + p.teams * p.rows_per_team, p.rows) : p.rows;
    const int64_t step = runs ? p.teams : (int64_t)gridDim.x * p.teams, first = t.id < p.teams ? (runs ? run + t.id : team) : p.rows;
    const int have = FULL ? V : max(0, min(V, (t.part_vecs - t.lane + L - 1) / L));   // vectors of this lane
    const float inv = 1.0f / (float)p.cols;
    const int S = p.stages, stage_bytes = Ring::kG + (p.gate_in_ring ? Ring::gate_bytes(p.gate_fp32) : 0);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring);
    float4 *const plane_cw = reinterpret_cast<float4 *>(s_ring + S * stage_bytes), *const plane_cb = plane_cw + (p.has_cw ? 2 * p.nvec : 0);
    float4 *const plane_pw = plane_cb + (p.has_cb ? 2 * p.nvec : 0), *const plane_pb = plane_pw + (p.pre.w ? 2 * p.nvec : 0);
    pdl_wait();

    const XT *xp = static_cast<const XT *>(p.x) + first * p.ldx + t.first_vec * 8;       // of the row that is fetched next
    const __nv_bfloat16 *fp = HAS_F ? p.f + first * p.ldf + t.first_vec * 8 : nullptr;
    const auto fetch = [&](int64_t row, uint32_t stage) {
        if (row < end) {
#pragma unroll
            for (int i = 0; i < V; i++)
                async_row8<XT, L>(stage + i * kSlots<XT> * N * 16, xp + i * L * 8, always<V, FULL, L>(i) ? L : t.part_vecs - i * L);
            if (HAS_F) {
#pragma unroll
                for (int i = 0; i < V; i++)
                    async_row8<__nv_bfloat16, L>(stage + Ring::kF + i * N * 16, fp + i * L * 8, always<V, FULL, L>(i) ? L : t.part_vecs - i * L);
                fp += step * p.ldf;
            }
            xp += step * p.ldx;
            if (HAS_F && p.gate_in_ring) {
                const int64_t g = (int64_t)((uint32_t)row / p.rows_per_gate) * p.ldg + t.first_vec * 8;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    if (p.gate_fp32) async_row8<float, L>(stage + Ring::kG + i * N * 32, static_cast<const float *>(p.gate) + g + i * L * 8, always<V, FULL, L>(i) ? L : t.part_vecs - i * L);
                    else async_row8<__nv_bfloat16, L>(stage + Ring::kG + i * N * 16, static_cast<const __nv_bfloat16 *>(p.gate) + g + i * L * 8, always<V, FULL, L>(i) ? L : t.part_vecs - i * L);
                }
            }
        }
        async_commit();
    };
    // the parameters' loads go first: behind the rows' they would wait for all of them (2 us)
    f2 pw[4], pb[4], cw[4], cb[4], g[4];
    const auto get_params = [&](int vec) {
        if (PRE) load_side8(p.pre, vec, pw, pb);
        if (HAS_F && p.has_cw) load_side8(POST ? p.post : NormSide{}, vec, cw, cb);
#pragma unroll
        for (int j = 0; j < 4; j++) g[j] = f2_of(1.0f, 1.0f);
        if (HAS_F && p.gate && !p.several) load_param8(p.gate, p.gate_fp32, vec * 8, g);
    };
    if (threadIdx.x < p.nvec) get_params(threadIdx.x);
    for (int k = 0; k < S - 1; k++) fetch(first + k * step, ring + k * stage_bytes);

    for (int vec = threadIdx.x; vec < p.nvec; vec += N) {
        if (vec >= N) get_params(vec);
        if (PRE && p.pre.w) plane_put(plane_pw, p.nvec, vec, pw);
        if (PRE && p.pre.b) plane_put(plane_pb, p.nvec, vec, pb);
        if (HAS_F && p.has_cw) {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                g[j] = f2_mul(g[j], f2_of(p.s, p.s));
                cw[j] = f2_mul(cw[j], g[j]), cb[j] = f2_mul(cb[j], g[j]);
            }
            plane_put(plane_cw, p.nvec, vec, cw);
            if (p.has_cb) plane_put(plane_cb, p.nvec, vec, cb);
        }
    }
    __syncthreads();

    bool bad = false;
    int slot = 0;
    int64_t at = first * p.nvec + t.first_vec;      // this row's place in a checkpoint
    XT *xo = static_cast<XT *>(p.xo) + first * p.ldxo + t.first_vec * 8;
    __nv_bfloat16 *h = p.h + first * p.ldh + t.first_vec * 8;
    const int turns = turns_of<L>(end, first, step);
    for (int k = 0; k < turns; k++) {
        const int64_t row = first + k * step;
        const bool live = L == 32 || row < end;
        if (sizeof(XT) == 4 || (HAS_F && p.gate_in_ring)) warp_sync();      // the others have read what is overwritten
        fetch(row + (S - 1) * step, ring + (slot == 0 ? S - 1 : slot - 1) * stage_bytes);
        const uint32_t stage = ring + slot * stage_bytes;
        slot = slot == S - 1 ? 0 : slot + 1;
        const int n = live ? have : 0;
        async_wait_all_but(S - 1);
        if (sizeof(XT) == 4 || (HAS_F && p.gate_in_ring)) warp_sync();
        f2 v[V][4];
        float r = 1.0f;
        if (HAS_F) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (always<V, FULL, L>(i) || i < n) ring_row8<__nv_bfloat16>(stage + Ring::kF + i * N * 16, v[i]);
                else zero8(v[i]);
            }
            if (POST) {
                float mean;
                normalize<V, FULL, L>(t, p.post, (float)p.cols, inv, n, v, mean, r);
                if (p.stats && live && t.leader) p.stats[2 * p.rows + row] = mean, p.stats[3 * p.rows + row] = r;
            }
            if (p.fc.codes) bad |= row_ckpt<V, FULL, L>(p.fc, t, n, v, r, at);
            if (p.has_cw) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    f2 w[4];
                    if (always<V, FULL, L>(i) || i < have) plane_get(plane_cw, p.nvec, i * L + t.first_vec, w);
                    else zero8(w);
#pragma unroll
                    for (int j = 0; j < 4; j++) v[i][j] = f2_mul(v[i][j], w[j]);
                }
                if (p.has_cb) {
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        f2 w[4];
                        if (always<V, FULL, L>(i) || i < have) plane_get(plane_cb, p.nvec, i * L + t.first_vec, w);
                        else zero8(w);
#pragma unroll
                        for (int j = 0; j < 4; j++) v[i][j] = f2_fma(v[i][j], f2_of(r, r), w[j]);
                    }
                }
                if (p.has_cb) r = 1.0f;
                if (p.several) {
                    const int64_t gate = live ? (int64_t)((uint32_t)row / p.rows_per_gate) * p.ldg + t.first_vec * 8 : 0;
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        f2 g[4];
                        if (!((L == 32 && always<V, FULL, L>(i)) || i < n)) zero8(g);
                        else if (!p.gate_in_ring) load_param8(p.gate, p.gate_fp32, gate + i * L * 8, g);
                        else if (p.gate_fp32) ring_row8<float>(stage + Ring::kG + i * N * 32, g);
                        else ring_row8<__nv_bfloat16>(stage + Ring::kG + i * N * 16, g);
#pragma unroll
                        for (int j = 0; j < 4; j++) v[i][j] = f2_mul(v[i][j], g[j]);
                    }
                }
            } else {
                r *= p.s;
            }
            // x' = a x + r v
#pragma unroll
            for (int i = 0; i < V; i++) {
                f2 xx[4];
                if (always<V, FULL, L>(i) || i < n) ring_row8<XT>(stage + i * kSlots<XT> * N * 16, xx);
                else zero8(xx);
                if (p.a != 1.0f) {
#pragma unroll
                    for (int j = 0; j < 4; j++) xx[j] = f2_mul(xx[j], f2_of(p.a, p.a));
                }
#pragma unroll
                for (int j = 0; j < 4; j++) v[i][j] = f2_fma(v[i][j], f2_of(r, r), xx[j]);
            }
            if (p.xo && live) {
#pragma unroll
                for (int i = 0; i < V; i++)
                    if (always<V, FULL, L>(i) || i < n) store8(xo + i * L * 8, v[i], p.wide);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (always<V, FULL, L>(i) || i < n) ring_row8<XT>(stage + i * kSlots<XT> * N * 16, v[i]);
                else zero8(v[i]);
            }
        }
        if (PRE) {
            float mean;
            normalize<V, FULL, L>(t, p.pre, (float)p.cols, inv, n, v, mean, r);
            if (p.stats && live && t.leader) p.stats[row] = mean, p.stats[p.rows + row] = r;
            if (p.xc.codes) bad |= row_ckpt<V, FULL, L>(p.xc, t, n, v, r, at);
            if (p.pre.w) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    f2 w[4];
                    if (always<V, FULL, L>(i) || i < have) plane_get(plane_pw, p.nvec, i * L + t.first_vec, w);
                    else zero8(w);
#pragma unroll
                    for (int j = 0; j < 4; j++) v[i][j] = f2_mul(v[i][j], w[j]);
                }
            }
            if (p.pre.b) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    f2 w[4];
                    if (always<V, FULL, L>(i) || i < have) plane_get(plane_pb, p.nvec, i * L + t.first_vec, w);
                    else zero8(w);
#pragma unroll
                    for (int j = 0; j < 4; j++) v[i][j] = f2_fma(v[i][j], f2_of(r, r), w[j]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) v[i][j] = f2_mul(v[i][j], f2_of(r, r));
            }
            uint4 q[V];
#pragma unroll
            for (int i = 0; i < V; i++) q[i] = pack8(v[i]);
            if (p.h && live) {
#pragma unroll
                for (int i = 0; i < V; i++)
                    if (always<V, FULL, L>(i) || i < n) *reinterpret_cast<uint4 *>(h + i * L * 8) = q[i];
            }
            if (p.hq) {      // Q1 of the bf16 result, as the row-wise quantizer makes it
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const int vec = i * L + t.first_vec;
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
                if (nblk + t.first_vec < p.nblk4 * 4) p.hq_scales[scale_offset(row, nblk + t.first_vec, p.nblk4)] = 0x7F;      // three blocks at most
                if (row == p.rows - 1)
                    for (int64_t r = p.rows; r & 127; r++)
                        for (int b = t.lane; b < p.nblk4 * 4; b += L) p.hq_scales[scale_offset(r, b, p.nblk4)] = 0x7F;
            }
        }
        at += step * p.nvec, xo += step * p.ldxo, h += step * p.ldh;
    }
    if (bad && p.dev_status) atomicOr(p.dev_status, MXFP4_DEV_NONFINITE);
}

// Launches the kernel for rows of type XT.
template <class XT> cudaError_t launch_norm_fwd(NormFwd &p, const RowPlan &plan, bool has_f, bool post, bool pre, cudaStream_t st)
{
    const auto go = [&](auto l, auto v, auto full) {
        constexpr int L = decltype(l)::value, V = decltype(v)::value;
        return with_bools(has_f, post, pre, [&](auto f, auto q, auto r) -> cudaError_t {
            constexpr bool F = decltype(f)::value, Q = decltype(q)::value, R = decltype(r)::value;
            if constexpr ((!F && (Q || !R)) || !some_width_has(V, L, decltype(full)::value, false)) {
                return cudaErrorInvalidValue;     // refused by the caller, or no width's plan
            } else {
                const size_t planes = (size_t)(p.has_cw + p.has_cb + (R && p.pre.w) + (R && p.pre.b)) * p.cols * 4;
                // two stages in half of an SM's shared memory, or as many as there is room for in all of it (one at least: 128 KB of planes
                // and 48 KB).  The row's gate travels with them if that does not take the second block's place (50432 x 1024 in FP32: 144 us
                // with it and one block per SM, 127 with two and the gate by way of L1; 50432 x 768 with 256 gates 91 with it and two blocks, 85 with three)
                using Ring = FwdRing<XT, V, F>;
                constexpr bool FULL = decltype(full)::value;
                const auto fits = [&](size_t stage, size_t room) { return planes + 2 * stage <= room; };
                const size_t gate = p.several ? Ring::gate_bytes(p.gate_fp32) : 0;
                const bool three = fwd_blocks_per_sm(V, sizeof(XT), Q, FULL) == 3 && fits(Ring::kG, kThirdRingBytes);
                p.gate_in_ring = p.several && fits(Ring::kG + gate, three ? kThirdRingBytes : kHalfRingBytes);
                const size_t stage = Ring::kG + (p.gate_in_ring ? gate : 0);
                const int per_sm = three ? 3 : fits(stage, kHalfRingBytes) ? 2 : 1;
                const size_t room = per_sm == 3 ? kThirdRingBytes : per_sm == 2 ? kHalfRingBytes : kRingBytes;
                p.stages = (int)std::min<size_t>((room - planes) / stage, kMostStages);
                // 50432 x 768 with one, two, three, five times as many blocks as are resident 74, 68, 69, 75 us, 8192 x 4096 48, 45, 44, 48,
                // 25216 x 384 (five rows with one) 20.3, 24.8, 25.2, 25.2
                RowPlan b = plan;
                deal(b, p.rows, per_sm, 3);
                p.rows_per_team = b.rows_per_team;
                return launch_ring<k_norm_fwd<XT, L, V, FULL, F, Q, R>, kFwdThreads>(b.blocks, p.stages * stage + planes, st, p);
            }
        });
    };
    if (plan.v == 3) return with_lanes<3>(plan, [&](auto l, auto full) { return go(l, std::integral_constant<int, 3>(), full); });
    return with_lanes<4>(plan, [&](auto l, auto full) { return go(l, std::integral_constant<int, 4>(), full); });
}

}  // namespace mx
