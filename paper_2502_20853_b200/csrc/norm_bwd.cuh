// Residual addition between two norms, backward: the kernel that goes over the rows.
//     t = dx' + r2 (d - mean d - x^ mean(d x^)), d = w2 dh;  dx = a t;  df = r1 (v - mean v - f^ mean(v f^)), v = s g w1 t
// One read of dh, dx', x^ and f^, one write of dx and df; two sums over each row's lanes at a time, and the sums over rows in registers.  With one
// norm it runs at 0.82 to 0.94 of the copy rate (50432 x 768 with biases 73 us, 50432 x 1024 RMS 75), with norms on both sides at 0.8 to 0.89 (50432 x
// 1024 layer norms 93 us in bf16, 125 in FP32; 0.55 to 0.7 where a row leaves lanes without work): the second sum of a row waits for the first, and
// the registers that hold the sums over rows leave eight to sixteen warps per SM.  Below some 40 000 rows the blocks' starts and sums tell, and
// the closing kernel (25216 x 768 between layer norms 41.5 us and 7.9, 0.6 of the copy rate).  Rows of more than 6144 columns have one team per block (6000 x
// 8192: 116 us, 0.65).
#pragma once
#include "norm.cuh"

namespace mx {

struct NormBwd {
    const __nv_bfloat16 *dh;
    const void *dxo;
    int64_t lddh, lddxo;
    const float *stats;
    const uint8_t *xcodes, *xscales, *fcodes, *fscales;
    const void *xo;
    const __nv_bfloat16 *f;
    int64_t ldxo, ldf;
    void *dx;
    __nv_bfloat16 *df;
    int64_t lddx, lddf;
    NormSide pre, post;
    const void *gate;
    int64_t ldg;
    uint32_t rows_per_gate;   // rows of one gate (all rows where there are not several)
    int gate_fp32;
    int wide;                 // dx in FP32 lies on 32 bytes
    int several;              // gates: A and B are kept apart by gate
    float a, s;
    float *part;              // [blocks][4][cols]: sums of dh x^, dh, t f^ (B), t (A)
    float *slots;             // several gates: [block + gate][2][cols]: B and A of a block's rows of a gate
    float *heads;             // and [team][2][cols]: of a team's rows of its first gate, where it goes on to another
    int64_t rows, rows_per_team;
    int cols, nvec, warps, teams;     // of a team; of a block
};

template <class XT, int V, int SUMS, bool EIGHT, bool NEED_F, bool PRE> struct BwdRing {
    // a stage: what is read of dx', dh, x^ (or x'), f^ (or f)
    static constexpr int N = bwd_threads(V, SUMS), kX = sizeof(XT) * 8, kRow = N * V;
    static constexpr int kDh = kX * kRow;
    static constexpr int kXh = kDh + (PRE ? 16 * kRow : 0);
    static constexpr int kFh = kXh + (PRE ? (EIGHT ? 8 : kX) * kRow : 0);
    static constexpr int kStage = kFh + (NEED_F ? (EIGHT ? 8 : 16) * kRow : 0);
    // behind the ring, also a lane's own: N_pre's weights, and s g w1 of the present gate, in FP32
    static constexpr int kW = PRE ? 32 * kRow : 0, kG = NEED_F ? 32 * kRow : 0;
    // and the fourth sum of four vectors, which the registers have no room for (21952 x 2048 between layer norms 175 us with 184 bytes of
    // spills, 93 so; 10944 x 4096 188, 104)
    static constexpr bool kKeepA = V < 4 || SUMS < 4;
    static constexpr int kA = kKeepA ? 0 : 32 * kRow;
    static constexpr int kRoom = (bwd_blocks_per_sm(V) == 2 ? kHalfRingBytes : kRingBytes) - kW - kG - kA;
    static constexpr int kDepth = kRoom / kStage < kMostStages ? kRoom / kStage : kMostStages;
    static constexpr int kSums = 6 * 4 * 8 * kRow;       // at the end: up to six sums per column for each warp (team)
    static constexpr int kBytes = kDepth * kStage + kW + kG + kA > kSums ? kDepth * kStage + kW + kG + kA : kSums;
};
template <int N> __device__ __forceinline__ void sts8(uint32_t slot, const f2 (&v)[4])
{
    asm volatile("st.shared.v2.u64 [%0], {%1, %2};" ::"r"(slot), "l"(v[0]), "l"(v[1]) : "memory");
    asm volatile("st.shared.v2.u64 [%0], {%1, %2};" ::"r"(slot + N * 16), "l"(v[2]), "l"(v[3]) : "memory");
}

// Each team keeps the sums over its rows of its lanes' columns in registers: of dh x^ and dh for N_pre's
// gradients, and of t f^ and t (t the gradient of x' in all) for those of N_post and the gate:  with g constant over the rows of a gate,
//     dg = s (w1 B + b1 A),   dw1 = s sum_g g B_g,   db1 = s sum_g g A_g,      B = sum t f^,  A = sum t.
// They go to memory once per block, A and B of several gates once per block and gate; k_norm_bwd_finish adds them up.
// SB, SA: the sums of dh and of t are wanted.
template <class XT, int L, int V, bool FULL, bool EIGHT, bool NEED_F, bool POST, bool PRE, bool SB, bool SA>
__global__ void __launch_bounds__(bwd_threads(V, 2 + SB + SA), bwd_blocks_per_sm(V)) k_norm_bwd(const __grid_constant__ NormBwd p)
{
    using Ring = BwdRing<XT, V, 2 + SB + SA, EIGHT, NEED_F, PRE>;
    constexpr int N = Ring::N, S = Ring::kDepth;
    __shared__ float4 s_sum[2 * (N / 32)];
    __shared__ uint2 s_gates[N / L < N / 32 ? N / 32 : N / L];     // each team's first and last gate
    extern __shared__ __align__(128) uint8_t s_ring[];
    pdl_launch_dependents();
    Team<L> t(p.warps, p.nvec, s_sum);
    const int64_t team = (int64_t)blockIdx.x * p.teams + t.id;
    // rows first, first + step, ...: side by side (see the forward pass), with several gates a run of rows for each team
    const int64_t first = t.id < p.teams ? min(p.several ? team * p.rows_per_team : team, p.rows) : p.rows, end = p.several ? min(first + p.rows_per_team, p.rows) : p.rows;
    const int64_t step = p.several ? 1 : (int64_t)gridDim.x * p.teams;
    const int have = FULL ? V : max(0, min(V, (t.part_vecs - t.lane + L - 1) / L));
    const float inv = 1.0f / (float)p.cols;
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(s_ring);
    const uint32_t at16 = threadIdx.x * 16, at8 = threadIdx.x * 8;
    pdl_wait();

    // the lane's places in the row that is fetched next
    const XT *dxo_at = static_cast<const XT *>(p.dxo) + first * p.lddxo + t.first_vec * 8, *xo_at = static_cast<const XT *>(p.xo) + first * p.ldxo + t.first_vec * 8;
    const __nv_bfloat16 *dh_at = p.dh + first * p.lddh + t.first_vec * 8, *f_at = p.f + first * p.ldf + t.first_vec * 8;
    const uint8_t *xc_at = p.xcodes + first * p.cols + t.first_vec * 8, *fc_at = p.fcodes + first * p.cols + t.first_vec * 8;
    const auto fetch = [&](int64_t row, uint32_t stage) {
        if (row < end) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const int l = always<V, FULL, L>(i) ? L : t.part_vecs - i * L;
                if (p.dxo) async_row8<XT, L>(stage + i * kSlots<XT> * N * 16, dxo_at + i * L * 8, l);
                if (PRE) {
                    async_row8<__nv_bfloat16, L>(stage + Ring::kDh + i * N * 16, dh_at + i * L * 8, l);
                    if (!EIGHT) async_row8<XT, L>(stage + Ring::kXh + i * kSlots<XT> * N * 16, xo_at + i * L * 8, l);
                    else if (always<V, FULL, L>(i) || i < have) async8(stage + Ring::kXh + at8 + i * N * 8, xc_at + i * L * 8);
                }
                if (NEED_F) {
                    if (!EIGHT) async_row8<__nv_bfloat16, L>(stage + Ring::kFh + i * N * 16, f_at + i * L * 8, l);
                    else if (always<V, FULL, L>(i) || i < have) async8(stage + Ring::kFh + at8 + i * N * 8, fc_at + i * L * 8);
                }
            }
            dxo_at += step * p.lddxo;
            if (PRE) dh_at += step * p.lddh;
            if (PRE && EIGHT) xc_at += step * p.cols;
            if (PRE && !EIGHT) xo_at += step * p.ldxo;
            if (NEED_F && EIGHT) fc_at += step * p.cols;
            if (NEED_F && !EIGHT) f_at += step * p.ldf;
        }
        async_commit();
    };
    // what is too small for the ring: statistics and scale bytes, one row ahead in registers
    float pm, pr, qm, qr;
    uint32_t xs[V], fs[V];
    const uint8_t *xs_at = p.xscales + first * (p.cols >> 5) + (t.first_vec >> 2), *fs_at = p.fscales + first * (p.cols >> 5) + (t.first_vec >> 2);
    const auto fetch_small = [&](int64_t row) {
        if (row >= end) return;
        if (PRE) pr = p.stats[p.rows + row];
        if (PRE && !EIGHT) pm = p.stats[row];
        if (POST) qr = p.stats[3 * p.rows + row];
        if (POST && !EIGHT) qm = p.stats[2 * p.rows + row];
        if (EIGHT) {
#pragma unroll
            for (int i = 0; i < V; i++)
                if (always<V, FULL, L>(i) || i < have) {
                    if (PRE) xs[i] = xs_at[i * (L / 4)];
                    if (NEED_F) fs[i] = fs_at[i * (L / 4)];
                }
            xs_at += step * (p.cols >> 5), fs_at += step * (p.cols >> 5);
        }
    };
    uint32_t gate = p.several ? (uint32_t)first / p.rows_per_gate : 0u;
    uint32_t left = p.several ? p.rows_per_gate - ((uint32_t)first - gate * p.rows_per_gate) : 0u;   // rows of this gate still to come
    pm = pr = qm = qr = 0.0f;
#pragma unroll
    for (int i = 0; i < V; i++) xs[i] = fs[i] = 0;
    // the parameters' loads go first: behind the rows' they would wait for all of them (2 us), and one after the other for each other
    f2 w1[V][4], w2[V][4], wg[V][4], none[4];
    const auto get_gate = [&](int64_t gate) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            zero8(w2[i]), zero8(wg[i]);
            if (i < have) {
                const int vec = i * L + t.first_vec;
                load_side8({POST ? p.post.w : nullptr, nullptr, p.post.fp32, 0, 0.0f}, vec, w2[i], none);
                if (p.gate) load_param8(p.gate, p.gate_fp32, gate * p.ldg + vec * 8, wg[i]);
            }
        }
    };
    if (PRE) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            zero8(w1[i]);
            if (i < have) load_side8({p.pre.w, nullptr, p.pre.fp32, 0, 0.0f}, i * L + t.first_vec, w1[i], none);
        }
    }
    if (NEED_F) get_gate(first < end ? gate : 0);
    fetch_small(first);
    if (!p.dxo) {       // nothing comes from further on: the slots stay zeros, each written by the lane that reads it (ring_row8), for no barrier follows
        for (int k = 0; k < S; k++)
#pragma unroll
            for (int i = 0; i < V; i++)
#pragma unroll
                for (int j = 0; j < kSlots<XT>; j++)
                    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(base + k * Ring::kStage + at16 * kSlots<XT> + (i * kSlots<XT> * N + j) * 16), "r"(0) : "memory");
    }
#pragma unroll
    for (int k = 0; k < S - 1; k++) fetch(first + k * step, base + k * Ring::kStage);

    const uint32_t w_at = base + S * Ring::kStage + at16, g_at = w_at + Ring::kW, a_at = g_at + Ring::kG;
    if (PRE) {
#pragma unroll
        for (int i = 0; i < V; i++) sts8<N>(w_at + i * N * 32, w1[i]);
    }
    const auto put_gate = [&]() {
#pragma unroll
        for (int i = 0; i < V; i++) {
#pragma unroll
            for (int j = 0; j < 4; j++) w2[i][j] = f2_mul(w2[i][j], f2_mul(p.gate ? wg[i][j] : f2_of(1.0f, 1.0f), f2_of(p.s, p.s)));
            sts8<N>(g_at + i * N * 32, w2[i]);
        }
    };

    f2 sw[V][4], sb[V][4], B[V][4], A[V][4];
#pragma unroll
    for (int i = 0; i < V; i++) zero8(sw[i]), zero8(sb[i]), zero8(B[i]), zero8(A[i]);
    const auto get_A = [&](int i) { if (!Ring::kKeepA) lds8f<N>(a_at + i * N * 32, A[i]); };
    const auto put_A = [&](int i) { if (!Ring::kKeepA) sts8<N>(a_at + i * N * 32, A[i]); };
#pragma unroll
    for (int i = 0; i < V; i++) put_A(i);
    if (NEED_F) put_gate();
    const uint32_t first_gate = gate;
    const auto flush = [&]() {     // the rows of a gate are done and the team goes on: its first one is left to the block's end, any other is whole
        float *o = gate == first_gate ? p.heads + team * 2 * p.cols : p.slots + ((int64_t)blockIdx.x + gate) * 2 * p.cols;
#pragma unroll
        for (int i = 0; i < V; i++)
            if (always<V, FULL, L>(i) || i < have) {
                const int c = (i * L + t.first_vec) * 8;
                store8(o + c, B[i]);
                get_A(i);
                if (SA) store8(o + p.cols + c, A[i]);
                zero8(B[i]), zero8(A[i]);
                put_A(i);
            }
    };

    uint32_t slot = 0;
    XT *dx = static_cast<XT *>(p.dx) + first * p.lddx + t.first_vec * 8;       // the lane's places in this row
    __nv_bfloat16 *df = p.df + first * p.lddf + t.first_vec * 8;
    const int turns = L < 32 ? (int)p.rows_per_team : first < end ? (int)((end - first + step - 1) / step) : 0;
    for (int k = 0; k < turns; k++, dx += step * p.lddx, df += step * p.lddf) {
        const int64_t row = first + k * step;
        const bool live = L == 32 || row < end;
        const int n = live ? have : 0;
        if (sizeof(XT) == 4) warp_sync();      // the others have read what is overwritten
        fetch(row + (S - 1) * step, base + (slot == 0 ? S - 1 : slot - 1) * Ring::kStage);
        const uint32_t stage = base + slot * Ring::kStage;
        slot = slot == S - 1 ? 0 : slot + 1;
        if (NEED_F && p.several && live) {
            if (left == 0) {
                flush();
                get_gate(++gate);
                put_gate();
                left = p.rows_per_gate;
            }
            left--;
        }
        const float pm0 = pm, pr0 = pr, qm0 = qm, qr0 = qr;
        float xsc[V], fsc[V];
#pragma unroll
        for (int i = 0; i < V; i++) xsc[i] = ckpt_scale(xs[i]), fsc[i] = ckpt_scale(fs[i]);
        fetch_small(row + step);
        async_wait<S - 1>();
        if (sizeof(XT) == 4) warp_sync();
        f2 xh[V][4], d[V][4];
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (PRE) {
                if (always<V, FULL, L>(i) || i < n) {
                    ring_row8<__nv_bfloat16>(stage + Ring::kDh + i * N * 16, d[i]);
                    if (EIGHT) {
                        e4m3_to8(lds8(stage + Ring::kXh + at8 + i * N * 8), xsc[i], xh[i]);
                    } else {
                        ring_row8<XT>(stage + Ring::kXh + i * kSlots<XT> * N * 16, xh[i]);
                        const f2 m2 = f2_of(-pm0, -pm0), r2 = f2_of(pr0, pr0);
#pragma unroll
                        for (int j = 0; j < 4; j++) xh[i][j] = f2_mul(f2_add(xh[i][j], m2), r2);
                    }
                } else {
                    zero8(d[i]), zero8(xh[i]);
                }
            }
        }
        if (L < 32 && PRE && !live) {       // what the ring holds for a row that is none: a lane of a team beside a longer one
#pragma unroll
            for (int i = 0; i < V; i++) zero8(d[i]), zero8(xh[i]);
        }
        float c[2] = {0, 0};
        if (PRE) {
            f2 c1[V], c2[V];
#pragma unroll
            for (int i = 0; i < V; i++) {
                f2 w[4];
                lds8f<N>(w_at + i * N * 32, w);
                c1[i] = c2[i] = 0;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    sw[i][j] = f2_fma(d[i][j], xh[i][j], sw[i][j]);
                    if (SB) sb[i][j] = f2_add(d[i][j], sb[i][j]);
                    d[i][j] = f2_mul(d[i][j], w[j]);
                    c1[i] = j ? f2_add(c1[i], d[i][j]) : d[i][j];
                    c2[i] = j ? f2_fma(d[i][j], xh[i][j], c2[i]) : f2_mul(d[i][j], xh[i][j]);
                }
            }
#pragma unroll
            for (int i = 1; i < V; i++) c1[0] = f2_add(c1[0], c1[i]), c2[0] = f2_add(c2[0], c2[i]);
            c[0] = f2_sum(c1[0]), c[1] = f2_sum(c2[0]);
            team_sum(t, c);
        }
        const float m1 = p.pre.rms ? 0.0f : -c[0] * inv, m2 = -c[1] * inv;
        // t = dx' + r (d + m1 + m2 x^)
        const f2 k1 = f2_of(m1 * pr0, m1 * pr0), k2 = f2_of(m2 * pr0, m2 * pr0), kr = f2_of(pr0, pr0);
        f2 e1[V], e2[V];
#pragma unroll
        for (int i = 0; i < V; i++) {
            const bool on = always<V, FULL, L>(i) ? live : i < n;
            f2 x[4];
            if (on) ring_row8<XT>(stage + i * kSlots<XT> * N * 16, x);
            else zero8(x);
            if (PRE && on) {
#pragma unroll
                for (int j = 0; j < 4; j++) x[j] = f2_add(x[j], f2_fma(d[i][j], kr, f2_fma(xh[i][j], k2, k1)));
            }
            if (on) {
                if (p.a == 1.0f) {
                    store8(dx + i * L * 8, x, p.wide);
                } else {
                    f2 y[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) y[j] = f2_mul(x[j], f2_of(p.a, p.a));
                    store8(dx + i * L * 8, y, p.wide);
                }
            }
            // the branch: from here on xh is f^, and d the gradient of f^, then of f
            e1[i] = e2[i] = 0;
            if (NEED_F) {
                if (!on) {
                    zero8(xh[i]);
                } else if (EIGHT) {
                    e4m3_to8(lds8(stage + Ring::kFh + at8 + i * N * 8), fsc[i], xh[i]);
                } else {
                    ring_row8<__nv_bfloat16>(stage + Ring::kFh + i * N * 16, xh[i]);
                    if (POST) {
                        const f2 n2 = f2_of(-qm0, -qm0), r2 = f2_of(qr0, qr0);
#pragma unroll
                        for (int j = 0; j < 4; j++) xh[i][j] = f2_mul(f2_add(xh[i][j], n2), r2);
                    }
                }
                f2 w[4];
                lds8f<N>(g_at + i * N * 32, w);
                get_A(i);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    B[i][j] = f2_fma(x[j], xh[i][j], B[i][j]);
                    if (SA) A[i][j] = f2_add(x[j], A[i][j]);
                    d[i][j] = f2_mul(x[j], w[j]);
                    if (POST) {
                        e1[i] = j ? f2_add(e1[i], d[i][j]) : d[i][j];
                        e2[i] = j ? f2_fma(d[i][j], xh[i][j], e2[i]) : f2_mul(d[i][j], xh[i][j]);
                    }
                }
                put_A(i);
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) d[i][j] = f2_mul(x[j], f2_of(p.s, p.s));
            }
        }
        if (NEED_F) {
            if (POST) {
#pragma unroll
                for (int i = 1; i < V; i++) e1[0] = f2_add(e1[0], e1[i]), e2[0] = f2_add(e2[0], e2[i]);
                float e[2] = {f2_sum(e1[0]), f2_sum(e2[0])};
                team_sum(t, e);
                const float n1 = p.post.rms ? 0.0f : -e[0] * inv, n2 = -e[1] * inv;
                const f2 a1 = f2_of(n1 * qr0, n1 * qr0), a2 = f2_of(n2 * qr0, n2 * qr0), r2 = f2_of(qr0, qr0);
#pragma unroll
                for (int i = 0; i < V; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) d[i][j] = f2_fma(d[i][j], r2, f2_fma(xh[i][j], a2, a1));
            }
        }
        if (p.df && live) {
#pragma unroll
            for (int i = 0; i < V; i++)
                if (always<V, FULL, L>(i) || i < n) store8(df + i * L * 8, d[i]);
        }
    }

    // the block's sums: teams of one warp by shuffles, then each warp's (team's) sums side by side in shared memory
    async_wait<0>();
#pragma unroll
    for (int i = 0; i < V; i++) get_A(i);
    __syncthreads();
    const int wide = p.warps * 32, parts = L < 32 ? N / 32 : p.teams, cols = p.cols;
    const bool in_team = L < 32 || t.id < p.teams;
    float *const mine = reinterpret_cast<float *>(s_ring) + (int64_t)(threadIdx.x / wide) * 4 * cols;
    const auto leave = [&](f2 (&v)[V][4], int which) {
#pragma unroll
        for (int i = 0; i < V; i++) {
#pragma unroll
            for (int o = L; o < 32; o <<= 1)
#pragma unroll
                for (int j = 0; j < 4; j++) v[i][j] = f2_add(v[i][j], __shfl_xor_sync(0xFFFFFFFFu, v[i][j], o));
            if (i < have && (threadIdx.x & 31) < L && in_team) store8(mine + which * cols + (i * L + t.first_vec) * 8, v[i]);
        }
    };
    const bool with_f = NEED_F && !p.several;
    if (PRE) leave(sw, 0);
    if (PRE && SB) leave(sb, 1);
    if (with_f) leave(B, 2);
    if (with_f && SA) leave(A, 3);
    float *const last = reinterpret_cast<float *>(s_ring) + (int64_t)parts * 4 * cols;     // [team][2][cols]: of each team's last gate
    if (NEED_F && p.several) {
        if (t.leader) s_gates[t.id] = make_uint2(first_gate, gate);
#pragma unroll
        for (int i = 0; i < V; i++)
            if ((always<V, FULL, L>(i) || i < have) && in_team) {
                float *o = last + (int64_t)t.id * 2 * cols + (i * L + t.first_vec) * 8;
                store8(o, B[i]);
                if (SA) store8(o + cols, A[i]);
            }
    }
    __syncthreads();
    float *part = p.part + (int64_t)blockIdx.x * 4 * cols;
    for (int c = threadIdx.x * 4; c < 4 * cols; c += N * 4) {
        const int which = c / cols;
        if (which < 2 ? !PRE || (which == 1 && !SB) : !with_f || (which == 3 && !SA)) continue;
        float4 v = make_float4(0, 0, 0, 0);
        for (int k = 0; k < parts; k++) {
            const float4 w = reinterpret_cast<const float4 *>(s_ring)[k * cols + c / 4];
            v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
        }
        *reinterpret_cast<float4 *>(part + c) = v;
    }
    if (NEED_F && p.several) {
        // along the block's teams: what they have of one gate follows each other, a team's first gate, (gates that are its own,) its last
        const int64_t row0 = (int64_t)blockIdx.x * p.teams * p.rows_per_team;
        const int with_rows = (int)min((int64_t)p.teams, (p.rows - row0 + p.rows_per_team - 1) / p.rows_per_team);
        for (int c = threadIdx.x * 4; c < (SA ? 2 : 1) * cols; c += N * 4) {
            float4 v = make_float4(0, 0, 0, 0);
            uint32_t now = s_gates[0].x;
            const auto add = [&](const float *at) {
                const float4 w = *reinterpret_cast<const float4 *>(at + c);
                v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
            };
            const auto put = [&](uint32_t next) {
                *reinterpret_cast<float4 *>(p.slots + ((int64_t)blockIdx.x + now) * 2 * cols + c) = v;
                v = make_float4(0, 0, 0, 0);
                now = next;
            };
            for (int k = 0; k < with_rows; k++) {
                const uint32_t a = s_gates[k].x, b = s_gates[k].y;
                if (a != now) put(a);
                if (b != a) add(p.heads + ((int64_t)blockIdx.x * p.teams + k) * 2 * cols), put(b);
                add(last + (int64_t)k * 2 * cols);
            }
            put(0);
        }
    }
}

// Launches the kernel for rows of type XT and x^, f^ from checkpoints (EIGHT) or made again.  `sb`, `sa`: whether the sums of dh and of t are wanted.
template <class XT, bool EIGHT> cudaError_t launch_norm_bwd(const NormBwd &p, const RowPlan &plan, bool need_f, bool post, bool pre, bool sb, bool sa, cudaStream_t st)
{
    const auto go = [&](auto l, auto v, auto full) {
        constexpr int L = decltype(l)::value, V = decltype(v)::value;
        return with_bools(need_f, post, pre, [&](auto f, auto q, auto r) -> cudaError_t {
            constexpr bool F = decltype(f)::value, Q = decltype(q)::value, R = decltype(r)::value;
            if constexpr ((Q && !F) || (!R && !F && EIGHT) || !some_width_has(V, L, decltype(full)::value, true)) {
                return cudaErrorInvalidValue;     // does not occur
            } else {
                return with_bools(sb, sa, false, [&](auto b, auto a, auto) -> cudaError_t {
                    constexpr bool B = decltype(b)::value, A = decltype(a)::value;
                    if constexpr ((B && !R) || (A && !Q)) return cudaErrorInvalidValue;     // does not occur
                    else
                        return launch_ring<k_norm_bwd<XT, L, V, decltype(full)::value, EIGHT, F, Q, R, B, A>, bwd_threads(V, 2 + B + A)>(
                            plan.blocks, BwdRing<XT, V, 2 + B + A, EIGHT, F, R>::kBytes, st, p);
                });
            }
        });
    };
    using L32 = std::integral_constant<int, 32>;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 3> three;
    const std::integral_constant<int, 4> four;
    if (plan.v == 2) return with_lanes<2>(plan, [&](auto l, auto full) { return go(l, two, full); });
    if (plan.v == 3) return with_lanes<3>(plan, [&](auto l, auto full) { return go(l, three, full); });
    return plan.full ? go(L32(), four, std::true_type()) : go(L32(), four, std::false_type());
}

}  // namespace mx
