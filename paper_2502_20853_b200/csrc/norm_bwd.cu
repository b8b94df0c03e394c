// Residual addition between two norms, backward.
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
    int several;              // gates: A and B are kept apart by gate
    float a, s;
    float *part;              // [blocks][4][cols]: sums of dh x^, dh, t f^ (B), t (A)
    float *slots;             // several gates: [team + gate][2][cols]: B and A of a team's rows of a gate
    int64_t rows, rows_per_team;
    int cols, nvec, log2_lanes;
};

template <class XT, int V, bool EIGHT, bool NEED_F, bool PRE> struct BwdRing {
    // a stage: what is read of dx', dh, x^ (or x'), f^ (or f)
    static constexpr int kX = sizeof(XT) * 8, kRow = kBwdThreads * V;
    static constexpr int kDh = kX * kRow;
    static constexpr int kXh = kDh + (PRE ? 16 * kRow : 0);
    static constexpr int kFh = kXh + (PRE ? (EIGHT ? 8 : kX) * kRow : 0);
    static constexpr int kStage = kFh + (NEED_F ? (EIGHT ? 8 : 16) * kRow : 0);
    // behind the ring, also a lane's own: N_pre's weights, and s g w1 of the present gate, in FP32
    static constexpr int kW = PRE ? 32 * kRow : 0, kG = NEED_F ? 32 * kRow : 0;
    static constexpr int kDepth = (kRingBytes - kW - kG) / kStage < kMostStages ? (kRingBytes - kW - kG) / kStage : kMostStages;
    static constexpr int kSums = 4 * 4 * 8 * kRow;       // at the end: four sums per column for each warp (team)
    static constexpr int kBytes = kDepth * kStage + kW + kG > kSums ? kDepth * kStage + kW + kG : kSums;
};
__device__ __forceinline__ void sts8(uint32_t slot, const f2 (&v)[4])
{
    asm volatile("st.shared.v2.u64 [%0], {%1, %2};" ::"r"(slot), "l"(v[0]), "l"(v[1]) : "memory");
    asm volatile("st.shared.v2.u64 [%0], {%1, %2};" ::"r"(slot + kBwdThreads * 16), "l"(v[2]), "l"(v[3]) : "memory");
}

// Each team takes a run of consecutive rows and keeps the sums over them of its lanes' columns in registers: of dh x^ and dh for N_pre's
// gradients, and of t f^ and t (t the gradient of x' in all) for those of N_post and the gate:  with g constant over the rows of a gate,
//     dg = s (w1 B + b1 A),   dw1 = s sum_g g B_g,   db1 = s sum_g g A_g,      B = sum t f^,  A = sum t.
// They go to memory once per block, A and B of several gates once per team and gate; k_norm_bwd_finish adds them up.  BIAS: the sums of
// dh and t are wanted (without biases they are not, and their registers are free).
template <class XT, int V, bool FULL, bool EIGHT, bool NEED_F, bool POST, bool PRE, bool BIAS>
__global__ void __launch_bounds__(kBwdThreads, 1) k_norm_bwd(const __grid_constant__ NormBwd p)
{
    using Ring = BwdRing<XT, V, EIGHT, NEED_F, PRE>;
    constexpr int N = kBwdThreads, S = Ring::kDepth;
    __shared__ float4 s_sum[2 * 8];
    extern __shared__ __align__(128) uint8_t s_ring[];
    pdl_launch_dependents();
    Team t = make_team(p.log2_lanes, s_sum);
    const int64_t team = (int64_t)blockIdx.x * (kBwdThreads >> p.log2_lanes) + t.id;
    const int64_t first = min(team * p.rows_per_team, p.rows), end = min(first + p.rows_per_team, p.rows);
    const int have = FULL ? V : max(0, min(V, (p.nvec - t.lane + t.lanes - 1) >> p.log2_lanes));
    const float inv = 1.0f / (float)p.cols;
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(s_ring);
    const uint32_t at16 = threadIdx.x * 16, at8 = threadIdx.x * 8;
    pdl_wait();

    const auto fetch = [&](int64_t row, uint32_t stage) {
        if (row < end) {
#pragma unroll
            for (int i = 0; i < V; i++)
                if (i < have) {
                    const int c = (i * t.lanes + t.lane) * 8;
                    if (p.dxo) async_row8<XT, N>(stage + at16 + i * kSlots<XT> * kBwdThreads * 16, static_cast<const XT *>(p.dxo) + row * p.lddxo + c);
                    if (PRE) {
                        async_row8<__nv_bfloat16, N>(stage + Ring::kDh + at16 + i * kBwdThreads * 16, p.dh + row * p.lddh + c);
                        if (EIGHT) async8(stage + Ring::kXh + at8 + i * kBwdThreads * 8, p.xcodes + row * p.cols + c);
                        else async_row8<XT, N>(stage + Ring::kXh + at16 + i * kSlots<XT> * kBwdThreads * 16, static_cast<const XT *>(p.xo) + row * p.ldxo + c);
                    }
                    if (NEED_F) {
                        if (EIGHT) async8(stage + Ring::kFh + at8 + i * kBwdThreads * 8, p.fcodes + row * p.cols + c);
                        else async_row8<__nv_bfloat16, N>(stage + Ring::kFh + at16 + i * kBwdThreads * 16, p.f + row * p.ldf + c);
                    }
                }
        }
        async_commit();
    };
    // what is too small for the ring: statistics and scale bytes, one row ahead in registers
    float pm, pr, qm, qr;
    uint32_t xs[V], fs[V];
    const auto fetch_small = [&](int64_t row) {
        if (row >= end) return;
        if (PRE) pr = p.stats[p.rows + row];
        if (PRE && !EIGHT) pm = p.stats[row];
        if (POST) qr = p.stats[3 * p.rows + row];
        if (POST && !EIGHT) qm = p.stats[2 * p.rows + row];
        if (EIGHT) {
#pragma unroll
            for (int i = 0; i < V; i++)
                if (i < have) {
                    const int64_t at = row * (p.cols >> 5) + ((i * t.lanes + t.lane) >> 2);
                    if (PRE) xs[i] = p.xscales[at];
                    if (NEED_F) fs[i] = p.fscales[at];
                }
        }
    };
#pragma unroll
    for (int k = 0; k < S - 1; k++) fetch(first + k, base + k * Ring::kStage);
    pm = pr = qm = qr = 0.0f;
#pragma unroll
    for (int i = 0; i < V; i++) xs[i] = fs[i] = 0;
    fetch_small(first);

    const uint32_t w_at = base + S * Ring::kStage + at16, g_at = w_at + Ring::kW;
    if (PRE) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            f2 w[4], none[4];
            zero8(w);
            if (i < have) load_side8({p.pre.w, nullptr, p.pre.fp32, 0, 0.0f}, i * t.lanes + t.lane, w, none);
            sts8(w_at + i * kBwdThreads * 32, w);
        }
    }
    const auto new_gate = [&](int64_t gate) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            f2 w[4], g[4];
            zero8(w);
            if (i < have) {
                const int vec = i * t.lanes + t.lane;
                load_side8({POST ? p.post.w : nullptr, nullptr, p.post.fp32, 0, 0.0f}, vec, w, g);
#pragma unroll
                for (int j = 0; j < 4; j++) g[j] = f2_of(1.0f, 1.0f);
                if (p.gate) load_param8(p.gate, p.gate_fp32, gate * p.ldg + vec * 8, g);
#pragma unroll
                for (int j = 0; j < 4; j++) w[j] = f2_mul(w[j], f2_mul(g[j], f2_of(p.s, p.s)));
            }
            sts8(g_at + i * kBwdThreads * 32, w);
        }
    };

    f2 sw[V][4], sb[V][4], B[V][4], A[V][4];
#pragma unroll
    for (int i = 0; i < V; i++) zero8(sw[i]), zero8(sb[i]), zero8(B[i]), zero8(A[i]);
    uint32_t gate = p.several ? (uint32_t)first / p.rows_per_gate : 0u;
    uint32_t left = p.several ? p.rows_per_gate - ((uint32_t)first - gate * p.rows_per_gate) : 0u;   // rows of this gate still to come
    if (NEED_F && first < end) new_gate(gate);
    const auto flush = [&]() {
        float *o = p.slots + (team + gate) * 2 * (int64_t)p.cols;
#pragma unroll
        for (int i = 0; i < V; i++)
            if (i < have) {
                const int c = (i * t.lanes + t.lane) * 8;
                store8(o + c, B[i]);
                if (BIAS) store8(o + p.cols + c, A[i]);
                zero8(B[i]), zero8(A[i]);
            }
    };

    uint32_t slot = 0;
    const int64_t turns = turns_of(t, p.rows_per_team, first, end);
    for (int64_t k = 0; k < turns; k++) {
        const int64_t row = first + k;
        const bool live = row < end;
        const int n = live ? have : 0;
        fetch(row + S - 1, base + (slot == 0 ? S - 1 : slot - 1) * Ring::kStage);
        const uint32_t stage = base + slot * Ring::kStage;
        slot = slot == S - 1 ? 0 : slot + 1;
        if (NEED_F && p.several && live) {
            if (left == 0) {
                flush();
                new_gate(++gate);
                left = p.rows_per_gate;
            }
            left--;
        }
        const float pm0 = pm, pr0 = pr, qm0 = qm, qr0 = qr;
        float xsc[V], fsc[V];
#pragma unroll
        for (int i = 0; i < V; i++) xsc[i] = ckpt_scale(xs[i]), fsc[i] = ckpt_scale(fs[i]);
        fetch_small(row + 1);
        async_wait<S - 1>();
        f2 xh[V][4], d[V][4];
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (PRE) {
                if (FULL || i < n) {
                    ring_row8<__nv_bfloat16, N>(stage + Ring::kDh + at16 + i * kBwdThreads * 16, d[i]);
                    if (EIGHT) {
                        e4m3_to8(lds8(stage + Ring::kXh + at8 + i * kBwdThreads * 8), xsc[i], xh[i]);
                    } else {
                        ring_row8<XT, N>(stage + Ring::kXh + at16 + i * kSlots<XT> * kBwdThreads * 16, xh[i]);
                        const f2 m2 = f2_of(-pm0, -pm0), r2 = f2_of(pr0, pr0);
#pragma unroll
                        for (int j = 0; j < 4; j++) xh[i][j] = f2_mul(f2_add(xh[i][j], m2), r2);
                    }
                } else {
                    zero8(d[i]), zero8(xh[i]);
                }
            }
        }
        if (FULL && PRE && !live) {       // what the ring holds for a row that is none: a lane of a team beside a longer one
#pragma unroll
            for (int i = 0; i < V; i++) zero8(d[i]), zero8(xh[i]);
        }
        float c[2] = {0, 0};
        if (PRE) {
            f2 c1[V], c2[V];
#pragma unroll
            for (int i = 0; i < V; i++) {
                f2 w[4];
                ring_row8<float, N>(w_at + i * kBwdThreads * 32, w);
                c1[i] = c2[i] = 0;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    sw[i][j] = f2_fma(d[i][j], xh[i][j], sw[i][j]);
                    if (BIAS) sb[i][j] = f2_add(d[i][j], sb[i][j]);
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
        const f2 k1 = f2_of(m1, m1), k2 = f2_of(m2, m2), kr = f2_of(pr0, pr0), ka = f2_of(p.a, p.a), ks = f2_of(p.s, p.s);
        f2 e1[V], e2[V];
        XT *const dx = static_cast<XT *>(p.dx) + row * p.lddx + t.lane * 8;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const bool on = FULL ? live : i < n;
            f2 x[4];
            zero8(x);
            if (p.dxo && on) ring_row8<XT, N>(stage + at16 + i * kSlots<XT> * N * 16, x);
            if (PRE && on) {
#pragma unroll
                for (int j = 0; j < 4; j++) x[j] = f2_fma(kr, f2_fma(xh[i][j], k2, f2_add(d[i][j], k1)), x[j]);
            }
            if (on) {
                f2 y[4];
#pragma unroll
                for (int j = 0; j < 4; j++) y[j] = f2_mul(x[j], ka);
                store8(dx + i * t.lanes * 8, y);
            }
            // the branch: from here on xh is f^, and d the gradient of f^, then of f
            e1[i] = e2[i] = 0;
            if (NEED_F) {
                if (!on) {
                    zero8(xh[i]);
                } else if (EIGHT) {
                    e4m3_to8(lds8(stage + Ring::kFh + at8 + i * N * 8), fsc[i], xh[i]);
                } else {
                    ring_row8<__nv_bfloat16, N>(stage + Ring::kFh + at16 + i * N * 16, xh[i]);
                    if (POST) {
                        const f2 n2 = f2_of(-qm0, -qm0), r2 = f2_of(qr0, qr0);
#pragma unroll
                        for (int j = 0; j < 4; j++) xh[i][j] = f2_mul(f2_add(xh[i][j], n2), r2);
                    }
                }
                f2 w[4];
                ring_row8<float, N>(g_at + i * N * 32, w);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    B[i][j] = f2_fma(x[j], xh[i][j], B[i][j]);
                    if (BIAS) A[i][j] = f2_add(x[j], A[i][j]);
                    d[i][j] = f2_mul(x[j], w[j]);
                    if (POST) {
                        e1[i] = j ? f2_add(e1[i], d[i][j]) : d[i][j];
                        e2[i] = j ? f2_fma(d[i][j], xh[i][j], e2[i]) : f2_mul(d[i][j], xh[i][j]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) d[i][j] = f2_mul(x[j], ks);
            }
        }
        if (NEED_F) {
            if (POST) {
#pragma unroll
                for (int i = 1; i < V; i++) e1[0] = f2_add(e1[0], e1[i]), e2[0] = f2_add(e2[0], e2[i]);
                float e[2] = {f2_sum(e1[0]), f2_sum(e2[0])};
                team_sum(t, e);
                const float n1 = p.post.rms ? 0.0f : -e[0] * inv, n2 = -e[1] * inv;
                const f2 a1 = f2_of(n1, n1), a2 = f2_of(n2, n2), r2 = f2_of(qr0, qr0);
#pragma unroll
                for (int i = 0; i < V; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) d[i][j] = f2_mul(r2, f2_fma(xh[i][j], a2, f2_add(d[i][j], a1)));
            }
        }
        if (p.df && live) {
            __nv_bfloat16 *o = p.df + row * p.lddf;
#pragma unroll
            for (int i = 0; i < V; i++)
                if (FULL || i < n) store8(o + (i * t.lanes + t.lane) * 8, d[i]);
        }
    }

    if (NEED_F && p.several && first < end) flush();
    // the block's sums: teams of one warp by shuffles, then each warp's (team's) sums side by side in shared memory
    async_wait<0>();
    __syncthreads();
    const int wide = max(t.lanes, 32);
    const int parts = kBwdThreads / wide, cols = p.cols;
    float *const mine = reinterpret_cast<float *>(s_ring) + (int64_t)(threadIdx.x / wide) * 4 * cols;
    const auto leave = [&](f2 (&v)[V][4], int which) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            for (int o = t.lanes; o < 32; o <<= 1)
#pragma unroll
                for (int j = 0; j < 4; j++) v[i][j] = f2_add(v[i][j], __shfl_xor_sync(0xFFFFFFFFu, v[i][j], o));
            if (i < have && (threadIdx.x & (wide - 1)) < t.lanes) store8(mine + which * cols + (i * t.lanes + t.lane) * 8, v[i]);
        }
    };
    const bool with_f = NEED_F && !p.several;
    if (PRE) leave(sw, 0);
    if (PRE && BIAS) leave(sb, 1);
    if (with_f) leave(B, 2);
    if (with_f && BIAS) leave(A, 3);
    __syncthreads();
    float *part = p.part + (int64_t)blockIdx.x * 4 * cols;
    for (int c = threadIdx.x * 4; c < 4 * cols; c += kBwdThreads * 4) {
        const int which = c / cols;
        if ((which & 1) > BIAS || (which < 2 ? !PRE : !with_f)) continue;
        float4 v = make_float4(0, 0, 0, 0);
        for (int k = 0; k < parts; k++) {
            const float4 w = reinterpret_cast<const float4 *>(s_ring)[k * cols + c / 4];
            v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
        }
        *reinterpret_cast<float4 *>(part + c) = v;
    }
}

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
    p.rows = rows, p.rows_per_team = plan.rows_per_team, p.cols = (int)cols, p.nvec = (int)(cols / 8), p.log2_lanes = plan.log2_lanes;
    const bool bias = b->db_pre || b->db_post || (n->gate && n->post.bias && post);
    MX_CHECK_CUDA(with_row(n->x_dtype == MXFP4_OUT_FP32, plan, [&](auto xt, auto vv, auto full) {
        using XT = decltype(xt);
        constexpr int V = decltype(vv)::value;
        return with_bools(eight, post, pre, [&](auto e, auto q, auto r) {
            constexpr bool E = decltype(e)::value, Q = decltype(q)::value, R = decltype(r)::value;
            return with_bools(need_f, bias, false, [&](auto nf, auto bi, auto) -> cudaError_t {
                constexpr bool F = decltype(nf)::value, B = decltype(bi)::value;
                if constexpr ((Q && !F) || (!R && !F && (B || E))) return cudaErrorInvalidValue;     // does not occur
                else return launch_ring<k_norm_bwd<XT, V, decltype(full)::value, E, F, Q, R, B>, kBwdThreads>(plan.blocks, BwdRing<XT, V, E, F, R>::kBytes, st, p);
            });
        });
    }));
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
