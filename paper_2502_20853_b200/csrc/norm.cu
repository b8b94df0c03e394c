// What stands between two branches of a transformer block: norm behind the branch, gate, residual addition, norm before the next branch,
// in one pass over the rows, forward and backward.
//
// A team of T lanes (a power of two from 4 to 256) holds a row in registers, each lane V vectors of eight columns: vector v * T + t.
// The sums over a row go through shuffles and, where a team has several warps, through shared memory and a barrier of the team.
// V is 3 or 4: with T a power of two these two reach every width within a third, and the usual widths (384 = 8 x 16 x 3, 768, 1024)
// exactly; long lanes keep the shuffles few (five for 768 or 1024 columns).
#include "ckpt.cuh"
#include "quant_tile.cuh"

namespace mx {

constexpr int kNormMaxCols = 8192;

// ---- teams --------------------------------------------------------------------------------------
struct Team {
    int lanes, lane;     // of the team
    int id;              // of the team in its block
    float4 *slots;       // several warps: where they leave their sums, two sets that take turns
    int turn;
};

__device__ __forceinline__ Team make_team(int log2_lanes, float4 *smem)
{
    Team t;
    t.lanes = 1 << log2_lanes;
    t.lane = threadIdx.x & (t.lanes - 1);
    t.id = threadIdx.x >> log2_lanes;
    t.slots = smem + t.id * 2 * (t.lanes >> 5);
    t.turn = 0;
    return t;
}

// The sums of N (1, 2) numbers over the lanes of the team, the same bits in each of them.  All lanes of the warp take part.
template <int N>
__device__ __forceinline__ void team_sum(Team &t, float (&v)[N])
{
    const int in_warp = min(t.lanes, 32);
    for (int o = in_warp >> 1; o; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; k++) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if (t.lanes > 32) {
        const int warps = t.lanes >> 5;
        float *s = reinterpret_cast<float *>(t.slots + t.turn * warps);
        t.turn ^= 1;     // a warp that is ahead writes the other set: nobody is more than one barrier ahead
        if ((t.lane & 31) == 0)
#pragma unroll
            for (int k = 0; k < N; k++) s[(t.lane >> 5) * 4 + k] = v[k];
        asm volatile("bar.sync %0, %1;" ::"r"(t.id + 1), "r"(t.lanes) : "memory");
#pragma unroll
        for (int k = 0; k < N; k++) v[k] = 0.0f;
        for (int w = 0; w < warps; w++)
#pragma unroll
            for (int k = 0; k < N; k++) v[k] += s[w * 4 + k];
    }
}

// ---- parameters ---------------------------------------------------------------------------------
struct NormSide {
    const void *w, *b;   // either may be missing
    int fp32;
    int rms;
    float eps;
};
__device__ __forceinline__ void load_param8(const void *p, int fp32, int64_t at, f2 (&o)[4])
{
    if (fp32) {
        const uint4 *q = reinterpret_cast<const uint4 *>(static_cast<const float *>(p) + at);
        const uint4 a = q[0], b = q[1];
        o[0] = (f2)a.y << 32 | a.x, o[1] = (f2)a.w << 32 | a.z, o[2] = (f2)b.y << 32 | b.x, o[3] = (f2)b.w << 32 | b.z;
    } else {
        unpack8(*reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p) + at), o);
    }
}

// ---- forward --------------------------------------------------------------------------------------
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
    int64_t rows;
    int cols, nvec, log2_lanes;
    uint32_t *dev_status;
};

// mean and 1 / sqrt(var + eps) of the row that the lanes hold (zeros behind its end), by two passes; then the row is normalized.
// `have`: vectors that this lane holds of the row.
template <int V>
__device__ __forceinline__ void normalize(Team &t, const NormSide &n, int cols, int have, f2 (&v)[V][4], float &mean, float &rstd)
{
    const float inv = 1.0f / (float)cols;
    float s[1];
    mean = 0.0f;
    if (!n.rms) {
        f2 acc = 0;
#pragma unroll
        for (int i = 0; i < V; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc = f2_add(acc, v[i][j]);
        s[0] = f2_sum(acc);
        team_sum(t, s);
        mean = s[0] * inv;
    }
    f2 acc = 0;
    const f2 m2 = f2_of(-mean, -mean);
#pragma unroll
    for (int i = 0; i < V; i++)
        if (i < have)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const f2 d = f2_add(v[i][j], m2);
                acc = f2_fma(d, d, acc);
            }
    s[0] = f2_sum(acc);
    team_sum(t, s);
    rstd = 1.0f / sqrtf(s[0] * inv + n.eps);
    const f2 r2 = f2_of(rstd, rstd);
#pragma unroll
    for (int i = 0; i < V; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) v[i][j] = i < have ? f2_mul(f2_add(v[i][j], m2), r2) : 0ull;     // zeros behind the row's end stay zeros
}

template <int V>
__device__ __forceinline__ void affine(const NormSide &n, int i, int vec, f2 (&v)[V][4])
{
    f2 w[4], b[4];
    if (n.w) {
        load_param8(n.w, n.fp32, (int64_t)vec * 8, w);
#pragma unroll
        for (int j = 0; j < 4; j++) v[i][j] = f2_mul(v[i][j], w[j]);
    }
    if (n.b) {
        load_param8(n.b, n.fp32, (int64_t)vec * 8, b);
#pragma unroll
        for (int j = 0; j < 4; j++) v[i][j] = f2_add(v[i][j], b[j]);
    }
}

// One row per team.
template <class XT, int V, bool HAS_F, bool POST, bool PRE>
__global__ void __launch_bounds__(256) k_norm_fwd(const __grid_constant__ NormFwd p)
{
    __shared__ float4 s_sum[2 * 16];
    pdl_launch_dependents();
    pdl_wait();
    Team t = make_team(p.log2_lanes, s_sum);
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x >> p.log2_lanes) + t.id;
    const bool live = row < p.rows;
    const int have = live ? max(0, min(V, (p.nvec - t.lane + t.lanes - 1) >> p.log2_lanes)) : 0;   // vectors of this lane
    const XT *x = static_cast<const XT *>(p.x) + row * p.ldx;
    Raw8<XT> rx[V];
    Raw8<__nv_bfloat16> rf[V];
#pragma unroll
    for (int i = 0; i < V; i++) {
        rx[i].zero(), rf[i].zero();
        if (i < have) {
            const int c = (i * t.lanes + t.lane) * 8;
            rx[i].load(x + c);
            if (HAS_F) rf[i].load(p.f + row * p.ldf + c);
        }
    }
    bool bad = false;
    f2 v[V][4];
    if (HAS_F) {
#pragma unroll
        for (int i = 0; i < V; i++) rf[i].get(v[i]);
        if (POST) {
            float mean, rstd;
            normalize(t, p.post, p.cols, have, v, mean, rstd);
            if (p.stats && live && t.lane == 0) p.stats[2 * p.rows + row] = mean, p.stats[3 * p.rows + row] = rstd;
        }
        const int64_t g = p.gate ? (int64_t)((uint32_t)row / p.rows_per_gate) * p.ldg : 0;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int vec = i * t.lanes + t.lane;
            if (p.fc.codes) {
                const uint32_t m = group_max4(amax8(v[i]));
                if (i < have) bad |= ckpt_write(p.fc, m, v[i], row * p.nvec + vec);
            }
            f2 xx[4];
            rx[i].get(xx);
            if (i < have) {
                if (POST) affine(p.post, i, vec, v);
                if (p.gate) {
                    f2 gg[4];
                    load_param8(p.gate, p.gate_fp32, g + vec * 8, gg);
#pragma unroll
                    for (int j = 0; j < 4; j++) v[i][j] = f2_mul(v[i][j], gg[j]);
                }
                const f2 a2 = f2_of(p.a, p.a), s2 = f2_of(p.s, p.s);
#pragma unroll
                for (int j = 0; j < 4; j++) v[i][j] = f2_fma(v[i][j], s2, f2_mul(xx[j], a2));
                if (p.xo) store8(static_cast<XT *>(p.xo) + row * p.ldxo + vec * 8, v[i]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; i++) rx[i].get(v[i]);
    }
    if (PRE) {
        float mean, rstd;
        normalize(t, p.pre, p.cols, have, v, mean, rstd);
        if (p.stats && live && t.lane == 0) p.stats[row] = mean, p.stats[p.rows + row] = rstd;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int vec = i * t.lanes + t.lane;
            if (p.xc.codes) {
                const uint32_t m = group_max4(amax8(v[i]));
                if (i < have) bad |= ckpt_write(p.xc, m, v[i], row * p.nvec + vec);
            }
            if (i < have) affine(p.pre, i, vec, v);
            const uint4 q = pack8(v[i]);
            if (i < have && p.h) *reinterpret_cast<uint4 *>(p.h + row * p.ldh + vec * 8) = q;
            if (p.hq) {      // Q1 of the bf16 result, as the row-wise quantizer makes it
                uint32_t am = absmax_fold(absmax_fold(absmax_fold(absmax_fold(0u, q.x), q.y), q.z), q.w);
                am = group_max4(hmax_halves(absmax_fold_end(am)));
                const bool odd = am >= 0x7F80u;
                const uint32_t byte = odd ? 0xFFu : scale_byte_from_amax(am, p.hq_tf_add);
                const uint32_t c = odd ? 0u : rne8(q, inv_scale_bf16x2(byte));
                if (i < have) {
                    bad |= odd;
                    *reinterpret_cast<uint32_t *>(p.hq + row * (p.cols >> 1) + vec * 4) = c;
                    if ((vec & 3) == 0) p.hq_scales[scale_offset(row, vec >> 2, p.nblk4)] = (uint8_t)byte;
                }
            }
        }
        if (p.hq) {          // the scales' padding: blocks to a multiple of 4, rows to one of 128
            const int nblk = p.cols >> 5;
            const int64_t rows_pad = (p.rows + 127) & ~(int64_t)127;
            if (live) {
                if (nblk + t.lane < p.nblk4 * 4) p.hq_scales[scale_offset(row, nblk + t.lane, p.nblk4)] = 0x7F;
            } else if (row < rows_pad) {
                for (int b = t.lane; b < p.nblk4 * 4; b += t.lanes) p.hq_scales[scale_offset(row, b, p.nblk4)] = 0x7F;
            }
        }
    }
    if (bad && p.dev_status) atomicOr(p.dev_status, MXFP4_DEV_NONFINITE);
}

// ---- backward -------------------------------------------------------------------------------------
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
    int need_f;               // f^ is read: there is N_post or a gate
    float a, s;
    float *part;              // [blocks][4][cols]: sums of dh x^, dh, t f^ (B), t (A)
    float *slots;             // several gates: [team + gate][2][cols]: B and A of a team's rows of a gate
    int64_t rows, rows_per_team;
    int cols, nvec, log2_lanes;
};

// One lane's share of a row, as loaded.
template <class XT, bool EIGHT, bool POST, bool PRE> struct RowIn {
    Raw8<__nv_bfloat16> dh, f;
    Raw8<XT> dxo, xo;
    RawCkpt xc, fc;
};

// Each team takes a run of consecutive rows and keeps the sums over them of its lanes' columns in registers: of dh x^ and dh for N_pre's
// gradients, and of t f^ and t (t the gradient of x' in all) for those of N_post and the gate:  with g constant over the rows of a gate,
//     dg = s (w1 B + b1 A),   dw1 = s sum_g g B_g,   db1 = s sum_g g A_g,      B = sum t f^,  A = sum t.
// They go to memory once per block, A and B of several gates once per team and gate; k_norm_bwd_finish adds them up.
template <class XT, int V, bool EIGHT, bool POST, bool PRE>
__global__ void __launch_bounds__(256) k_norm_bwd(const __grid_constant__ NormBwd p)
{
    __shared__ float4 s_sum[2 * 16];
    extern __shared__ float s_cols[];     // [2][cols], where a block has several teams
    pdl_launch_dependents();
    pdl_wait();
    Team t = make_team(p.log2_lanes, s_sum);
    const int teams = blockDim.x >> p.log2_lanes;
    const int64_t team = (int64_t)blockIdx.x * teams + t.id;
    const int64_t first = min(team * p.rows_per_team, p.rows), end = min(first + p.rows_per_team, p.rows);
    const int have = max(0, min(V, (p.nvec - t.lane + t.lanes - 1) >> p.log2_lanes));
    const float inv = 1.0f / (float)p.cols;
    f2 sw[V][4], sb[V][4], B[V][4], A[V][4];
#pragma unroll
    for (int i = 0; i < V; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) sw[i][j] = sb[i][j] = B[i][j] = A[i][j] = 0;

    uint32_t gate = p.several ? (uint32_t)first / p.rows_per_gate : 0u;
    uint32_t left = p.several ? p.rows_per_gate - ((uint32_t)first - gate * p.rows_per_gate) : 0u;   // rows of this gate still to come
    const auto flush = [&]() {
        float *o = p.slots + (team + gate) * 2 * (int64_t)p.cols;
#pragma unroll
        for (int i = 0; i < V; i++)
            if (i < have) {
                const int c = (i * t.lanes + t.lane) * 8;
                store8(o + c, B[i]);
                store8(o + p.cols + c, A[i]);
#pragma unroll
                for (int j = 0; j < 4; j++) B[i][j] = A[i][j] = 0;
            }
    };

    for (int64_t k = 0; k < p.rows_per_team; k++) {       // the same number of turns for all teams of a warp: the shuffles need all lanes
        const int64_t row = first + k;
        const bool live = row < end;
        const int n = live ? have : 0;
        if (p.several && live) {
            if (left == 0) {
                flush();
                gate++;
                left = p.rows_per_gate;
            }
            left--;
        }
        float pm = 0, pr = 0, qm = 0, qr = 0;
        if (live) {
            if (PRE) pm = p.stats[row], pr = p.stats[p.rows + row];
            if (POST) qm = p.stats[2 * p.rows + row], qr = p.stats[3 * p.rows + row];
        }
        f2 xh[V][4], d[V][4], tt[V][4];
        float c[2] = {0, 0};
        if (PRE) {
            f2 c1 = 0, c2 = 0;
#pragma unroll
            for (int i = 0; i < V; i++) {
                const int vec = i * t.lanes + t.lane;
                Raw8<__nv_bfloat16> rd;
                rd.zero();
                if (i < n) rd.load(p.dh + row * p.lddh + vec * 8);
                rd.get(d[i]);
                if (EIGHT) {
                    RawCkpt r;
                    r.zero();
                    if (i < n) r.load(p.xcodes, p.xscales, row * p.nvec + vec);
                    r.get(xh[i]);
                } else {
                    Raw8<XT> r;
                    r.zero();
                    if (i < n) r.load(static_cast<const XT *>(p.xo) + row * p.ldxo + vec * 8);
                    r.get(xh[i]);
                    const f2 m2 = f2_of(-pm, -pm), r2 = f2_of(pr, pr);
#pragma unroll
                    for (int j = 0; j < 4; j++) xh[i][j] = f2_mul(f2_add(xh[i][j], m2), r2);
                }
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    sw[i][j] = f2_fma(d[i][j], xh[i][j], sw[i][j]);
                    sb[i][j] = f2_add(d[i][j], sb[i][j]);
                }
                if (p.pre.w) {
                    f2 w[4] = {0, 0, 0, 0};
                    if (i < n) load_param8(p.pre.w, p.pre.fp32, (int64_t)vec * 8, w);
#pragma unroll
                    for (int j = 0; j < 4; j++) d[i][j] = f2_mul(d[i][j], w[j]);
                }
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    c1 = f2_add(c1, d[i][j]);
                    c2 = f2_fma(d[i][j], xh[i][j], c2);
                }
            }
            c[0] = f2_sum(c1), c[1] = f2_sum(c2);
            team_sum(t, c);
        }
        const float m1 = p.pre.rms ? 0.0f : -c[0] * inv, m2 = -c[1] * inv;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int vec = i * t.lanes + t.lane;
            Raw8<XT> r;
            r.zero();
            if (i < n && p.dxo) r.load(static_cast<const XT *>(p.dxo) + row * p.lddxo + vec * 8);
            r.get(tt[i]);
            if (PRE) {
                const f2 a1 = f2_of(m1, m1), a2 = f2_of(m2, m2), r2 = f2_of(pr, pr);
#pragma unroll
                for (int j = 0; j < 4; j++) tt[i][j] = i < n ? f2_fma(r2, f2_fma(xh[i][j], a2, f2_add(d[i][j], a1)), tt[i][j]) : 0ull;
            }
            if (i < n) {
                const f2 a2 = f2_of(p.a, p.a);
                f2 o[4];
#pragma unroll
                for (int j = 0; j < 4; j++) o[j] = f2_mul(tt[i][j], a2);
                store8(static_cast<XT *>(p.dx) + row * p.lddx + vec * 8, o);
            }
        }
        // the branch: xh and d are used again for f^ and for the gradient of the normalized row
        f2 e1 = 0, e2 = 0;
        const int64_t g = p.gate ? (int64_t)gate * p.ldg : 0;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int vec = i * t.lanes + t.lane;
            if (p.need_f) {
                if (EIGHT) {
                    RawCkpt r;
                    r.zero();
                    if (i < n) r.load(p.fcodes, p.fscales, row * p.nvec + vec);
                    r.get(xh[i]);
                } else {
                    Raw8<__nv_bfloat16> r;
                    r.zero();
                    if (i < n) r.load(p.f + row * p.ldf + vec * 8);
                    r.get(xh[i]);
                    if (POST) {
                        const f2 m2 = f2_of(-qm, -qm), r2 = f2_of(qr, qr);
#pragma unroll
                        for (int j = 0; j < 4; j++) xh[i][j] = f2_mul(f2_add(xh[i][j], m2), r2);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    B[i][j] = f2_fma(tt[i][j], xh[i][j], B[i][j]);
                    A[i][j] = f2_add(tt[i][j], A[i][j]);
                }
            }
            const f2 s2 = f2_of(p.s, p.s);
#pragma unroll
            for (int j = 0; j < 4; j++) d[i][j] = f2_mul(tt[i][j], s2);
            if (i < n) {
                f2 w[4];
                if (p.gate) {
                    load_param8(p.gate, p.gate_fp32, g + vec * 8, w);
#pragma unroll
                    for (int j = 0; j < 4; j++) d[i][j] = f2_mul(d[i][j], w[j]);
                }
                if (POST && p.post.w) {
                    load_param8(p.post.w, p.post.fp32, (int64_t)vec * 8, w);
#pragma unroll
                    for (int j = 0; j < 4; j++) d[i][j] = f2_mul(d[i][j], w[j]);
                }
            }
            if (POST) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    e1 = f2_add(e1, d[i][j]);
                    e2 = f2_fma(d[i][j], xh[i][j], e2);
                }
            }
        }
        if (POST) {
            float e[2] = {f2_sum(e1), f2_sum(e2)};
            team_sum(t, e);
            const float n1 = p.post.rms ? 0.0f : -e[0] * inv, n2 = -e[1] * inv;
            const f2 a1 = f2_of(n1, n1), a2 = f2_of(n2, n2), r2 = f2_of(qr, qr);
#pragma unroll
            for (int i = 0; i < V; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) d[i][j] = f2_mul(r2, f2_fma(xh[i][j], a2, f2_add(d[i][j], a1)));
        }
        if (p.df) {
#pragma unroll
            for (int i = 0; i < V; i++)
                if (i < n) store8(p.df + row * p.lddf + (i * t.lanes + t.lane) * 8, d[i]);
        }
    }

    if (p.several && first < end) flush();
    // the block's sums: team by team into shared memory, two of the four at a time
    float *part = p.part + (int64_t)blockIdx.x * 4 * p.cols;
#pragma unroll
    for (int half = 0; half < 2; half++) {
        if (half == 0 ? !PRE : (p.several || !p.need_f)) continue;
        for (int k = 0; k < teams; k++) {
            if (k == t.id) {
#pragma unroll
                for (int i = 0; i < V; i++)
                    if (i < have) {
                        const int c = (i * t.lanes + t.lane) * 8;
                        f2 u[4], w[4];
#pragma unroll
                        for (int j = 0; j < 4; j++) u[j] = half ? B[i][j] : sw[i][j], w[j] = half ? A[i][j] : sb[i][j];
                        if (k > 0) {
#pragma unroll
                            for (int j = 0; j < 4; j++) {
                                u[j] = f2_add(u[j], *reinterpret_cast<f2 *>(s_cols + c + 2 * j));
                                w[j] = f2_add(w[j], *reinterpret_cast<f2 *>(s_cols + p.cols + c + 2 * j));
                            }
                        }
                        float *o = k + 1 < teams ? s_cols : part + half * 2 * p.cols;
                        store8(o + c, u);
                        store8(o + p.cols + c, w);
                    }
            }
            __syncthreads();
        }
    }
}

struct NormBwdFinish {
    const float *part, *slots;
    NormSide post;
    const void *gate;
    int64_t ldg, gates;
    int gate_fp32, several;
    float s;
    int blocks, pre, use_f, has_post;
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
            add(b, *reinterpret_cast<const float4 *>(s + p.cols));
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
                    add(A, *reinterpret_cast<const float4 *>(s + p.cols));
                }
            } else {
                for (int k = sub; k < p.blocks; k += p.split) {
                    const float *s = p.part + (int64_t)k * 4 * p.cols + 2 * p.cols + c;
                    add(B, *reinterpret_cast<const float4 *>(s));
                    add(A, *reinterpret_cast<const float4 *>(s + p.cols));
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

// ---- host -----------------------------------------------------------------------------------------
// Lanes and vectors per lane of a row: the least of T * V >= cols / 8 with V = 3 or 4.
static void team_of(int64_t cols, int *log2_lanes, int *v)
{
    const int64_t nvec = cols / 8;
    int l3 = 2, l4 = 2;
    while ((3ll << l3) < nvec) l3++;
    while ((4ll << l4) < nvec) l4++;
    const bool three = (3ll << l3) <= (4ll << l4);
    *log2_lanes = three ? l3 : l4;
    *v = three ? 3 : 4;
}

// Blocks of the backward pass and the rows of one of its teams: depends on the shape alone (the workspace is laid out by it).
constexpr int kBwdBlocks = 296;
struct BwdPlan {
    int log2_lanes, v, threads, teams, blocks;
    int64_t rows_per_team, part_floats, slot_floats;
};
static BwdPlan bwd_plan(int64_t rows, int64_t cols, int64_t gates)
{
    BwdPlan b;
    team_of(cols, &b.log2_lanes, &b.v);
    b.threads = 256;
    b.teams = b.threads >> b.log2_lanes;
    const int64_t most = ceil_div(rows, b.teams);
    b.blocks = (int)(most < kBwdBlocks ? most : kBwdBlocks);
    b.rows_per_team = ceil_div(rows, (int64_t)b.blocks * b.teams);
    b.blocks = (int)ceil_div(ceil_div(rows, b.rows_per_team), b.teams);     // blocks that have rows
    b.part_floats = (int64_t)b.blocks * 4 * cols;
    b.slot_floats = gates > 1 ? ((int64_t)b.blocks * b.teams + gates) * 2 * cols : 0;
    return b;
}

static mxfp4_status_t check_side(const mxfp4_norm_t &n)
{
    if (n.kind < MXFP4_NORM_NONE || n.kind > MXFP4_NORM_RMS) return MXFP4_INVALID_ARG;
    if (n.kind == MXFP4_NORM_NONE) return MXFP4_OK;
    if ((n.dtype != MXFP4_OUT_BF16 && n.dtype != MXFP4_OUT_FP32) || !(n.eps >= 0.0f)) return MXFP4_INVALID_ARG;
    return aligned16(n.weight) && aligned16(n.bias) ? MXFP4_OK : MXFP4_MISALIGNED;
}
static NormSide side_of(const mxfp4_norm_t &n) { return {n.weight, n.bias, n.dtype == MXFP4_OUT_FP32, n.kind == MXFP4_NORM_RMS, n.eps}; }

// What the two directions check alike; `done`: there is nothing to do.
static mxfp4_status_t check_plan(const mxfp4_residual_norm_t *n)
{
    if (!n || n->rows < 0 || n->cols <= 0 || n->gates < 0) return MXFP4_INVALID_ARG;
    if (n->x_dtype != MXFP4_OUT_BF16 && n->x_dtype != MXFP4_OUT_FP32) return MXFP4_INVALID_ARG;
    if (n->cols % 32 != 0 || n->cols > kNormMaxCols || n->rows > 0x7FFFFFFF) return MXFP4_BAD_SHAPE;
    mxfp4_status_t s;
    if ((s = check_side(n->pre)) || (s = check_side(n->post))) return s;
    if ((n->gates > 0) != (n->gate != nullptr)) return MXFP4_INVALID_ARG;
    if (n->gate) {
        if (n->gate_dtype != MXFP4_OUT_BF16 && n->gate_dtype != MXFP4_OUT_FP32) return MXFP4_INVALID_ARG;
        if (n->rows % n->gates != 0) return MXFP4_BAD_SHAPE;
        if (n->gates > 1 && n->ld_gate < n->cols) return MXFP4_BAD_SHAPE;
        if (!aligned16(n->gate) || (n->gates > 1 && (n->ld_gate * dtype_bytes(n->gate_dtype)) % 16 != 0)) return MXFP4_MISALIGNED;
    }
    return MXFP4_OK;
}

// Outputs may lie over the input that is read in the same place (the same address and pitch), or apart from it.
static bool over_or_apart(const Span &out, int64_t ldo, int64_t out_bytes, const Span &in, int64_t ldi, int64_t in_bytes)
{
    return !meet(out, in) || (out.lo == in.lo && ldo == ldi && out_bytes == in_bytes);
}

// Calls go(std::integral_constant for each of the kernel's template arguments).
template <class F> static cudaError_t with_bools(bool a, bool b, bool c, F &&f)
{
    using T = std::true_type;
    using N = std::false_type;
    if (a) return b ? (c ? f(T(), T(), T()) : f(T(), T(), N())) : (c ? f(T(), N(), T()) : f(T(), N(), N()));
    return b ? (c ? f(N(), T(), T()) : f(N(), T(), N())) : (c ? f(N(), N(), T()) : f(N(), N(), N()));
}
template <class F> static cudaError_t with_row(bool fp32, int v, F &&f)
{
    using Three = std::integral_constant<int, 3>;
    using Four = std::integral_constant<int, 4>;
    if (fp32) return v == 3 ? f(float(), Three()) : f(float(), Four());
    return v == 3 ? f(__nv_bfloat16(), Three()) : f(__nv_bfloat16(), Four());
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
    if (!over_or_apart(so, ldxo, xb, sx, ldx, xb) || !over_or_apart(so, ldxo, xb, sf, ldf, 2) || !over_or_apart(sh, ldh, 2, sx, ldx, xb) ||
        !over_or_apart(sh, ldh, 2, sf, ldf, 2) || meet(so, sh))
        return MXFP4_INVALID_ARG;
    NormFwd p = {};
    int v;
    team_of(cols, &p.log2_lanes, &v);
    p.x = x, p.f = static_cast<const __nv_bfloat16 *>(f_bf16), p.xo = x_out, p.h = static_cast<__nv_bfloat16 *>(h_bf16);
    p.ldx = ldx, p.ldf = ldf, p.ldxo = ldxo, p.ldh = ldh;
    p.pre = side_of(n->pre), p.post = side_of(n->post);
    p.gate = n->gate, p.ldg = n->ld_gate, p.gate_fp32 = n->gate_dtype == MXFP4_OUT_FP32;
    p.rows_per_gate = n->gate ? (uint32_t)(rows / n->gates) : 1u;
    p.a = n->residual_scale, p.s = n->branch_scale, p.stats = stats;
    p.xc = {x_ckpt.codes, x_ckpt.scales, ckpt_tf_add(scale_mode)};
    p.fc = {f_ckpt.codes, f_ckpt.scales, ckpt_tf_add(scale_mode)};
    p.nblk4 = (int)ceil_div(cols / 32, 4);
    if (hq) p.hq = static_cast<uint8_t *>(hq->data), p.hq_scales = hq->scales, p.hq_tf_add = scale_mode == MXFP4_SCALE_FLOOR ? 0u : 63u;
    p.rows = rows, p.cols = (int)cols, p.nvec = (int)(cols / 8), p.dev_status = dev_status;
    constexpr int threads = 256;
    const int64_t all = hq ? (rows + 127) / 128 * 128 : rows;
    const unsigned blocks = (unsigned)ceil_div(all, threads >> p.log2_lanes);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    MX_CHECK_CUDA(with_row(n->x_dtype == MXFP4_OUT_FP32, v, [&](auto xt, auto vv) {
        using XT = decltype(xt);
        constexpr int V = decltype(vv)::value;
        return with_bools(has_f, post, pre, [&](auto f, auto q, auto r) -> cudaError_t {
            constexpr bool F = decltype(f)::value, Q = decltype(q)::value, R = decltype(r)::value;
            if constexpr ((!F && (Q || !R))) return cudaErrorInvalidValue;     // refused above
            else return launch_pdl(k_norm_fwd<XT, V, F, Q, R>, blocks, 1, threads, 0, st, p);
        });
    }));
    return MXFP4_OK;
}

size_t mxfp4_residual_norm_workspace_bytes(int64_t rows, int64_t cols, int64_t gates)
{
    if (rows <= 0 || cols <= 0 || cols > kNormMaxCols || gates < 0) return 0;
    const BwdPlan b = bwd_plan(rows, cols, gates);
    return (size_t)(b.part_floats + b.slot_floats) * 4;
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
    const bool eight = pre ? b->x_ckpt.codes != nullptr : b->f_ckpt.codes != nullptr;
    if (pre && eight && (s = check_ckpt(b->x_ckpt, rows, cols))) return s;
    if (need_f && eight && (s = check_ckpt(b->f_ckpt, rows, cols))) return s;
    if (pre && !eight && (s = check_rows(b->x_out, b->ldxo, cols, n->x_dtype))) return s;
    if (need_f && !eight && (s = check_rows(b->f_bf16, b->ldf, cols, MXFP4_OUT_BF16))) return s;
    if (!workspace) return MXFP4_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return MXFP4_MISALIGNED;
    const BwdPlan plan = bwd_plan(rows, cols, n->gates);
    if (workspace_bytes < (size_t)(plan.part_floats + plan.slot_floats) * 4) return MXFP4_WORKSPACE_TOO_SMALL;
    {
        // dx and df are written row by row while later rows are still to be read
        const Span dx = span_of_rows(b->dx, b->lddx, rows, cols, xb), df = span_of_rows(b->df_bf16, b->lddf, rows, cols, 2);
        const Span dxo = span_of_rows(b->dx_out, b->lddxo, rows, cols, xb), dh = span_of_rows(b->dh_bf16, b->lddh, rows, cols, 2);
        if (meet(dx, df) || !over_or_apart(dx, b->lddx, xb, dxo, b->lddxo, xb) || !over_or_apart(dx, b->lddx, xb, dh, b->lddh, 2) ||
            !over_or_apart(df, b->lddf, 2, dxo, b->lddxo, xb) || !over_or_apart(df, b->lddf, 2, dh, b->lddh, 2))
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
    p.need_f = need_f, p.a = n->residual_scale, p.s = n->branch_scale;
    p.part = static_cast<float *>(workspace), p.slots = p.part + plan.part_floats;
    p.rows = rows, p.rows_per_team = plan.rows_per_team, p.cols = (int)cols, p.nvec = (int)(cols / 8), p.log2_lanes = plan.log2_lanes;
    const size_t smem = plan.teams > 1 ? (size_t)cols * 8 : 0;
    MX_CHECK_CUDA(with_row(n->x_dtype == MXFP4_OUT_FP32, plan.v, [&](auto xt, auto vv) {
        using XT = decltype(xt);
        constexpr int V = decltype(vv)::value;
        return with_bools(eight, post, pre, [&](auto e, auto q, auto r) {
            return launch_pdl(k_norm_bwd<XT, V, decltype(e)::value, decltype(q)::value, decltype(r)::value>, (unsigned)plan.blocks, 1, (unsigned)plan.threads, smem, st, p);
        });
    }));
    if (!b->dw_pre && !b->db_pre && !b->dw_post && !b->db_post && !b->dgate) return MXFP4_OK;
    NormBwdFinish e = {};
    e.part = p.part, e.slots = p.slots, e.post = p.post, e.gate = p.gate, e.ldg = p.ldg, e.gate_fp32 = p.gate_fp32;
    e.gates = n->gates > 1 ? n->gates : 1, e.several = p.several, e.s = p.s, e.blocks = plan.blocks, e.pre = pre, e.use_f = need_f, e.has_post = post;
    e.rows = rows, e.rows_per_gate = p.rows_per_gate, e.rows_per_team = plan.rows_per_team, e.cols = (int)cols;
    e.split = 64;
    while (e.split > 1 && 64 / e.split < e.gates) e.split >>= 1;
    e.dw_pre = b->dw_pre, e.db_pre = b->db_pre, e.dw_post = b->dw_post, e.db_post = b->db_post, e.dgate = b->dgate;
    MX_CHECK_CUDA(launch_pdl(k_norm_bwd_finish, (unsigned)(cols / 16), 1, 256, 0, st, e));
    return MXFP4_OK;
}

}  // extern "C"
