// What the two directions of the residual addition between norms share: teams, the ring of rows, parameters, the host's plan.
//
// A team of lanes (4, 8, 16, or a number of warps) holds a row in registers, each lane V vectors of eight columns.  The sums over a row go
// through shuffles and, where a team has several warps, through shared memory and a barrier of the team.  V (2 to 4
// backward, 3 or 4 forward) and the lanes are chosen so that a block's lanes have the most to do (row_plan); the usual widths are reached
// exactly.
// Two or three blocks per SM, and for long matrices forward several times as many blocks as fit: the SMs do not get equal shares of the memory's bandwidth (in
// a kernel of one block per SM the mean SM was done at 81 % of the last one's time), so what is left is dealt out as they finish.  A block's
// lanes keep their columns from row to row: what belongs to a column (weights, a gate, sums over rows) is fetched once.  The few warps
// cannot hide the memory's latency by themselves; a lane's share of the next rows travels into shared memory meanwhile (cp.async, mostly
// into slots that only this lane reads: no barriers of the block).
// FULL: the lanes' vectors are exactly a row.  Without the masks of a partly filled lane the loops over V are straight code (25216 x 384
// forward: 343 warp instructions per 256 columns with them, 213 without).  Otherwise teams are such that only a lane's last vector may be
// missing, and the others have no masks either (47039 x 960 backward: 130 us with masks for all, 98 so; 50432 x 1056 forward: 138, 130); 32 and
// 64 columns, on 4 lanes, have them.
#pragma once
#include <algorithm>

#include "ckpt.cuh"
#include "quant_tile.cuh"
#include "tma.cuh"

namespace mx {

constexpr int kNormMaxCols = 8192;
constexpr int kFwdThreads = 256;
// Three blocks per SM where 80 registers and 74 KB each are enough and there is more to compute than a norm of full rows (50432 x 768 between two
// layer norms 82 us with two, 73 with three, 50432 x 1056 with one 130, 114; 50432 x 768 with one, which has four stages of two blocks, 69, 71).
constexpr int fwd_blocks_per_sm(int v, int x_bytes, bool post, bool full) { return v == 3 && x_bytes == 2 && (post || !full) ? 3 : 2; }
// Backward: as many warps as the registers allow for v vectors of a lane and `sums` sums over rows (8 v registers each).  A kernel that
// spills is twice as slow (50432 x 768: 80 us with eight warps, 158 with twelve and 200 bytes of spills): the ring leaves no L1 for them.
constexpr int bwd_threads(int v, int sums) { return v == 4 ? 256 : v == 2 ? (sums == 2 ? 256 : 192) : sums == 2 ? 192 : 128; }
constexpr int bwd_blocks_per_sm(int v) { return v == 4 ? 1 : 2; }

// ---- a lane's ring of rows in shared memory ----------------------------------------------------
__device__ __forceinline__ void async16(uint32_t dst, const void *src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void async8(uint32_t dst, const void *src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void warp_sync() { asm volatile("bar.warp.sync 0xffffffff;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
// Eight elements of type T: slots of 16 bytes per lane, one (bf16) or two (fp32) of them.  The block's lanes lie side by side in `slots`.  FP32 elements are copied in the order of memory, half of the L lanes' share at a time, which are not each lane's own
// (a lane that copied both of its own would have the L2 read every sector twice, and so would any other order in shared memory): they
// become visible by the warp's barrier.  `lanes`: the first so many have something to copy.
template <class T> constexpr int kSlots = sizeof(T) / 2;
template <class T, int L> __device__ __forceinline__ void async_row8(uint32_t slots, const T *src, int lanes)
{
    const int tid = threadIdx.x, l = tid & (L - 1);
    if (sizeof(T) == 2) {
        if (l < lanes) async16(slots + tid * 16, src);
    } else {
        const uint32_t to = slots + tid * 32 - l * 16;
        if (l >> 1 < lanes) async16(to, src - 4 * l);
        if ((l >> 1) + L / 2 < lanes) async16(to + L * 16, src - 4 * l + 4 * L);
    }
}
template <class T> __device__ __forceinline__ void ring_row8(uint32_t slots, f2 (&o)[4])
{
    const uint4 a = lds16(slots + threadIdx.x * (sizeof(T) == 2 ? 16 : 32));
    if (sizeof(T) == 2) {
        unpack8(a, o);
    } else {
        const uint4 b = lds16(slots + threadIdx.x * 32 + 16);
        o[0] = (f2)a.y << 32 | a.x, o[1] = (f2)a.w << 32 | a.z, o[2] = (f2)b.y << 32 | b.x, o[3] = (f2)b.w << 32 | b.z;
    }
}
// A lane's own eight FP32 elements.
template <int N> __device__ __forceinline__ void lds8f(uint32_t slot, f2 (&o)[4])
{
    const uint4 a = lds16(slot), b = lds16(slot + N * 16);
    o[0] = (f2)a.y << 32 | a.x, o[1] = (f2)a.w << 32 | a.z, o[2] = (f2)b.y << 32 | b.x, o[3] = (f2)b.w << 32 | b.z;
}
constexpr int kRingBytes = 226 * 1024, kHalfRingBytes = 112 * 1024, kThirdRingBytes = 74 * 1024, kMostStages = 4;     // of an SM's one block, of one of two
// Waits until at most `left` (0 to 3) of this lane's groups of copies are under way.
__device__ __forceinline__ void async_wait_all_but(int left)
{
    if (left == 3) async_wait<3>();
    else if (left == 2) async_wait<2>();
    else if (left == 1) async_wait<1>();
    else async_wait<0>();
}
// A parameter of all columns in shared memory: two planes, the first and the second four of every eight columns.
__device__ __forceinline__ void plane_put(float4 *plane, int nvec, int vec, const f2 (&v)[4])
{
    *reinterpret_cast<ulonglong2 *>(plane + vec) = make_ulonglong2(v[0], v[1]);
    *reinterpret_cast<ulonglong2 *>(plane + nvec + vec) = make_ulonglong2(v[2], v[3]);
}
__device__ __forceinline__ void plane_get(const float4 *plane, int nvec, int vec, f2 (&v)[4])
{
    const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(plane + vec), b = *reinterpret_cast<const ulonglong2 *>(plane + nvec + vec);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}
__device__ __forceinline__ void zero8(f2 (&o)[4]) { o[0] = o[1] = o[2] = o[3] = 0; }

// ---- teams --------------------------------------------------------------------------------------
// L: its lanes of one warp (32, or fewer where a warp holds several teams).  Lane l of a warp whose part of the row starts at vector a holds
// a + i L + l, i < V, as far as they are in that part; the warps' parts differ by at most one group of 32 columns.
template <int L> struct Team {
    int warps, lane;     // of the team; of the warp's part of it
    int id, first_vec;   // of the team in its block; of the lane
    int part_vecs;       // vectors of the warp's part
    bool leader;
    float4 *slots;       // several warps: where they leave their sums, two sets that take turns
    int turn;

    __device__ __forceinline__ Team(int team_warps, int nvec, float4 *smem) : warps(team_warps), lane(threadIdx.x & (L - 1)), part_vecs(nvec), turn(0)
    {
        const int part = L < 32 ? threadIdx.x / L : threadIdx.x >> 5;     // of a team, in the block
        id = L < 32 ? part : part / team_warps;
        first_vec = lane;
        if (L == 32 && team_warps > 1) {
            const int w = part - id * team_warps, groups = nvec >> 2, each = groups / team_warps, more = groups - each * team_warps;
            first_vec += (w * each + min(w, more)) * 4;
            part_vecs = (each + (w < more)) * 4;
        }
        leader = first_vec == 0;
        slots = smem + id * 2 * team_warps;
    }
};

// Whether a lane of a team has its vector i whatever its place: if not, that goes by the number that it has.
template <int V, bool FULL, int L> __device__ __forceinline__ bool always(int i) { return FULL || (L > 4 && i < V - 1); }

// Rows of which a team of several in a warp has none left take part in its shuffles; `turns` is the same for all teams of a warp.
// (A warp that is in no team has no rows.)
template <int L> __device__ __forceinline__ int turns_of(int64_t end, int64_t first, int64_t step)
{
    const int64_t at = L < 32 ? first - first % step : first;     // (of the first team of several)
    return at < end ? (int)((end - at + step - 1) / step) : 0;
}

// The sums of N (1, 2) numbers over the lanes of the team, the same bits in each of them.  All lanes of the warp take part.
template <int N, int L>
__device__ __forceinline__ void team_sum(Team<L> &t, float (&v)[N])
{
#pragma unroll
    for (int o = L / 2; o; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; k++) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if (L == 32 && t.warps > 1) {
        float *s = reinterpret_cast<float *>(t.slots + t.turn * t.warps);
        t.turn ^= 1;     // a warp that is ahead writes the other set: nobody is more than one barrier ahead
        if (t.lane == 0)
#pragma unroll
            for (int k = 0; k < N; k++) s[((threadIdx.x >> 5) - t.id * t.warps) * 4 + k] = v[k];
        asm volatile("bar.sync %0, %1;" ::"r"(t.id + 1), "r"(t.warps * 32) : "memory");
#pragma unroll
        for (int k = 0; k < N; k++) v[k] = 0.0f;
        for (int w = 0; w < t.warps; w++)
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

// One column's factor and summand of a norm as pairs; 1 and 0 where there are none.
__device__ __forceinline__ void load_side8(const NormSide &n, int vec, f2 (&w)[4], f2 (&b)[4])
{
#pragma unroll
    for (int j = 0; j < 4; j++) w[j] = f2_of(1.0f, 1.0f), b[j] = 0;
    if (n.w) load_param8(n.w, n.fp32, (int64_t)vec * 8, w);
    if (n.b) load_param8(n.b, n.fp32, (int64_t)vec * 8, b);
}

// ---- host -----------------------------------------------------------------------------------------
constexpr int kSms = 148;      // of a B200; the plan goes by the shape alone, for the backward pass's workspace is laid out by it

// A matrix's rows on teams.
struct RowPlan {
    int lanes, v, teams, blocks;    // lanes of a team, vectors of a lane, teams of a block
    bool full;
    int64_t rows_per_team;

    int warps() const { return lanes <= 32 ? 1 : lanes / 32; }
};
// Of 3 or 4 vectors per lane, and the fewest lanes that hold a row then, whatever leaves the fewest of a block's vectors without work; of both
// 4 (fewer shuffles).  Backward (sums > 0) of 2, 3 or 4, of two alike 2 (43904 x 1024 with an RMS norm 68 us with 2, 70 with 4), or 3 if a block
// has several teams (35136 x 1280 between layer norms 133 with 2, 116 with 3; 17536 x 2560, one team, 118 with 2, 125 with 3), and of all four
// sums 4 (between layer norms 43904 x 1024 94 with 2, 84 with 4, 56192 x 800 135, 105; in FP32 from the inputs 141, 133 and 127, 152; if fewer
// of its vectors have work it is not: 29248 x 1536 96, 118).
// More than 4 lanes only if each has its first k - 1 vectors.
constexpr RowPlan row_plan(int64_t cols, int sums)
{
    RowPlan b = {};
    const int64_t nvec = cols / 8;
    int best = 0;
    for (int k = sums ? 2 : 3; k <= 4; k++) {
        const int threads = sums ? bwd_threads(k, sums) : kFwdThreads;
        int lanes = sums && k == 4 ? 32 : 4;
        while (lanes * k < nvec) lanes += lanes < 32 ? lanes : 32;
        if (lanes > 4 && (lanes <= 32 ? nvec <= (k - 1) * lanes : nvec / 4 / (lanes / 32) < 8 * (k - 1))) continue;
        const int teams = threads / lanes, used = (int)(teams * nvec * 1000 / (threads * k));     // in thousandths
        const bool of_two = !sums || (k == 3 && teams > 1) || (k == 4 && sums == 4);
        if (teams > 0 && (used > best || (used == best && of_two))) b.v = k, b.lanes = lanes, b.teams = teams, best = used;
    }
    b.full = (int64_t)b.v * b.lanes * 8 == cols;
    return b;
}
constexpr bool each_width_has_a_plan()
{
    for (int64_t cols = 32; cols <= kNormMaxCols; cols += 32)
        for (int sums = 0; sums <= 4; sums += sums ? 1 : 2)
            if (row_plan(cols, sums).teams == 0 || row_plan(cols, sums).v * row_plan(cols, sums).lanes * 8 < cols) return false;
    return true;
}
static_assert(each_width_has_a_plan());
// Whether any width's plan has v vectors per lane on `lanes` lanes of a warp, full or not: the kernels of the others are not made (backward 2 on 8 lanes
// and 3 on 4, forward 4 on 4, not full: 102 of 988).
constexpr bool some_width_has(int v, int lanes, bool full, bool backward)
{
    for (int64_t cols = 32; cols <= kNormMaxCols; cols += 32)
        for (int sums = backward ? 2 : 0; sums <= (backward ? 4 : 0); sums++) {
            const RowPlan b = row_plan(cols, sums);
            if (b.v == v && (b.lanes < 32 ? b.lanes : 32) == lanes && b.full == full) return true;
        }
    return false;
}
// Deals the rows to as many blocks as are resident, or `times` as many as long as a team keeps six rows.
inline void deal(RowPlan &b, int64_t rows, int blocks_per_sm, int64_t times)
{
    const int64_t resident = (int64_t)kSms * blocks_per_sm, most = ceil_div(rows, b.teams);
    times = std::min<int64_t>(std::max<int64_t>(rows / (resident * b.teams * 6), 1), times);
    b.rows_per_team = ceil_div(rows, std::min(most, resident * times) * b.teams);
    b.blocks = (int)ceil_div(ceil_div(rows, b.rows_per_team), b.teams);     // blocks that have rows
}
// Backward each block has sums to leave, and more blocks than are resident do not pay: 50432 x 768 with one, two, three times as many 75, 84, 92 us.
inline RowPlan bwd_plan(int64_t rows, int64_t cols, int sums)
{
    RowPlan b = row_plan(cols, sums);
    deal(b, rows, bwd_blocks_per_sm(b.v), 1);
    return b;
}
inline int64_t part_floats(const RowPlan &b, int64_t cols) { return (int64_t)b.blocks * 4 * cols; }
inline int64_t slot_floats(const RowPlan &b, int64_t cols, int64_t gates) { return gates > 1 ? ((int64_t)b.blocks * (b.teams + 1) + gates) * 2 * cols : 0; }

inline mxfp4_status_t check_side(const mxfp4_norm_t &n)
{
    if (n.kind < MXFP4_NORM_NONE || n.kind > MXFP4_NORM_RMS) return MXFP4_INVALID_ARG;
    if (n.kind == MXFP4_NORM_NONE) return MXFP4_OK;
    if ((n.dtype != MXFP4_OUT_BF16 && n.dtype != MXFP4_OUT_FP32) || !(n.eps >= 0.0f)) return MXFP4_INVALID_ARG;
    return aligned16(n.weight) && aligned16(n.bias) ? MXFP4_OK : MXFP4_MISALIGNED;
}
// The parameters, as memory that is read.
inline void read_plan(Memory &m, const mxfp4_residual_norm_t &n)
{
    for (const mxfp4_norm_t *s : {&n.pre, &n.post})
        if (s->kind != MXFP4_NORM_NONE) m.read(s->weight, n.cols * dtype_bytes(s->dtype)), m.read(s->bias, n.cols * dtype_bytes(s->dtype));
    m.read(span_of_rows(n.gate, n.gates > 1 ? n.ld_gate : n.cols, n.gates, n.cols, dtype_bytes(n.gate_dtype)));
}
inline NormSide side_of(const mxfp4_norm_t &n) { return {n.weight, n.bias, n.dtype == MXFP4_OUT_FP32, n.kind == MXFP4_NORM_RMS, n.eps}; }

// What the two directions check alike.
inline mxfp4_status_t check_plan(const mxfp4_residual_norm_t *n)
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
inline bool rows_over_or_apart(const Span &out, int64_t ldo, int64_t out_bytes, const Span &in, int64_t ldi, int64_t in_bytes)
{
    return !meet(out, in) || (out.lo == in.lo && ldo == ldi && out_bytes == in_bytes);
}

// Call f with the arguments as types, for a kernel's template arguments.
template <class F> inline cudaError_t with_bools(bool a, bool b, bool c, F &&f)
{
    using T = std::true_type;
    using N = std::false_type;
    if (a) return b ? (c ? f(T(), T(), T()) : f(T(), T(), N())) : (c ? f(T(), N(), T()) : f(T(), N(), N()));
    return b ? (c ? f(N(), T(), T()) : f(N(), T(), N())) : (c ? f(N(), N(), T()) : f(N(), N(), N()));
}
// Launches a kernel of THREADS per block that may take up to kRingBytes of shared memory.
template <auto KERNEL, int THREADS, class P> inline cudaError_t launch_ring(int blocks, size_t smem, cudaStream_t st, const P &p)
{
    static bool attr_set[kMaxDevices];
    const cudaError_t e = set_smem_once(attr_set, KERNEL, kRingBytes);
    return e != cudaSuccess ? e : launch_pdl(KERNEL, (unsigned)blocks, 1, THREADS, smem, st, p);
}
template <int V, class F> inline cudaError_t with_lanes(const RowPlan &plan, F &&f)     // f(lanes of a warp's part of a team, full)
{
    return with_bools(plan.full, false, false, [&](auto full, auto, auto) {
        return plan.lanes == 4    ? f(std::integral_constant<int, 4>(), full)
               : plan.lanes == 8  ? f(std::integral_constant<int, 8>(), full)
               : plan.lanes == 16 ? f(std::integral_constant<int, 16>(), full)
                                  : f(std::integral_constant<int, 32>(), full);
    });
}

}  // namespace mx
