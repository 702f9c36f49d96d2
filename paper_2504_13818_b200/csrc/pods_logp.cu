// pods_logp_chunk, pods_logp_grad_chunk - log-probability and entropy of each row's token, and the gradient of any objective on
// them carried back to the logits.
//
// Mathematics, c = log2 e / temperature:  log2 sum_v 2^(z_v c) = R + log2 S,  S = sum_v 2^(z_v c - R)  for any reference R.
// R is an integer kept per thread, so parts are brought together by exact powers of two, and it only follows the data where a
// block's sum shows that the reference lies far below it: no maximum is taken of every element.  Entropy needs
// U = sum_v 2^(z_v c - R) (z_v c - R) beside S:  H = ln 2 (log2 S - U / S).
// The gradient's exponentials are relative to the integer part of lse log2 e; the fraction goes into the row's coefficient.
//
// Bound: HBM; a read of the logits (forward), a read and a write (gradient).
#include <float.h>

#include <type_traits>

#include "pods_logp.cuh"
#include "row_plan.cuh"

namespace {

using namespace pods_row;
using pods_logp::FwdArgs;
using pods_logp::GradArgs;
using pods_logp::kBatch;
using pods_logp::kFewRows;

constexpr int kThreads = 256;
constexpr int kBlockVecs = 4;          // vectors a thread takes at once
constexpr float kSumLimit = 1024.0f;   // a block's sum above this moves the reference
constexpr int kNoRef = -(1 << 28);
// ex2.approx comes out low by 3.5e-8 in the mean over evenly spread fractions (measured: 3.4e-8 to 3.7e-8 on rows of 1000 to 150000
// logits), which sums of many terms show and sums over many tokens keep: added to the logarithm of a row's sum.
constexpr double kExponentialsLow = 3.5e-8 * 1.4426950408889634;
constexpr int kFar = 1 << 22;          // references from here on leave fp32 too few fractional bits: the row is taken in fp64

// A part of a row: S and U relative to 2^R.  R == kNoRef: nothing above -kFar so far.
struct Part {
    double s, u;
    int R;
    int bad;                           // 1: NaN or +inf, 2: far above 0
};

__device__ __forceinline__ double pow2_int(int n) {    // n <= 0
    return n < -1000 ? 0.0 : __hiloint2double((1023 + n) << 20, 0);
}

// Adds what a lane left of a row to `p`, whose reference is at least the lane's: a product with a power of two, then fp64.
template <bool ENT>
__device__ __forceinline__ void add_left(Part& p, uint2 l, float lu) {
    const float s = __uint_as_float(l.x);
    const int d = ((int)l.y >> 2) - p.R;
    const double f = pow2_int(d);
    // 2^(y - R) (y - R) = 2^(y - Rl) 2^(Rl - R) (y - Rl + Rl - R); a lane without anything adds nothing
    if (ENT) p.u += s != 0.0f ? ((double)lu + (double)s * (double)d) * f : 0.0;
    p.s += (double)s * f;
    p.bad |= (int)(l.y & 3u);
}
__device__ __forceinline__ int ref_of(uint2 l) { return (int)l.y >> 2; }

// What a thread holds while it goes through its elements of a row.  R starts as the row before left it, and is looked at once
// more if the first block shows it far from this row's logits: a reference of the row's own would cost each row a block twice.
template <int DT, bool ENT>
struct Sums {
    using El = Elem<DT>;
    static constexpr int E = El::E;
    float s, u;
    int R = kNoRef, bad;
    bool fresh;                        // nothing has been added yet

    __device__ __forceinline__ void start() {
        s = u = 0.0f;
        bad = 0;
        fresh = true;
    }
    // e = 2^(x c - R) of a vector, added to the pairs of sums; with ENT also e (x c - R)
    __device__ __forceinline__ void add(const uint4& q, float c, float c_lo, float ref, unsigned long long& acc, unsigned long long& accu) const {
        float x[E];
        El::unpack(q, x);
        const unsigned long long c2 = pack2(c, c), lo2 = pack2(c_lo, c_lo), off2 = pack2(-ref, -ref);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const unsigned long long x2 = pack2(x[i], x[i + 1]), d2 = fma2(x2, lo2, fma2(x2, c2, off2));
            float d0, d1;
            unpack2(d2, d0, d1);
            const unsigned long long e2 = pack2(ex2_approx(d0), ex2_approx(d1));
            acc = add2(acc, e2);
            if (ENT) accu = fma2(e2, pack2(fmaxf(d0, -1e4f), fmaxf(d1, -1e4f)), accu);   // 2^-inf (-inf) counts 0
        }
    }
    template <int N>
    __device__ __forceinline__ void add_all(const uint4 (&q)[N], float c, float c_lo, float& bs, float& bu) const {
        const float ref = (float)R;
        unsigned long long acc = 0ull, accu = 0ull;
#pragma unroll
        for (int k = 0; k < N; ++k) add(q[k], c, c_lo, ref, acc, accu);
        float a, b;
        unpack2(acc, a, b);
        bs = a + b;
        bu = 0.0f;
        if (ENT) {
            unpack2(accu, a, b);
            bu = a + b;
        }
    }
    template <int N>
    __device__ __forceinline__ void take(const uint4 (&q)[N], float c, float c_lo) {
        float bs, bu;
        add_all(q, c, c_lo, bs, bu);
        if (!(bs < kSumLimit) || (fresh && !(bs > 1.0f / kSumLimit))) {
            // rare: the reference lies far from the first block or below a later one; NaN, +inf, nothing but ids ruled out
            float m = -INFINITY;
#pragma unroll
            for (int k = 0; k < N; ++k) m = max_nan(m, El::vec_max(q[k]));
            bs = bu = 0.0f;
            if (fresh) R = kNoRef;
            if (!(m < INFINITY)) bad |= 1;
            else if (m > -INFINITY) {
                const float top = ceilf(m * c);
                if (!(top < (float)kFar)) bad |= 2;
                else if (top > -(float)kFar) {         // below: nothing so far, see finish_rows
                    const int to = (int)top;
                    if (to > R) {
                        const float f = R - to < -126 ? 0.0f : __uint_as_float((uint32_t)(127 + R - to) << 23);
                        if (ENT) u = f == 0.0f ? 0.0f : (u + s * (float)(R - to)) * f;
                        s *= f;
                        R = to;
                    }
                    add_all(q, c, c_lo, bs, bu);
                }
            }
            if (R == kNoRef && !bad) return;           // still nothing
        }
        fresh = false;
        s += bs;
        if (ENT) u += bu;
    }
    // What a lane leaves of a row, 8 bytes and with ENT 8 more.  Nothing so far: the reference is still that of the row before.
    __device__ __forceinline__ uint2 left() const {
        return make_uint2(__float_as_uint(s), (uint32_t)(fresh ? kNoRef : R) << 2 | (uint32_t)bad);
    }
};

template <typename T, typename Op>
__device__ __forceinline__ T warp_reduce(T v, Op op) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(PODS_FULL_MASK, v, d));
    return v;
}

// A row in fp64 by one warp: what is left where fp32 has no fractional bits for the exponents.  top: the largest logit.
template <int DT>
__device__ __noinline__ Part far_row(const typename Elem<DT>::raw* row, int V, double inv_tau, int lane, float& top) {
    using El = Elem<DT>;
    float m = -INFINITY;
    for (int i = lane; i < V; i += 32) m = max_nan(m, El::to_float(row[i]));
    m = warp_reduce(m, MaxNan());
    top = m;
    Part p = {0.0, 0.0, 0, m < INFINITY ? 0 : 1};
    if (!(fabsf(m) < INFINITY)) return p;
    for (int i = lane; i < V; i += 32) {
        const double d = ((double)El::to_float(row[i]) - (double)m) * inv_tau, e = exp64(d);
        p.s += e;
        if (e != 0.0) p.u += e * d;
    }
    p.s = warp_reduce(p.s, Plus());
    p.u = warp_reduce(p.u, Plus());
    return p;
}

// What a lane knows of its row's token: its logit.
template <int DT>
__device__ __forceinline__ float token_logit(const FwdArgs& a, int64_t t) {
    int token = a.tokens[t];
    if ((unsigned)token >= (unsigned)a.V) {
        pods_raise(a.status, PODS_STATUS_TOKEN_RANGE);
        token = 0;
    }
    return Elem<DT>::to_float((static_cast<const typename Elem<DT>::raw*>(a.logits) + t * a.ldl)[token]);
}

// A warp's lanes each hold the sums of a row of their own (t < 0: none), and its token's logit: writes the rows' outputs.
template <int DT, bool ENT>
__device__ __forceinline__ void finish_rows(const FwdArgs& a, int64_t t, Part p, float z, int lane) {
    // far, or nothing near 0: a thread leaves out blocks below -kFar (ids ruled out by a large negative number), which are nothing beside
    // a reference above -kFar / 2; without one fp64 also tells huge negative logits from a row of -inf.  2048 bf16 rows of 151936 logits
    // with nine in ten at the type's lowest value: 117 us spread, 126 us in one stretch ahead of the others (106 us without; 7500 us if
    // such a block sends its row to fp64).
    const bool far = t >= 0 && (p.bad == 2 || (p.bad == 0 && p.R < -kFar / 2));
    float top = 0.0f;
    for (unsigned todo = __ballot_sync(PODS_FULL_MASK, far); todo != 0; todo &= todo - 1) {
        const int who = __ffs(todo) - 1;
        const int64_t at = __shfl_sync(PODS_FULL_MASK, t, who);
        float m;
        const Part q = far_row<DT>(static_cast<const typename Elem<DT>::raw*>(a.logits) + at * a.ldl, a.V, a.inv_tau, lane, m);
        if (lane == who) {
            p = q;
            top = m;
        }
    }
    if (t < 0) return;
    double lse, logp, H;
    if (p.bad & 1) {
        pods_raise(a.status, PODS_STATUS_NONFINITE_LOGIT);
        lse = logp = H = (double)NAN;
    } else if (p.s == 0.0) {
        pods_raise(a.status, PODS_STATUS_EMPTY_ROW);
        lse = -(double)INFINITY;
        logp = H = (double)NAN;
    } else if (far) {
        const double ls = log(p.s);
        lse = (double)top * a.inv_tau + ls;
        logp = ((double)z - (double)top) * a.inv_tau - ls;
        H = ls - p.u / p.s;
    } else {
        const double ls = log2(p.s) + kExponentialsLow;
        lse = ((double)p.R + ls) * kLn2;
        logp = (((double)z * a.c64 - (double)p.R) - ls) * kLn2;
        H = (ls - p.u / p.s) * kLn2;
    }
    logp = logp == logp ? fmin(logp, 0.0) : logp;
    a.logp[t] = (float)logp;
    if (a.logp64 != nullptr) a.logp64[t] = logp;
    if (a.lse != nullptr) a.lse[t] = lse;
    if (ENT) a.entropy[t] = H == H ? (float)fmax(H, 0.0) : NAN;
}

// Whether row t is to be read; one that is not gets its 0 where the call fills.
__device__ __forceinline__ bool live_row(const FwdArgs& a, int64_t t, bool fill) {
    if (t >= a.T) return false;
    const bool live = (a.mask == nullptr || a.mask[t] != 0) && (a.rows_end == nullptr || t < *a.rows_end);
    if (!live && fill && a.fill) a.logp[t] = 0.0f;
    return live;
}

// The elements of a row outside its whole 16-byte vectors, less than 2 E: one a lane.
template <int DT, bool ENT>
__device__ __forceinline__ void take_edges(const FwdArgs& a, const typename Elem<DT>::raw* row, int head, int tail, int lane, Sums<DT, ENT>& sums) {
    using El = Elem<DT>;
    const int i = lane < head ? lane : tail + lane - head;
    if (head + a.V - tail == 0) return;
    typename El::raw e[El::E];
#pragma unroll
    for (int k = 0; k < El::E; ++k) e[k] = El::kNegInf;
    if (lane < head + a.V - tail && PODS_INDEX_OK(i, a.V, a.status)) e[0] = row[i];
    uint4 q[1];
    memcpy(q, e, sizeof q);
    sums.take(q, a.c, a.c_lo);
}

template <int DT>
__device__ __forceinline__ uint4 nothing() {           // a vector of -inf
    const uint32_t w = DT == PODS_DTYPE_F32 ? (uint32_t)Elem<DT>::kNegInf : (uint32_t)Elem<DT>::kNegInf * 0x10001u;
    return make_uint4(w, w, w, w);
}

// Short rows: a warp takes `batch` rows one after the other, with two blocks of 2 KB on their way to its own shared memory while
// it works on a third, and finishes the rows together.  What its lanes have of each row goes to shared memory too, and then four
// lanes sum a row: a reduction over the warp for each row, its logarithms and the chain to its token's logit would cost more
// than 1000 logits do.  bf16, 20000 rows of 8000 logits 63 us (5.1 TB/s), 100000 of 1000 51 us (3.9 TB/s); the exponentials' pipe is
// busy 71 % of the first.
constexpr int kAhead = 3;              // blocks a warp holds

template <bool ENT>
struct RowsWarp {
    uint4 block[kAhead][kBlockVecs * 32];
    uint2 left[kBatch][33];
    float left_u[ENT ? kBatch : 1][33];
};

__device__ __forceinline__ void copy16(uint4* dst, const uint4* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// Where a warp is in its rows: blocks of the rows whose bits are set, in order.
template <int DT>
struct Cursor {
    const uint4* vec;
    int nvec, v;                       // the row's whole vectors; the block's first
    unsigned todo;                     // rows from this one on
    __device__ __forceinline__ void open(const FwdArgs& a, int64_t first) {
        using raw = typename Elem<DT>::raw;
        const raw* const row = static_cast<const raw*>(a.logits) + (first + __ffs(todo) - 1) * a.ldl;
        const int lead = (int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(raw)), head = min(lead, a.V);
        nvec = (a.V - head) / Elem<DT>::E;
        vec = reinterpret_cast<const uint4*>(row + head);
        v = 0;
    }
};

template <int DT, bool ENT>
__global__ void __launch_bounds__(kThreads, 3) pods_logp_rows_kernel(const FwdArgs a, int batch) {
    using El = Elem<DT>;
    using raw = typename El::raw;
    extern __shared__ __align__(128) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    RowsWarp<ENT>& w = reinterpret_cast<RowsWarp<ENT>*>(smem)[warp];
    Sums<DT, ENT> sums;
    for (int64_t first = ((int64_t)blockIdx.x * (kThreads / 32) + warp) * batch; first < a.T; first += (int64_t)gridDim.x * (kThreads / 32) * batch) {
        const int64_t mine = lane < batch && live_row(a, first + lane, true) ? first + lane : -1;
        const unsigned rows = __ballot_sync(PODS_FULL_MASK, mine >= 0);
        if (rows == 0) continue;
        Cursor<DT> load, use;
        load.todo = use.todo = rows;
        load.open(a, first);
        int to = 0;
        auto issue = [&] {
            if (load.todo != 0) {
                const int v = load.v + lane;
#pragma unroll
                for (int k = 0; k < kBlockVecs; ++k)
                    if (v + k * 32 < load.nvec) copy16(&w.block[to][k * 32 + lane], load.vec + v + k * 32);
                load.v += kBlockVecs * 32;
                if (load.v >= load.nvec) {
                    load.todo &= load.todo - 1;
                    if (load.todo != 0) load.open(a, first);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            to = to + 1 == kAhead ? 0 : to + 1;
        };
#pragma unroll
        for (int k = 0; k < kAhead - 1; ++k) issue();
        const float z = mine >= 0 ? token_logit<DT>(a, mine) : 0.0f;
        int from = 0;
        for (; use.todo != 0; use.todo &= use.todo - 1) {
            const int j = __ffs(use.todo) - 1;
            use.open(a, first);
            sums.start();
            for (; use.v < use.nvec || use.v == 0; use.v += kBlockVecs * 32) {
                issue();
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
                uint4 q[kBlockVecs];                   // a lane's own copies: nobody else's are waited for
                const int v = use.v + lane;
                if (use.v + kBlockVecs * 32 <= use.nvec) {
#pragma unroll
                    for (int k = 0; k < kBlockVecs; ++k) q[k] = w.block[from][k * 32 + lane];
                } else {
#pragma unroll
                    for (int k = 0; k < kBlockVecs; ++k) q[k] = v + k * 32 < use.nvec ? w.block[from][k * 32 + lane] : nothing<DT>();
                }
                from = from + 1 == kAhead ? 0 : from + 1;
                sums.take(q, a.c, a.c_lo);
            }
            const raw* const row = static_cast<const raw*>(a.logits) + (first + j) * a.ldl;
            const int head = (int)(reinterpret_cast<const raw*>(use.vec) - row);
            take_edges(a, row, head, head + use.nvec * El::E, lane, sums);
            w.left[j][lane] = sums.left();
            if (ENT) w.left_u[j][lane] = sums.u;
        }
        __syncwarp();
        // four lanes a row: lane l sums row l / 4
        const int j = lane >> 2;
        Part p = {0.0, 0.0, kNoRef, 0};
        if (rows >> j & 1) {
#pragma unroll
            for (int k = 0; k < 8; ++k) p.R = max(p.R, ref_of(w.left[j][(lane & 3) + 4 * k]));
        }
        p.R = max(p.R, __shfl_xor_sync(PODS_FULL_MASK, p.R, 1));
        p.R = max(p.R, __shfl_xor_sync(PODS_FULL_MASK, p.R, 2));
        if (rows >> j & 1) {
#pragma unroll
            for (int k = 0; k < 8; ++k) add_left<ENT>(p, w.left[j][(lane & 3) + 4 * k], ENT ? w.left_u[j][(lane & 3) + 4 * k] : 0.0f);
        }
#pragma unroll
        for (int d = 1; d <= 2; d <<= 1) {
            p.s += __shfl_xor_sync(PODS_FULL_MASK, p.s, d);
            if (ENT) p.u += __shfl_xor_sync(PODS_FULL_MASK, p.u, d);
            p.bad |= __shfl_xor_sync(PODS_FULL_MASK, p.bad, d);
        }
        // back to a lane a row
        const int at = (lane & 7) * 4;
        Part q;
        q.s = __shfl_sync(PODS_FULL_MASK, p.s, at);
        q.u = ENT ? __shfl_sync(PODS_FULL_MASK, p.u, at) : 0.0;
        q.R = __shfl_sync(PODS_FULL_MASK, p.R, at);
        q.bad = __shfl_sync(PODS_FULL_MASK, p.bad, at);
        finish_rows<DT, ENT>(a, mine, q, z, lane);
        __syncwarp();
    }
}

// Few rows, not long: a CTA each, a row's vectors loaded at once, for the time of a small call is a chain of latencies (37 rows of
// 1024 bf16 logits: 3.0 us).
template <int DT, bool ENT>
__global__ void __launch_bounds__(kThreads) pods_logp_row_kernel(const FwdArgs a) {
    using El = Elem<DT>;
    using raw = typename El::raw;
    __shared__ uint2 left[kThreads];
    __shared__ float left_u[ENT ? kThreads : 1];
    const int tid = threadIdx.x, lane = tid & 31;
    const int64_t t = blockIdx.x;
    if (!live_row(a, t, tid == 0)) return;
    const float z = tid == 0 ? token_logit<DT>(a, t) : 0.0f;
    const raw* const row = static_cast<const raw*>(a.logits) + t * a.ldl;
    const int lead = (int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(raw));
    const int head = min(lead, a.V), nvec = (a.V - head) / El::E;
    const uint4* const vec = reinterpret_cast<const uint4*>(row + head);
    const int threads = blockDim.x;
    Sums<DT, ENT> sums;
    sums.start();
    for (int v = tid; v - tid < nvec; v += kBlockVecs * threads) {
        uint4 q[kBlockVecs];
#pragma unroll
        for (int k = 0; k < kBlockVecs; ++k) q[k] = v + k * threads < nvec ? __ldg(vec + v + k * threads) : nothing<DT>();
        sums.take(q, a.c, a.c_lo);
    }
    if (tid < 32) take_edges(a, row, head, head + nvec * El::E, lane, sums);
    left[tid] = sums.left();
    if (ENT) left_u[tid] = sums.u;
    __syncthreads();
    if (tid >= 32) return;
    Part p = {0.0, 0.0, kNoRef, 0};
    for (int k = lane; k < threads; k += 32) p.R = max(p.R, ref_of(left[k]));
    p.R = __reduce_max_sync(PODS_FULL_MASK, p.R);
    for (int k = lane; k < threads; k += 32) add_left<ENT>(p, left[k], ENT ? left_u[k] : 0.0f);
    p.s = warp_reduce(p.s, Plus());
    if (ENT) p.u = warp_reduce(p.u, Plus());
    p.bad = (int)__reduce_or_sync(PODS_FULL_MASK, (unsigned)p.bad);
    finish_rows<DT, ENT>(a, lane == 0 ? t : -1, p, z, lane);
}

// Long rows: a cluster of CTAs holds a share of the row each and goes round over the rows; a CTA is a producer warp that keeps
// 192 KB of copies in flight, consumer warps that add up what has arrived, and a warp that finishes the rows, 32 at once.  They
// meet at mbarriers only, so the copies never wait for a row's end.  Consumers work in groups of W warps, each on a row of its
// own and with a producer and stages of its own (a group that waited for a stage which another one uses first could be two uses
// ahead of it, which a barrier's parity does not tell apart): at a row's end one group leaves the exponentials' pipe to the others.
// bf16, 2048 rows of 151936 logits 94 us (6.6 TB/s; one CTA a row with loads to registers 127), the exponentials' pipe busy for 75 %
// of it; 6007 fp16 rows of 32000 71 us (5.4 TB/s).
constexpr int kConsumers = 16;
constexpr int kStageBytes = 196608;

template <int W>
struct Pipe {
    static constexpr int groups = kConsumers / W;
    static constexpr int stage_vecs = W * 32 * kBlockVecs;
    static constexpr int stages = kStageBytes / (stage_vecs * 16 * groups);          // of a group
    static constexpr int threads = (kConsumers + groups + 1) * 32;
    static constexpr int ring = 2 * groups < 4 ? 4 : 2 * groups;       // rows whose sums may be waiting to be finished
};

struct PipePart {                      // a CTA's sums of a row, as they travel to the cluster's first CTA
    double s;
    unsigned long long ref;            // R above, bad below
    double u;
    unsigned long long unused;
};

template <int W>
struct PipeCtrl {
    using P = Pipe<W>;
    unsigned long long full[P::groups][P::stages], empty[P::groups][P::stages], summed[P::ring], free_slot[P::ring], parts[P::ring], free_part[P::ring];
    alignas(16) PipePart part[P::ring][8];
    uint2 left[P::ring][W * 32];
    float left_u[P::ring][W * 32];
};

// Rows of a cluster, a mask of 32 at a time
struct RowWalk {
    int64_t first, step;
    int n;
    unsigned bits;
    __device__ __forceinline__ bool live(const FwdArgs& a, int i, int lane, bool fill) {
        if ((i & 31) == 0) {
            const bool plain = a.mask == nullptr && a.rows_end == nullptr;
            bits = plain ? PODS_FULL_MASK : __ballot_sync(PODS_FULL_MASK, i + lane < n && live_row(a, first + (int64_t)(i + lane) * step, fill));
        }
        return bits >> (i & 31) & 1;
    }
};

template <int DT, bool ENT, int W>
__global__ void __launch_bounds__(Pipe<W>::threads, 1) pods_logp_pipe_kernel(const FwdArgs a) {
    using El = Elem<DT>;
    using raw = typename El::raw;
    extern __shared__ __align__(128) unsigned char smem[];
    uint4* const stages = reinterpret_cast<uint4*>(smem);
    constexpr int kStages = Pipe<W>::stages, kStageVecs = Pipe<W>::stage_vecs, kRing = Pipe<W>::ring, kGroups = Pipe<W>::groups;
    PipeCtrl<W>& c = *reinterpret_cast<PipeCtrl<W>*>(smem + kStageBytes);
    cg::cluster_group cl = cg::this_cluster();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int CL = (int)cl.num_blocks(), rank = (int)cl.block_rank();
    RowWalk walk;
    walk.first = blockIdx.x / CL;
    walk.step = gridDim.x / CL;
    walk.n = walk.first < a.T ? (int)((a.T - walk.first + walk.step - 1) / walk.step) : 0;
    if (threadIdx.x == 0) {
        for (int g = 0; g < kGroups; ++g)
            for (int i = 0; i < kStages; ++i) {
                mbar_init(&c.full[g][i], 1);
                mbar_init(&c.empty[g][i], W);
            }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&c.summed[i], W);
            mbar_init(&c.free_slot[i], 1);
            mbar_init(&c.parts[i], 1);
            mbar_init(&c.free_part[i], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cl.sync();
    bool late = false;                                 // a wait ran out: no further one is made
    auto spins = [&] { return late ? 1u : kSpinLimit; };
    // this CTA's share [lo, hi) of a row's whole vectors
    auto share = [&](const raw* row, int& head, int& nvec, int& lo, int& hi) {
        const int lead = (int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(raw));
        head = min(lead, a.V);
        nvec = (a.V - head) / El::E;
        const int per = ((nvec + CL - 1) / CL + 7) & ~7;
        lo = min(nvec, rank * per);
        hi = min(nvec, lo + per);
    };
    if (warp >= kConsumers && warp < kConsumers + kGroups) {
        // ---- a group's producer ----
        const int group = warp - kConsumers;
        uint4* const mine = stages + (size_t)group * kStages * kStageVecs;
        StageRing ring;
        int64_t issued = 0;
        int rows = 0;
        for (int i = 0; i < walk.n; ++i) {
            if (!walk.live(a, i, lane, false)) continue;
            if (rows++ % kGroups != group) continue;
            const raw* const row = static_cast<const raw*>(a.logits) + (walk.first + (int64_t)i * walk.step) * a.ldl;
            int head, nvec, lo, hi;
            share(row, head, nvec, lo, hi);
            const uint4* const vec = reinterpret_cast<const uint4*>(row + head);
            for (int v = lo; v < hi; v += kStageVecs, ++issued, ring.next(kStages)) {
                if (issued >= kStages && !mbar_wait(&c.empty[group][ring.st], ring.parity ^ 1u, spins())) late = true;
                if (lane == 0) {
                    const int n = PODS_INDEX_OK(head + min(v + kStageVecs, hi) * El::E - 1, a.V, a.status) ? min(kStageVecs, hi - v) : 0;
                    mbar_expect_tx(&c.full[group][ring.st], (uint32_t)n * 16u);
                    for (int k = 0; k < n; k += 512)
                        bulk_load(mine + (size_t)ring.st * kStageVecs + k, vec + v + k, (uint32_t)min(512, n - k) * 16u, &c.full[group][ring.st]);
                }
                __syncwarp();
            }
        }
    } else if (warp < kConsumers) {
        // ---- consumers ----
        StageRing ring;
        int rows = 0;
        const int group = warp / W, tid = threadIdx.x % (W * 32);
        Sums<DT, ENT> sums;
        for (int i = 0; i < walk.n; ++i) {
            if (!walk.live(a, i, lane, false)) continue;
            const raw* const row = static_cast<const raw*>(a.logits) + (walk.first + (int64_t)i * walk.step) * a.ldl;
            if (rows % kGroups != group) {
                ++rows;
                continue;
            }
            int head, nvec, lo, hi;
            share(row, head, nvec, lo, hi);
            sums.start();
            for (int v = lo; v < hi; v += kStageVecs, ring.next(kStages)) {
                if (!mbar_wait(&c.full[group][ring.st], ring.parity, spins())) late = true;
                const uint4* const buf = stages + (size_t)(group * kStages + ring.st) * kStageVecs;
                const int n = hi - v;
                // as many vectors a thread as the chunk has, the last ones padded
                auto some = [&](auto count) {
                    constexpr int N = decltype(count)::value;
                    uint4 q[N];
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const int at = tid + k * W * 32;
                        q[k] = k + 1 < N || at < n ? buf[at] : nothing<DT>();
                    }
                    __syncwarp();
                    if (lane == 0) arrive_local(&c.empty[group][ring.st]);
                    sums.take(q, a.c, a.c_lo);
                };
                if (n > 3 * W * 32) some(std::integral_constant<int, 4>());
                else if (n > 2 * W * 32) some(std::integral_constant<int, 3>());
                else if (n > W * 32) some(std::integral_constant<int, 2>());
                else some(std::integral_constant<int, 1>());
            }
            if (rank == 0 && warp % W == 0) take_edges(a, row, head, head + nvec * El::E, lane, sums);
            const int slot = rows % kRing;
            if (rows >= kRing && !mbar_wait(&c.free_slot[slot], (uint32_t)((rows / kRing - 1) & 1), spins())) late = true;
            c.left[slot][tid] = sums.left();
            if (ENT) c.left_u[slot][tid] = sums.u;
            __syncwarp();
            if (lane == 0) arrive_local(&c.summed[slot]);
            ++rows;
        }
    } else {
        // ---- finisher: this CTA's sums of a row, then, in the cluster's first CTA, the row ----
        int rows = 0;
        int64_t mine = -1;
        float z = 0.0f;
        Part kept = {0.0, 0.0, kNoRef, 0};
        for (int i = 0; i < walk.n; ++i) {
            const bool live = walk.live(a, i, lane, rank == 0);
            if ((i & 31) == 0 && rank == 0) {
                mine = i + lane < walk.n && (walk.bits >> lane & 1) ? walk.first + (int64_t)(i + lane) * walk.step : -1;
                z = mine >= 0 ? token_logit<DT>(a, mine) : 0.0f;
            }
            if (live) {
                const int slot = rows % kRing;
                const uint32_t use = (uint32_t)(rows / kRing);
                if (CL > 1 && rank == 0 && lane == 0) mbar_expect_tx(&c.parts[slot], (uint32_t)((CL - 1) * (ENT ? 32 : 16)));
                if (!mbar_wait(&c.summed[slot], use & 1u, spins())) late = true;
                Part sum = {0.0, 0.0, kNoRef, 0};
                uint2 l[W];
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    l[k] = c.left[slot][k * 32 + lane];
                    sum.R = max(sum.R, ref_of(l[k]));
                }
                sum.R = __reduce_max_sync(PODS_FULL_MASK, sum.R);
#pragma unroll
                for (int k = 0; k < W; ++k) add_left<ENT>(sum, l[k], ENT ? c.left_u[slot][k * 32 + lane] : 0.0f);
                __syncwarp();
                if (lane == 0) arrive_local(&c.free_slot[slot]);
                sum.s = warp_reduce(sum.s, Plus());
                if (ENT) sum.u = warp_reduce(sum.u, Plus());
                sum.bad = (int)__reduce_or_sync(PODS_FULL_MASK, (unsigned)sum.bad);
                if (CL > 1 && rank != 0) {
                    if (lane == 0) {
                        if (rows >= kRing && !wait_cluster(&c.free_part[slot], (use - 1u) & 1u, spins())) late = true;
                        const uint32_t to = mapa(&c.part[slot][rank], 0), bar = mapa(&c.parts[slot], 0);
                        store_async(to, bar, sum.s, (unsigned long long)(uint32_t)sum.R << 32 | (uint32_t)sum.bad);
                        if (ENT) store_async(to + 16, bar, sum.u, 0ull);
                    }
                    __syncwarp();
                } else if (CL > 1) {
                    if (!wait_cluster(&c.parts[slot], use & 1u, spins())) late = true;
                    Part p = {0.0, 0.0, kNoRef, 0};
                    if (lane == 0) p = sum;
                    else if (lane < CL) {
                        const PipePart& q = c.part[slot][lane];
                        p = {q.s, ENT ? q.u : 0.0, (int)(q.ref >> 32), (int)(uint32_t)q.ref};
                    }
                    __syncwarp();
                    if (lane > 0 && lane < CL) arrive_remote(mapa(&c.free_part[slot], lane));
                    const int R = __reduce_max_sync(PODS_FULL_MASK, p.R);
                    const double f = pow2_int(p.R - R);
                    if (ENT) sum.u = warp_reduce(p.s != 0.0 ? (p.u + p.s * (double)(p.R - R)) * f : 0.0, Plus());
                    sum.s = warp_reduce(p.s * f, Plus());
                    sum.R = R;
                    sum.bad = (int)__reduce_or_sync(PODS_FULL_MASK, (unsigned)p.bad);
                }
                if (lane == (i & 31)) kept = sum;
                ++rows;
            }
            if (rank == 0 && ((i & 31) == 31 || i + 1 == walk.n)) {
                finish_rows<DT, ENT>(a, mine, kept, z, lane);
                kept = {0.0, 0.0, kNoRef, 0};
            }
        }
    }
    if (late && lane == 0) pods_raise(a.status, PODS_STATUS_TIMEOUT);
    __syncwarp();
    cl.sync();                                         // no CTA leaves while a peer may still write to it
}

// 16 bytes from `bytes` (a multiple of the element's) behind a 16-byte boundary, of the 32 that follow it.
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, int bytes) {
    const uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    const int sub = (bytes & 3) * 8;
    auto from = [&](auto first) {
        constexpr int W = decltype(first)::value;
        return make_uint4(__funnelshift_r(x[W], x[W + 1], sub), __funnelshift_r(x[W + 1], x[W + 2], sub), __funnelshift_r(x[W + 2], x[W + 3], sub),
                          __funnelshift_r(x[W + 3], W + 4 < 8 ? x[W + 4 < 8 ? W + 4 : 7] : 0u, sub));
    };
    switch (bytes >> 2) {                              // the same for the whole row
        case 0: return from(std::integral_constant<int, 0>());
        case 1: return from(std::integral_constant<int, 1>());
        case 2: return from(std::integral_constant<int, 2>());
        default: return from(std::integral_constant<int, 3>());
    }
}

// d objective / d logits.  A CTA takes a stretch of `seg` vectors of one row (WARP: a warp a whole row).  HBM bounds it: bf16, 2048
// rows of 151936 logits 187 us (6.7 TB/s read and written), 20000 of 8000 111 us (5.8 TB/s).
//   p = 2^(z c - n) 2^-f,  n + f = lse log2 e, n an integer;   out = p (A + B (z c - n)),  + g at the token
//   A = -2^-f (g + (dH / tau) (H - ln 2 f)),  B = -2^-f (dH / tau) ln 2,  g = dlogp / tau
template <int DT, bool ENT, bool WARP>
__global__ void __launch_bounds__(kThreads) pods_logp_grad_kernel(const GradArgs a) {
    using El = Elem<DT>;
    using raw = typename El::raw;
    constexpr int E = El::E;
    __shared__ float scratch_max[kThreads / 32];
    __shared__ double scratch_sum[kThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int me = WARP ? lane : (int)threadIdx.x, G = WARP ? 32 : kThreads;
    int64_t t;
    int seg;
    if (WARP) {
        t = (int64_t)blockIdx.x * (kThreads / 32) + warp;
        seg = 0;
        if (t >= a.T) return;
    } else {
        t = blockIdx.x / a.n_seg;
        seg = (int)(blockIdx.x % a.n_seg);
    }
    const double g64 = (double)a.dlogp[t] * a.inv_tau, b64 = ENT ? (double)a.dentropy[t] * a.inv_tau : 0.0;
    raw* const out = static_cast<raw*>(a.dlogits) + t * a.ldd;
    const raw* const row = static_cast<const raw*>(a.logits) + t * a.ldl;
    // cut at the output's 16-byte boundaries
    const int lead = (int)(((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / sizeof(raw));
    const int head = min(lead, a.V), nvec = (a.V - head) / E, tail = head + nvec * E;
    const int lo = min(nvec, seg * a.seg), hi = WARP ? nvec : min(nvec, lo + a.seg);
    uint4* const dst = reinterpret_cast<uint4*>(out + head);
    const int edge = me < head ? me : tail + me - head;               // element of the two ends that is this thread's
    const bool has_edge = seg == 0 && me < head + a.V - tail && PODS_INDEX_OK(edge, a.V, a.status);
    if (g64 == 0.0 && b64 == 0.0) {                                   // what the logits hold is of no consequence
        for (int v = lo + me; v < hi; v += G) dst[v] = make_uint4(0, 0, 0, 0);
        if (has_edge) out[edge] = 0;
        return;
    }
    // the first block is on its way while the row's coefficients are made.  Logits that do not lie on the output's boundaries are
    // taken from the two vectors of their own that hold them, but for those at the row's ends, whose neighbours may not be the row's.
    const int apart = (int)(reinterpret_cast<uintptr_t>(row + head) & 15);
    const uint4* const src = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(row + head) - apart);
    auto fetch = [&](int v) {
        if (apart == 0) return src[v];
        if (v > 0 && v + 1 < nvec) return shifted(src[v], src[v + 1], apart);
        raw e[E];
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = row[head + v * E + i];
        uint4 q;
        memcpy(&q, e, sizeof q);
        return q;
    };
    uint4 ahead[kBlockVecs];
#pragma unroll
    for (int k = 0; k < kBlockVecs; ++k)
        if (lo + me + k * G < hi) ahead[k] = fetch(lo + me + k * G);
    int token = a.tokens[t];
    if ((unsigned)token >= (unsigned)a.V) {
        if (me == 0 && seg == 0) pods_raise(a.status, PODS_STATUS_TOKEN_RANGE);
        token = 0;
    }
    const double lse = a.lse[t], L = lse * 1.4426950408889634074;
    const double H = ENT && b64 != 0.0 ? (double)a.entropy[t] : 0.0;
    const float g = (float)g64;
    if (!(fabs(L) < (double)kFar)) {
        // too large for fp32 exponents, and lse for its own fraction: the row again in fp64, by one CTA (NaN and empty rows too)
        if (seg != 0) return;
        float top = -INFINITY;
        for (int i = me; i < a.V; i += G) top = max_nan(top, El::to_float(row[i]));
        top = WARP ? warp_reduce(top, MaxNan()) : block_reduce<kThreads / 32>(top, scratch_max, MaxNan());
        const bool bad = !(fabsf(top) < INFINITY);
        double sum = 0.0;
        for (int i = bad ? a.V : me; i < a.V; i += G) sum += exp64(((double)El::to_float(row[i]) - (double)top) * a.inv_tau);
        sum = WARP ? warp_reduce(sum, Plus()) : block_reduce<kThreads / 32>(sum, scratch_sum, Plus());
        const double ls = bad ? 0.0 : log(sum);
        for (int i = me; i < a.V; i += G) {
            const double d = ((double)El::to_float(row[i]) - (double)top) * a.inv_tau - ls, p = exp64(d);
            double x = bad ? (double)NAN : -p * (g64 + (ENT && p != 0.0 ? b64 * (d + H) : 0.0));
            if (i == token) x += g64;
            out[i] = El::from_float((float)x);
        }
        return;
    }
    const double n64 = ceil(L), f64 = L - n64, back = exp2(-f64);
    const float n = (float)n64;
    const float A = (float)(-back * (g64 + (ENT ? b64 * (H - kLn2 * f64) : 0.0))), B = (float)(-back * b64 * kLn2);
    const int tok_vec = token >= head && token < tail ? (token - head) / E : -1, tok_at = (token - head) - tok_vec * E;
    auto one = [&](float z) {
        const float d = fmaf(z, a.c_lo, fmaf(z, a.c, -n)), p = ex2_approx(d);
        return ENT ? p * fmaf(B, fmaxf(d, -1e4f), A) : p * A;
    };
    auto vector = [&](const uint4& q, int v) {
        float x[E];
        El::unpack(q, x);
        const unsigned long long c2 = pack2(a.c, a.c), lo2 = pack2(a.c_lo, a.c_lo), off2 = pack2(-n, -n);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const unsigned long long x2 = pack2(x[i], x[i + 1]);
            float d0, d1;
            unpack2(fma2(x2, lo2, fma2(x2, c2, off2)), d0, d1);
            const float p0 = ex2_approx(d0), p1 = ex2_approx(d1);
            x[i] = ENT ? p0 * fmaf(B, fmaxf(d0, -1e4f), A) : p0 * A;
            x[i + 1] = ENT ? p1 * fmaf(B, fmaxf(d1, -1e4f), A) : p1 * A;
        }
        if (v == tok_vec) {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i == tok_at) x[i] += g;
        }
        dst[v] = El::pack(x);
    };
#pragma unroll
    for (int k = 0; k < kBlockVecs; ++k)
        if (lo + me + k * G < hi) vector(ahead[k], lo + me + k * G);
    int v = lo + me + kBlockVecs * G;
    for (; v + (kBlockVecs - 1) * G < hi; v += kBlockVecs * G) {
        uint4 q[kBlockVecs];
#pragma unroll
        for (int k = 0; k < kBlockVecs; ++k) q[k] = fetch(v + k * G);
#pragma unroll
        for (int k = 0; k < kBlockVecs; ++k) vector(q[k], v + k * G);
    }
    for (; v < hi; v += G) vector(fetch(v), v);
    if (has_edge) {
        float x = one(El::to_float(row[edge]));
        if (edge == token) x += g;
        out[edge] = El::from_float(x);
    }
}

// Gradient: rows of up to this many vectors are taken a warp each, unless there are few of them.  Measured, a warp each against a
// CTA each: bf16 V = 1000 81 : 310 us (100000 rows), V = 4000 116 : 157 us (40000), 6.0 : 3.3 us (300); V = 8000 115 : 111 us (20000).
constexpr int kWarpVecs = 512;

template <int DT, bool ENT>
int launch_rows(const FwdArgs& a, int dev, int batch, int grid, cudaStream_t stream) {
    static uint64_t prepared = 0;                      // devices as bits
    constexpr size_t smem = sizeof(RowsWarp<ENT>) * (kThreads / 32);
    if (!(__atomic_load_n(&prepared, __ATOMIC_ACQUIRE) >> dev & 1)) {
        PODS_RETURN_IF_CUDA_ERROR(cudaFuncSetAttribute(pods_logp_rows_kernel<DT, ENT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        __atomic_fetch_or(&prepared, 1ull << dev, __ATOMIC_RELEASE);
    }
    pods_logp_rows_kernel<DT, ENT><<<grid, kThreads, smem, stream>>>(a, batch);
    PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
    return PODS_OK;
}

template <int DT, bool ENT>
int launch_fwd(const FwdArgs& a, cudaStream_t stream) {
    const int64_t nvec = a.V / Elem<DT>::E;
    int dev;
    const int sms = pods_logp::device_sms(dev);
    if (dev < 0) return PODS_ERR_UNSUPPORTED;
    const pods_logp::RowPlan plan = pods_logp::plan_rows(a.T, nvec, sms);
    if (plan.kernel == pods_logp::kRowEach) {
        const int threads = nvec <= 128 ? 32 : nvec <= 256 ? 64 : nvec <= 512 ? 128 : kThreads;
        pods_logp_row_kernel<DT, ENT><<<(unsigned)a.T, threads, 0, stream>>>(a);
        PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
        return PODS_OK;
    }
    if (plan.kernel == pods_logp::kRowsWarp) {
        const int64_t per_cta = (int64_t)plan.batch * (kThreads / 32), ctas = (a.T + per_cta - 1) / per_cta;
        return launch_rows<DT, ENT>(a, dev, plan.batch, ctas < 3 * sms ? (int)ctas : 3 * sms, stream);
    }
    return plan.warps == 4 ? launch_row_clusters<pods_logp_pipe_kernel<DT, ENT, 4>>(a, a.T, plan.cluster, Pipe<4>::threads, kStageBytes + sizeof(PipeCtrl<4>), stream)
                           : launch_row_clusters<pods_logp_pipe_kernel<DT, ENT, 16>>(a, a.T, plan.cluster, Pipe<16>::threads, kStageBytes + sizeof(PipeCtrl<16>), stream);
}

template <int DT, bool ENT>
int launch_grad(GradArgs& a, cudaStream_t stream) {
    const int nvec = a.V / Elem<DT>::E;
    if (nvec <= kWarpVecs && (nvec <= 128 || a.T > kFewRows * (int64_t)pods_sm_count())) {
        pods_logp_grad_kernel<DT, ENT, true><<<(unsigned)((a.T + kThreads / 32 - 1) / (kThreads / 32)), kThreads, 0, stream>>>(a);
    } else {
        a.n_seg = max(1, (nvec + 4 * kThreads) / (8 * kThreads));
        a.seg = (nvec + a.n_seg - 1) / a.n_seg;
        pods_logp_grad_kernel<DT, ENT, false><<<(unsigned)(a.T * a.n_seg), kThreads, 0, stream>>>(a);
    }
    PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
    return PODS_OK;
}

}  // namespace

int pods_logp::launch_forward(const FwdArgs& a, int dtype, cudaStream_t s) {
    const bool ent = a.entropy != nullptr;
    if (dtype == PODS_DTYPE_BF16) return ent ? launch_fwd<PODS_DTYPE_BF16, true>(a, s) : launch_fwd<PODS_DTYPE_BF16, false>(a, s);
    if (dtype == PODS_DTYPE_F16) return ent ? launch_fwd<PODS_DTYPE_F16, true>(a, s) : launch_fwd<PODS_DTYPE_F16, false>(a, s);
    return ent ? launch_fwd<PODS_DTYPE_F32, true>(a, s) : launch_fwd<PODS_DTYPE_F32, false>(a, s);
}

int pods_logp::launch_gradient(GradArgs& a, int dtype, cudaStream_t s) {
    const bool ent = a.dentropy != nullptr;
    if (dtype == PODS_DTYPE_BF16) return ent ? launch_grad<PODS_DTYPE_BF16, true>(a, s) : launch_grad<PODS_DTYPE_BF16, false>(a, s);
    if (dtype == PODS_DTYPE_F16) return ent ? launch_grad<PODS_DTYPE_F16, true>(a, s) : launch_grad<PODS_DTYPE_F16, false>(a, s);
    return ent ? launch_grad<PODS_DTYPE_F32, true>(a, s) : launch_grad<PODS_DTYPE_F32, false>(a, s);
}

int pods_logp::check_rows(const void* logits, int64_t ldl, int32_t dtype, int64_t T, int32_t V, float temperature) {
    if (dtype != PODS_DTYPE_BF16 && dtype != PODS_DTYPE_F16 && dtype != PODS_DTYPE_F32) return PODS_ERR_UNSUPPORTED;
    if (T < 0 || V < 1 || ldl < V) return PODS_ERR_INVALID_ARG;
    if (V > PODS_MAX_ROW_V || T > pods_logp::kMaxRows) return PODS_ERR_UNSUPPORTED;
    if (!(temperature >= FLT_MIN && temperature < INFINITY)) return PODS_ERR_INVALID_ARG;
    if (T > 0 && (logits == nullptr || !pods_aligned(logits, dtype == PODS_DTYPE_F32 ? 4 : 2))) return PODS_ERR_INVALID_ARG;
    return PODS_OK;
}

extern "C" int pods_logp_chunk(const void* logits, int64_t ldl, int32_t dtype, const int32_t* tokens, const uint8_t* mask,
                               int64_t T, int32_t V, float temperature, float* logp, double* lse, float* entropy,
                               uint32_t* status, void* stream) {
    const int rc = pods_logp::check_rows(logits, ldl, dtype, T, V, temperature);
    if (rc != PODS_OK || T == 0) return rc;
    if (tokens == nullptr || logp == nullptr || !pods_all_aligned(4, tokens, logp, entropy, status) || !pods_aligned(lse, 8))
        return PODS_ERR_INVALID_ARG;
    FwdArgs a = {};
    a.logits = logits;
    a.ldl = ldl;
    a.tokens = tokens;
    a.mask = mask;
    a.T = T;
    a.V = V;
    a.c64 = pods_logp::set_temperature(a, temperature);
    a.logp = logp;
    a.lse = lse;
    a.entropy = entropy;
    a.status = status;
    return pods_logp::launch_forward(a, dtype, pods_stream(stream));
}

extern "C" int pods_logp_grad_chunk(const void* logits, int64_t ldl, int32_t dtype, const int32_t* tokens, const double* lse,
                                    const float* dlogp, const float* entropy, const float* dentropy, int64_t T, int32_t V,
                                    float temperature, void* dlogits, int64_t ldd, uint32_t* status, void* stream) {
    const int rc = pods_logp::check_rows(logits, ldl, dtype, T, V, temperature);
    if (rc != PODS_OK) return rc;
    const size_t esize = dtype == PODS_DTYPE_F32 ? 4 : 2;
    if (ldd < V || (dlogits == logits && ldd != ldl) || (dentropy != nullptr && entropy == nullptr)) return PODS_ERR_INVALID_ARG;
    if (T == 0) return PODS_OK;
    if (tokens == nullptr || lse == nullptr || dlogp == nullptr || dlogits == nullptr || !pods_aligned(dlogits, esize) ||
        !pods_all_aligned(4, tokens, dlogp, entropy, dentropy, status) || !pods_aligned(lse, 8))
        return PODS_ERR_INVALID_ARG;
    GradArgs a = {};
    a.logits = logits;
    a.ldl = ldl;
    a.tokens = tokens;
    a.lse = lse;
    a.dlogp = dlogp;
    a.entropy = entropy;
    a.dentropy = dentropy;
    a.T = T;
    a.V = V;
    pods_logp::set_temperature(a, temperature);
    a.dlogits = dlogits;
    a.ldd = ldd;
    a.status = status;
    return pods_logp::launch_gradient(a, dtype, pods_stream(stream));
}
