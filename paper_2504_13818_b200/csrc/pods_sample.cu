// pods_sample and pods_topk: one token a row drawn from logits, and the first K logits of a row with its log-normaliser.
//
// With z the row, d_v = (z_v - max z) / tau and e_v = exp(d_v), the kept set of every filter (top-k, top-p, min-p) is a
// prefix of the row's order "larger logit first, then lower id", so it is described by one threshold: a value and the
// highest id kept among the logits equal to it.  The token is the first kept id, ids ascending, whose running sum of e
// exceeds u times the kept sum.
//
// A cluster of CL CTAs holds the row in shared memory (row_cluster.cuh): HBM is read once whatever the filters ask for.
// Lanes own contiguous vectors of the CTA's segment, so a lane's, a warp's and a CTA's sums are stretches of the running sum.
//
//   all rows  each warp reduces its part to a sum of exponentials relative to 2^R, R the integer above its maximum's exponent,
//            and hands the pair to every CTA; parts are then brought together by powers of two, exactly and without an
//            exponential.  After this one cluster barrier every warp knows all parts in id order.
//   no filter  the warp whose part holds the drawn point takes the lane from the lane sums that it kept, and evaluates that
//            lane's few vectors again; every other warp goes on to the next row.
//   filters  one warp of each CTA also finds the r-th largest of the CTA's lanes' maxima; the least of these over the cluster is
//            a value that at least `want` logits reach, so the logits reaching it contain the first `want` of the order.  They are
//            listed (in the typical row a few hundred), every CTA ranks its own among all of them into the first CTA's list, and
//            the rest is fp64 arithmetic on that list.
//   wide nucleus  where the list does not reach far enough, or the lanes' maxima hold so little of the row's mass that it cannot
//            (then it is not made), a histogram of the row's mass over kBins stretches of logit brackets the border within a few
//            stretches; one sweep takes the sums above the bracket and lists what lies in it, and the list settles the border.
//            The sweep is fast at first, and in fp64 where the border is too close to call.
//   the rest  (a bracket full of ties, a top_k above the list) bisects the order-preserving keys of the values with counts and
//            fp64 sums over the resident row.
//
// Which token is drawn must not depend on how sums are split or rounded: a draw or a border that lies nearer to its
// neighbours than the error of the fast sums (fp32 exponentials, summed eight at a time in fp32 and then in fp64; see
// draw_margin) is taken again with fp64 exponentials throughout, so the outcome is that of fp64 arithmetic.
//
// What it takes on one B200 (6.54 TB/s measured copy rate; rows of 151936 bf16 unless said), and what bounds it:
//   512 rows, no filter   77 us = 2.0 TB/s: the pipeline 53 us (44 % of the issue slots, 48 % of the special-function pipe, the
//            rest waits of one row for its slowest part), then 5 % of these flat rows in fp64, 16 to 28 us
//   512 rows, nuclei of thousands   427 us: 82 K cycles a row, of which the histogram's shared-memory atomics 22 K, the bracket
//            sweep 14 K, ranking and border 16 K, first sweep and load 10 K, about ten cluster barriers the rest
//   512 rows, top_k 50 and top_p 0.95   139 us: the chain of one row, with its load ahead of it and nothing to overlap them
//   512 rows of 32000, top_k 300   249 to 290 us, 700   294 us: the lanes' maxima bound so many ids that the list overflows, and
//            the threshold is bisected with a sweep and a cluster barrier for each bit of the key
//   one row, top_k and top_p   19 us: a chain of cluster barriers, rankings and fp64 exponentials, not bandwidth; 64 fp32 rows
//            with settings of their own   43 us: two such chains, as clusters of eight hold only about 33 rows at a time
//   pods_topk, 1024 rows, K = 64   179 us = 1.7 TB/s; 16 fp32 rows of 32000, K = 20   12 us: the same chain, fewer steps
//   33554 rows of 1000, no filter   419 us = 0.16 TB/s: a CTA and its barriers for 2 KB

#include <float.h>
#include <stddef.h>

#include "row_cluster.cuh"

using namespace pods_row;

namespace {

constexpr int W = 8;                          // warps of a CTA (12 and 16 were slower on three of the four filter cases)
constexpr int kThreads = W * 32;
constexpr float kGreedyBelow = 0x1p-20f;      // temperatures below this are the arg-max
constexpr int kSampleList = 1024;             // entries that the sampler's first CTA orders
constexpr int kBins = 2048;                   // stretches of the mass histogram, as many as fit the ordered list's place
constexpr int kNoCut = 0x7fffffff;
constexpr int kMarked = -2;                   // token of a row that the pipeline leaves to fp64
constexpr int kRedoRows = 8192;               // rows of a cluster between two visits of the marked ones

// Errors of the fast sums, rigorously bounded.  An exponential e_v is off by at most (slope |d_v| + kFlat) of itself: the
// rounding of the fused multiply-add (2^-24 of the exponent; `far` rows take a difference first, 2^-24 more) and of log2e / tau,
// |d_v| deep (and ln 2 more, as R lies up to one above the maximum's exponent); the hardware exponential (2^-22.5) and the three
// roundings of a vector's sum, flat.  The mean of |d| under the row's distribution is at most ln V - ln Z (its entropy,
// ln Z + mean |d|, is at most ln V).
constexpr double kFlat = 3.6e-7;
__device__ __forceinline__ double deep_error(int V, double Z, float c, double tau_inv, bool far) {
    const float depth = fmaxf(0.0f, __logf((float)V) - __logf((float)Z)) + 0.7f;
    const double log2e = fabs((double)c / tau_inv * 0.6931471805599453 - 1.0);
    return ((far ? 1.2e-7 : 6e-8) + log2e) * (double)depth;
}
// How near an edge C of the running sum a drawn point u Z may lie before fp64 decides: the error of u Z - C, which with
// Z = C + rest is that of u rest - (1 - u) C where C is about u Z.
__device__ __forceinline__ double draw_margin(double u, double Z, double deep) {
    return (fmax(u, 1.0 - u) * deep + 2.1 * u * (1.0 - u) * kFlat + 1e-12) * Z;
}
// A point below this share of the kept sum is always fp64's: there a fast running sum of 0 need not be the row's start.  What
// it may hide of the ids ahead: exponentials below 2^-126 of their part's reference, which become 0 (at most 2^19 2^-125 of
// the sum), and what bracket_sum and fp64 additions round off (together below 3e-13).
constexpr double kFastFrom = 1e-12;
// Whether a drawn point `target` = u Z between the edges lo and hi of the fast running sum is sure to lie between the exact ones.
__device__ __forceinline__ bool draw_is_sure(double u, double target, double lo, double hi, double margin) {
    return u > kFastFrom && (target - lo > margin || lo == 0.0) && hi - target > margin;
}

struct SampleArgs {
    const void* logits;
    int64_t ldl, T;
    int V, seg, n_stages;
    const float* u;
    const float *temperature_row, *top_p_row, *min_p_row;
    const int32_t* top_k_row;
    float temperature, top_p, min_p;
    int32_t top_k;
    const uint8_t* mask;
    int32_t* tokens;
    float *logp, *logq;
    // pods_topk
    int K;
    int32_t* ids;
    float *values, *lse;
    int marked;                               // rows are marked for fp64
    int list_cap, own_cap;                    // entries of one CTA: its share of all lists, its own list
    uint32_t* status;
};

struct Part {                                 // of one warp
    double s;             // sum relative to the part's reference (to its maximum in fp64 rows)
    float m;              // its maximum
    float lim;            // a value that enough of its logits reach
    float near;           // mass of the lanes' maxima alone, relative to the part's reference
    int pad;
};

struct Xch {                                  // one CTA's word in an exchange
    double a, b;
    float m;
    int i, n;
};

struct RowCtrl {
    unsigned long long full;                  // the segment's copy
    Part part[2][kMaxCluster * W];            // exchanges alternate between two places, so that one barrier each is enough
    uint32_t redo[kRedoRows / 32];
    uint32_t top[kThreads];                   // the lanes' maxima, as keys
};
struct FilterCtrl {
    Xch x[2][kMaxCluster];
    double dpart[W];
    int ipart[W];
    int n_list, found, sure;
    int start[kMaxCluster], count[kMaxCluster];  // the CTAs' lists within `all`
    double weight;
};
// Shared memory: RowCtrl, the row's segment, FilterCtrl, lists.  Reached through the array's name wherever it is used, so that
// every access is known to be to shared memory.
extern __shared__ __align__(128) unsigned char smem_[];
constexpr int kRowCtrlBytes = (sizeof(RowCtrl) + 127) & ~127;
__device__ __forceinline__ RowCtrl& row_ctrl() { return *reinterpret_cast<RowCtrl*>(smem_); }
__device__ __forceinline__ uint4* row_buf() { return reinterpret_cast<uint4*>(smem_ + kRowCtrlBytes); }
__device__ __forceinline__ FilterCtrl& filter_ctrl(const SampleArgs& a) { return *reinterpret_cast<FilterCtrl*>(smem_ + kRowCtrlBytes + a.seg * 16); }
constexpr int kFilterCtrlBytes = (sizeof(FilterCtrl) + 127) & ~127;

// Sum of the threads ahead, in thread order; *total is the sum of all.  Never a difference of an inclusive sum and one's own
// part: a large part would round off what lies ahead of it, which a small u may ask for.
__device__ __forceinline__ double block_scan_ahead(double v, double* part, double* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_scan(v, lane);
    const double ahead = scan_ahead(v, lane);
    __syncthreads();
    if (lane == 31) part[warp] = v;
    __syncthreads();
    double before = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        if (w < warp) before += part[w];
        all += part[w];
    }
    *total = all;
    return ahead + before;
}

// Sorts list[0, n) ascending, n <= kSampleList; keys differ.  Few entries are ranked, each against all; many go through a
// bitonic network in registers (four a thread), of which only the steps across warps need shared memory.
__device__ __forceinline__ void sort_list(unsigned long long* list, int n) {
    const int tid = threadIdx.x;
    if (n <= kThreads) {
        int P = 1;
        while (P < 32 && n * P * 2 <= kThreads) P *= 2;
        const int i = tid / P, sub = tid & (P - 1);
        const unsigned long long key = i < n ? list[i] : 0ull;
        int r = 0;
#pragma unroll 4
        for (int k = sub; k < n; k += P) r += list[k] < key ? 1 : 0;
        for (int d = 1; d < P; d <<= 1) r += __shfl_xor_sync(PODS_FULL_MASK, r, d);
        __syncthreads();
        if (i < n && sub == 0) list[r] = key;
        __syncthreads();
        return;
    }
    constexpr int PT = kSampleList / kThreads;
    int m = 1;
    while (m < n) m <<= 1;
    unsigned long long v[PT];
#pragma unroll
    for (int k = 0; k < PT; ++k) v[k] = tid * PT + k < n ? list[tid * PT + k] : ~0ull;
    for (int size = 2; size <= m; size <<= 1) {
        for (int d = size >> 1; d >= PT; d >>= 1) {
            if (d >= 32 * PT) {
                __syncthreads();
#pragma unroll
                for (int k = 0; k < PT; ++k) list[tid * PT + k] = v[k];
                __syncthreads();
            }
#pragma unroll
            for (int k = 0; k < PT; ++k) {
                const int i = tid * PT + k;
                const unsigned long long o = d >= 32 * PT ? list[i ^ d] : __shfl_xor_sync(PODS_FULL_MASK, v[k], d / PT);
                const bool small = ((i & d) == 0) == ((i & size) == 0);
                v[k] = (o < v[k]) == small ? o : v[k];
            }
        }
#pragma unroll
        for (int d = PT / 2; d > 0; d >>= 1)
            if (d < size) {
#pragma unroll
                for (int k = 0; k < PT; ++k)
                    if ((k & d) == 0) {
                        const bool up = ((tid * PT + k) & size) == 0;
                        const unsigned long long x = v[k], y = v[k | d];
                        if ((x > y) == up) { v[k] = y; v[k | d] = x; }
                    }
            }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PT; ++k) list[tid * PT + k] = v[k];
    __syncthreads();
}

// A lane's vectors of a segment dealt out to NW warps: a warp's share is contiguous, and so is a lane's - an odd number, so
// that eight lanes of a 16-byte access touch all 32 banks once.
template <int NW>
__device__ __forceinline__ void lane_vectors(int cnt, int warp, int lane, int* v0, int* v1) {
    const int share = (cnt + NW - 1) / NW, per = ((share + 31) / 32) | 1, end = min(cnt, (warp + 1) * share);
    *v0 = min(end, warp * share + lane * per);
    *v1 = min(end, *v0 + per);
}

// Fast sum of e over vectors [v0, v1).
template <int DT, bool FAR>
__device__ __forceinline__ double lane_exp_sum(const uint4* buf, int v0, int v1, const PartRef& ref) {
    double sum = 0.0;
#pragma unroll 2
    for (int j = v0; j < v1; ++j) {
        float x[Elem<DT>::E];
        Elem<DT>::unpack(buf[j], x);
        ref.template exps<FAR>(x);
        sum += (double)vec_add(x);
    }
    return sum;
}

// A row and its cluster.
template <int DT>
struct Rows {
    using El = Elem<DT>;
    static constexpr int E = El::E;
    const SampleArgs& a;
    cg::cluster_group cl;
    int CL, rank, tid, lane, warp;
    uint32_t phase = 0;
    int parity = 0;       // of the next exchange of parts
    Segment s;
    int v0, v1;           // my vectors

    __device__ __forceinline__ explicit Rows(const SampleArgs& a_) : a(a_), cl(cg::this_cluster()) {
        CL = (int)cl.num_blocks();
        rank = (int)cl.block_rank();
        tid = threadIdx.x;
        lane = tid & 31;
        warp = tid >> 5;
        if (tid == 0) {
            mbar_init(&row_ctrl().full, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        for (int i = tid; i < kRedoRows / 32; i += kThreads) row_ctrl().redo[i] = 0;
        __syncthreads();
        cl.sync();                                     // every CTA runs before its shared memory is written
    }

    __device__ __forceinline__ void start(int64_t t) {
        s = make_segment<DT>(a.logits, a.ldl, t, a.V, rank, a.seg);
        if (tid == 0) start_load<DT>(s, a.V, row_buf(), &row_ctrl().full);
        lane_vectors<W>(s.cnt, warp, lane, &v0, &v1);
    }
    __device__ __forceinline__ void wait() {
        if (!mbar_wait(&row_ctrl().full, phase, kSpinLimit) && lane == 0) pods_raise(a.status, PODS_STATUS_TIMEOUT);
        phase ^= 1u;
        __syncthreads();
    }
    __device__ __forceinline__ void done() {
        fence_async_proxy();                           // the buffer is refilled by bulk copies
        __syncthreads();
    }
    __device__ __forceinline__ int id_of(int j, int e) const { return s.id0 + j * E + e; }
    __device__ __forceinline__ bool is_id(int id) const { return id >= 0 && id < a.V; }

    __device__ __forceinline__ float lane_max() const {
        float m = -INFINITY;
#pragma unroll 4
        for (int j = v0; j < v1; ++j) m = max_nan(m, El::vec_max(row_buf()[j]));
        return m;
    }
    static __device__ __forceinline__ float warp_max(float m) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(PODS_FULL_MASK, m, d));
        return m;
    }

    // e of one logit: fast relative to ref, or fp64 relative to ref's maximum
    template <bool PREC>
    __device__ __forceinline__ double weight(float x, const PartRef& ref, double tau_inv) const {
        return PREC ? exp64(((double)x - (double)ref.m) * tau_inv) : ref.exp1(x);
    }
    static __device__ __forceinline__ bool kept(float x, int id, float thr, int cut) { return x > thr || (x == thr && id <= cut); }

    // sum of e over my vectors, of the kept ids only if FILT
    template <bool PREC, bool FILT>
    __device__ __forceinline__ double lane_sum(const PartRef& ref, double tau_inv, float thr, int cut) const {
        double sum = 0.0;
        if constexpr (PREC) {
#pragma unroll 1
            for (int j = v0; j < v1; ++j) {
                const uint4 q = row_buf()[j];
                if (FILT && El::vec_max(q) < thr) continue;
                float x[E];
                El::unpack(q, x);
#pragma unroll
                for (int h = 0; h < E; h += 4) {
                    double d[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[i] = ((double)x[h + i] - (double)ref.m) * tau_inv;
                    exp64x4(d);
                    if (FILT)
#pragma unroll
                        for (int i = 0; i < 4; ++i) d[i] = kept(x[h + i], id_of(j, h + i), thr, cut) ? d[i] : 0.0;
                    sum += (d[0] + d[1]) + (d[2] + d[3]);
                }
            }
        } else if constexpr (!FILT) {
            sum = ref.far ? lane_exp_sum<DT, true>(row_buf(), v0, v1, ref) : lane_exp_sum<DT, false>(row_buf(), v0, v1, ref);
        } else {
#pragma unroll 1
            for (int j = v0; j < v1; ++j) {
                const uint4 q = row_buf()[j];
                if (El::vec_max(q) < thr) continue;
                float x[E], p[E];
                El::unpack(q, x);
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] = x[e];
                if (ref.far) ref.template exps<true>(p);
                else ref.template exps<false>(p);
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] = kept(x[e], id_of(j, e), thr, cut) ? p[e] : 0.0f;
                sum += (double)vec_add(p);
            }
        }
        return sum;
    }

    // Hands my warp's part to every CTA; returns the cluster's parts.
    __device__ __forceinline__ const Part* publish(const Part& p) {
        Part* const at = row_ctrl().part[parity];
        parity ^= 1;
        if (lane < CL) *cl.map_shared_rank(at + rank * W + warp, lane) = p;
        cl.sync();
        return at;
    }

    // All parts of a row; lane l of every warp holds parts [l n, (l + 1) n).
    static constexpr int N = kMaxCluster * W / 32;
    struct Sums {
        double v[N], mine, incl, total;
    };
    // ONE_REF: the parts are relative to one reference already
    template <bool PREC, bool ONE_REF>
    __device__ __forceinline__ Sums sum_parts(const Part* part, const PartRef& top, double tau_inv) const {
        const int n_parts = CL * W, n = (n_parts + 31) / 32;
        Sums r;
        r.mine = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            r.v[i] = 0.0;
            if (i < n && lane * n + i < n_parts) {
                const Part q = part[lane * n + i];
                if (q.s > 0.0)
                    r.v[i] = ONE_REF ? q.s
                             : q.s * (PREC ? exp64(((double)q.m - (double)top.m) * tau_inv) : PartRef(q.m, top.c).scale_to(top));
            }
            r.mine += r.v[i];
        }
        r.incl = warp_scan(r.mine, lane);
        r.total = __shfl_sync(PODS_FULL_MASK, r.incl, 31);
        return r;
    }
    // The part that holds `target` < total, and the sum ahead of it.
    __device__ __forceinline__ int owner_of(const Sums& r, double target, double* before) const {
        const int n = (CL * W + 31) / 32;
        const uint32_t hit = __ballot_sync(PODS_FULL_MASK, r.incl > target && r.mine > 0.0);
        const int from = hit ? __ffs(hit) - 1 : 0;
        int owner = -1;
        double b = scan_ahead(r.incl, lane), at = b;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (r.v[i] > 0.0 && (owner < 0 || !(b > target))) {    // the first that passes the target, else the last
                owner = lane * n + i;
                at = b;
                b += r.v[i];
            }
        *before = __shfl_sync(PODS_FULL_MASK, at, from);
        return __shfl_sync(PODS_FULL_MASK, owner, from);
    }
    // Within my warp's part, whose lane sums are `sum` and their scan `incl`: the first id whose running sum exceeds `goal`
    // (relative to ref).  One lane returns true, with the element, the sum ahead of it and its own e.
    template <bool PREC, bool FILT>
    __device__ __forceinline__ bool search(double goal, double sum, double incl, const PartRef& ref, double tau_inv, float thr, int cut,
                                           int* element, double* lo, double* ev) const {
        uint32_t hit = __ballot_sync(PODS_FULL_MASK, incl > goal && sum > 0.0);
        const uint32_t any = __ballot_sync(PODS_FULL_MASK, sum > 0.0);
        if (any == 0) return false;
        const int from = hit ? __ffs(hit) - 1 : 31 - __clz(any);
        const double ahead = __shfl_sync(PODS_FULL_MASK, scan_ahead(incl, lane), from);
        // the elements of that lane's vectors, k a lane
        const int e0 = __shfl_sync(PODS_FULL_MASK, v0, from) * E, e1 = __shfl_sync(PODS_FULL_MASK, v1, from) * E;
        const int k = (e1 - e0 + 31) / 32;
        const int k0 = min(e1, e0 + lane * k), k1 = min(e1, k0 + k);
        const typename El::raw* el = reinterpret_cast<const typename El::raw*>(row_buf());
        auto at = [&](int i) {
            const float x = El::to_float(el[i]);
            return !FILT || kept(x, s.id0 + i, thr, cut) ? weight<PREC>(x, ref, tau_inv) : 0.0;
        };
        double own = 0.0;
        for (int i = k0; i < k1; ++i) own += at(i);
        const double eincl = warp_scan(own, lane), eahead = scan_ahead(eincl, lane);
        hit = __ballot_sync(PODS_FULL_MASK, ahead + eincl > goal && own > 0.0);
        const uint32_t some = __ballot_sync(PODS_FULL_MASK, own > 0.0);
        if (some == 0) return false;
        if (lane != (hit ? __ffs(hit) - 1 : 31 - __clz(some))) return false;
        double run = ahead + eahead;
        for (int i = k0; i < k1; ++i) {
            const double w = at(i);
            if (!(w > 0.0)) continue;
            *element = i;
            *lo = run;
            *ev = w;
            run += w;
            if (run > goal) break;
        }
        return true;
    }
    // An edge of the running sum nearer than the margin is decided in fp64 (the row's start is no edge where u is no smaller
    // than the fast sums see).
    __device__ __forceinline__ bool certain(double u, double target, double lo, double ev, double total, const PartRef& top, double tau_inv) const {
        const double margin = draw_margin(u, total, deep_error(a.V, total, top.c, tau_inv, top.near_far()));
        return draw_is_sure(u, target, lo, lo + ev, margin);
    }

    // A value that at least ceil(want / CL) logits of the segment reach, so the least one of the cluster is reached by `want`
    // logits of the row: that many lanes' maxima reach it.  The first warp finds it among the lanes' maxima by bisection, on
    // the upper half of the keys (a slightly lower value is as good); the other warps get +inf and go on.
    __device__ __forceinline__ float reach(float lane_m, int want) const {
        constexpr int M = kThreads / 32;
        const int r = (want + CL - 1) / CL;
        row_ctrl().top[tid] = order32(lane_m) >> 16;
        __syncthreads();
        if (warp != 0) return INFINITY;
        if (r > kThreads) return -INFINITY;
        uint32_t key[M];
#pragma unroll
        for (int k = 0; k < M; ++k) key[k] = row_ctrl().top[lane + 32 * k];
        uint32_t lo = key[0], hi = key[0];
#pragma unroll
        for (int k = 1; k < M; ++k) {
            lo = min(lo, key[k]);
            hi = max(hi, key[k]);
        }
        lo = __reduce_min_sync(PODS_FULL_MASK, lo);    // reached by all lanes, so by r
        hi = __reduce_max_sync(PODS_FULL_MASK, hi) + 1;
#pragma unroll 1
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            int n = 0;
#pragma unroll
            for (int k = 0; k < M; ++k) n += (int)(key[k] >= mid);
            if ((int)__reduce_add_sync(PODS_FULL_MASK, (unsigned)n) >= r) lo = mid; else hi = mid;
        }
        const float v = unorder32(lo << 16);
        return v >= -3.4028235e38f ? v : -INFINITY;    // below the finite numbers: every id
    }
    __device__ __forceinline__ float row_max(const Part* part) const {
        float z = -INFINITY;
        for (int i = lane; i < CL * W; i += 32) z = max_nan(z, part[i].m);
        return warp_max(z) + 0.0f;
    }
    __device__ __forceinline__ float limit(const Part* part) const {
        float l = INFINITY;
        for (int i = lane; i < CL; i += 32) l = fminf(l, part[i * W].lim);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) l = fminf(l, __shfl_xor_sync(PODS_FULL_MASK, l, d));
        return l;
    }
};

// What is found by lists, counts and sums over the cluster.  Every method is called by the whole cluster.
template <int DT>
struct Finder {
    using El = Elem<DT>;
    static constexpr int E = El::E;
    Rows<DT>& w;
    int parity = 0;

    __device__ __forceinline__ explicit Finder(Rows<DT>& w_) : w(w_) {}
    __device__ __forceinline__ FilterCtrl& ctrl() const { return filter_ctrl(w.a); }
    // the CTA's own list [own_cap]; all CTAs' lists [CL list_cap]; the sampler's ordered list or its histogram
    __device__ __forceinline__ unsigned long long* own() const {
        return reinterpret_cast<unsigned long long*>(smem_ + kRowCtrlBytes + w.a.seg * 16 + kFilterCtrlBytes);
    }
    __device__ __forceinline__ unsigned long long* all() const { return own() + w.a.own_cap; }
    __device__ __forceinline__ unsigned long long* list() const { return all() + w.CL * w.a.list_cap; }
    __device__ __forceinline__ uint32_t* hist() const { return reinterpret_cast<uint32_t*>(list()); }

    // Hands `mine` to every CTA of the cluster; returns the CL words.
    __device__ const Xch* exchange(const Xch& mine) {
        Xch* const slot = ctrl().x[parity];
        parity ^= 1;
        if (w.tid < w.CL) *w.cl.map_shared_rank(slot + w.rank, w.tid) = mine;
        w.cl.sync();
        return slot;
    }

    // ids with value > thr and == thr
    __device__ void row_count(float thr, long long* above, long long* equal) {
        int n = 0, m = 0;
        for (int j = w.v0; j < w.v1; ++j) {
            const uint4 q = row_buf()[j];
            if (El::vec_max(q) < thr) continue;
            float x[E];
            El::unpack(q, x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool ok = w.is_id(w.id_of(j, e));
                n += (ok && x[e] > thr) ? 1 : 0;
                m += (ok && x[e] == thr) ? 1 : 0;
            }
        }
        Xch mine = {};
        mine.n = block_reduce<W>(n, ctrl().ipart, Plus());
        mine.i = block_reduce<W>(m, ctrl().ipart, Plus());
        const Xch* x = exchange(mine);
        *above = *equal = 0;
        for (int q = 0; q < w.CL; ++q) { *above += x[q].n; *equal += x[q].i; }
    }

    // id of the nth (from 0) id, ascending, whose value is thr
    __device__ int nth_equal(float thr, long long nth) {
        int m = 0;
        for (int j = w.v0; j < w.v1; ++j) {
            float x[E];
            El::unpack(row_buf()[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) m += (x[e] == thr && w.is_id(w.id_of(j, e))) ? 1 : 0;
        }
        const int incl = warp_scan(m, w.lane);
        __syncthreads();
        if (w.lane == 31) ctrl().ipart[w.warp] = incl;
        if (w.tid == 0) ctrl().found = -1;
        __syncthreads();
        Xch mine = {};
        int before = incl - m;
        for (int q = 0; q < W; ++q) {
            mine.n += ctrl().ipart[q];
            if (q < w.warp) before += ctrl().ipart[q];
        }
        const Xch* x = exchange(mine);
        long long at = before;
        for (int q = 0; q < w.rank; ++q) at += x[q].n;
        if (nth >= at && nth < at + m) {
            const typename El::raw* el = reinterpret_cast<const typename El::raw*>(row_buf());
            for (int i = w.v0 * E; i < w.v1 * E; ++i)
                if (El::to_float(el[i]) == thr && w.is_id(w.s.id0 + i)) {
                    if (at == nth) ctrl().found = w.s.id0 + i;
                    ++at;
                }
        }
        __syncthreads();
        Xch out = {};
        out.i = ctrl().found;
        x = exchange(out);
        int id = -1;
        for (int q = 0; q < w.CL; ++q) id = max(id, x[q].i);
        return id;
    }

    // Threshold of the first `count` ids of the order: value and highest id kept among the ids equal to it.
    __device__ void count_threshold(long long count, float zmax, float* thr, int* cut) {
        uint32_t lo = El::to_key(-INFINITY), hi = El::to_key(zmax) + 1;        // ids >= lo: all; >= hi: none
        long long above, equal;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            row_count(El::from_key(mid), &above, &equal);
            if (above + equal >= count) lo = mid; else hi = mid;
        }
        *thr = El::from_key(lo);
        row_count(*thr, &above, &equal);
        const long long need = count - above;
        *cut = need >= equal ? kNoCut : nth_equal(*thr, need - 1);
    }

    // sum of e over the kept ids, relative to top's maximum, in fp64
    __device__ double kept_sum(float thr, int cut, const PartRef& top, double tau_inv) {
        double sum = w.template lane_sum<true, true>(top, tau_inv, thr, cut);
        Xch mine = {};
        mine.a = block_reduce<W>(sum, ctrl().dpart, Plus());
        const Xch* x = exchange(mine);
        double total = 0.0;
        for (int q = 0; q < w.CL; ++q) total += x[q].a;
        return total;
    }

    // Shrinks (thr, cut) to the smallest prefix of the kept ids whose sum of e reaches `mass`, by bisection.
    __device__ void mass_threshold(double mass, const PartRef& top, double tau_inv, float* thr, int* cut) {
        uint32_t lo = El::to_key(*thr), hi = El::to_key(top.m) + 1;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (kept_sum(El::from_key(mid), kNoCut, top, tau_inv) >= mass) lo = mid; else hi = mid;
        }
        const float v = El::from_key(lo);
        long long above, equal;
        row_count(v, &above, &equal);
        // everything above v: v itself with no id of its own
        const double more = mass - kept_sum(v, -1, top, tau_inv);
        const double ev = exp64(((double)v - (double)top.m) * tau_inv);
        double need = ev > 0.0 ? ceil(more / ev) : (double)equal;
        if (need < 1.0) need = 1.0;
        if (v > *thr) {
            *thr = v;
            *cut = need >= (double)equal ? kNoCut : nth_equal(v, (long long)need - 1);
        } else if (need < (double)equal) {
            const int id = nth_equal(v, (long long)need - 1);
            *cut = min(*cut, id);
        }
    }

    // Lists hold (order32(value) << 32) | ~id: larger first is the row's order, and no two entries are equal.
    __device__ __forceinline__ void list_add(float x, int id) {
        const int at = atomicAdd(&ctrl().n_list, 1);
        if (at < w.a.own_cap) own()[at] = ((unsigned long long)order32(x) << 32) | (uint32_t)~id;
    }
    // Lists those elements of vector j whose bit is set: as many steps as the warp's busiest lane has, not one an element.
    __device__ __forceinline__ void list_hits(int j, uint32_t hits) {
        const typename El::raw* const el = reinterpret_cast<const typename El::raw*>(row_buf());
        while (hits) {
            const int e = __ffs(hits) - 1;
            hits &= hits - 1;
            if (w.is_id(w.id_of(j, e))) list_add(El::to_float(el[j * E + e]), w.id_of(j, e));
        }
    }
    // Hands my list to every CTA, with `mine`; returns the CL words and the lists' length together.  Each list has a room of
    // list_cap; -1 if one is longer.  PACKED: the lengths are exchanged first and the lists laid end to end, for lists that are
    // known to fit together but may all come from one CTA.
    template <bool PACKED>
    __device__ const Xch* share_list(Xch mine, int* total) {
        __syncthreads();
        mine.n = ctrl().n_list;
        int at = w.rank * w.a.list_cap;
        if (PACKED) {
            const Xch* x = exchange(mine);
            at = 0;
            for (int q = 0; q < w.rank; ++q) at += x[q].n;
        }
        const int n = min(mine.n, PACKED ? w.a.own_cap : w.a.list_cap);
        for (int q = w.warp; q < w.CL; q += W) {
            unsigned long long* const peer = w.cl.map_shared_rank(all() + at, q);
            for (int k = w.lane; k < n; k += 32)
                if (PODS_INDEX_OK(at + k, w.CL * w.a.list_cap, w.a.status)) peer[k] = own()[k];
        }
        const Xch* x = exchange(mine);
        int sum = 0;
        bool fits = true;
        for (int q = 0; q < w.CL; ++q) {
            if (w.tid == 0) {
                ctrl().start[q] = PACKED ? sum : q * w.a.list_cap;
                ctrl().count[q] = x[q].n;
            }
            sum += x[q].n;
            fits = fits && (PACKED || x[q].n <= w.a.list_cap);
        }
        __syncthreads();
        *total = fits ? sum : -1;
        return x;
    }
    __device__ __forceinline__ void add_kept(float thr, int cut) {
        __syncthreads();
        if (w.tid == 0) ctrl().n_list = 0;
        __syncthreads();
        for (int j = w.v0; j < w.v1; ++j) {
            const uint4 q = row_buf()[j];
            if (El::vec_max(q) < thr) continue;
            float x[E];
            El::unpack(q, x);
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) hits |= w.kept(x[e], w.id_of(j, e), thr, cut) ? 1u << e : 0u;
            list_hits(j, hits);
        }
    }
    // Lists the kept ids of the row; returns how many, -1 if they do not fit.
    template <bool PACKED>
    __device__ __forceinline__ int list_kept(float thr, int cut) {
        add_kept(thr, cut);
        const Xch none = {};
        int total;
        share_list<PACKED>(none, &total);
        return total;
    }
    // The same for the sampler, with the sum of e over all lists, relative to top's maximum.
    __device__ __forceinline__ int list_kept_mass(float thr, const PartRef& top, double tau_inv, double* mass) {
        add_kept(thr, kNoCut);
        __syncthreads();
        Xch mine = {};
        for (int i = w.tid; i < min(ctrl().n_list, w.a.own_cap); i += kThreads)
            mine.a += exp64(((double)unorder32((uint32_t)(own()[i] >> 32)) - (double)top.m) * tau_inv);
        mine.a = block_reduce<W>(mine.a, ctrl().dpart, Plus());
        int total;
        const Xch* x = share_list<false>(mine, &total);
        *mass = 0.0;
        for (int q = 0; q < w.CL; ++q) *mass += x[q].a;
        return total;
    }
    // Calls put(rank, key) for the entries of CTAs [q0, q1), the rank being the number of entries of all lists ahead of it: the
    // whole CTA.  Few entries are looked at by P neighbouring lanes each, many by a thread R at a time.
    template <int R, typename Put>
    __device__ __forceinline__ void rank_entries(int q0, int i0, int n, int P, Put put) const {
        const int sub = w.tid & (P - 1);
        unsigned long long key[R];
        bool live[R];
        int r[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            int i = i0 + w.tid / P + k * kThreads, q = q0;
            live[k] = i < n;
            if (live[k])
                while (i >= ctrl().count[q]) i -= ctrl().count[q++];
            key[k] = live[k] ? all()[ctrl().start[q] + i] : ~0ull;
            r[k] = 0;
        }
        for (int q = 0; q < w.CL; ++q) {
            const unsigned long long* const at = all() + ctrl().start[q];
            const int m = ctrl().count[q];
#pragma unroll 4
            for (int j = sub; j < m; j += P) {
                const unsigned long long o = at[j];
#pragma unroll
                for (int k = 0; k < R; ++k) r[k] += o > key[k] ? 1 : 0;
            }
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            for (int d = 1; d < P; d <<= 1) r[k] += __shfl_xor_sync(PODS_FULL_MASK, r[k], d);
            if (live[k] && sub == 0) put(r[k], key[k]);
        }
    }
    template <typename Put>
    __device__ __forceinline__ void rank_lists(int q0, int q1, Put put) const {
        int n = 0;
        for (int q = q0; q < q1; ++q) n += ctrl().count[q];
        if (n <= kThreads) {
            int P = 1;
            while (P < 32 && n * P * 2 <= kThreads) P *= 2;
            rank_entries<1>(q0, 0, n, P, put);
        } else {
            for (int i0 = 0; i0 < n; i0 += 4 * kThreads) rank_entries<4>(q0, i0, n, 1, put);
        }
    }
    // The sampler: all lists in the row's order in the first CTA's `list`, every CTA placing its own entries; n <= kSampleList.
    __device__ __forceinline__ void order_lists() {
        unsigned long long* const first = w.cl.map_shared_rank(list(), 0);
        rank_lists(w.rank, w.rank + 1, [&](int r, unsigned long long key) {
            if (PODS_INDEX_OK(r, kSampleList, w.a.status)) first[r] = key;
        });
        w.cl.sync();
    }

    // Shrinks (thr, cut) to the smallest prefix of the kept ids whose sum of e reaches top_p of theirs, where the border is
    // found in one bracket of the mass histogram; S: their sum, by fast exponentials or (exact_S) in fp64.  false: the bracket
    // does not fit the lists.
    // lane_above: see bracket_sum; negative where there is none.
    __device__ bool nucleus_threshold(float top_p, double S, bool exact_S, const PartRef& top, double tau_inv, float* thr, int* cut, double* lane_above) {
        // logits below this have less than 1 - top_p of the mass together, so the border lies above
        const double deep = log(fmax((1.0 - (double)top_p) * S, 1e-30) / (double)w.a.V) - 1e-3;
        const float low = fmaxf(*thr, __double2float_rd((double)top.m + deep / tau_inv));
        const float range = top.m - low;
        const float scale = (float)kBins / range;      // stretches a unit of logit
        if (!(range > 0.0f) || !(scale < INFINITY)) return false;
        const float h2 = (float)(1.4426950408889634 * tau_inv * (double)range / kBins);     // exponent of two a stretch, < 0.05
        const bool all_ids = *thr == -INFINITY;        // no top_k in force
        for (int i = w.tid; i < kBins; i += kThreads) hist()[i] = 0;
        __syncthreads();
        // mass in units of 2^-12 of the weight at the stretch's upper end: at most 2^19 ids make 2^31; each is off by 1.3e-4
        for (int j = w.v0; j < w.v1; ++j) {
            const uint4 q = row_buf()[j];
            if (El::vec_max(q) < low) continue;
            float x[E];
            uint32_t b[E], mass[E];
            El::unpack(q, x);
            // the eight chains overlap, and rounding by a large addend keeps them off the pipe that converts and exponentiates:
            // 2^-y for y <= 0.05 by its quadratic (the next term is 7e-6)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float pos = (top.m - fmaxf(x[e], low)) * scale;
                const float t = (pos - 0.5f) + 12582912.0f, y = (pos - (t - 12582912.0f)) * (h2 * 0.6931472f);     // 1.5 * 2^23
                b[e] = min((uint32_t)kBins - 1u, __float_as_uint(t) & 0x3fffffu);
                mass[e] = __float_as_uint(fmaf(fmaf(y, 2048.0f, -4096.0f), y, 4096.0f + 8388608.0f)) & 0x7fffffu;
            }
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] >= low && (all_ids || w.kept(x[e], w.id_of(j, e), *thr, *cut))) atomicAdd(&hist()[b[e]], mass[e]);
        }
        w.cl.sync();
        constexpr int PB = kBins / kThreads;
        uint32_t n[PB] = {};
        for (int q = 0; q < w.CL; ++q) {
            const uint32_t* const peer = w.cl.map_shared_rank(hist() + w.tid * PB, q);
#pragma unroll
            for (int k = 0; k < PB; k += 4) {
                const uint4 h = *reinterpret_cast<const uint4*>(peer + k);
                n[k] += h.x;
                n[k + 1] += h.y;
                n[k + 2] += h.z;
                n[k + 3] += h.w;
            }
        }
        static_assert(PB % 4 == 0, "16 bytes a read");
        static_assert(kBins * 4 <= kSampleList * 8, "the histogram lies where the list does");
        double run[PB], sum = 0.0;
#pragma unroll
        for (int k = 0; k < PB; ++k) {
            sum += (double)n[k] * (1.0 / 4096.0) * (double)ex2_approx(-(float)(w.tid * PB + k) * h2);
            run[k] = sum;
        }
        double all;
        const double base = block_scan_ahead(sum, ctrl().dpart, &all);
        const double goal = (double)top_p * S, tol = 2e-4 * S;     // 1.3e-4 of rounding, the quadratic, the fast sum S
        int below = 0, first = kBins - 1;
#pragma unroll
        for (int k = 0; k < PB; ++k) {
            if (base + run[k] <= goal - tol) ++below;              // a prefix of the stretches
            if (base + run[k] >= goal + tol) first = min(first, w.tid * PB + k);
        }
        const int b1 = block_reduce<W>(below, ctrl().ipart, Plus()), b2 = block_reduce<W>(first, ctrl().ipart, Min());

        // the sums above the bracket, and the bracket's ids listed; fast first, then, where the border is too close to call, in fp64
        *lane_above = 0.0;
        // its ends in logits, a hundredth of a stretch further out than the stretches, whose own ends are rounded
        const float x_hi = top.m - ((float)b1 - 0.01f) / scale, x_lo = fmaxf(low, top.m - ((float)b2 + 1.01f) / scale);
        int answer = bracket<false>(top_p, S, exact_S, x_hi, x_lo, b1 == 0, top, tau_inv, thr, cut, lane_above);
        if (answer == 2) {
            *lane_above = -1.0;
            answer = bracket<true>(top_p, S, exact_S, x_hi, x_lo, b1 == 0, top, tau_inv, thr, cut, lane_above);
        }
        return answer == 1;
    }

    // One sweep for nucleus_threshold.  1: (thr, cut) is the border; 2: too close to call; 0: the bracket misses it or does not
    // fit the lists.  The fast sweep leaves the lane's sum above the bracket (relative to top) in lane_above.
    template <bool PREC>
    __device__ __forceinline__ int bracket(float top_p, double S, bool exact_S, float x_hi, float x_lo, bool from_top, const PartRef& top,
                                           double tau_inv, float* thr, int* cut, double* lane_above) {
        __syncthreads();
        if (w.tid == 0) ctrl().n_list = 0;
        __syncthreads();
        double above = 0.0, total = 0.0;
        const bool all_ids = *thr == -INFINITY;
        if (from_top) x_hi = INFINITY;                 // the bracket begins with the largest logit
#pragma unroll 1
        for (int j = w.v0; j < w.v1; ++j) {
            const uint4 q = row_buf()[j];
            const float vmax = El::vec_max(q);
            if (vmax < (PREC ? *thr : x_lo)) continue;
            float x[E];
            El::unpack(q, x);
            if (!all_ids)                              // ids that top_k left out weigh nothing
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = w.kept(x[e], w.id_of(j, e), *thr, *cut) ? x[e] : -INFINITY;
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) hits |= x[e] >= x_lo && x[e] <= x_hi ? 1u << e : 0u;
            if (PREC) {
#pragma unroll
                for (int h = 0; h < E; h += 4) {
                    double d[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[i] = ((double)x[h + i] - (double)top.m) * tau_inv;
                    exp64x4(d);
                    double a[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        a[i] = x[h + i] > x_hi ? d[i] : 0.0;
                    }
                    total += (d[0] + d[1]) + (d[2] + d[3]);
                    above += (a[0] + a[1]) + (a[2] + a[3]);
                }
            } else {
                float p[E];
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] = x[e];
                if (top.far) top.template exps<true>(p);
                else top.template exps<false>(p);
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] = x[e] > x_hi ? p[e] : 0.0f;
                above += (double)vec_add(p);
            }
            list_hits(j, hits);
        }
        if (!PREC) *lane_above = above;
        // relative to e^zmax
        const double unit = PREC || top.far ? 1.0 : exp2((double)top.R - (double)top.m * (double)top.c);
        Xch mine = {};
        mine.a = block_reduce<W>(above, ctrl().dpart, Plus()) * unit;
        if (PREC) mine.b = block_reduce<W>(total, ctrl().dpart, Plus());
        int len;
        const Xch* x = share_list<false>(mine, &len);  // past its barrier the histogram is read: its room is the list's again
        double A = 0.0, Z = 0.0;
        for (int q = 0; q < w.CL; ++q) { A += x[q].a; Z += x[q].b; }
        if (!PREC) Z = S;
        const double goal = (double)top_p * Z;
        const double deep = deep_error(w.a.V, Z, top.c, tau_inv, top.near_far());
        const double margin = PREC ? 0.0 : exact_S ? (deep + kFlat) * goal + 1e-12 * Z : draw_margin((double)top_p, Z, deep);
        Xch out = {};
        const bool fits = len > 0 && len <= kSampleList;
        if (fits) order_lists();
        if (w.rank == 0 && fits) {
            const int per = (len + kThreads - 1) / kThreads;
            double own = 0.0;
            for (int k = 0; k < per; ++k) {
                const int i = w.tid * per + k;
                if (i < len) own += exp64(((double)unorder32((uint32_t)(list()[i] >> 32)) - (double)top.m) * tau_inv);
            }
            double sum_all;
            double at = A + block_scan_ahead(own, ctrl().dpart, &sum_all);
            int pick = kNoCut, unsure = w.tid == 0 && !from_top && fabs(A - goal) <= margin;
            for (int k = 0; k < per; ++k) {
                const int i = w.tid * per + k;
                if (i < len) {
                    at += exp64(((double)unorder32((uint32_t)(list()[i] >> 32)) - (double)top.m) * tau_inv);
                    if (at >= goal && pick == kNoCut) pick = i;
                    if (fabs(at - goal) <= margin) unsure = 1;
                }
            }
            pick = block_reduce<W>(pick, ctrl().ipart, Min());
            unsure = block_reduce<W>(unsure, ctrl().ipart, Plus());
            if (!PREC && unsure) {
                out.n = 2;
            } else if (pick < len && (A < goal || from_top)) {
                out.n = 1;
                out.m = unorder32((uint32_t)(list()[pick] >> 32));
                out.i = (int)~(uint32_t)list()[pick];
            }
        }
        x = exchange(out);
        if (x[0].n == 1) {
            *thr = x[0].m;
            *cut = x[0].i;
        }
        return x[0].n;
    }
    // The lane's fast sum over the kept ids, from its sum above the bracket and the bracket's entries: a thread an entry, added
    // to the lane that holds it in units of 2^-53, so that their order does not matter (each lane walking all entries took 5000
    // cycles of a row's 80000).  e is at most 1 and the entries of the cluster at most 1024: no overflow, and 1.2e-13 of rounding.
    __device__ __forceinline__ double bracket_sum(double lane_above, float thr, int cut, const PartRef& top) {
        unsigned long long* const extra = reinterpret_cast<unsigned long long*>(hist());
        extra[w.tid] = 0ull;
        __syncthreads();
        const int n = min(ctrl().n_list, w.a.own_cap), share = (w.s.cnt + W - 1) / W, per = ((share + 31) / 32) | 1;
        for (int k = w.tid; k < n; k += kThreads) {
            const unsigned long long key = own()[k];
            const float x = unorder32((uint32_t)(key >> 32));
            const int id = (int)~(uint32_t)key, j = (id - w.s.id0) / E;
            if (w.kept(x, id, thr, cut)) atomicAdd(&extra[j / share * 32 + j % share / per], (unsigned long long)(top.exp1(x) * 0x1p53));
        }
        __syncthreads();
        return lane_above + (double)extra[w.tid] * 0x1p-53;
    }

    // Draws over the kept ids; the whole cluster gets the token, its logit and the kept sum relative to top's maximum.
    template <bool PREC>
    __device__ bool draw(double u, float thr, int cut, const PartRef& top, double tau_inv, double lane_above, int* token, float* logit, double* total) {
        const double sum = !PREC && lane_above >= 0.0 ? bracket_sum(lane_above, thr, cut, top)
                                                      : w.template lane_sum<PREC, true>(top, tau_inv, thr, cut);
        const double incl = warp_scan(sum, w.lane);
        Part p = {};
        p.s = __shfl_sync(PODS_FULL_MASK, incl, 31);
        if (w.tid == 0) ctrl().found = -1;
        const Part* part = w.publish(p);
        const typename Rows<DT>::Sums r = w.template sum_parts<PREC, true>(part, top, tau_inv);
        const double target = u * r.total;
        double before;
        const int owner = w.owner_of(r, target, &before);
        if (u == 0.0) {                                // the lowest kept id, however little its weight
            const typename El::raw* el = reinterpret_cast<const typename El::raw*>(row_buf());
            int id = kNoCut;
            for (int i = w.v0 * E; i < w.v1 * E && id == kNoCut; ++i) {
                const float x = El::to_float(el[i]);
                if (x > -INFINITY && w.kept(x, w.s.id0 + i, thr, cut)) id = w.s.id0 + i;
            }
            id = block_reduce<W>(id, ctrl().ipart, Min());
            if (w.tid == 0 && id != kNoCut) {
                ctrl().found = id;
                ctrl().sure = 1;
                ctrl().weight = (double)El::to_float(el[id - w.s.id0]);
            }
        } else if (owner == w.rank * W + w.warp) {
            int at = 0;
            double lo = 0.0, ev = 0.0;
            if (w.template search<PREC, true>(target - before, sum, incl, top, tau_inv, thr, cut, &at, &lo, &ev)) {
                ctrl().found = w.s.id0 + at;
                ctrl().sure = PREC || w.certain(u, target, before + lo, ev, r.total, top, tau_inv);
                ctrl().weight = (double)El::to_float(reinterpret_cast<const typename El::raw*>(row_buf())[at]);
            }
        }
        __syncthreads();
        Xch out = {};
        out.i = ctrl().found;
        out.n = ctrl().found >= 0 ? ctrl().sure : 0;
        out.m = ctrl().found >= 0 ? (float)ctrl().weight : 0.0f;
        const Xch* x = exchange(out);
        bool sure = false;
        *token = -1;
        for (int q = w.CL - 1; q >= 0; --q)
            if (x[q].i >= 0) { *token = x[q].i; *logit = x[q].m; sure = x[q].n != 0; }
        *total = PREC ? r.total : r.total * exp2(top.far ? 0.0 : (double)top.R - (double)top.m * (double)top.c);
        return sure;
    }
};

// A row's settings, checked.
struct Settings {
    float tau, u, top_p, min_p;
    long long top_k;
    bool greedy, nucleus, floor, filtered, odd;
    __device__ __forceinline__ Settings(const SampleArgs& a, int64_t t, bool filters) {
        tau = a.temperature_row ? a.temperature_row[t] : a.temperature;
        u = a.u[t];
        odd = false;
        if (!(tau >= 0.0f) || tau == INFINITY) { tau = 1.0f; odd = true; }
        if (!(u >= 0.0f)) { u = 0.0f; odd = true; }
        if (!(u < 1.0f)) { u = 0x1.fffffep-1f; odd = true; }
        greedy = tau < kGreedyBelow;
        if (greedy) tau = 1.0f;
        top_k = 0;
        nucleus = floor = filtered = false;
        if (filters) {
            top_p = a.top_p_row ? a.top_p_row[t] : a.top_p;
            min_p = a.min_p_row ? a.min_p_row[t] : a.min_p;
            const int k = a.top_k_row ? a.top_k_row[t] : a.top_k;
            if (top_p != top_p) { top_p = 1.0f; odd = true; }
            if (min_p != min_p) { min_p = 0.0f; odd = true; }
            top_k = (k <= 0 || k >= a.V) ? 0 : k;
            min_p = fminf(min_p, 1.0f);
            nucleus = top_p < 1.0f;
            floor = min_p > 0.0f;
            filtered = !greedy && (top_k > 0 || nucleus || floor);
        }
    }
};

// One row.  PREC: the second time, in fp64, for rows without filters.  `mark`: the row's bit among the marked ones.
template <int DT, bool PREC, bool FILTERS>
__device__ __forceinline__ void sample_row(Rows<DT>& w, Finder<DT>* f, int64_t t, int mark) {
    using El = Elem<DT>;
    const SampleArgs& a = w.a;
    const int tid = w.tid, lane = w.lane, CL = w.CL;
    w.start(t);
    const Settings g(a, t, FILTERS);
    if (g.odd && w.rank == 0 && tid == 0) pods_raise(a.status, PODS_STATUS_PARAM_RANGE);
    const double tau_inv = 1.0 / (double)g.tau;
    const float c = (float)(1.4426950408889634 * tau_inv);
    w.wait();

    const float lm = w.lane_max();
    Part p;
    p.m = w.warp_max(lm);
    const PartRef ref(p.m, c);
    const double sum = w.template lane_sum<PREC, false>(ref, tau_inv, 0.0f, 0);
    const double incl = warp_scan(sum, lane);
    p.s = __shfl_sync(PODS_FULL_MASK, incl, 31);
    const int want = (int)(g.top_k > 0 ? (g.top_k < 512 ? g.top_k : 512) : 256);
    p.lim = FILTERS && g.filtered ? w.reach(lm, want) : 0.0f;
    p.near = 0.0f;
    p.pad = 0;
    if (FILTERS && g.nucleus) {
        p.near = lm > -INFINITY ? (float)ref.exp1(lm) : 0.0f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) p.near += __shfl_xor_sync(PODS_FULL_MASK, p.near, d);
    }
    const Part* const part = w.publish(p);
    const float zmax = w.row_max(part);
    if (!(fabsf(zmax) < INFINITY)) {
        if (w.rank == 0 && tid == 0) {
            const bool empty = zmax == -INFINITY;
            a.tokens[t] = -1;
            const float v = empty ? -INFINITY : NAN;
            if (a.logp) a.logp[t] = v;
            if (a.logq) a.logq[t] = v;
            pods_raise(a.status, empty ? PODS_STATUS_EMPTY_ROW : PODS_STATUS_NONFINITE_LOGIT);
        }
        return;
    }
    const PartRef top(zmax, c);
    const typename Rows<DT>::Sums r = w.template sum_parts<PREC, false>(part, top, tau_inv);
    const double Z = r.total;                          // relative to 2^R of top (to e^zmax in fp64 rows)

    if (!FILTERS || !g.filtered) {
        const int mine = w.rank * W + w.warp;
        if (g.greedy || g.u == 0.0f) {
            // the lowest id of the maximum; u = 0: the lowest id of all that can be drawn, however little its weight
            int from = kNoCut, id = kNoCut;
            for (int i = lane; i < CL * W; i += 32)
                if (g.greedy ? part[i].m == zmax : part[i].m > -INFINITY) from = min(from, i);
            if ((int)__reduce_min_sync(PODS_FULL_MASK, from) != mine) return;
            const float least = g.greedy ? zmax : -FLT_MAX;
            for (int j = w.v0; j < w.v1; ++j) {
                float x[El::E];
                El::unpack(row_buf()[j], x);
#pragma unroll
                for (int e = El::E - 1; e >= 0; --e)
                    if (x[e] >= least) id = min(id, w.id_of(j, e));
            }
            id = __reduce_min_sync(PODS_FULL_MASK, id);
            if (lane == 0) {
                const float x = El::to_float(reinterpret_cast<const typename El::raw*>(row_buf())[id - w.s.id0]);
                const float d = (float)(((double)x - (double)zmax) * tau_inv - (log(Z) + (PREC ? 0.0 : top.log_offset())));
                a.tokens[t] = id;
                if (a.logp) a.logp[t] = d;
                if (a.logq) a.logq[t] = g.greedy ? 0.0f : d;
            }
            return;
        }
        const double target = (double)g.u * Z;
        double before;
        if (w.owner_of(r, target, &before) != mine) return;
        const double scale = PREC ? exp64(((double)p.m - (double)zmax) * tau_inv) : ref.scale_to(top);
        int at = 0;
        double lo = 0.0, ev = 0.0;
        if (w.template search<PREC, false>((target - before) / scale, sum, incl, ref, tau_inv, 0.0f, 0, &at, &lo, &ev)) {
            if (PREC || w.certain((double)g.u, target, before + lo * scale, ev * scale, Z, top, tau_inv)) {
                const float x = El::to_float(reinterpret_cast<const typename El::raw*>(row_buf())[at]);
                const float d = (float)(((double)x - (double)zmax) * tau_inv - (log(Z) + (PREC ? 0.0 : top.log_offset())));
                a.tokens[t] = w.s.id0 + at;
                if (a.logp) a.logp[t] = d;
                if (a.logq) a.logq[t] = d;
            } else {
                for (int q = 0; q < CL; ++q) atomicOr(w.cl.map_shared_rank(&row_ctrl().redo[mark >> 5], q), 1u << (mark & 31));
            }
        }
        return;
    }

    if constexpr (FILTERS) {
        unsigned long long* const list = f->list();
        FilterCtrl& ctl = f->ctrl();
        // relative to e^zmax, as everything below is
        const double lz = log(Z) + top.log_offset(), Zm = Z * exp2(top.far ? 0.0 : (double)top.R - (double)top.m * (double)top.c);
        // the lowest value that min_p admits
        const float zfloor = g.floor ? __double2float_ru((double)zmax + (double)g.tau * log((double)g.min_p)) : -INFINITY;
        float lim = w.limit(part);
        // top_p is a share of the whole top-k sum, so min_p may not shorten the list where both are set
        if (g.floor && !(g.top_k > 0 && g.nucleus)) lim = (g.top_k > 0 || g.nucleus) ? fmaxf(lim, zfloor) : zfloor;
        // a nucleus of thousands shows in the maxima of the lanes: where they hold much less than top_p of the row, the list,
        // which holds hardly more than they do, cannot reach the border
        bool wide = false;
        if (g.nucleus && g.top_k == 0) {
            double near = 0.0;
            for (int i = lane; i < CL * W; i += 32)
                if (part[i].s > 0.0) near += (double)part[i].near * PartRef(part[i].m, c).scale_to(top);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) near += __shfl_xor_sync(PODS_FULL_MASK, near, d);
            wide = near < 0.7 * (double)g.top_p * Z;
        }
        double list_mass = 0.0;
        const int n = wide ? -1 : f->list_kept_mass(lim, top, tau_inv, &list_mass);
        const bool whole = n == a.V;                   // the list is the row
        const bool to_floor = g.floor && lim == zfloor;  // the list holds all that min_p admits
        int token = -1;
        float logit = 0.0f;
        double kept_total = 1.0;
        // can the list settle the kept set?  (a nucleus that ends at its very end is found out below)
        const bool over_list = g.top_k > 0 || whole;   // what top_p is a share of
        const double slack = over_list ? 0.0 : (deep_error(a.V, Zm, c, tau_inv, top.near_far()) + kFlat) * (double)g.top_p * Zm + 1e-12 * Zm;
        const bool listed = n > 0 && n <= kSampleList && (g.top_k == 0 || n >= g.top_k || whole || (to_floor && !g.nucleus)) &&
                            (!g.nucleus || over_list || to_floor || list_mass > (double)g.top_p * Zm + slack);
        if (listed) f->order_lists();
        if (w.rank == 0 && listed) {
            bool ok = true;
            {
                // running sums in the row's order
                const int lim_n = g.top_k > 0 && g.top_k < n ? (int)g.top_k : n;
                constexpr int PT = kSampleList / kThreads;
                const int per = (lim_n + kThreads - 1) / kThreads;
                double run[PT];
                double own = 0.0;
#pragma unroll
                for (int k = 0; k < PT; ++k) {
                    const int i = tid * per + k;
                    if (k < per && i < lim_n) own += exp64(((double)unorder32((uint32_t)(list[i] >> 32)) - (double)zmax) * tau_inv);
                    run[k] = own;
                }
                double total;
                const double base = block_scan_ahead(own, ctl.dpart, &total);
                // the nucleus: the first entry whose running sum reaches top_p of the (top-k) sum
                int count = lim_n;
                if (g.nucleus) {
                    const double goal = (double)g.top_p * (over_list ? total : Zm);
                    int first = kNoCut, unsure = 0;
#pragma unroll
                    for (int k = 0; k < PT; ++k) {
                        const int i = tid * per + k;
                        if (k < per && i < lim_n) {
                            const double at = base + run[k];
                            if (at >= goal && first == kNoCut) first = i;
                            if (slack > 0.0 && fabs(at - goal) <= slack) unsure = 1;
                        }
                    }
                    first = block_reduce<W>(first, ctl.ipart, Min());
                    unsure = block_reduce<W>(unsure, ctl.ipart, Plus());
                    if (unsure) ok = false;
                    if (first < kNoCut) count = first + 1;
                    else if (!over_list && !to_floor) ok = false;    // the nucleus goes on below the list
                }
                // min_p: entries are sorted, so the admitted ones are a prefix
                if (g.floor) {
                    int m = 0;
#pragma unroll
                    for (int k = 0; k < PT; ++k) {
                        const int i = tid * per + k;
                        if (k < per && i < count && unorder32((uint32_t)(list[i] >> 32)) >= zfloor) ++m;
                    }
                    m = block_reduce<W>(m, ctl.ipart, Plus());
                    count = max(1, min(count, m));
                }
                if (ok) {
                    // back into id order, and the draw
                    __syncthreads();
                    for (int i = tid; i < count; i += kThreads) {
                        const unsigned long long k = list[i];
                        list[i] = ((unsigned long long)~(uint32_t)k << 32) | (k >> 32);
                    }
                    __syncthreads();
                    if (count > 1) sort_list(list, count);
                    const int per2 = (count + kThreads - 1) / kThreads;
                    double s2 = 0.0;
#pragma unroll
                    for (int k = 0; k < PT; ++k) {
                        const int i = tid * per2 + k;
                        if (k < per2 && i < count) s2 += exp64(((double)unorder32((uint32_t)list[i]) - (double)zmax) * tau_inv);
                        run[k] = s2;
                    }
                    const double base2 = block_scan_ahead(s2, ctl.dpart, &kept_total);
                    const double target = (double)g.u * kept_total;
                    int pick = kNoCut;
#pragma unroll
                    for (int k = 0; k < PT; ++k) {
                        const int i = tid * per2 + k;
                        if (k < per2 && i < count && pick == kNoCut &&
                            (g.u == 0.0f ? unorder32((uint32_t)list[i]) > -INFINITY : base2 + run[k] > target))
                            pick = i;
                    }
                    pick = block_reduce<W>(pick, ctl.ipart, Min());
                    if (pick >= count) pick = count - 1;
                    token = (int)(uint32_t)(list[pick] >> 32);
                    logit = unorder32((uint32_t)list[pick]);
                }
            }
            if (!ok) token = -1;
        }
        bool settled = false;
        if (listed) {
            Xch out = {};
            out.i = token;
            settled = f->exchange(out)[0].i >= 0;
        }
        if (!settled) {
            float thr = -INFINITY;
            int cut = kNoCut;
            double lane_above = -1.0;
            if (g.top_k > 0) f->count_threshold(g.top_k, zmax, &thr, &cut);
            if (g.nucleus) {
                const double S = g.top_k > 0 ? f->kept_sum(thr, cut, top, tau_inv) : Zm;
                if (!f->nucleus_threshold(g.top_p, S, g.top_k > 0, top, tau_inv, &thr, &cut, &lane_above)) {
                    lane_above = -1.0;
                    const double total = f->kept_sum(thr, cut, top, tau_inv);
                    f->mass_threshold((double)g.top_p * total, top, tau_inv, &thr, &cut);
                }
            }
            if (zfloor > thr) { thr = zfloor; cut = kNoCut; lane_above = -1.0; }
            if (!f->template draw<false>((double)g.u, thr, cut, top, tau_inv, lane_above, &token, &logit, &kept_total))
                f->template draw<true>((double)g.u, thr, cut, top, tau_inv, -1.0, &token, &logit, &kept_total);
        }
        if (w.rank == 0 && tid == 0) {
            const double d = ((double)logit - (double)zmax) * tau_inv;
            a.tokens[t] = token;
            if (a.logp) a.logp[t] = (float)(d - lz);
            if (a.logq) a.logq[t] = (float)(d - log(kept_total));
        }
    }
}

template <int DT, bool FILTERS>
__global__ void __launch_bounds__(kThreads, 2)
pods_sample_kernel(const SampleArgs a) {
    Rows<DT> w(a);
    Finder<DT> f(w);

    const int64_t n_clusters = gridDim.x / w.CL;
    for (int64_t t0 = blockIdx.x / w.CL; t0 < a.T; t0 += kRedoRows * n_clusters) {
        for (int k = 0; k < kRedoRows; ++k) {
            const int64_t t = t0 + k * n_clusters;
            if (t >= a.T) break;
            if (a.mask != nullptr && a.mask[t] == 0) continue;
            sample_row<DT, false, FILTERS>(w, &f, t, k);
            w.done();
        }
        w.cl.sync();                                   // the marks are in place, the same in every CTA
        static_assert(kRedoRows / 32 <= kThreads, "a word of marks a thread");
        if (__syncthreads_or(w.tid < kRedoRows / 32 && row_ctrl().redo[w.tid] != 0)) {
            const int64_t left = (a.T - t0 + n_clusters - 1) / n_clusters;           // rows of this cluster from t0 on
            const int words = (int)((left < kRedoRows ? left : kRedoRows) + 31) / 32;
            for (int i = 0; i < words; ++i) {
                uint32_t bits = row_ctrl().redo[i];
                while (bits) {
                    const int k = 32 * i + __ffs(bits) - 1;
                    bits &= bits - 1;
                    sample_row<DT, true, false>(w, nullptr, t0 + k * n_clusters, 0);
                    w.done();
                }
            }
            __syncthreads();
            if (w.tid < kRedoRows / 32) row_ctrl().redo[w.tid] = 0;
        }
        if (t0 + kRedoRows * n_clusters < a.T) w.cl.sync();      // cleared before the next mark
    }
}

// ---- many rows without filters: a pipeline -----------------------------------------------------------------------------
// The same arithmetic where rows come by the hundred and every SM holds two CTAs: three kinds of warps that meet only at
// mbarriers, so that no warp waits for the cluster with its hands full (with a cluster barrier a row, 512 rows of 151936 took
// 135 us, two thirds of the instructions being every warp's own copy of what one needs to know).
//   producer  one thread: the row's segment into one of three stages, as soon as the consumers have left it
//   consumer  eight warps: maximum, sum, lane sums kept in a ring; the part goes to every CTA of the cluster by asynchronous
//            stores that count on the receiver's mbarrier; then the stage is free - no consumer waits for the exchange
//   exchange  one warp: all parts of the row, the owner of the drawn point, and, where that is a warp of this CTA, the search
//            among the lane sums and of one lane's elements, read again from global memory
// A row's slots are used again four rows later, when every exchange warp of the cluster has said that it is done with them.
// Close draws are marked by a token of kMarked; pods_sample_marked_kernel takes them in fp64.
constexpr int PW = 8;                         // consumer warps
constexpr int kPolicyThreads = (PW + 2) * 32;
constexpr int kMaxStages = 3, kRing = 4;

struct SumPart {                              // 16 bytes, sent as one store
    double s;
    float m;
    int pad;
};

struct PolicyCtrl {
    unsigned long long full[kMaxStages], empty[kMaxStages];
    unsigned long long parts[kRing];          // a row's parts have arrived
    unsigned long long ready[kRing];          // this CTA's lane sums are there
    unsigned long long done[kRing];           // every exchange warp is done with the slots
    double lanes[kRing][PW][32];              // lane sums, scanned
    alignas(16) SumPart part[1];              // [kRing][CL PW]
};
// control block of a CTA in a cluster of cl
__host__ __device__ constexpr int policy_ctrl_bytes(int cl) {
    return ((int)offsetof(PolicyCtrl, part) + kRing * cl * PW * (int)sizeof(SumPart) + 127) & ~127;
}

template <int DT>
__global__ void __launch_bounds__(kPolicyThreads, 2)
pods_sample_policy_kernel(const SampleArgs a) {
    const int n_stages = a.n_stages;
    using El = Elem<DT>;
    constexpr int E = El::E;
    PolicyCtrl& c = *reinterpret_cast<PolicyCtrl*>(smem_);
    cg::cluster_group cl = cg::this_cluster();
    const int CL = (int)cl.num_blocks();
    uint4* const stages = reinterpret_cast<uint4*>(smem_ + policy_ctrl_bytes(CL));
    const int rank = (int)cl.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t n_clusters = gridDim.x / CL, first = blockIdx.x / CL;
    const int n_rows = first < a.T ? (int)((a.T - first + n_clusters - 1) / n_clusters) : 0;
    if (tid == 0) {
        for (int i = 0; i < kMaxStages; ++i) {
            mbar_init(&c.full[i], 1);
            mbar_init(&c.empty[i], PW);
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&c.parts[i], 1);
            mbar_init(&c.ready[i], PW);
            mbar_init(&c.done[i], (uint32_t)CL);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    cl.sync();                                         // every CTA's barriers are there before anyone reaches for them

    const float tau = a.temperature;
    const double tau_inv = 1.0 / (double)tau;
    const float cexp = (float)(1.4426950408889634 * tau_inv);
    bool late = false;                                 // a wait ran out: no further one is worth its time
    auto spins = [&]() { return late ? 1u : kSpinLimit; };

    if (warp == PW) {
        // ---- producer ----
        if (lane == 0) {
            StageRing ring;
            for (int i = 0; i < n_rows; ++i) {
                const int st = ring.st;
                if (i >= n_stages && !mbar_wait(&c.empty[st], ring.parity ^ 1u, spins())) late = true;
                const Segment s = make_segment<DT>(a.logits, a.ldl, first + i * n_clusters, a.V, rank, a.seg);
                uint4* const buf = stages + (size_t)st * a.seg;
                fill_edges<DT>(s, a.V, buf);
                fence_async_proxy();                   // edges of an earlier row may lie where this row's copy goes
                start_copy(s, buf, &c.full[st]);
                ring.next(n_stages);
            }
            // every copy has landed before the CTA ends, also one that a consumer gave up on
            for (int k = 0; k < n_stages && k < n_rows; ++k) {
                ring.st = ring.st == 0 ? n_stages - 1 : ring.st - 1;           // from the last row back
                if (ring.st == n_stages - 1) ring.parity ^= 1u;
                if (!mbar_wait(&c.full[ring.st], ring.parity, kSpinLimit)) late = true;
            }
        }
    } else if (warp < PW) {
        // ---- consumers ----
        StageRing ring;
        for (int i = 0; i < n_rows; ++i, ring.next(n_stages)) {
            const int st = ring.st, slot = i % kRing;
            const Segment s = make_segment<DT>(a.logits, a.ldl, first + i * n_clusters, a.V, rank, a.seg);
            int v0, v1;
            lane_vectors<PW>(s.cnt, warp, lane, &v0, &v1);
            const uint4* const buf = stages + (size_t)st * a.seg;
            if (!mbar_wait(&c.full[st], ring.parity, spins())) late = true;
            float m = -INFINITY;
#pragma unroll 4
            for (int j = v0; j < v1; ++j) m = max_nan(m, El::vec_max(buf[j]));
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(PODS_FULL_MASK, m, d));
            const PartRef ref(m, cexp);
            const double sum = ref.far ? lane_exp_sum<DT, true>(buf, v0, v1, ref) : lane_exp_sum<DT, false>(buf, v0, v1, ref);
            __syncwarp();
            if (lane == 0) arrive_local(&c.empty[st]);
            const double incl = warp_scan(sum, lane);
            const double total = __shfl_sync(PODS_FULL_MASK, incl, 31);
            if (i >= kRing && !wait_cluster(&c.done[slot], (uint32_t)((i / kRing - 1) & 1), spins())) late = true;
            c.lanes[slot][warp][lane] = incl;
            __syncwarp();
            if (lane == 0) arrive_local(&c.ready[slot]);
            if (lane < CL)
                store_async(mapa(c.part + slot * CL * PW + rank * PW + warp, lane), mapa(&c.parts[slot], lane), total,
                            (unsigned long long)__float_as_uint(m));
        }
    } else {
        // ---- exchange ----
        float u_next = n_rows > 0 ? a.u[first] : 0.0f;
        for (int i = 0; i < n_rows; ++i) {
            const int slot = i % kRing;
            const int64_t t = first + i * n_clusters;
            float u = u_next;
            if (i + 1 < n_rows) u_next = a.u[t + n_clusters];
            bool odd = false;
            if (!(u >= 0.0f)) { u = 0.0f; odd = true; }
            if (!(u < 1.0f)) { u = 0x1.fffffep-1f; odd = true; }
            if (lane == 0) {
                mbar_expect_tx(&c.parts[slot], (uint32_t)(CL * PW * 16));
                if (odd && rank == 0) pods_raise(a.status, PODS_STATUS_PARAM_RANGE);
            }
            if (!wait_cluster(&c.parts[slot], (uint32_t)((i / kRing) & 1), spins())) late = true;

            // lane l holds parts [l n, (l + 1) n)
            constexpr int N = kMaxCluster * PW / 32;
            const int n_parts = CL * PW, n = (n_parts + 31) / 32;
            double v[N], mine = 0.0;
            float pm[N], z = -INFINITY;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = 0.0;
                pm[k] = -INFINITY;
                if (k < n && lane * n + k < n_parts) {
                    const SumPart p = c.part[slot * n_parts + lane * n + k];
                    v[k] = p.s;
                    pm[k] = p.m;
                }
                z = max_nan(z, pm[k]);
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) z = max_nan(z, __shfl_xor_sync(PODS_FULL_MASK, z, d));
            const float zmax = z + 0.0f;
            if (fabsf(z) < INFINITY) {
                const PartRef top(zmax, cexp);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    if (v[k] > 0.0) v[k] *= PartRef(pm[k], cexp).scale_to(top);
                    mine += v[k];
                }
                const double incl = warp_scan(mine, lane);
                const double Z = __shfl_sync(PODS_FULL_MASK, incl, 31), target = (double)u * Z;
                const uint32_t hit = __ballot_sync(PODS_FULL_MASK, incl > target && mine > 0.0);
                const int from = hit ? __ffs(hit) - 1 : 0;
                int owner = -1;
                double b = incl - mine, before = b;
                float om = 0.0f;
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (v[k] > 0.0 && (owner < 0 || !(b > target))) {  // the first that passes the target, else the last
                        owner = lane * n + k;
                        om = pm[k];
                        before = b;
                        b += v[k];
                    }
                owner = __shfl_sync(PODS_FULL_MASK, owner, from);
                before = __shfl_sync(PODS_FULL_MASK, before, from);
                om = __shfl_sync(PODS_FULL_MASK, om, from);
                if (u == 0.0f) {                       // needs every id's own logit: left to the other kernel
                    if (rank == 0 && lane == 0) a.tokens[t] = kMarked;
                } else if (owner / PW == rank) {
                    const int w = owner % PW;
                    const PartRef ref(om, cexp);
                    const double scale = ref.scale_to(top), goal = (target - before) / scale;
                    if (!mbar_wait(&c.ready[slot], (uint32_t)((i / kRing) & 1), spins())) late = true;
                    const double lincl = c.lanes[slot][w][lane], up = __shfl_up_sync(PODS_FULL_MASK, lincl, 1);
                    const double lsum = lincl - (lane ? up : 0.0);
                    const uint32_t past = __ballot_sync(PODS_FULL_MASK, lincl > goal && lsum > 0.0);
                    const uint32_t any = __ballot_sync(PODS_FULL_MASK, lsum > 0.0);
                    const int l = past ? __ffs(past) - 1 : 31 - __clz(any | 1u);
                    const double ahead = __shfl_sync(PODS_FULL_MASK, lane ? up : 0.0, l);
                    const Segment s = make_segment<DT>(a.logits, a.ldl, t, a.V, rank, a.seg);
                    int v0, v1;
                    lane_vectors<PW>(s.cnt, w, l, &v0, &v1);
                    const int e0 = max(v0 * E, -s.id0), e1 = min(v1 * E, a.V - s.id0), K = (max(0, e1 - e0) + 31) / 32;
                    const int k0 = min(e1, e0 + lane * K), k1 = min(e1, k0 + K);
                    const typename El::raw* const row = static_cast<const typename El::raw*>(a.logits) + t * a.ldl + s.id0;
                    double own = 0.0;
                    for (int k = k0; k < k1; ++k) own += ref.exp1(El::to_float(row[k]));
                    const double eincl = warp_scan(own, lane);
                    const uint32_t over = __ballot_sync(PODS_FULL_MASK, ahead + eincl > goal && own > 0.0);
                    const uint32_t some = __ballot_sync(PODS_FULL_MASK, own > 0.0);
                    if (lane == (over ? __ffs(over) - 1 : 31 - __clz(some | 1u))) {
                        double run = ahead + eincl - own, lo = run, ev = 0.0;
                        int at = -1;
                        float x = 0.0f;
                        for (int k = k0; k < k1; ++k) {
                            const float y = El::to_float(row[k]);
                            const double wgt = ref.exp1(y);
                            if (!(wgt > 0.0)) continue;
                            at = s.id0 + k;
                            x = y;
                            lo = run;
                            ev = wgt;
                            run += wgt;
                            if (run > goal) break;
                        }
                        const double edge = before + lo * scale, next = edge + ev * scale;
                        const double margin = draw_margin((double)u, Z, deep_error(a.V, Z, cexp, tau_inv, top.near_far()));
                        if (at >= 0 && draw_is_sure((double)u, target, edge, next, margin)) {
                            const float d = (float)(((double)x - (double)zmax) * tau_inv - (log(Z) + top.log_offset()));
                            a.tokens[t] = at;
                            if (a.logp) a.logp[t] = d;
                            if (a.logq) a.logq[t] = d;
                        } else {
                            a.tokens[t] = kMarked;
                        }
                    }
                }
            } else if (rank == 0 && lane == 0) {
                const bool empty = zmax == -INFINITY;
                const float d = empty ? -INFINITY : NAN;
                a.tokens[t] = -1;
                if (a.logp) a.logp[t] = d;
                if (a.logq) a.logq[t] = d;
                pods_raise(a.status, empty ? PODS_STATUS_EMPTY_ROW : PODS_STATUS_NONFINITE_LOGIT);
            }
            __syncwarp();
            if (lane < CL) arrive_remote(mapa(&c.done[slot], lane));
        }
    }
    if (late && lane == 0) pods_raise(a.status, PODS_STATUS_TIMEOUT);
    __syncwarp();
    cl.sync();                                         // no CTA leaves while a peer may still reach its shared memory
}

// Numbers the marked rows, so that they can be dealt out evenly: kMarked becomes kMarked - 1 - number.  One CTA.
__global__ void __launch_bounds__(1024)
number_marks_kernel(int32_t* tokens, int64_t T) {
    __shared__ int part[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int count = 0;
    for (int64_t t0 = 0; t0 < T; t0 += 1024) {
        const int64_t t = t0 + threadIdx.x;
        const bool marked = t < T && tokens[t] == kMarked;
        if (!__syncthreads_or(marked)) continue;
        const uint32_t bits = __ballot_sync(PODS_FULL_MASK, marked);
        if (lane == 0) part[warp] = __popc(bits);
        __syncthreads();
        int before = count;
        for (int w = 0; w < 32; ++w) {
            if (w < warp) before += part[w];
            count += part[w];
        }
        if (marked) tokens[t] = kMarked - 1 - (before + __popc(bits & ((1u << lane) - 1u)));
        __syncthreads();
    }
}

// The marked rows in fp64, each cluster the numbers that fall to it.  Other clusters put tokens in place of other numbers
// meanwhile, which changes nothing for this one; its own rows are found before any of them is taken.
template <int DT>
__global__ void __launch_bounds__(kThreads, 2)
pods_sample_marked_kernel(const SampleArgs a) {
    Rows<DT> w(a);
    const int n_clusters = (int)(gridDim.x / w.CL), mine = (int)(blockIdx.x / w.CL);
    uint32_t* const bits = row_ctrl().redo;
    for (int64_t t0 = 0; t0 < a.T; t0 += kRedoRows) {
        const int rows = (int)(a.T - t0 < kRedoRows ? a.T - t0 : kRedoRows), words = (rows + 31) / 32;
        bool any = false;
        for (int k0 = 0; k0 < rows; k0 += kThreads) {
            const int k = k0 + w.tid;
            const int token = k < rows ? a.tokens[t0 + k] : 0;
            const bool hit = token < kMarked && (kMarked - 1 - token) % n_clusters == mine;
            const uint32_t b = __ballot_sync(PODS_FULL_MASK, hit);
            if (w.lane == 0 && (k >> 5) < words) bits[k >> 5] = b;
            any |= hit;
        }
        w.cl.sync();
        if (__syncthreads_or(any))
            for (int i = 0; i < words; ++i) {
                uint32_t b = bits[i];
                while (b) {
                    const int k = 32 * i + __ffs(b) - 1;
                    b &= b - 1;
                    sample_row<DT, true, false>(w, nullptr, t0 + k, 0);
                    w.done();
                }
            }
        __syncthreads();
    }
}

template <int DT>
__global__ void __launch_bounds__(kThreads, 3)
pods_topk_kernel(const SampleArgs a) {
    Rows<DT> w(a);
    Finder<DT> f(w);
    const int tid = w.tid;

    const double tau_inv = 1.0 / (double)a.temperature;
    const float c = (float)(1.4426950408889634 * tau_inv);
    const int64_t n_clusters = gridDim.x / w.CL;
    for (int64_t t = blockIdx.x / w.CL; t < a.T; t += n_clusters) {
        if (a.mask != nullptr && a.mask[t] == 0) continue;
        w.start(t);
        w.wait();
        const float lm = w.lane_max();
        Part p = {};
        p.m = w.warp_max(lm);
        if (a.lse != nullptr) {
            const PartRef ref(p.m, c);
            p.s = warp_scan(w.template lane_sum<false, false>(ref, tau_inv, 0.0f, 0), w.lane);
            p.s = __shfl_sync(PODS_FULL_MASK, p.s, 31);
        }
        p.lim = w.reach(lm, a.K);
        const Part* const part = w.publish(p);
        const float zmax = w.row_max(part);
        if (zmax != zmax || zmax == INFINITY) {
            if (w.rank == 0) {
                for (int i = tid; i < a.K; i += kThreads) {
                    a.ids[t * a.K + i] = -1;
                    a.values[t * a.K + i] = NAN;
                }
                if (tid == 0) {
                    if (a.lse) a.lse[t] = NAN;
                    pods_raise(a.status, PODS_STATUS_NONFINITE_LOGIT);
                }
            }
        } else {
            if (f.template list_kept<false>(w.limit(part), kNoCut) < a.K) {      // too many reach it: the exact threshold
                float thr;
                int cut;
                f.count_threshold(a.K, zmax, &thr, &cut);
                f.template list_kept<true>(thr, cut);
            }
            // every CTA ranks its own entries and writes those within K
            f.rank_lists(w.rank, w.rank + 1, [&](int r, unsigned long long k) {
                if (r < a.K) {
                    a.ids[t * a.K + r] = (int32_t)~(uint32_t)k;
                    a.values[t * a.K + r] = unorder32((uint32_t)(k >> 32));
                }
            });
            if (w.rank == 0) {
                if (w.warp == 0 && a.lse != nullptr) {
                    const PartRef top(zmax, c);
                    const double Z = w.template sum_parts<false, false>(part, top, tau_inv).total;
                    if (tid == 0) a.lse[t] = zmax == -INFINITY ? -INFINITY : (float)((double)zmax * tau_inv + log(Z) + top.log_offset());
                }
                if (tid == 0 && zmax == -INFINITY) pods_raise(a.status, PODS_STATUS_EMPTY_ROW);
            }
        }
        w.done();
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

constexpr size_t kMaxSmem = 227 * 1024;
// Segments of at most this size let two CTAs share an SM, and the smallest such cluster has the fewest partners to wait for.
// With twice the CTAs a row: 64 fp32 rows of 151936 with their own settings 43 -> 94 us, 512 bf16 rows with wide nuclei 427 ->
// 877, pods_topk of 1024 bf16 rows 179 -> 276; with half of them, one CTA an SM, all three were slower too.
// A cluster wide enough for a bound on top_k above 128, as K gets one, does not pay: V = 32000, 512 rows, top_k = 300 264 -> 223
// us, but 700 270 -> 356 us, and V = 4000, 300 86 -> 222 us.
constexpr size_t kSegmentBytes = 80 * 1024;

constexpr size_t kHalfSmBytes = 233472 / 2 - 1024;     // what a CTA may hold for two of them to share an SM

// CTAs a row: segments of at most kSegmentBytes, and enough lanes for a list of K, whose bound comes from their maxima.
int row_cluster_size(int64_t V, int64_t T, int esize, int K) {
    int cl = 1;
    while (cl < kMaxCluster && ((size_t)segment_vectors(V, esize, cl) * 16 > kSegmentBytes || cl * kThreads < 2 * K)) cl *= 2;
    // few rows: spread over idle SMs down to a vector a thread.  One row of 32000 bf16: top_k = 200 45 -> 21 us, 700 121 -> 31 us,
    // top_k = 50 21 -> 19 us; of 151936: 700 41 -> 33 us, 50 19 -> 20 us
    while (cl < kMaxCluster && 2 * cl * T <= 128 && segment_vectors(V, esize, 2 * cl) >= kThreads) cl *= 2;
    return cl;
}

// room: bytes besides the segment
template <auto KERNEL>
int launch_rows(SampleArgs& a, int esize, int cl, size_t room, cudaStream_t stream) {
    a.seg = segment_vectors(a.V, esize, cl);
    const size_t smem = room + (size_t)a.seg * 16;
    if (smem > kMaxSmem) return PODS_ERR_UNSUPPORTED;
    return launch_row_clusters<KERNEL>(a, a.T, cl, kThreads, smem, stream);
}

// The pipeline where there are rows enough for it; sets `marked` if it ran.  Measured, pipeline (its three launches) against the
// kernel for few rows, bf16: 27.0 : 22.9 us at 16 MB of logits of 151936, 30.9 : 37.0 at 32 MB, 41.2 : 45.3 at 64 MB, 71.3 : 78.2
// at 128 MB; V = 32000 34.0 : 35.0 at 32 MB, 45.5 : 47.3 at 64 MB; V = 1000 213 : 209 at 32 MB, 394 : 409 at 64 MB.  One limit for all
// V, where none loses: long rows would gain from 32 MB on.  Rows with a mask or temperatures of their own do not come here: 512
// rows of 151936 102 us by the kernel for few rows against 71, half of them masked 56; V = 32000, 2048 rows 77 against 74, 512
// rows 29 both.  (The marks' numbers fit 32 bits with kMarked for the rows that are admitted.)
constexpr int64_t kPipelineMinBytes = 64 << 20;
template <int DT>
int launch_policy(SampleArgs& a, int esize, cudaStream_t stream) {
    if (a.T * a.V * esize < kPipelineMinBytes || a.T > 0x7ffffff0) return PODS_OK;
    // the smallest cluster whose stages fit twice on an SM: few partners, and few places of the GPU left empty by its size
    static const int kSizes[] = {1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 12, 16};
    int cl = 0;
    size_t smem = 0;
    for (a.n_stages = kMaxStages; a.n_stages >= 2 && cl == 0; --a.n_stages)    // the longest rows make do with two stages
        for (int size : kSizes) {
            a.seg = segment_vectors(a.V, esize, size);
            smem = policy_ctrl_bytes(size) + (size_t)a.n_stages * a.seg * 16;
            if (smem <= kHalfSmBytes) { cl = size; break; }
        }
    ++a.n_stages;
    if (cl == 0) return PODS_OK;
    const int rc = launch_row_clusters<pods_sample_policy_kernel<DT>>(a, a.T, cl, kPolicyThreads, smem, stream);
    if (rc == PODS_OK) a.marked = 1;
    return rc;
}

int check_rows(const void* logits, int64_t ldl, int32_t dtype, int64_t T, int32_t V, int* esize) {
    if (dtype != PODS_DTYPE_BF16 && dtype != PODS_DTYPE_F16 && dtype != PODS_DTYPE_F32) return PODS_ERR_UNSUPPORTED;
    *esize = dtype == PODS_DTYPE_F32 ? 4 : 2;
    if (T < 0 || V < 1 || ldl < V) return PODS_ERR_INVALID_ARG;
    if (V > PODS_MAX_ROW_V) return PODS_ERR_UNSUPPORTED;
    if (!pods_aligned(logits, *esize)) return PODS_ERR_INVALID_ARG;
    return PODS_OK;
}

}  // namespace

extern "C" int pods_sample(const void* logits, int64_t ldl, int32_t dtype, int64_t T, int32_t V, const float* u,
                           const float* temperature_row, float temperature, const int32_t* top_k_row, int32_t top_k,
                           const float* top_p_row, float top_p, const float* min_p_row, float min_p,
                           const uint8_t* mask, int32_t* tokens, float* logp, float* logq, uint32_t* status,
                           void* stream) {
    int esize = 0;
    const int rc = check_rows(logits, ldl, dtype, T, V, &esize);
    if (rc != PODS_OK) return rc;
    if (!temperature_row && !(temperature >= 0.0f && temperature < INFINITY)) return PODS_ERR_INVALID_ARG;
    if (!top_p_row && !(top_p == top_p)) return PODS_ERR_INVALID_ARG;
    if (!min_p_row && !(min_p == min_p)) return PODS_ERR_INVALID_ARG;
    if (T == 0) return PODS_OK;
    if (logits == nullptr || u == nullptr || tokens == nullptr) return PODS_ERR_INVALID_ARG;
    if (!pods_all_aligned(4, u, temperature_row, top_k_row, top_p_row, min_p_row, tokens, logp, logq, status)) return PODS_ERR_INVALID_ARG;
    SampleArgs a = {};
    a.logits = logits;
    a.ldl = ldl;
    a.T = T;
    a.V = V;
    a.u = u;
    a.temperature_row = temperature_row;
    a.top_p_row = top_p_row;
    a.min_p_row = min_p_row;
    a.top_k_row = top_k_row;
    a.temperature = temperature;
    a.top_p = top_p;
    a.min_p = min_p;
    a.top_k = top_k;
    a.mask = mask;
    a.tokens = tokens;
    a.logp = logp;
    a.logq = logq;
    a.status = status;
    cudaStream_t s = pods_stream(stream);
    int cl = row_cluster_size(V, T, esize, 0);
    if (!top_k_row && !top_p_row && !min_p_row && (top_k <= 0 || top_k >= V) && top_p >= 1.0f && min_p <= 0.0f) {
        if (mask == nullptr && temperature_row == nullptr && temperature >= kGreedyBelow) {
            const int rc_pipe = dtype == PODS_DTYPE_BF16  ? launch_policy<PODS_DTYPE_BF16>(a, esize, s)
                                : dtype == PODS_DTYPE_F16 ? launch_policy<PODS_DTYPE_F16>(a, esize, s)
                                                          : launch_policy<PODS_DTYPE_F32>(a, esize, s);
            if (rc_pipe != PODS_OK) return rc_pipe;
        }
        if (a.marked) {
            number_marks_kernel<<<1, 1024, 0, s>>>(tokens, T);
            PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
            if (cl < 8) cl *= 2;                       // marked rows are few: twice as many CTAs each
            if (dtype == PODS_DTYPE_BF16) return launch_rows<pods_sample_marked_kernel<PODS_DTYPE_BF16>>(a, esize, cl, kRowCtrlBytes, s);
            if (dtype == PODS_DTYPE_F16) return launch_rows<pods_sample_marked_kernel<PODS_DTYPE_F16>>(a, esize, cl, kRowCtrlBytes, s);
            return launch_rows<pods_sample_marked_kernel<PODS_DTYPE_F32>>(a, esize, cl, kRowCtrlBytes, s);
        }
        if (dtype == PODS_DTYPE_BF16) return launch_rows<pods_sample_kernel<PODS_DTYPE_BF16, false>>(a, esize, cl, kRowCtrlBytes, s);
        if (dtype == PODS_DTYPE_F16) return launch_rows<pods_sample_kernel<PODS_DTYPE_F16, false>>(a, esize, cl, kRowCtrlBytes, s);
        return launch_rows<pods_sample_kernel<PODS_DTYPE_F32, false>>(a, esize, cl, kRowCtrlBytes, s);
    }
    // a CTA may list more than its share of what is ordered: the ids of a row's top need not be spread evenly
    a.list_cap = a.own_cap = cl <= 4 ? kSampleList / cl : 2 * kSampleList / cl;
    const size_t ctrl = kRowCtrlBytes + kFilterCtrlBytes + (size_t)(1 + cl) * a.list_cap * 8 + (size_t)kSampleList * 8;
    if (dtype == PODS_DTYPE_BF16) return launch_rows<pods_sample_kernel<PODS_DTYPE_BF16, true>>(a, esize, cl, ctrl, s);
    if (dtype == PODS_DTYPE_F16) return launch_rows<pods_sample_kernel<PODS_DTYPE_F16, true>>(a, esize, cl, ctrl, s);
    return launch_rows<pods_sample_kernel<PODS_DTYPE_F32, true>>(a, esize, cl, ctrl, s);
}

extern "C" int pods_topk(const void* logits, int64_t ldl, int32_t dtype, int64_t T, int32_t V, int32_t K,
                         float temperature, const uint8_t* mask, int32_t* ids, float* values, float* lse,
                         uint32_t* status, void* stream) {
    int esize = 0;
    const int rc = check_rows(logits, ldl, dtype, T, V, &esize);
    if (rc != PODS_OK) return rc;
    if (K < 1 || K > V || !(temperature >= FLT_MIN && temperature < INFINITY)) return PODS_ERR_INVALID_ARG;
    if (K > PODS_MAX_TOPK) return PODS_ERR_UNSUPPORTED;
    if (T == 0) return PODS_OK;
    if (logits == nullptr || ids == nullptr || values == nullptr) return PODS_ERR_INVALID_ARG;
    if (!pods_all_aligned(4, ids, values, lse, status)) return PODS_ERR_INVALID_ARG;
    SampleArgs a = {};
    a.logits = logits;
    a.ldl = ldl;
    a.T = T;
    a.V = V;
    a.temperature = temperature;
    a.mask = mask;
    a.K = K;
    a.ids = ids;
    a.values = values;
    a.lse = lse;
    a.status = status;
    cudaStream_t s = pods_stream(stream);
    const int cl = row_cluster_size(V, T, esize, K);
    // the first bound leaves one to four times K entries, fewer the larger K is; the exact threshold K, maybe all in one CTA
    a.list_cap = 128;
    while (a.list_cap * cl < 4 * K || a.list_cap * cl < 1024) a.list_cap *= 2;
    a.own_cap = a.list_cap > K ? a.list_cap : K;
    const size_t ctrl = kRowCtrlBytes + kFilterCtrlBytes + ((size_t)a.own_cap + (size_t)cl * a.list_cap) * 8;
    if (dtype == PODS_DTYPE_BF16) return launch_rows<pods_topk_kernel<PODS_DTYPE_BF16>>(a, esize, cl, ctrl, s);
    if (dtype == PODS_DTYPE_F16) return launch_rows<pods_topk_kernel<PODS_DTYPE_F16>>(a, esize, cl, ctrl, s);
    return launch_rows<pods_topk_kernel<PODS_DTYPE_F32>>(a, esize, cl, ctrl, s);
}
