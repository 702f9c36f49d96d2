// pods_sample and pods_topk: one token a row drawn from logits, and the first K logits of a row with its log-normaliser.
//
// With z the row, d_v = (z_v - max z) / tau and e_v = exp(d_v), the kept set of every filter (top-k, top-p, min-p) is a
// prefix of the row's order "larger logit first, then lower id", so it is described by one threshold: a value and the
// highest id kept among the logits equal to it.  The token is the first kept id, ids ascending, whose running sum of e
// exceeds u times the kept sum.
//
// A cluster of CL CTAs holds the row in shared memory (row_cluster.cuh): HBM is read once whatever the filters ask for.
//
//   pass 1   the segment's maximum; pass 2 its sum of exponentials relative to that maximum, one exponential an element;
//            one exchange of (maximum, sum) over the cluster gives every CTA the row's maximum and normaliser.
//   no filter  the CTA whose part of the running sum holds the target finds the token: warps own contiguous parts of the
//            segment, so the search narrows from CTA to warp to 32 vectors to the element.
//   filters  every warp takes the r-th largest of its lanes' maxima; the least of these over the cluster is a value that at
//            least `want` logits reach, so the logits reaching it contain the first `want` of the order.  They are listed
//            (in the typical row a few hundred), the cluster's first CTA sorts them, and the rest is arithmetic on the
//            list in fp64.
//   general  where the list does not reach far enough (a nucleus of thousands, a list full of ties), the threshold is
//            bisected on the order-preserving keys of the values, counts and fp64 sums taken over the resident row.
//
// Which token is drawn must not depend on how sums are split or rounded: a draw or a border that lies nearer to its
// neighbours than the error of the fast sums (fp32 exponentials, summed eight at a time in fp32 and then in fp64; see
// draw_margin) is taken again with fp64 exponentials throughout, so the outcome is that of fp64 arithmetic.

#include "row_cluster.cuh"

using namespace pods_row;

namespace {

constexpr int W = 8;                          // warps of a CTA
constexpr int kThreads = W * 32;
constexpr float kGreedyBelow = 0x1p-20f;      // temperatures below this are the arg-max
constexpr int kSampleList = 1024;             // entries of the sampler's list
constexpr int kNoCut = 0x7fffffff;

// How near an edge of the fast running sum a drawn point may lie before fp64 decides: twice the error of a fast sum.  That
// is (2^-24 + 2^-24 + 2^-25) of the exponent (difference, product, log2e / tau), whose mean |d| under the row's distribution
// is at most ln V - ln Z (its entropy, ln Z + mean |d|, is at most ln V), and 4e-7 for the hardware exponential (2^-22.5)
// and the three roundings of a vector's sum.
__device__ __forceinline__ double draw_margin(int V, double Z) {
    const float depth = fmaxf(0.0f, __logf((float)V) - __logf((float)Z)) + 0.01f;
    return 2.0 * (1.5e-7 * (double)depth + 4e-7) * Z;
}

struct SampleArgs {
    const void* logits;
    int64_t ldl, T;
    int V, seg;
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
    int list_cap;                             // entries of the list in shared memory (a power of two)
    uint32_t* status;
};

struct Xch {                                  // one CTA's word in an exchange
    double a, b;
    float m, lim;
    int i, n;
};

struct Ctrl {
    unsigned long long full;                  // the segment's copy
    Xch x[2][kMaxCluster];                    // exchanges alternate between the two, so that one barrier each is enough
    double dpart[W], dwarp[W];
    float fpart[W];
    int ipart[W], iwarp[W];
    int n_list;
    int found;
    double found_before;
    double found_e;
};
constexpr int kCtrlBytes = (sizeof(Ctrl) + 127) & ~127;

// Everything of a row that the steps share; the same in every thread of the cluster.
struct Row {
    double tau_inv;       // 1 / tau
    float c;              // log2e / tau
    float zmax;
    double Z;             // fast sum of e over the row
    int t_ok;
};

template <int DT>
struct Worker {
    using El = Elem<DT>;
    static constexpr int E = El::E;
    const SampleArgs& a;
    Ctrl& c;
    uint4* buf;
    unsigned long long* list;
    cg::cluster_group cl;
    int CL, rank, tid, lane, warp;
    int parity = 0;       // of the next exchange
    Segment s;
    int w0, w1;           // my warp's vectors

    __device__ Worker(const SampleArgs& a_, Ctrl& c_, uint4* buf_, unsigned long long* list_)
        : a(a_), c(c_), buf(buf_), list(list_), cl(cg::this_cluster()) {
        CL = (int)cl.num_blocks();
        rank = (int)cl.block_rank();
        tid = threadIdx.x;
        lane = tid & 31;
        warp = tid >> 5;
    }

    // Hands `mine` to every CTA of the cluster; returns the CL words.  Call with the whole CTA.
    __device__ const Xch* exchange(const Xch& mine) {
        Xch* slot = c.x[parity];
        parity ^= 1;
        if (tid < CL) *cl.map_shared_rank(slot + rank, tid) = mine;
        cl.sync();
        return slot;
    }

    __device__ int id_of(int j, int e) const { return s.id0 + j * E + e; }
    __device__ bool is_id(int id) const { return id >= 0 && id < a.V; }

    // e of one value relative to `ref`, fast or in fp64
    template <bool PREC>
    __device__ static double weight(float x, float ref, const Row& r) {
        if (PREC) return exp(((double)x - (double)ref) * r.tau_inv);
        return (double)ex2_approx((x - ref) * r.c);
    }

    // sum of e over a vector, of the kept elements only if FILT
    template <bool PREC, bool FILT>
    __device__ double vec_sum(int j, float ref, float thr, int cut, const Row& r) const {
        if constexpr (PREC) {
            double sum = 0.0;
#pragma unroll 1
            for (int e = 0; e < E; ++e) {
                const float v = El::to_float(reinterpret_cast<const typename El::raw*>(buf + j)[e]);
                if (!FILT || v > thr || (v == thr && id_of(j, e) <= cut)) sum += weight<true>(v, ref, r);
            }
            return sum;
        } else {
            float x[E], p[E];
            El::unpack(buf[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                p[e] = ex2_approx((x[e] - ref) * r.c);
                if (FILT && !(x[e] > thr || (x[e] == thr && id_of(j, e) <= cut))) p[e] = 0.0f;
            }
#pragma unroll
            for (int d = E / 2; d > 0; d >>= 1)
#pragma unroll
                for (int e = 0; e < d; ++e) p[e] += p[e + d];
            return (double)p[0];
        }
    }

    // per-warp sums of e into c.dwarp; returns the segment's sum
    template <bool PREC, bool FILT>
    __device__ double segment_sum(float ref, float thr, int cut, const Row& r) {
        double sum = 0.0;
        if (ref != -INFINITY)
            for (int j = w0 + lane; j < w1; j += 32) sum += vec_sum<PREC, FILT>(j, ref, thr, cut, r);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(PODS_FULL_MASK, sum, d);
        __syncthreads();
        if (lane == 0) c.dwarp[warp] = sum;
        __syncthreads();
        double total = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w) total += c.dwarp[w];
        return total;
    }

    // cluster-wide sum of e over the kept elements, relative to zmax, in fp64
    __device__ double row_sum_exact(float thr, int cut, const Row& r) {
        Xch mine = {};
        mine.a = segment_sum<true, true>(r.zmax, thr, cut, r);
        const Xch* x = exchange(mine);
        double total = 0.0;
        for (int q = 0; q < CL; ++q) total += x[q].a;
        return total;
    }

    // cluster-wide number of ids with value > thr and == thr
    __device__ void row_count(float thr, long long* above, long long* equal) {
        int n = 0, m = 0;
        for (int j = w0 + lane; j < w1; j += 32) {
            float x[E];
            El::unpack(buf[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool ok = is_id(id_of(j, e));
                n += (ok && x[e] > thr) ? 1 : 0;
                m += (ok && x[e] == thr) ? 1 : 0;
            }
        }
        Xch mine = {};
        mine.n = block_reduce<W>(n, c.ipart, Plus());
        mine.i = block_reduce<W>(m, c.ipart, Plus());
        const Xch* x = exchange(mine);
        *above = *equal = 0;
        for (int q = 0; q < CL; ++q) { *above += x[q].n; *equal += x[q].i; }
    }

    // id of the nth (from 0) id, ascending, whose value is thr
    __device__ int nth_equal(float thr, long long nth) {
        int m = 0;
        for (int j = w0 + lane; j < w1; j += 32) {
            float x[E];
            El::unpack(buf[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) m += (x[e] == thr && is_id(id_of(j, e))) ? 1 : 0;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m += __shfl_xor_sync(PODS_FULL_MASK, m, d);
        __syncthreads();
        if (lane == 0) c.iwarp[warp] = m;
        if (tid == 0) c.found = -1;
        __syncthreads();
        Xch mine = {};
        for (int w = 0; w < W; ++w) mine.n += c.iwarp[w];
        const Xch* x = exchange(mine);
        long long before = 0;
        for (int q = 0; q < rank; ++q) before += x[q].n;
        for (int w = 0; w < warp; ++w) before += c.iwarp[w];
        if (nth >= before && nth < before + c.iwarp[warp]) {
            for (int k = w0; k < w1; k += 32) {
                const int j = k + lane;
                int mine_n = 0;
                float x[E];
                if (j < w1) {
                    El::unpack(buf[j], x);
#pragma unroll
                    for (int e = 0; e < E; ++e) mine_n += (x[e] == thr && is_id(id_of(j, e))) ? 1 : 0;
                }
                int incl = mine_n;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int o = __shfl_up_sync(PODS_FULL_MASK, incl, d);
                    if (lane >= d) incl += o;
                }
                const int total = __shfl_sync(PODS_FULL_MASK, incl, 31);
                if (nth < before + total) {
                    long long at = before + incl - mine_n;
                    if (nth >= at && nth < at + mine_n)
                        for (int e = 0; e < E; ++e) {
                            const float v = El::to_float(reinterpret_cast<const typename El::raw*>(buf + j)[e]);
                            if (v == thr && is_id(id_of(j, e))) {
                                if (at == nth) c.found = id_of(j, e);
                                ++at;
                            }
                        }
                    break;
                }
                before += total;
            }
        }
        __syncthreads();
        Xch out = {};
        out.i = c.found;
        x = exchange(out);
        int id = -1;
        for (int q = 0; q < CL; ++q) id = max(id, x[q].i);
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

    // Shrinks (thr, cut) to the smallest prefix whose sum of e reaches `mass`.
    __device__ void mass_threshold(double mass, const Row& r, float* thr, int* cut) {
        uint32_t lo = El::to_key(*thr), hi = El::to_key(r.zmax) + 1;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (row_sum_exact(El::from_key(mid), kNoCut, r) >= mass) lo = mid; else hi = mid;
        }
        const float v = El::from_key(lo);
        long long above, equal;
        row_count(v, &above, &equal);
        // everything above v: v itself with no id of its own
        const double more = mass - row_sum_exact(v, -1, r);
        const double ev = exp(((double)v - (double)r.zmax) * r.tau_inv);
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

    // The first kept id whose running sum exceeds `target`; warp sums in c.dwarp are relative to `ref`, `target` and
    // `before` (the sum ahead of this segment) too.  Result in c.found (-1: not in this segment), with the sums around it.
    template <bool PREC, bool FILT>
    __device__ void locate(double target, double before, float ref, float thr, int cut, const Row& r) {
        if (tid == 0) c.found = -1;
        __syncthreads();
        int last = -1;                                          // the last warp with any weight takes what rounding leaves
        for (int w = 0; w < W; ++w)
            if (c.dwarp[w] > 0.0) last = w;
        double b = before;
        int mine = -1;
        for (int w = 0; w <= last; ++w) {
            if (target < b + c.dwarp[w] || w == last) { mine = w; break; }
            b += c.dwarp[w];
        }
        if (warp == mine) {
            int best = -1;
            double best_before = 0.0, best_e = 0.0;
            bool done = false;
            for (int k = w0; k < w1 && !done; k += 32) {
                const int j = k + lane;
                const double sum = j < w1 ? vec_sum<PREC, FILT>(j, ref, thr, cut, r) : 0.0;
                double incl = sum;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const double o = __shfl_up_sync(PODS_FULL_MASK, incl, d);
                    if (lane >= d) incl += o;
                }
                const double total = __shfl_sync(PODS_FULL_MASK, incl, 31);
                const bool past = b + incl > target && sum > 0.0;
                const uint32_t hit = __ballot_sync(PODS_FULL_MASK, past);
                const uint32_t any = __ballot_sync(PODS_FULL_MASK, sum > 0.0);
                // the vector that crosses the target; otherwise remember the last one with weight
                const int from = hit ? __ffs(hit) - 1 : (any ? 31 - __clz(any) : -1);
                if (from >= 0) {
                    if (lane == from) {
                        double run = b + incl - sum;
                        for (int e = 0; e < E; ++e) {
                            const float v = El::to_float(reinterpret_cast<const typename El::raw*>(buf + j)[e]);
                            const int id = id_of(j, e);
                            if (!is_id(id) || (FILT && !(v > thr || (v == thr && id <= cut)))) continue;
                            const double ev = weight<PREC>(v, ref, r);
                            if (!(ev > 0.0)) continue;
                            best = id;
                            best_before = run;
                            best_e = ev;
                            run += ev;
                            if (run > target) break;
                        }
                    }
                    best = __shfl_sync(PODS_FULL_MASK, best, from);
                    best_before = __shfl_sync(PODS_FULL_MASK, best_before, from);
                    best_e = __shfl_sync(PODS_FULL_MASK, best_e, from);
                }
                done = hit != 0;
                b += total;
            }
            if (lane == 0) {
                c.found = best;
                c.found_before = best_before;
                c.found_e = best_e;
            }
        }
        __syncthreads();
    }

    // Draw over the kept set in fp64; every thread of the cluster gets the token and the kept sum.
    __device__ int draw_exact(double u, float thr, int cut, const Row& r, double* kept) {
        Xch mine = {};
        mine.a = segment_sum<true, true>(r.zmax, thr, cut, r);
        const Xch* x = exchange(mine);
        double total = 0.0;
        for (int q = 0; q < CL; ++q) total += x[q].a;
        const double target = u * total;
        double before = 0.0;
        int last = -1, owner = -1;
        for (int q = 0; q < CL; ++q)
            if (x[q].a > 0.0) last = q;
        for (int q = 0; q <= last; ++q) {
            if (target < before + x[q].a || q == last) { owner = q; break; }
            before += x[q].a;
        }
        if (rank == owner) locate<true, true>(target, before, r.zmax, thr, cut, r);
        __syncthreads();
        Xch out = {};
        out.i = rank == owner ? c.found : -1;
        x = exchange(out);
        int id = -1;
        for (int q = 0; q < CL; ++q) id = max(id, x[q].i);
        *kept = total;
        return id;
    }

    // Lists the kept (value, id) pairs of the segment: (order32(value) << 32) | ~id, larger first in the row's order.
    // The count may exceed the room; only list_cap entries are stored.
    __device__ void list_segment(float thr, int cut) {
        __syncthreads();
        if (tid == 0) c.n_list = 0;
        __syncthreads();
        for (int j = w0 + lane; j < w1; j += 32) {
            const uint4 q = buf[j];
            if (El::vec_max(q) < thr) continue;
            float x[E];
            El::unpack(q, x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int id = id_of(j, e);
                if (is_id(id) && (x[e] > thr || (x[e] == thr && id <= cut))) {
                    const int at = atomicAdd(&c.n_list, 1);
                    if (at < a.list_cap) list[at] = ((unsigned long long)order32(x[e]) << 32) | (uint32_t)~id;
                }
            }
        }
        __syncthreads();
    }

    // The cluster's list in the first CTA, sorted in the row's order; returns its length, or -1 if it does not fit.
    // Ends without a barrier after the first CTA's reads of its peers: an exchange has to follow.
    __device__ int gather_sorted(float thr, int cut) {
        list_segment(thr, cut);
        Xch mine = {};
        mine.n = c.n_list;
        const Xch* x = exchange(mine);
        long long total = 0;
        for (int q = 0; q < CL; ++q) total += x[q].n;
        if (total > a.list_cap) return -1;
        if (rank == 0) {
            int at = x[0].n;
            for (int q = 1; q < CL; ++q) {
                const unsigned long long* peer = cl.map_shared_rank(list, q);
                for (int k = tid; k < x[q].n; k += kThreads) list[at + k] = peer[k];
                at += x[q].n;
            }
            sort_list((int)total, true);
        }
        return (int)total;
    }

    // Bitonic sort of list[0, n), padded with the value that sorts last; the whole CTA.
    __device__ void sort_list(int n, bool descending) {
        int m = 1;
        while (m < n) m <<= 1;
        for (int k = n + tid; k < m; k += kThreads) list[k] = descending ? 0ull : ~0ull;
        __syncthreads();
        for (int size = 2; size <= m; size <<= 1)
            for (int d = size >> 1; d > 0; d >>= 1) {
                for (int k = tid; k < m / 2; k += kThreads) {
                    const int i = 2 * k - (k & (d - 1)), p = i + d;
                    const unsigned long long x = list[i], y = list[p];
                    const bool up = ((i & size) == 0) != descending;
                    if ((x > y) == up) { list[i] = y; list[p] = x; }
                }
                __syncthreads();
            }
    }

    // The value that at least `want` ids of the row reach (over the CTAs' minimum): my CTA's part of it.
    __device__ float reach(float lane_max, int want) {
        const int r = min(32, (want + CL * W - 1) / (CL * W));
        // lanes sorted by value, descending; lane r-1 holds the r-th largest
        uint32_t k = order32(lane_max);
#pragma unroll
        for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
            for (int d = size >> 1; d > 0; d >>= 1) {
                const uint32_t o = __shfl_xor_sync(PODS_FULL_MASK, k, d);
                const bool keep_big = ((lane & size) == 0) == ((lane & d) == 0);
                k = keep_big ? max(k, o) : min(k, o);
            }
        const float v = unorder32(__shfl_sync(PODS_FULL_MASK, k, r - 1));
        return block_reduce<W>(want > CL * W * 32 ? -INFINITY : v, c.fpart, Min());
    }
};

// ---- what both kernels begin with -------------------------------------------------------------------------------------

template <int DT>
__device__ __forceinline__ void load_row(Worker<DT>& w, int64_t t, uint32_t phase) {
    w.s = make_segment<DT>(w.a.logits, w.a.ldl, t, w.a.V, w.rank, w.a.seg);
    const int per = (w.s.cnt + W - 1) / W;
    w.w0 = min(w.s.cnt, w.warp * per);
    w.w1 = min(w.s.cnt, w.w0 + per);
    if (w.tid == 0) start_load<DT>(w.s, w.a.V, w.buf, &w.c.full);
    if (!mbar_wait(&w.c.full, phase, kSpinLimit) && w.lane == 0) pods_raise(w.a.status, PODS_STATUS_TIMEOUT);
    __syncthreads();
}

template <int DT>
__device__ __forceinline__ float lane_max(const Worker<DT>& w) {
    float m = -INFINITY;
    for (int j = w.w0 + w.lane; j < w.w1; j += 32) m = max_nan(m, Elem<DT>::vec_max(w.buf[j]));
    return m;
}

// Cluster-wide maximum and fast sum from the CTAs' (maximum, sum relative to it).
__device__ __forceinline__ void combine(const Xch* x, int CL, Row* r) {
    float m = x[0].m;
    for (int q = 1; q < CL; ++q) m = max_nan(m, x[q].m);
    r->zmax = m + 0.0f;
    double Z = 0.0;
    if (fabsf(m) < INFINITY)
        for (int q = 0; q < CL; ++q)
            if (x[q].m > -INFINITY) Z += x[q].a * exp(((double)x[q].m - (double)r->zmax) * r->tau_inv);
    r->Z = Z;
}

// Inclusive scan of v over the CTA in thread order; *total is the sum.
__device__ __forceinline__ double block_scan(double v, double* part, double* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const double o = __shfl_up_sync(PODS_FULL_MASK, v, d);
        if (lane >= d) v += o;
    }
    __syncthreads();
    if (lane == 31) part[warp] = v;
    __syncthreads();
    double before = 0.0, all = 0.0;
    for (int w = 0; w < W; ++w) {
        if (w < warp) before += part[w];
        all += part[w];
    }
    *total = all;
    return v + before;
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
pods_sample_kernel(const SampleArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    Ctrl& c = *reinterpret_cast<Ctrl*>(smem);
    unsigned long long* const list = reinterpret_cast<unsigned long long*>(smem + kCtrlBytes);
    uint4* const buf = reinterpret_cast<uint4*>(smem + kCtrlBytes + (size_t)a.list_cap * 8);
    Worker<DT> w(a, c, buf, list);
    const int CL = w.CL, tid = w.tid;
    if (tid == 0) {
        mbar_init(&c.full, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    w.cl.sync();                                       // every CTA of the cluster runs before its shared memory is written

    const int64_t n_clusters = gridDim.x / CL;
    uint32_t phase = 0;
    for (int64_t t = blockIdx.x / CL; t < a.T; t += n_clusters) {
        if (a.mask != nullptr && a.mask[t] == 0) continue;
        load_row(w, t, phase);
        phase ^= 1u;

        // the row's settings
        float tau = a.temperature_row ? a.temperature_row[t] : a.temperature;
        float top_p = a.top_p_row ? a.top_p_row[t] : a.top_p;
        float min_p = a.min_p_row ? a.min_p_row[t] : a.min_p;
        const int top_k_in = a.top_k_row ? a.top_k_row[t] : a.top_k;
        float u = a.u[t];
        bool odd = false;
        if (!(tau >= 0.0f) || tau == INFINITY) { tau = 1.0f; odd = true; }
        if (top_p != top_p) { top_p = 1.0f; odd = true; }
        if (min_p != min_p) { min_p = 0.0f; odd = true; }
        if (!(u >= 0.0f)) { u = 0.0f; odd = true; }
        if (!(u < 1.0f)) { u = 0x1.fffffep-1f; odd = true; }
        if (odd && w.rank == 0 && tid == 0) pods_raise(a.status, PODS_STATUS_PARAM_RANGE);
        const bool greedy = tau < kGreedyBelow;
        if (greedy) tau = 1.0f;
        const long long top_k = (top_k_in <= 0 || top_k_in >= a.V) ? 0 : top_k_in;
        min_p = fminf(min_p, 1.0f);
        const bool nucleus = top_p < 1.0f, floor = min_p > 0.0f;
        const bool filtered = !greedy && (top_k > 0 || nucleus || floor);

        Row r;
        r.tau_inv = 1.0 / (double)tau;
        r.c = (float)(1.4426950408889634 * r.tau_inv);

        const float lm = lane_max(w);
        Xch mine = {};
        mine.m = block_reduce<W>(lm, c.fpart, MaxNan());
        const float ref = fabsf(mine.m) < INFINITY ? mine.m : -INFINITY;     // no sums where they mean nothing
        mine.a = w.template segment_sum<false, false>(ref, 0.0f, 0, r);
        const int want = (int)(top_k > 0 ? (top_k < 512 ? top_k : 512) : 256);
        mine.lim = filtered ? w.reach(lm, want) : 0.0f;
        const Xch* x = w.exchange(mine);
        combine(x, CL, &r);

        int token = -1;
        double logq = 0.0;
        bool have = false;                             // token and logq are valid in the first CTA
        if (!(r.zmax < INFINITY) || r.zmax == -INFINITY) {
            const bool empty = r.zmax == -INFINITY;
            if (w.rank == 0 && tid == 0) {
                a.tokens[t] = -1;
                const float v = empty ? -INFINITY : NAN;
                if (a.logp) a.logp[t] = v;
                if (a.logq) a.logq[t] = v;
                pods_raise(a.status, empty ? PODS_STATUS_EMPTY_ROW : PODS_STATUS_NONFINITE_LOGIT);
            }
        } else {
            if (greedy) {
                int id = kNoCut;
                for (int j = w.w0 + w.lane; j < w.w1; j += 32) {
                    if (Elem<DT>::vec_max(buf[j]) != r.zmax) continue;
                    float v[Elem<DT>::E];
                    Elem<DT>::unpack(buf[j], v);
#pragma unroll
                    for (int e = Elem<DT>::E - 1; e >= 0; --e)
                        if (v[e] == r.zmax) id = min(id, w.id_of(j, e));
                }
                Xch out = {};
                out.i = block_reduce<W>(id, c.ipart, Min());
                x = w.exchange(out);
                token = kNoCut;
                for (int q = 0; q < CL; ++q) token = min(token, x[q].i);
                logq = 0.0;
                have = true;
            } else if (!filtered) {
                // the CTA that holds the target
                const double target = (double)u * r.Z;
                double before = 0.0, scale = 1.0;
                int owner = -1, last = -1;
                for (int q = 0; q < CL; ++q)
                    if (x[q].a > 0.0) last = q;
                for (int q = 0; q <= last; ++q) {
                    scale = exp(((double)x[q].m - (double)r.zmax) * r.tau_inv);
                    if (target < before + x[q].a * scale || q == last) { owner = q; break; }
                    before += x[q].a * scale;
                }
                Xch out = {};
                out.i = -1;
                out.n = 0;
                if (w.rank == owner) {
                    w.template locate<false, false>(target / scale, before / scale, ref, 0.0f, 0, r);
                    const double lo = c.found_before * scale, hi = lo + c.found_e * scale;
                    // an edge of the running sum closer than the margin is decided in fp64 (the row's start is no edge)
                    out.n = (target - lo > draw_margin(a.V, r.Z) || lo == 0.0) && hi - target > draw_margin(a.V, r.Z) ? 1 : 0;
                    out.i = c.found;
                }
                x = w.exchange(out);
                int sure = 0;
                for (int q = 0; q < CL; ++q) { token = max(token, x[q].i); sure |= x[q].n; }
                double kept = r.Z;
                if (!sure) token = w.draw_exact((double)u, -INFINITY, kNoCut, r, &kept);
                logq = -log(kept);
                have = true;
            } else {
                float lim = x[0].lim;
                for (int q = 1; q < CL; ++q) lim = fminf(lim, x[q].lim);
                // the lowest value that min_p admits
                const float zfloor = floor ? __double2float_ru((double)r.zmax + (double)tau * log((double)min_p)) : -INFINITY;
                // top_p is a share of the whole top-k sum, so min_p may not shorten the list where both are set
                if (floor && !(top_k > 0 && nucleus)) lim = (top_k > 0 || nucleus) ? fmaxf(lim, zfloor) : zfloor;
                const int n = w.gather_sorted(lim, kNoCut);
                const bool whole = n == a.V;                                 // the list is the row
                const bool to_floor = floor && lim == zfloor;                // the list holds all that min_p admits
                if (w.rank == 0) {
                    if (tid == 0) c.found = -1;
                    __syncthreads();
                    // does the list settle the kept set?  (a nucleus that it does not reach is found out below)
                    bool ok = n > 0 && (top_k == 0 || n >= top_k || whole || (to_floor && !nucleus));
                    if (ok) {
                        // prefix sums in the row's order, 4 entries a thread and step
                        const int lim_n = top_k > 0 && top_k < n ? (int)top_k : n;
                        constexpr int PT = kSampleList / kThreads;
                        const int per = PT;
                        double run[PT];
                        double sum = 0.0;
#pragma unroll
                        for (int k = 0; k < PT; ++k) {
                            const int i = tid * per + k;
                            if (i < lim_n) sum += exp(((double)unorder32((uint32_t)(list[i] >> 32)) - (double)r.zmax) * r.tau_inv);
                            run[k] = sum;
                        }
                        double total;
                        const double incl = block_scan(sum, c.dpart, &total);
                        const double base = incl - sum;
                        // the nucleus: the first entry whose running sum reaches top_p of the (top-k) sum
                        int count = lim_n;
                        if (nucleus) {
                            const bool over_list = top_k > 0 || whole;
                            const double goal = (double)top_p * (over_list ? total : r.Z);
                            const double slack = over_list ? 0.0 : draw_margin(a.V, r.Z);
                            int first = kNoCut, unsure = 0;
#pragma unroll
                            for (int k = 0; k < PT; ++k) {
                                const int i = tid * per + k;
                                if (i < lim_n) {
                                    const double at = base + run[k];
                                    if (at >= goal && first == kNoCut) first = i;
                                    if (slack > 0.0 && fabs(at - goal) <= slack) unsure = 1;
                                }
                            }
                            first = block_reduce<W>(first, c.ipart, Min());
                            unsure = block_reduce<W>(unsure, c.ipart, Plus());
                            if (unsure) ok = false;
                            if (first < kNoCut) count = first + 1;
                            else if (!over_list && !to_floor) ok = false;    // the nucleus goes on below the list
                        }
                        // min_p: entries are sorted, so the admitted ones are a prefix
                        if (floor) {
                            int m = 0;
#pragma unroll
                            for (int k = 0; k < PT; ++k) {
                                const int i = tid * per + k;
                                if (i < count && unorder32((uint32_t)(list[i] >> 32)) >= zfloor) ++m;
                            }
                            m = block_reduce<W>(m, c.ipart, Plus());
                            count = max(1, min(count, m));
                        }
                        if (ok) {
                            // back into id order, and the draw
                            __syncthreads();
                            for (int i = tid; i < count; i += kThreads) {
                                const unsigned long long k = list[i];
                                list[i] = ((unsigned long long)~(uint32_t)k << 32) | (k >> 32);
                            }
                            w.sort_list(count, false);
                            double s2 = 0.0;
#pragma unroll
                            for (int k = 0; k < PT; ++k) {
                                const int i = tid * per + k;
                                if (i < count) s2 += exp(((double)unorder32((uint32_t)list[i]) - (double)r.zmax) * r.tau_inv);
                                run[k] = s2;
                            }
                            const double incl2 = block_scan(s2, c.dpart, &total);
                            const double target = (double)u * total;
                            int pick = kNoCut;
#pragma unroll
                            for (int k = 0; k < PT; ++k) {
                                const int i = tid * per + k;
                                if (i < count && pick == kNoCut && incl2 - s2 + run[k] > target) pick = i;
                            }
                            pick = block_reduce<W>(pick, c.ipart, Min());
                            if (pick >= count) pick = count - 1;
                            token = (int)(uint32_t)(list[pick] >> 32);
                            logq = -log(total);
                        }
                    }
                    if (tid == 0) c.found = ok ? token : -1;
                    __syncthreads();
                }
                Xch out = {};
                out.i = w.rank == 0 ? c.found : -1;
                x = w.exchange(out);
                if (x[0].i < 0) {
                    float thr = -INFINITY;
                    int cut = kNoCut;
                    if (top_k > 0) w.count_threshold(top_k, r.zmax, &thr, &cut);
                    if (nucleus) {
                        const double total = w.row_sum_exact(thr, cut, r);
                        w.mass_threshold((double)top_p * total, r, &thr, &cut);
                    }
                    if (zfloor > thr) { thr = zfloor; cut = kNoCut; }
                    double kept;
                    token = w.draw_exact((double)u, thr, cut, r, &kept);
                    logq = -log(kept);
                }
                have = true;
            }
            // the owner of the token's logit writes the row's results
            if (have && w.rank == 0 && tid == 0) {
                a.tokens[t] = token;
                const typename Elem<DT>::raw* row = static_cast<const typename Elem<DT>::raw*>(a.logits) + t * a.ldl;
                const int safe = token < 0 ? 0 : token;
                const double d = ((double)Elem<DT>::to_float(row[PODS_CLAMPED(safe, a.V, a.status)]) - (double)r.zmax) * r.tau_inv;
                if (a.logp) a.logp[t] = (float)(d - log(r.Z));
                if (a.logq) a.logq[t] = greedy ? 0.0f : (float)(d + logq);
            }
        }
        fence_async_proxy();                           // the buffer is refilled by bulk copies
        __syncthreads();
    }
    w.cl.sync();                                       // no CTA leaves while a peer may still reach its shared memory
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
pods_topk_kernel(const SampleArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    Ctrl& c = *reinterpret_cast<Ctrl*>(smem);
    unsigned long long* const list = reinterpret_cast<unsigned long long*>(smem + kCtrlBytes);
    uint4* const buf = reinterpret_cast<uint4*>(smem + kCtrlBytes + (size_t)a.list_cap * 8);
    Worker<DT> w(a, c, buf, list);
    const int CL = w.CL, tid = w.tid;
    if (tid == 0) {
        mbar_init(&c.full, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    w.cl.sync();

    const int64_t n_clusters = gridDim.x / CL;
    uint32_t phase = 0;
    for (int64_t t = blockIdx.x / CL; t < a.T; t += n_clusters) {
        if (a.mask != nullptr && a.mask[t] == 0) continue;
        load_row(w, t, phase);
        phase ^= 1u;
        Row r;
        r.tau_inv = 1.0 / (double)a.temperature;
        r.c = (float)(1.4426950408889634 * r.tau_inv);
        const float lm = lane_max(w);
        Xch mine = {};
        mine.m = block_reduce<W>(lm, c.fpart, MaxNan());
        const float ref = fabsf(mine.m) < INFINITY ? mine.m : -INFINITY;
        if (a.lse != nullptr) mine.a = w.template segment_sum<false, false>(ref, 0.0f, 0, r);
        mine.lim = w.reach(lm, a.K);
        const Xch* x = w.exchange(mine);
        combine(x, CL, &r);
        if (r.zmax != r.zmax || r.zmax == INFINITY) {
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
            float lim = x[0].lim;
            for (int q = 1; q < CL; ++q) lim = fminf(lim, x[q].lim);
            int n = w.gather_sorted(lim, kNoCut);
            if (n < a.K) {                             // too many reach it: the exact threshold
                float thr;
                int cut;
                w.count_threshold(a.K, r.zmax, &thr, &cut);
                n = w.gather_sorted(thr, cut);
            }
            if (w.rank == 0) {
                for (int i = tid; i < a.K; i += kThreads) {
                    const unsigned long long k = list[i];
                    if (PODS_INDEX_OK(i, n, a.status)) {
                        a.ids[t * a.K + i] = (int32_t)~(uint32_t)k;
                        a.values[t * a.K + i] = unorder32((uint32_t)(k >> 32));
                    }
                }
                if (tid == 0 && a.lse) a.lse[t] = r.zmax == -INFINITY ? -INFINITY : (float)((double)r.zmax * r.tau_inv + log(r.Z));
                if (tid == 0 && r.zmax == -INFINITY) pods_raise(a.status, PODS_STATUS_EMPTY_ROW);
            }
            w.exchange(mine);                          // the first CTA has read its peers' lists
        }
        fence_async_proxy();
        __syncthreads();
    }
    w.cl.sync();
}

// ---- no filters: the whole policy -------------------------------------------------------------------------------------
// Lanes own contiguous vectors of the segment, so a lane's, a warp's and a CTA's sums are stretches of the running sum.
// Each warp reduces its part to a sum relative to 2^R, R the integer above its maximum's exponent, and hands the pair to
// every CTA of the cluster; parts are then brought together by powers of two, exactly and without an exponential.  After
// the one cluster barrier of a row every warp knows all parts in id order, and so whether the drawn point is in its own;
// the warp that has it takes the lane from the lane sums that it kept and evaluates that lane's few vectors again.  Rows
// whose draw lies within draw_margin of an edge are marked in every CTA of the cluster and taken in fp64 at the end.
// 152 K bf16 vocabulary, 512 rows: ORIGINAL

struct Part {
    double s;             // sum relative to the part's reference (to its maximum, the second time round)
    float m;              // its maximum
    int pad;
};

constexpr int kRedoRows = 8192;               // rows of a cluster between two visits of the marked ones

struct PolicyCtrl {
    unsigned long long full;
    Part part[2][kMaxCluster * W];
    uint32_t redo[kRedoRows / 32];
};
constexpr int kPolicyCtrlBytes = (sizeof(PolicyCtrl) + 127) & ~127;

__device__ __forceinline__ double pow2(int n) {       // n <= 0; below the normal numbers: 0
    return n < -1000 ? 0.0 : __hiloint2double((1023 + n) << 20, 0);
}

// e = 2^(x c - R).  R is an integer, at least m c; where the product is so large that floats have no fractions, the
// difference to the maximum is taken first and `far` parts are related by fp64 exponentials.
struct PartRef {
    float m, R, c;
    bool far;
    __device__ __forceinline__ PartRef(float m_, float c_) : c(c_) {
        m = fabsf(m_) < INFINITY ? m_ : 0.0f;
        R = ceilf(__fmul_ru(m, c));
        far = !(fabsf(R) < 0x1p23f);
    }
    template <int E>
    __device__ __forceinline__ void exps(float (&x)[E]) const {
        const unsigned long long c2 = pack2(c, c), off2 = far ? pack2(-m, -m) : pack2(-R, -R);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const unsigned long long v = pack2(x[i], x[i + 1]);
            float p, q;
            unpack2(far ? mul2(add2(v, off2), c2) : fma2(v, c2, off2), p, q);
            x[i] = ex2_approx(p);
            x[i + 1] = ex2_approx(q);
        }
    }
    __device__ __forceinline__ double exp1(float x) const { return (double)ex2_approx(far ? (x - m) * c : fmaf(x, c, -R)); }
    // what sums relative to this reference are multiplied with to be relative to that of `top`, the row's
    __device__ __forceinline__ double scale_to(const PartRef& top) const {
        if (!top.far) return pow2((int)fmaxf(R - top.R, -2000.0f));
        return exp2((far ? (double)m * (double)c : (double)R) - (double)top.m * (double)c);
    }
};

// Inclusive scan over a warp.
__device__ __forceinline__ double warp_scan(double v, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const double o = __shfl_up_sync(PODS_FULL_MASK, v, d);
        if (lane >= d) v += o;
    }
    return v;
}

template <int DT>
struct Policy {
    using El = Elem<DT>;
    static constexpr int E = El::E;
    const SampleArgs& a;
    PolicyCtrl& ctl;
    uint4* const buf;
    cg::cluster_group cl;
    int CL, rank, tid, lane, warp;
    uint32_t phase = 0;
    int parity = 0;

    __device__ Policy(const SampleArgs& a_, PolicyCtrl& c_, uint4* b_) : a(a_), ctl(c_), buf(b_), cl(cg::this_cluster()) {
        CL = (int)cl.num_blocks();
        rank = (int)cl.block_rank();
        tid = threadIdx.x;
        lane = tid & 31;
        warp = tid >> 5;
    }

    // One row; `mark`: the bit of the row in the marked ones.
    template <bool PREC>
    __device__ void row(int64_t t, int mark) {
        const Segment s = make_segment<DT>(a.logits, a.ldl, t, a.V, rank, a.seg);
        if (tid == 0) start_load<DT>(s, a.V, buf, &ctl.full);
        float tau = a.temperature_row ? a.temperature_row[t] : a.temperature;
        float u = a.u[t];
        bool odd = false;
        if (!(tau >= 0.0f) || tau == INFINITY) { tau = 1.0f; odd = true; }
        if (!(u >= 0.0f)) { u = 0.0f; odd = true; }
        if (!(u < 1.0f)) { u = 0x1.fffffep-1f; odd = true; }
        if (odd && rank == 0 && tid == 0) pods_raise(a.status, PODS_STATUS_PARAM_RANGE);
        const bool greedy = tau < kGreedyBelow;
        if (greedy) tau = 1.0f;
        const double tau_inv = 1.0 / (double)tau;
        const float c = (float)(1.4426950408889634 * tau_inv);
        // an odd number of vectors a lane: eight lanes of a 16-byte access then touch all 32 banks once
        const int per = ((s.cnt + kThreads - 1) / kThreads) | 1;
        const int v0 = min(s.cnt, tid * per), v1 = min(s.cnt, v0 + per);
        if (!mbar_wait(&ctl.full, phase, kSpinLimit) && lane == 0) pods_raise(a.status, PODS_STATUS_TIMEOUT);
        phase ^= 1u;
        __syncthreads();

        float m = -INFINITY;
#pragma unroll 4
        for (int j = v0; j < v1; ++j) m = max_nan(m, El::vec_max(buf[j]));
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(PODS_FULL_MASK, m, d));
        const PartRef ref(m, c);
        double sum = 0.0;
        if (PREC) {
            for (int j = v0; j < v1; ++j) {
                float x[E];
                El::unpack(buf[j], x);
#pragma unroll
                for (int e = 0; e < E; ++e) sum += exp(((double)x[e] - (double)ref.m) * tau_inv);
            }
        } else {
#pragma unroll 2
            for (int j = v0; j < v1; ++j) {
                float x[E];
                El::unpack(buf[j], x);
                ref.exps(x);
                sum += (double)vec_add(x);
            }
        }
        const double incl = warp_scan(sum, lane);
        Part p;
        p.s = __shfl_sync(PODS_FULL_MASK, incl, 31);
        p.m = m;
        p.pad = 0;
        const int mine = rank * W + warp, n_parts = CL * W;
        if (lane < CL) *cl.map_shared_rank(&ctl.part[parity][mine], lane) = p;
        cl.sync();

        // lane l holds parts [l n, (l + 1) n)
        const Part* const part = ctl.part[parity];
        parity ^= 1;
        constexpr int N = kMaxCluster * W / 32;
        const int n = (n_parts + 31) / 32;
        float z = -INFINITY;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n && lane * n + i < n_parts) z = max_nan(z, part[lane * n + i].m);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) z = max_nan(z, __shfl_xor_sync(PODS_FULL_MASK, z, d));
        const float zmax = z + 0.0f;
        if (!(fabsf(z) < INFINITY)) {
            if (rank == 0 && tid == 0) {
                const bool empty = z == -INFINITY;
                a.tokens[t] = -1;
                const float v = empty ? -INFINITY : NAN;
                if (a.logp) a.logp[t] = v;
                if (a.logq) a.logq[t] = v;
                pods_raise(a.status, empty ? PODS_STATUS_EMPTY_ROW : PODS_STATUS_NONFINITE_LOGIT);
            }
            return;
        }
        const PartRef top(zmax, c);
        double v[N], psum = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0;
            if (i < n && lane * n + i < n_parts) {
                const Part q = part[lane * n + i];
                if (q.s > 0.0) v[i] = q.s * (PREC ? exp(((double)q.m - (double)zmax) * tau_inv) : PartRef(q.m, c).scale_to(top));
            }
            psum += v[i];
        }
        const double pincl = warp_scan(psum, lane);
        const double Z = __shfl_sync(PODS_FULL_MASK, pincl, 31);
        const double target = (double)u * Z;
        int owner = -1;
        double before = 0.0;
        if (greedy) {
            int first = kNoCut;
            for (int i = lane; i < n_parts; i += 32)
                if (part[i].m == zmax) first = min(first, i);
            owner = __reduce_min_sync(PODS_FULL_MASK, first);
        } else {
            const uint32_t hit = __ballot_sync(PODS_FULL_MASK, pincl > target && psum > 0.0);
            const int from = __ffs(hit) - 1;               // there is one: target < Z
            double b = pincl - psum, at = b;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (v[i] > 0.0 && (owner < 0 || !(b > target))) {  // the first that passes the target, else the last
                    owner = lane * n + i;
                    at = b;
                    b += v[i];
                }
            owner = __shfl_sync(PODS_FULL_MASK, owner, from);
            before = __shfl_sync(PODS_FULL_MASK, at, from);
        }
        if (owner != mine) return;

        // ---- the warp with the drawn point ----
        if (greedy) {
            int id = kNoCut;
            for (int j = v0; j < v1; ++j) {
                float x[E];
                El::unpack(buf[j], x);
#pragma unroll
                for (int e = E - 1; e >= 0; --e)
                    if (x[e] == zmax) id = min(id, s.id0 + j * E + e);
            }
            id = __reduce_min_sync(PODS_FULL_MASK, id);
            if (lane == 0) {
                // the sum is relative to 2^R: ln Z over e^zmax
                const double lz = log(Z) + (PREC || top.far ? 0.0 : ((double)top.R - (double)zmax * (double)c) * 0.6931471805599453);
                a.tokens[t] = id;
                if (a.logp) a.logp[t] = (float)-lz;
                if (a.logq) a.logq[t] = 0.0f;
            }
            return;
        }
        const double scale = PREC ? exp(((double)m - (double)zmax) * tau_inv) : ref.scale_to(top);
        const double goal = (target - before) / scale;
        uint32_t hit = __ballot_sync(PODS_FULL_MASK, incl > goal && sum > 0.0);
        const uint32_t any = __ballot_sync(PODS_FULL_MASK, sum > 0.0);
        const int from = hit ? __ffs(hit) - 1 : 31 - __clz(any);
        const double lane_before = __shfl_sync(PODS_FULL_MASK, incl - sum, from);
        // the elements of that lane's vectors, K a lane
        const int e0 = __shfl_sync(PODS_FULL_MASK, v0, from) * E, e1 = __shfl_sync(PODS_FULL_MASK, v1, from) * E;
        const int K = (e1 - e0 + 31) / 32;
        const typename El::raw* el = reinterpret_cast<const typename El::raw*>(buf);
        const int k0 = min(e1, e0 + lane * K), k1 = min(e1, k0 + K);
        auto weight = [&](int i) {
            const float x = El::to_float(el[i]);
            return PREC ? exp(((double)x - (double)ref.m) * tau_inv) : ref.exp1(x);
        };
        double own = 0.0;
        for (int i = k0; i < k1; ++i) own += weight(i);
        const double eincl = warp_scan(own, lane);
        hit = __ballot_sync(PODS_FULL_MASK, lane_before + eincl > goal && own > 0.0);
        const uint32_t some = __ballot_sync(PODS_FULL_MASK, own > 0.0);
        const int last = hit ? __ffs(hit) - 1 : 31 - __clz(some);
        if (lane == last) {
            double run = lane_before + eincl - own, lo = run, ev = 0.0;
            int at = -1;
            for (int i = k0; i < k1; ++i) {
                const double w = weight(i);
                if (!(w > 0.0)) continue;
                at = i;
                lo = run;
                ev = w;
                run += w;
                if (run > goal) break;
            }
            // an edge of the running sum within the margin is decided in fp64 (the row's start is no edge)
            const double edge = before + lo * scale, next = edge + ev * scale, margin = draw_margin(a.V, Z);
            if (PREC || ((target - edge > margin || edge == 0.0) && next - target > margin)) {
                const double lz = log(Z) + (PREC || top.far ? 0.0 : ((double)top.R - (double)zmax * (double)c) * 0.6931471805599453);
                const float d = (float)(((double)El::to_float(el[at]) - (double)zmax) * tau_inv - lz);
                a.tokens[t] = s.id0 + at;
                if (a.logp) a.logp[t] = d;
                if (a.logq) a.logq[t] = d;
            } else {
                for (int q = 0; q < CL; ++q) atomicOr(cl.map_shared_rank(&ctl.redo[mark >> 5], q), 1u << (mark & 31));
            }
        }
    }
};

template <int DT>
__global__ void __launch_bounds__(kThreads, 5)
pods_sample_policy_kernel(const SampleArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    PolicyCtrl& ctl = *reinterpret_cast<PolicyCtrl*>(smem);
    Policy<DT> w(a, ctl, reinterpret_cast<uint4*>(smem + kPolicyCtrlBytes));
    const int tid = w.tid;
    if (tid == 0) {
        mbar_init(&ctl.full, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < kRedoRows / 32; i += kThreads) ctl.redo[i] = 0;
    __syncthreads();
    w.cl.sync();                                       // every CTA runs before its shared memory is written

    const int64_t n_clusters = gridDim.x / w.CL;
    for (int64_t t0 = blockIdx.x / w.CL; t0 < a.T; t0 += kRedoRows * n_clusters) {
        for (int k = 0; k < kRedoRows; ++k) {
            const int64_t t = t0 + k * n_clusters;
            if (t >= a.T) break;
            if (a.mask != nullptr && a.mask[t] == 0) continue;
            w.template row<false>(t, k);
            fence_async_proxy();                       // the buffer is refilled by bulk copies
            __syncthreads();
        }
        w.cl.sync();                                   // the marks are in place, the same in every CTA
        static_assert(kRedoRows / 32 == kThreads, "a word of marks a thread");
        if (__syncthreads_or(ctl.redo[tid] != 0)) {
            for (int i = 0; i < kRedoRows / 32; ++i) {
                uint32_t bits = ctl.redo[i];
                while (bits) {
                    const int k = 32 * i + __ffs(bits) - 1;
                    bits &= bits - 1;
                    w.template row<true>(t0 + k * n_clusters, 0);
                    fence_async_proxy();
                    __syncthreads();
                }
            }
            __syncthreads();
            ctl.redo[tid] = 0;
        }
        if (t0 + kRedoRows * n_clusters < a.T) w.cl.sync();      // cleared before the next mark
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

constexpr size_t kMaxSmem = 227 * 1024;
constexpr size_t kSegmentBytes = 40 * 1024;            // segments of about this size let five CTAs share an SM

template <typename Kernel>
int launch_rows(Kernel kernel, SampleArgs& a, int esize, size_t ctrl_bytes, cudaStream_t stream) {
    int cl = 1;
    while (cl < kMaxCluster && (size_t)segment_vectors(a.V, esize, cl) * 16 > kSegmentBytes) cl *= 2;
    a.seg = segment_vectors(a.V, esize, cl);
    const size_t smem = ctrl_bytes + (size_t)a.seg * 16;
    if (smem > kMaxSmem) return PODS_ERR_UNSUPPORTED;
    PODS_RETURN_IF_CUDA_ERROR(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    if (cl > 8) PODS_RETURN_IF_CUDA_ERROR(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cl;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)cl, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)(row_clusters(a.T, cl, smem) * cl), 1, 1);
    PODS_RETURN_IF_CUDA_ERROR(cudaLaunchKernelEx(&cfg, kernel, a));
    return PODS_OK;
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
    a.list_cap = kSampleList;
    a.status = status;
    cudaStream_t s = pods_stream(stream);
    if (!top_k_row && !top_p_row && !min_p_row && (top_k <= 0 || top_k >= V) && top_p >= 1.0f && min_p <= 0.0f) {
        if (dtype == PODS_DTYPE_BF16) return launch_rows(pods_sample_policy_kernel<PODS_DTYPE_BF16>, a, esize, kPolicyCtrlBytes, s);
        if (dtype == PODS_DTYPE_F16) return launch_rows(pods_sample_policy_kernel<PODS_DTYPE_F16>, a, esize, kPolicyCtrlBytes, s);
        return launch_rows(pods_sample_policy_kernel<PODS_DTYPE_F32>, a, esize, kPolicyCtrlBytes, s);
    }
    const size_t ctrl = kCtrlBytes + (size_t)a.list_cap * 8;
    if (dtype == PODS_DTYPE_BF16) return launch_rows(pods_sample_kernel<PODS_DTYPE_BF16>, a, esize, ctrl, s);
    if (dtype == PODS_DTYPE_F16) return launch_rows(pods_sample_kernel<PODS_DTYPE_F16>, a, esize, ctrl, s);
    return launch_rows(pods_sample_kernel<PODS_DTYPE_F32>, a, esize, ctrl, s);
}

extern "C" int pods_topk(const void* logits, int64_t ldl, int32_t dtype, int64_t T, int32_t V, int32_t K,
                         float temperature, const uint8_t* mask, int32_t* ids, float* values, float* lse,
                         uint32_t* status, void* stream) {
    int esize = 0;
    const int rc = check_rows(logits, ldl, dtype, T, V, &esize);
    if (rc != PODS_OK) return rc;
    if (K < 1 || K > V || !(temperature > 0.0f && temperature < INFINITY)) return PODS_ERR_INVALID_ARG;
    if (K > PODS_MAX_TOPK) return PODS_ERR_UNSUPPORTED;
    if (T == 0) return PODS_OK;
    if (logits == nullptr || ids == nullptr || values == nullptr) return PODS_ERR_INVALID_ARG;
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
    a.list_cap = 1024;
    while (a.list_cap < 4 * K) a.list_cap *= 2;
    a.status = status;
    cudaStream_t s = pods_stream(stream);
    const size_t ctrl = kCtrlBytes + (size_t)a.list_cap * 8;
    if (dtype == PODS_DTYPE_BF16) return launch_rows(pods_topk_kernel<PODS_DTYPE_BF16>, a, esize, ctrl, s);
    if (dtype == PODS_DTYPE_F16) return launch_rows(pods_topk_kernel<PODS_DTYPE_F16>, a, esize, ctrl, s);
    return launch_rows(pods_topk_kernel<PODS_DTYPE_F32>, a, esize, ctrl, s);
}
