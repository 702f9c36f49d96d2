// pods_distill_chunk: divergence from a teacher's top-K list to the policy's logits, with its gradient.
//
// With z the row, zl its listed logits, the other logits are summed apart: m2 their maximum, S2 = sum exp((z - m2)/tau).
// Then  Z = S2 e^{(m2-zmax)/tau} + sum_listed e^{(z-zmax)/tau},  1 - s = S2 e^{(m2-zmax)/tau} / Z  (no difference is ever
// taken, so a policy that is sure of the list keeps its accuracy), and every id outside the list has the gradient
//   e^{(z_v - m2)/tau} * g ((Q + r) e^{(m2-zmax)/tau} / Z - r / S2),
// one factor for the row.  What concerns the list is fp64: K exponentials a CTA, against V / CL fp32 ones twice.
//
// A cluster of CTAs holds the row in shared memory (row_cluster.cuh): one read and one write per element.  The listed
// logits are taken out first (their slots become -inf), so the sweeps run over the segment without asking about the list:
// maximum, sum, and after one exchange over the cluster the gradient; the listed entries are written over it.  Two kernels:
//   32 MB of logits and more, K <= 128   pods_distill_pipe_kernel: every warp one task, rows overlap, only mbarriers.
//             4096 x 151936 bf16 with K = 64: 549 to 557 us = 4.5 TB/s of one read and one write, 0.69 of the measured copy rate;
//             one exponential an element (the gradient scales what the sum's sweep kept).  Nothing is full (issue slots 53 %):
//             its consumers sweep the stage for the maximum and again for the exponentials, and add to an fp64 sum once a vector,
//             where the kernel of grpo_loss_cluster.cu holds its slice in registers and moves the same bytes at 0.95.
//             512 x 151936 fp32 with K = 128: 144 to 148 us = 4.2 TB/s, 0.65, 9 % of it idle SMs.  1024 x 151936 with K = 64:
//             bf16 153 us, fp16, which keeps nothing and takes two exponentials an element, 169.  600 x 50257 fp16, the loss
//             alone: 33 us = 1.8 TB/s, six rows a cluster: filling and draining, and the launches around.
//   all others   pods_distill_kernel: every warp does everything, a dozen CTA barriers a row, which bound it, and two
//             exponentials an element.  1024 x 151936 bf16 with K = 200: 199 us = 3.1 TB/s, K = 1024: 284; 37 rows of 1024:
//             13 us, four dependent launches of 2 to 5 us.

#include <float.h>
#include <stddef.h>

#include "grpo_loss_common.cuh"
#include "row_cluster.cuh"

using namespace pods_row;

namespace {

constexpr int W = 8;
constexpr int kThreads = W * 32;

struct DistillArgs {
    const void* logits;
    int64_t ldl;
    const int32_t* ids;
    const float* values;
    int64_t ldk;
    int K;
    const float* teacher_lse;
    const double* seq_weight;
    const int64_t* cu_seqlens;
    int64_t M, row0;
    const uint8_t* mask;
    int64_t T;
    int V, seg;
    float temperature;
    int rest;
    float grad_scale;
    float* kl;
    void* dlogits;
    int64_t ldd;
    double* row_loss;
    struct RowPrep* prep;                              // workspace: what a row needs besides its logits (many rows)
    uint32_t* status;
};

struct alignas(16) RowPrep {
    double w;                                          // mask_t w_i
    double L, Q, H;                                    // the list's log-normaliser, sum q, sum q log q
};

struct Xch {
    double s_out, s_in, a;                             // sums outside and inside the list, sum of q z / tau
    float m_out, m_in;
};

struct Ctrl {
    unsigned long long full;
    Xch x[2][kMaxCluster];
    double dpart[W][3];
    float fpart[W];
    double weight;                                     // mask_t w_i of the row
    double coef, p_scale, g;                           // of the row's gradient, see below
    float m2, zmax;
    int bad;
};
constexpr int kCtrlBytes = (sizeof(Ctrl) + 127) & ~127;

// N sums over the CTA in one go; every thread gets them.
template <int N>
__device__ __forceinline__ void block_sums(double (&v)[N], double (*part)[3]) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) v[n] += __shfl_xor_sync(PODS_FULL_MASK, v[n], d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < N; ++n) part[threadIdx.x >> 5][n] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        v[n] = part[0][n];
#pragma unroll
        for (int w = 1; w < W; ++w) v[n] += part[w][n];
    }
}

// Rollout of packed row r by a whole warp: 32 probes a step.
__device__ __forceinline__ int64_t find_rollout_warp(const int64_t* cu, int64_t M, int64_t r) {
    const int lane = threadIdx.x & 31;
    int64_t lo = 0, hi = M;                            // cu[lo] <= r, answer in [lo, hi)
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + 31) / 32;
        const int64_t at = lo + lane * step;
        const bool le = at < hi && cu[at] <= r;        // a prefix of the lanes, lane 0 always
        const int n = __popc(__ballot_sync(PODS_FULL_MASK, le));
        lo += (int64_t)(n > 0 ? n - 1 : 0) * step;
        hi = hi < lo + step ? hi : lo + step;
    }
    return lo;
}

// KP: list entries a thread holds at most, so K <= KP * kThreads.
template <int DT, int KP>
__global__ void __launch_bounds__(kThreads, KP == 1 ? 4 : 2)
pods_distill_kernel(const DistillArgs a) {
    using El = Elem<DT>;
    using raw = typename El::raw;
    constexpr int E = El::E;
    extern __shared__ __align__(128) unsigned char smem[];
    Ctrl& c = *reinterpret_cast<Ctrl*>(smem);
    uint4* const buf = reinterpret_cast<uint4*>(smem + kCtrlBytes);
    raw* const elems = reinterpret_cast<raw*>(buf);
    cg::cluster_group cl = cg::this_cluster();
    const int CL = (int)cl.num_blocks(), rank = (int)cl.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        mbar_init(&c.full, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    bool started = false;

    const double tau_inv = 1.0 / (double)a.temperature;
    const float cexp = (float)(1.4426950408889634 * tau_inv);
    const int64_t n_clusters = gridDim.x / CL;
    uint32_t phase = 0;
    int parity = 0;
    for (int64_t t = blockIdx.x / CL; t < a.T; t += n_clusters) {
        const Segment s = make_segment<DT>(a.logits, a.ldl, t, a.V, rank, a.seg);
        const bool masked = a.mask != nullptr && a.mask[t] == 0;
        if (!masked) {
            if (tid == 0) start_load<DT>(s, a.V, buf, &c.full);
            if (!started) { cl.sync(); started = true; }       // every CTA runs before its shared memory is written
            if (warp == 1) {
                const int64_t i = find_rollout_warp(a.cu_seqlens, a.M, a.row0 + t);
                if (lane == 0) c.weight = a.seq_weight[i];
            }
        } else if (tid == 0) {
            c.weight = 0.0;
        }

        // ---- the teacher's list: every CTA holds all of it ------------------------------------------------------
        int id[KP];
        float y[KP];
        double q[KP];
        double Q = 0.0, H = 0.0, L = 0.0;              // sum q, sum q log q, log-normaliser
        bool odd = false;                              // an id out of range
        if (!masked) {
            const int32_t* ids = a.ids + t * a.ldk;
            const float* vals = a.values + t * a.ldk;
            float ymax = -INFINITY;
#pragma unroll
            for (int k = 0; k < KP; ++k) {
                const int j = tid + k * kThreads;
                id[k] = -1;
                y[k] = -INFINITY;
                if (j < a.K) {
                    const int v = ids[j];
                    if (v >= 0 && v < a.V) {
                        id[k] = v;
                        y[k] = vals[j];
                        ymax = max_nan(ymax, y[k]);
                    } else if (v != -1) {
                        odd = true;
                    }
                }
            }
            if (a.teacher_lse != nullptr) {
                L = (double)a.teacher_lse[t];
            } else {
                ymax = block_reduce<W>(ymax, c.fpart, MaxNan());
                const double ref = ymax == -INFINITY ? 0.0 : (double)ymax;     // no entry at all: every q is 0
                double sum[1] = {0.0};
#pragma unroll
                for (int k = 0; k < KP; ++k)
                    if (id[k] >= 0) sum[0] += exp(((double)y[k] - ref) * tau_inv);
                block_sums(sum, c.dpart);
                L = ref * tau_inv + (sum[0] > 0.0 || sum[0] != sum[0] ? log(sum[0]) : 0.0);
            }
            double two[2] = {0.0, 0.0};
#pragma unroll
            for (int k = 0; k < KP; ++k) {
                q[k] = 0.0;
                if (id[k] >= 0) {
                    const double lq = (double)y[k] * tau_inv - L;
                    q[k] = exp(lq);
                    two[0] += q[k];
                    if (q[k] != 0.0) two[1] += q[k] * lq;
                }
            }
            block_sums(two, c.dpart);
            Q = two[0];
            H = two[1];
            if (!mbar_wait(&c.full, phase, kSpinLimit) && lane == 0) pods_raise(a.status, PODS_STATUS_TIMEOUT);
            phase ^= 1u;
        }
        __syncthreads();
        const double w = c.weight;
        if (odd && rank == 0 && w != 0.0) pods_raise(a.status, PODS_STATUS_TOKEN_RANGE);

        // the part of the gradient row that is mine
        const int id_lo = max(0, s.id0), id_hi = min(a.V, s.id0 + s.cnt * E);
        raw* const drow = a.dlogits != nullptr ? static_cast<raw*>(a.dlogits) + t * a.ldd : nullptr;
        const int dlead = (int)((reinterpret_cast<uintptr_t>(drow) & 15) / sizeof(raw));
        // gradient vectors (16-byte boundaries of dlogits) whole inside [id_lo, id_hi): ids v * E - dlead ...
        const int v_lo = (id_lo + dlead + E - 1) / E, v_hi = max(v_lo, (id_hi + dlead) / E);

        if (w == 0.0) {                                // masked row, or one of an empty rollout
            if (drow != nullptr && id_lo < id_hi) {
                const raw zero = 0;
                uint4* const dvec = reinterpret_cast<uint4*>(drow - dlead);
                for (int v = v_lo + tid; v < v_hi; v += kThreads) dvec[v] = make_uint4(0u, 0u, 0u, 0u);
                for (int i = id_lo + tid; i < min(id_hi, v_lo * E - dlead); i += kThreads) drow[i] = zero;
                for (int i = max(id_lo, v_hi * E - dlead) + tid; i < id_hi; i += kThreads) drow[i] = zero;
            }
            if (rank == 0 && tid == 0) {
                a.kl[t] = 0.0f;
                a.row_loss[t] = 0.0;
            }
            fence_async_proxy();
            __syncthreads();
            continue;
        }

        // ---- the listed logits of my segment leave it -----------------------------------------------------------
        float z[KP];
        int slot[KP];                                // element of my segment, -1 where the entry is not mine
#pragma unroll
        for (int k = 0; k < KP; ++k) {
            const int at = id[k] - s.id0;
            slot[k] = id[k] >= 0 && at >= 0 && at < s.cnt * E ? at : -1;
            z[k] = slot[k] >= 0 ? El::to_float(elems[slot[k]]) : -INFINITY;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < KP; ++k)
            if (slot[k] >= 0) elems[slot[k]] = (raw)(tid + k * kThreads);      // one entry of an id stays visible
        __syncthreads();
        int twice = 0;
#pragma unroll
        for (int k = 0; k < KP; ++k)
            if (slot[k] >= 0 && elems[slot[k]] != (raw)(tid + k * kThreads)) twice = 1;
        twice = __syncthreads_or(twice);
        double qsum[KP];                             // teacher mass of the entry's id
        unsigned first = 0;                            // bit k: the entry speaks for its id
#pragma unroll
        for (int k = 0; k < KP; ++k) {
            qsum[k] = q[k];
            if (slot[k] >= 0) {
                elems[slot[k]] = El::kNegInf;
                first |= 1u << k;
            }
        }
        if (twice) {
            // an id in several entries: the first speaks for it, with their mass added in list order
            const int32_t* ids = a.ids + t * a.ldk;
            const float* vals = a.values + t * a.ldk;
#pragma unroll
            for (int k = 0; k < KP; ++k)
                if (slot[k] >= 0) {
                    const int j = tid + k * kThreads;
                    for (int o = 0; o < a.K; ++o)
                        if (o != j && ids[o] == id[k]) {
                            if (o < j) first &= ~(1u << k);
                            else qsum[k] += exp((double)vals[o] * tau_inv - L);
                        }
                }
        }
        __syncthreads();

        // ---- maxima and sums -------------------------------------------------------------------------------------
        float m_out = -INFINITY, m_in = -INFINITY;
        for (int j = tid; j < s.cnt; j += kThreads) m_out = max_nan(m_out, El::vec_max(buf[j]));
#pragma unroll
        for (int k = 0; k < KP; ++k)
            if (first >> k & 1u) m_in = max_nan(m_in, z[k]);
        Xch mine;                                      // the last thing a row asks of its peers is the exchange's barrier
        mine.m_out = block_reduce<W>(m_out, c.fpart, MaxNan());
        mine.m_in = block_reduce<W>(m_in, c.fpart, MaxNan());
        double three[3] = {0.0, 0.0, 0.0};
        {
            const ExpRef ref(mine.m_out, cexp);
            for (int j = tid; j < s.cnt; j += kThreads) {
                float x[E];
                El::unpack(buf[j], x);
                ref.exps(x);
                three[0] += (double)vec_add(x);
            }
        }
#pragma unroll
        for (int k = 0; k < KP; ++k) {
            if (first >> k & 1u)
                if (mine.m_in > -INFINITY) three[1] += exp(((double)z[k] - (double)mine.m_in) * tau_inv);
            if (slot[k] >= 0 && q[k] != 0.0) three[2] += q[k] * ((double)z[k] * tau_inv);
        }
        block_sums(three, c.dpart);
        mine.s_out = three[0];
        mine.s_in = three[1];
        mine.a = three[2];
        Xch* const xs = c.x[parity];
        parity ^= 1;
        if (tid < CL) *cl.map_shared_rank(xs + rank, tid) = mine;
        cl.sync();

        // ---- the row's scalars: one CTA a lane of the first warp ---------------------------------------------------
        if (warp == 0) {
            Xch x = {0.0, 0.0, 0.0, -INFINITY, -INFINITY};
            if (lane < CL) x = xs[lane];
            float m2 = x.m_out, m1 = x.m_in;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                m2 = max_nan(m2, __shfl_xor_sync(PODS_FULL_MASK, m2, d));
                m1 = max_nan(m1, __shfl_xor_sync(PODS_FULL_MASK, m1, d));
            }
            const float zmax = max_nan(m1, m2);
            const bool bad = !(fabsf(zmax) < INFINITY);
            double S2 = 0.0, S1 = 0.0, A = x.a;
            if (!bad) {
                if (x.m_out > -INFINITY) S2 = x.s_out * ExpRef(x.m_out, cexp).scale_to(m2, cexp);
                if (x.m_in > -INFINITY) S1 = x.s_in * exp(((double)x.m_in - (double)zmax) * tau_inv);
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                S2 += __shfl_xor_sync(PODS_FULL_MASK, S2, d);
                S1 += __shfl_xor_sync(PODS_FULL_MASK, S1, d);
                A += __shfl_xor_sync(PODS_FULL_MASK, A, d);
            }
            const double part = m2 > -INFINITY ? exp(((double)m2 - (double)zmax) * tau_inv) : 0.0;
            const double Z = S2 * part + S1;
            const double r = a.rest && m2 > -INFINITY ? fmax(0.0, 1.0 - Q) : 0.0;
            const double g = (double)a.grad_scale * w * tau_inv;
            if (lane == 0) {
                const double f = bad ? (double)NAN : (Q + r) / Z;
                // relative to 2^-R of the sweep's reference, as the exponentials of the gradient are
                const double per_e = ExpRef(m2, cexp).scale_to(m2 > -INFINITY ? m2 : 0.0f, cexp);
                c.coef = g * (f * part - (r > 0.0 ? r / S2 : 0.0)) * per_e;
                c.p_scale = f;
                c.g = g;
                c.m2 = m2;
                c.zmax = zmax;
                c.bad = bad;
            }
            __syncwarp();
            if (rank == 0 && lane == 0) {              // nobody waits for these
                double kl = NAN;
                if (!bad) {
                    const double lz = log(Z);
                    kl = H - A + Q * ((double)zmax * tau_inv + lz);
                    if (r > 0.0) kl += r * (log(r) - (((double)m2 - (double)zmax) * tau_inv + log(S2) - lz));
                } else {
                    pods_raise(a.status, zmax == -INFINITY ? PODS_STATUS_EMPTY_ROW : PODS_STATUS_NONFINITE_LOGIT);
                }
                a.kl[t] = (float)kl;
                a.row_loss[t] = w * kl;
            }
        }
        __syncthreads();

        // ---- the gradient ------------------------------------------------------------------------------------------
        if (drow != nullptr && id_lo < id_hi) {
            const ExpRef ref(c.m2, cexp);
            const float coef = (float)c.coef;
            uint4* const dvec = reinterpret_cast<uint4*>(drow - dlead);
            const int shift = v_lo * E - dlead - s.id0 - (v_lo * E - dlead - s.id0) / E * E;
            if (shift == 0) {
                const int to_buf = -(dlead + s.id0) / E;                       // gradient vector v is vector v + to_buf here
                for (int v = v_lo + tid; v < v_hi; v += kThreads)
                    if (PODS_INDEX_OK(v + to_buf, s.cnt, a.status)) {
                        float x[E];
                        El::unpack(buf[v + to_buf], x);
                        ref.exps(x);
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] *= coef;
                        dvec[v] = El::pack(x);
                    }
            } else {
                for (int v = v_lo + tid; v < v_hi; v += kThreads) {
                    const int at = v * E - dlead - s.id0;
                    if (PODS_INDEX_OK(at, s.cnt * E - E + 1, a.status)) {
                        float x[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] = El::to_float(elems[at + e]);
                        ref.exps(x);
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] *= coef;
                        dvec[v] = El::pack(x);
                    }
                }
            }
            for (int i = id_lo + tid; i < min(id_hi, v_lo * E - dlead); i += kThreads)
                drow[i] = El::from_float(coef * ref.exp1(El::to_float(elems[i - s.id0]), cexp));
            for (int i = max(id_lo, v_hi * E - dlead) + tid; i < id_hi; i += kThreads)
                drow[i] = El::from_float(coef * ref.exp1(El::to_float(elems[i - s.id0]), cexp));
            __syncthreads();
#pragma unroll
            for (int k = 0; k < KP; ++k)
                if (first >> k & 1u) {
                    const double p = exp(((double)z[k] - (double)c.zmax) * tau_inv) * c.p_scale;      // (Q + r) p
                    drow[id[k]] = El::from_float((float)(c.g * (p - qsum[k])));
                }
        }
        fence_async_proxy();                           // the buffer is refilled by bulk copies
        __syncthreads();
    }
}

// One warp a row: its weight and what the teacher's list says by itself.
__global__ void __launch_bounds__(256)
distill_prep_kernel(const DistillArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (t >= a.T) return;
    RowPrep p = {0.0, 0.0, 0.0, 0.0};
    if (a.mask == nullptr || a.mask[t] != 0) {
        p.w = a.seq_weight[find_rollout_warp(a.cu_seqlens, a.M, a.row0 + t)];
        const double tau_inv = 1.0 / (double)a.temperature;
        const int32_t* const ids = a.ids + t * a.ldk;
        const float* const vals = a.values + t * a.ldk;
        bool odd = false;
        float ymax = -INFINITY;
        for (int j = lane; j < a.K; j += 32) {
            const int id = ids[j];
            if (id >= 0 && id < a.V) ymax = max_nan(ymax, vals[j]);
            else odd |= id != -1;
        }
        if (__any_sync(PODS_FULL_MASK, odd) && lane == 0 && p.w != 0.0) pods_raise(a.status, PODS_STATUS_TOKEN_RANGE);
        if (a.teacher_lse != nullptr) {
            p.L = (double)a.teacher_lse[t];
        } else {
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) ymax = max_nan(ymax, __shfl_xor_sync(PODS_FULL_MASK, ymax, d));
            const double ref = ymax == -INFINITY ? 0.0 : (double)ymax;         // no entry at all: every q is 0
            double sum = 0.0;
            for (int j = lane; j < a.K; j += 32)
                if (ids[j] >= 0 && ids[j] < a.V) sum += exp(((double)vals[j] - ref) * tau_inv);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(PODS_FULL_MASK, sum, d);
            p.L = ref * tau_inv + (sum > 0.0 || sum != sum ? log(sum) : 0.0);
        }
        for (int j = lane; j < a.K; j += 32)
            if (ids[j] >= 0 && ids[j] < a.V) {
                const double lq = (double)vals[j] * tau_inv - p.L, q = exp(lq);
                p.Q += q;
                if (q != 0.0) p.H += q * lq;
            }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            p.Q += __shfl_xor_sync(PODS_FULL_MASK, p.Q, d);
            p.H += __shfl_xor_sync(PODS_FULL_MASK, p.H, d);
        }
    }
    if (lane == 0) a.prep[t] = p;
}

// ---- many rows: a pipeline ------------------------------------------------------------------------------------------------
// The same arithmetic where rows come by the hundred and every SM holds two CTAs (lists of up to kPipeK entries): warps with one
// task each that meet only at mbarriers.  With every warp doing everything and a dozen CTA barriers a row, 4096 rows of 151936
// took 731 us, half the time waiting at barriers.
//   producer  one thread: the row's segment into one of three stages, as soon as the consumers have left it
//   list      one warp: the listed logits out of the stage (their slots become -inf), their sums to every CTA of the cluster;
//            it works a row ahead of the others
//   consumer  eight warps: front(i) maximum and sum of their slice, sent to every CTA; back(i - 1) the gradient of the row
//            before, whose factors have had a whole sweep to arrive, and the listed entries of their slice
//   exchange  one warp: all parts of a row into the row's factors, loss and status
// What the list says by itself (its normaliser, Q, sum q log q) and the row's weight are made beforehand, a warp a row: done by
// the list warp of each CTA they took 7200 of a row's 9900 cycles, and every other warp waited for that one.
// Parts and factors have four slots each.  A part of row i is sent after its sender has seen the factors of row i - 2, which
// took every CTA's parts of row i - 2, which were sent after the factors of row i - 4 were made: the slot of row i - 4 is free.
// PW: consumer warps, 8 where two CTAs share an SM, 16 where one has it alone.
constexpr int kStages = 3, kRing = 4;
// Entries of a list: four a lane.  Pipeline against the other kernel at K = 128: 1024 rows of 151936 bf16 182 : 195 us, 2048 of
// 32000 88 : 98, 512 fp32 rows of 151936 142 : 188.  With room for 256 (eight a lane) K = 129 took 200 : 196, 95 : 97 and 144 : 187 us,
// K = 256 202 : 201, 126 : 101 and 150 : 190, and K = 64, which every list would pay, 166 instead of 153 (bf16, 1024 rows).
constexpr int kPipeK = 128;

struct PipePart {                             // of one consumer warp
    double s;
    float m;
    int pad;
};
struct PipeList {                             // of one CTA's part of the list
    double s, a;
    float m;
    int pad;
    double unused;
};
struct Entry {                                // a listed id of my segment
    double q;                                 // its teacher mass
    float z;
    int id;
};
struct Factors {
    double p_scale, g;                        // listed ids: g (p_scale e^((z - zmax)/tau) - q)
    float coef, m2, zmax;                     // the others: coef 2^(x c - R(m2))
    int mode;                                 // 0: a row of zeros
};
struct PipeCtrl {
    unsigned long long full[kStages], done[kStages];   // the stage is loaded; its consumers have left it
    unsigned long long listed[kRing];         // the listed logits are out of the stage
    unsigned long long parts[kRing];          // all parts of the cluster have arrived
    unsigned long long ready[kRing];          // the factors are there
    Factors f[kRing];
    int n_entry[kRing];
    alignas(16) PipeList list[kRing][kMaxCluster];
    alignas(16) Entry entry[1];               // [kRing][K], then PipePart [kRing][CL PW]
};
__host__ __device__ constexpr int pipe_part_offset(int K) { return (int)offsetof(PipeCtrl, entry) + kRing * K * (int)sizeof(Entry); }
__host__ __device__ constexpr int pipe_ctrl_bytes(int cl, int K, int pw) {
    return (pipe_part_offset(K) + kRing * cl * pw * (int)sizeof(PipePart) + 127) & ~127;
}

extern __shared__ __align__(128) unsigned char smem_[];

template <int DT, int PW>
__global__ void __launch_bounds__((PW + 3) * 32, 16 / PW)
pods_distill_pipe_kernel(const DistillArgs a) {
    using El = Elem<DT>;
    using raw = typename El::raw;
    constexpr int E = El::E;
    PipeCtrl& c = *reinterpret_cast<PipeCtrl*>(smem_);
    cg::cluster_group cl = cg::this_cluster();
    const int CL = (int)cl.num_blocks(), rank = (int)cl.block_rank();
    PipePart* const part = reinterpret_cast<PipePart*>(smem_ + pipe_part_offset(a.K));
    uint4* const stages = reinterpret_cast<uint4*>(smem_ + pipe_ctrl_bytes(CL, a.K, PW));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t n_clusters = gridDim.x / CL, first = blockIdx.x / CL;
    const int n_rows = first < a.T ? (int)((a.T - first + n_clusters - 1) / n_clusters) : 0;
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&c.full[i], 1);
            mbar_init(&c.done[i], PW);
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&c.listed[i], 1);
            mbar_init(&c.parts[i], 1);
            mbar_init(&c.ready[i], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    cl.sync();                                         // every CTA's barriers are there before anyone reaches for them

    const double tau_inv = 1.0 / (double)a.temperature;
    const float cexp = (float)(1.4426950408889634 * tau_inv);
    bool late = false;                                 // a wait ran out: no further one is worth its time
    auto spins = [&]() { return late ? 1u : kSpinLimit; };
    auto wait_ready = [&](int i) {
        if (!mbar_wait(&c.ready[i % kRing], (uint32_t)((i / kRing) & 1), spins())) late = true;
    };

    if (warp == PW) {
        // ---- producer ----
        if (lane == 0) {
            StageRing ring;
            for (int i = 0; i < n_rows; ++i) {
                const int st = ring.st;
                if (i >= kStages && !mbar_wait(&c.done[st], ring.parity ^ 1u, spins())) late = true;
                const Segment s = make_segment<DT>(a.logits, a.ldl, first + i * n_clusters, a.V, rank, a.seg);
                uint4* const buf = stages + (size_t)st * a.seg;
                fill_edges<DT>(s, a.V, buf);
                fence_async_proxy();                   // edges of an earlier row may lie where this row's copy goes
                start_copy(s, buf, &c.full[st]);
                ring.next(kStages);
            }
            // every copy has landed before the CTA ends, also one that a consumer gave up on
            for (int k = 0; k < kStages && k < n_rows; ++k) {
                ring.st = ring.st == 0 ? kStages - 1 : ring.st - 1;           // from the last row back
                if (ring.st == kStages - 1) ring.parity ^= 1u;
                if (!mbar_wait(&c.full[ring.st], ring.parity, kSpinLimit)) late = true;
            }
        }
    } else if (warp == PW + 1) {
        // ---- list ----
        constexpr int KP = kPipeK / 32;
        int id_next[KP];
        float y_next[KP];
        double L_next = 0.0;
        auto fetch = [&](int64_t t) {
#pragma unroll
            for (int k = 0; k < KP; ++k) {
                const int j = lane + 32 * k;
                id_next[k] = j < a.K ? a.ids[t * a.ldk + j] : -1;
                y_next[k] = j < a.K ? a.values[t * a.ldk + j] : -INFINITY;
            }
            L_next = a.prep[t].L;
        };
        if (n_rows > 0) fetch(first);
        StageRing ring;
        for (int i = 0; i < n_rows; ++i, ring.next(kStages)) {
            const int st = ring.st, slot = i % kRing;
            const int64_t t = first + i * n_clusters;
            const Segment s = make_segment<DT>(a.logits, a.ldl, t, a.V, rank, a.seg);
            raw* const elems = reinterpret_cast<raw*>(stages + (size_t)st * a.seg);
            Entry* const entry = c.entry + slot * a.K;
            const double L = L_next;
            const int id_lo = max(0, s.id0), id_hi = min(a.V, s.id0 + s.cnt * E);
            int id[KP];
            float y[KP], z[KP];
#pragma unroll
            for (int k = 0; k < KP; ++k) {
                id[k] = id_next[k];
                y[k] = y_next[k];
            }
            if (i + 1 < n_rows) fetch(t + n_clusters);
            if (!mbar_wait(&c.full[st], ring.parity, spins())) late = true;
            float m_in = -INFINITY;
#pragma unroll
            for (int k = 0; k < KP; ++k) {
                if (id[k] < id_lo || id[k] >= id_hi) id[k] = -1;
                z[k] = id[k] >= 0 ? El::to_float(elems[id[k] - s.id0]) : -INFINITY;
                m_in = max_nan(m_in, z[k]);
            }
            __syncwarp();
#pragma unroll
            for (int k = 0; k < KP; ++k)
                if (id[k] >= 0) elems[id[k] - s.id0] = (raw)(lane + 32 * k);   // one entry of an id stays visible
            __syncwarp();
            bool twice = false;
#pragma unroll
            for (int k = 0; k < KP; ++k) twice |= id[k] >= 0 && elems[id[k] - s.id0] != (raw)(lane + 32 * k);
            twice = __any_sync(PODS_FULL_MASK, twice);                         // (and everyone has looked)
#pragma unroll
            for (int k = 0; k < KP; ++k)
                if (id[k] >= 0) elems[id[k] - s.id0] = El::kNegInf;
            fence_async_proxy();                       // what was written to the stage lies where a later copy goes
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) m_in = max_nan(m_in, __shfl_xor_sync(PODS_FULL_MASK, m_in, d));
            // entry slots of row i - 4 were read by back(i - 4), before the parts of row i - 2 that made its factors
            if (i >= 2) wait_ready(i - 2);
            // the entries together, the teacher's value in place of its mass
            int n = 0;
#pragma unroll
            for (int k = 0; k < KP; ++k) {
                const uint32_t b = __ballot_sync(PODS_FULL_MASK, id[k] >= 0);
                if (id[k] >= 0) {
                    Entry e;
                    e.q = (double)y[k];
                    e.z = z[k];
                    e.id = id[k];
                    entry[n + __popc(b & ((1u << lane) - 1u))] = e;
                }
                n += __popc(b);
            }
            __syncwarp();
            double A = 0.0, sum = 0.0;
            for (int k = lane; k < n; k += 32) {
                const Entry e = entry[k];
                const double lq = e.q * tau_inv - L, q = exp(lq);
                if (q != 0.0) A += q * ((double)e.z * tau_inv);
                if (m_in > -INFINITY && !twice) sum += exp64(((double)e.z - (double)m_in) * tau_inv);
                entry[k].q = q;
            }
            if (twice) {
                // an id in several entries (kept in list order): the first speaks for it, with their mass added; the others are
                // taken off the list of entries
                __syncwarp();
                if (lane == 0) {
                    int kept = 0;
                    for (int k = 0; k < n; ++k) {
                        const Entry e = entry[k];
                        int o = 0;
                        while (o < kept && entry[o].id != e.id) ++o;
                        if (o < kept) {
                            entry[o].q += e.q;
                        } else {
                            entry[kept++] = e;
                            if (m_in > -INFINITY) sum += exp64(((double)e.z - (double)m_in) * tau_inv);
                        }
                    }
                    n = kept;
                }
                n = __shfl_sync(PODS_FULL_MASK, n, 0);
            }
            if (lane == 0) c.n_entry[slot] = n;
            __syncwarp();
            if (lane == 0) arrive_local(&c.listed[slot]);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                A += __shfl_xor_sync(PODS_FULL_MASK, A, d);
                sum += __shfl_xor_sync(PODS_FULL_MASK, sum, d);
            }
            if (lane < CL) {
                const uint32_t to = mapa(&c.list[slot][rank], lane), bar = mapa(&c.parts[slot], lane);
                store_async(to, bar, sum, (unsigned long long)__double_as_longlong(A));
                store_async(to + 16, bar, __longlong_as_double((long long)__float_as_uint(m_in)), 0ull);
            }
        }
    } else if (warp == PW + 2) {
        // ---- exchange ----
        RowPrep next = {0.0, 0.0, 0.0, 0.0};
        if (n_rows > 0) next = a.prep[first];
        for (int i = 0; i < n_rows; ++i) {
            const int slot = i % kRing;
            const int64_t t = first + i * n_clusters;
            if (lane == 0) mbar_expect_tx(&c.parts[slot], (uint32_t)(CL * (PW * 16 + 32)));
            const double w = next.w, Q = next.Q, H = next.H;
            if (i + 1 < n_rows) next = a.prep[t + n_clusters];
            if (!wait_cluster(&c.parts[slot], (uint32_t)((i / kRing) & 1), spins())) late = true;
            constexpr int N = kMaxCluster * PW / 32;
            double v[N], S2 = 0.0, S1 = 0.0, A = 0.0;
            float pm[N], m2 = -INFINITY, m1 = -INFINITY, lm = -INFINITY;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = 0.0;
                pm[k] = -INFINITY;
                if (lane + 32 * k < CL * PW) {
                    const PipePart p = part[slot * CL * PW + lane + 32 * k];
                    v[k] = p.s;
                    pm[k] = p.m;
                }
                m2 = max_nan(m2, pm[k]);
            }
            if (lane < CL) {
                const PipeList l = c.list[slot][lane];
                S1 = l.s;
                A = l.a;
                m1 = lm = l.m;
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                m2 = max_nan(m2, __shfl_xor_sync(PODS_FULL_MASK, m2, d));
                m1 = max_nan(m1, __shfl_xor_sync(PODS_FULL_MASK, m1, d));
            }
            const float zmax = max_nan(m1, m2);
            const bool bad = !(fabsf(zmax) < INFINITY);
            const PartRef top(m2, cexp);
            if (!bad) {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (v[k] > 0.0) S2 += v[k] * PartRef(pm[k], cexp).scale_to(top);
                S1 = lm > -INFINITY ? S1 * exp64(((double)lm - (double)zmax) * tau_inv) : 0.0;
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                S2 += __shfl_xor_sync(PODS_FULL_MASK, S2, d);
                S1 += __shfl_xor_sync(PODS_FULL_MASK, S1, d);
                A += __shfl_xor_sync(PODS_FULL_MASK, A, d);
            }
            // the reference's weight over e^(zmax / tau), and its logarithm
            const double lpart = top.far ? ((double)m2 - (double)zmax) * (double)cexp * kLn2 : ((double)top.R - (double)zmax * (double)cexp) * kLn2;
            const double pw = m2 > -INFINITY ? exp64(lpart) : 0.0;
            const double Z = S2 * pw + S1;
            const double r = a.rest && m2 > -INFINITY ? fmax(0.0, 1.0 - Q) : 0.0;
            const double g = (double)a.grad_scale * w * tau_inv;
            if (lane == 0) {
                Factors f;
                f.p_scale = bad ? (double)NAN : (Q + r) / Z;
                f.g = g;
                f.coef = (float)(g * (f.p_scale * pw - (r > 0.0 ? r / S2 : 0.0)));
                f.m2 = m2;
                f.zmax = zmax;
                f.mode = w != 0.0;
                c.f[slot] = f;
                arrive_local(&c.ready[slot]);
                if (rank == 0) {                       // nobody waits for these
                    double kl = 0.0;
                    if (w != 0.0) {
                        kl = NAN;
                        if (!bad) {
                            const double lz = log(Z);
                            kl = H - A + Q * ((double)zmax * tau_inv + lz);
                            if (r > 0.0) kl += r * (log(r) - (lpart + log(S2) - lz));
                        } else {
                            pods_raise(a.status, zmax == -INFINITY ? PODS_STATUS_EMPTY_ROW : PODS_STATUS_NONFINITE_LOGIT);
                        }
                    }
                    a.kl[t] = (float)kl;
                    a.row_loss[t] = w != 0.0 ? w * kl : 0.0;
                }
            }
            __syncwarp();
        }
    } else {
        // ---- consumers ----
        // Where the gradient's vectors lie on the logits' (shift 0) and the exponents are of ordinary size, the sweep of front()
        // serves back() too: an fp32 row keeps e in the stage, a bf16 row bf16(e), which back() scales with two-term bf16
        // factors.  In bf16 that is a second rounding of the ids outside the list, half a step each time, as in
        // grpo_loss_chunk's gradient; it saves the exponentials' second pass, which with the first fills half of the
        // special-function pipe (4096 x 151936 bf16: 731 us without, with the preparation apart 564).  fp16 could not hold e.
        constexpr bool kKeep = DT != PODS_DTYPE_F16;
        struct Slice { float R; bool kept; };
        auto aligned = [&](const Segment& s, int64_t t) {
            const int dlead = (int)((reinterpret_cast<uintptr_t>(static_cast<raw*>(a.dlogits) + t * a.ldd) & 15) / sizeof(raw));
            return ((s.id0 + dlead) % E) == 0;
        };
        auto back = [&](int i, int st, const Slice& slice) {
            const int slot = i % kRing;
            const int64_t t = first + i * n_clusters;
            wait_ready(i);
            if (a.dlogits != nullptr) {
                const Segment s = make_segment<DT>(a.logits, a.ldl, t, a.V, rank, a.seg);
                const uint4* const buf = stages + (size_t)st * a.seg;
                const raw* const elems = reinterpret_cast<const raw*>(buf);
                const Factors f = c.f[slot];
                raw* const drow = static_cast<raw*>(a.dlogits) + t * a.ldd;
                const int share = (s.cnt + PW - 1) / PW, lo = min(s.cnt, warp * share), hi = min(s.cnt, lo + share);
                const PartRef ref(f.m2, cexp);
                // what the slice kept is relative to its own reference
                const float to_ref = !(kKeep && slice.kept) ? 1.0f
                                     : ref.far ? (float)exp64(((double)slice.R - (double)f.m2 * (double)cexp) * kLn2)
                                               : pow2_any(slice.R - ref.R);
                // element k of the segment, alone
                auto one = [&](int k) {
                    if (f.mode == 0) return (raw)0;
                    const float x = El::to_float(elems[k]);
                    return El::from_float(f.coef * (kKeep && slice.kept ? x * to_ref : (float)ref.exp1(x)));
                };
                if (aligned(s, t)) {
                    uint4* const dvec = reinterpret_cast<uint4*>(drow + s.id0);
                    const unsigned long long coef2 = pack2(f.coef, f.coef);
                    const int whole_lo = max(lo, s.full0), whole_hi = min(hi, s.full1);
                    if (f.mode == 0) {
                        for (int j = whole_lo + lane; j < whole_hi; j += 32) dvec[j] = make_uint4(0u, 0u, 0u, 0u);
                    } else if (kKeep && slice.kept) {
                        const float coef = f.coef * to_ref;
                        if constexpr (DT == PODS_DTYPE_F32) {
                            const unsigned long long c2 = pack2(coef, coef);
#pragma unroll 4
                            for (int j = whole_lo + lane; j < whole_hi; j += 32) {
                                float x[E];
                                El::unpack(buf[j], x);
#pragma unroll
                                for (int e = 0; e < E; e += 2) unpack2(mul2(pack2(x[e], x[e + 1]), c2), x[e], x[e + 1]);
                                dvec[j] = El::pack(x);
                            }
                        } else {
                            const uint16_t hi16 = pods_loss::to_bf16_bits(coef);
                            const uint16_t lo16 = pods_loss::to_bf16_bits(coef - __uint_as_float((uint32_t)hi16 << 16));
                            const uint32_t c_hi = (uint32_t)hi16 * 0x10001u, c_lo = (uint32_t)lo16 * 0x10001u;
#pragma unroll 4
                            for (int j = whole_lo + lane; j < whole_hi; j += 32) {
                                uint4 q = buf[j];
                                pods_loss::scale_vec(q, c_hi, c_lo);
                                dvec[j] = q;
                            }
                        }
                    } else {
#pragma unroll 2
                        for (int j = whole_lo + lane; j < whole_hi; j += 32) {
                            float x[E];
                            El::unpack(buf[j], x);
                            if (ref.far) ref.template exps<true>(x);
                            else ref.template exps<false>(x);
#pragma unroll
                            for (int e = 0; e < E; e += 2) unpack2(mul2(pack2(x[e], x[e + 1]), coef2), x[e], x[e + 1]);
                            dvec[j] = El::pack(x);
                        }
                    }
                    // the vectors that the row covers in part: its first and last
                    for (int j = lo; j < hi; ++j) {
                        if (j >= s.full0 && j < s.full1) { j = s.full1 - 1; continue; }
                        const int id = s.id0 + j * E + lane;
                        if (lane < E && id >= 0 && id < a.V) drow[id] = one(j * E + lane);
                    }
                    __syncwarp();                      // the listed ids of my slice over what was just stored there
                } else {
                    // gradient vectors (16-byte boundaries of dlogits) whole inside the segment's ids, dealt out anew
                    const int id_lo = max(0, s.id0), id_hi = max(id_lo, min(a.V, s.id0 + s.cnt * E));
                    const int dlead = (int)((reinterpret_cast<uintptr_t>(drow) & 15) / sizeof(raw));
                    const int v_lo = (id_lo + dlead + E - 1) / E, v_hi = max(v_lo, (id_hi + dlead) / E);
                    const int vshare = (v_hi - v_lo + PW - 1) / PW;
                    const int w_lo = min(v_hi, v_lo + warp * vshare), w_hi = min(v_hi, w_lo + vshare);
                    uint4* const dvec = reinterpret_cast<uint4*>(drow - dlead);
                    for (int v = w_lo + lane; v < w_hi; v += 32) {
                        const int at = v * E - dlead - s.id0;
                        float x[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] = PODS_INDEX_OK(at + e, s.cnt * E, a.status) ? El::to_float(elems[at + e]) : 0.0f;
                        if (ref.far) ref.template exps<true>(x);
                        else ref.template exps<false>(x);
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] = f.mode ? x[e] * f.coef : 0.0f;
                        dvec[v] = El::pack(x);
                    }
                    if (warp == 0) {                   // the ids outside whole vectors: less than 2 E
                        const int head = min(id_hi, v_lo * E - dlead), tail = max(head, v_hi * E - dlead);
                        if (id_lo + lane < head) drow[id_lo + lane] = one(id_lo + lane - s.id0);
                        if (tail + lane < id_hi) drow[tail + lane] = one(tail + lane - s.id0);
                    }
                    // all warps of the CTA have stored before any listed id goes over it
                    asm volatile("bar.sync 1, %0;" ::"n"(PW * 32) : "memory");
                }
                if (f.mode)
                    for (int k = lane; k < c.n_entry[slot]; k += 32) {
                        const Entry e = c.entry[slot * a.K + k];
                        if ((e.id - s.id0) / E / share == warp) {
                            const double p = exp64(((double)e.z - (double)f.zmax) * tau_inv) * f.p_scale;    // (Q + r) p
                            drow[e.id] = El::from_float((float)(f.g * (p - e.q)));
                        }
                    }
            }
            fence_async_proxy();                       // the stage was written to, and copies refill it
            __syncwarp();
            if (lane == 0) arrive_local(&c.done[st]);
        };
        Slice before = {0.0f, false};
        int st_before = 0;
        StageRing ring;
        for (int i = 0; i < n_rows; ++i, ring.next(kStages)) {
            const int st = ring.st, slot = i % kRing;
            const int64_t t = first + i * n_clusters;
            const Segment s = make_segment<DT>(a.logits, a.ldl, t, a.V, rank, a.seg);
            uint4* const buf = stages + (size_t)st * a.seg;
            const int share = (s.cnt + PW - 1) / PW, lo = min(s.cnt, warp * share), hi = min(s.cnt, lo + share);
            if (!mbar_wait(&c.full[st], ring.parity, spins())) late = true;
            if (!mbar_wait(&c.listed[slot], (uint32_t)((i / kRing) & 1), spins())) late = true;
            float m = -INFINITY;
#pragma unroll 4
            for (int j = lo + lane; j < hi; j += 32) m = max_nan(m, El::vec_max(buf[j]));
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(PODS_FULL_MASK, m, d));
            const PartRef ref(m, cexp);
            const Slice now = {ref.R, kKeep && !ref.far && a.dlogits != nullptr && aligned(s, t)};
            double sum = 0.0;
            if (!ref.far) {
#pragma unroll 2
                for (int j = lo + lane; j < hi; j += 32) {
                    float x[E];
                    El::unpack(buf[j], x);
                    ref.template exps<false>(x);
                    if (kKeep && now.kept) buf[j] = El::pack(x);
                    sum += (double)vec_add(x);
                }
            } else {
                for (int j = lo + lane; j < hi; j += 32) {
                    float x[E];
                    El::unpack(buf[j], x);
                    ref.template exps<true>(x);
                    sum += (double)vec_add(x);
                }
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(PODS_FULL_MASK, sum, d);
            if (lane < CL)
                store_async(mapa(part + slot * CL * PW + rank * PW + warp, lane), mapa(&c.parts[slot], lane), sum,
                            (unsigned long long)__float_as_uint(m));
            if (i > 0) back(i - 1, st_before, before);
            before = now;
            st_before = st;
        }
        if (n_rows > 0) back(n_rows - 1, st_before, before);
    }
    if (late && lane == 0) pods_raise(a.status, PODS_STATUS_TIMEOUT);
    __syncwarp();
    cl.sync();                                         // no CTA leaves while a peer may still write its parts
}

size_t align_up(size_t v, size_t n) { return (v + n - 1) / n * n; }

constexpr size_t kMaxSmem = 227 * 1024;
constexpr size_t kHalfSmBytes = 233472 / 2 - 1024;     // what a CTA may hold for two of them to share an SM
// The pipeline from this much of logits on.  Measured, pipeline (with its preparation) against the kernel above, at 16, 32
// and 64 MB: bf16 V = 1000 88 : 94, 162 : 180, 306 : 385 us; V = 8000 25 : 25, 37 : 39, 69 : 75; V = 32000 21 : 19, 29 : 31,
// 49 : 57; V = 151936 19 : 21, 27 : 29, 46 : 54; fp32 V = 1000 47 : 53, 83 : 96, 150 : 198; V = 8000 18 : 17, 25 : 25, 43 : 53;
// V = 32000 19 : 17, 25 : 25, 43 : 51; V = 151936 21 : 19, 26 : 27, 44 : 53.
constexpr int64_t kPipeMinBytes = 32 << 20;

template <int DT, int KP>
int launch_distill(DistillArgs& a, cudaStream_t stream) {
    const int esize = DT == PODS_DTYPE_F32 ? 4 : 2;
    if (a.K <= kPipeK && a.T * a.V * esize >= kPipeMinBytes && a.T <= 0x7fffffff) {
        // the smallest cluster whose stages fit twice on an SM: few partners, few places of the GPU left empty by its size;
        // for rows too long for that the smallest that fits an SM once, with twice the consumers.  (512 fp32 rows of
        // 151936: 144 us on clusters of 9, 178 of 10, 236 of 12, 226 of 16; 218 with two stages twice an SM; 198 by the kernel above.
        // One CTA an SM where two fit: 602 us for 4096 bf16 rows of 151936 against 551.)
        static const int kSizes[] = {1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 12, 16};
        for (int pw = 8; pw <= 16; pw *= 2)
            for (int size : kSizes) {
                a.seg = segment_vectors(a.V, esize, size);
                const size_t smem = pipe_ctrl_bytes(size, a.K, pw) + (size_t)kStages * a.seg * 16;
                if (smem > (pw == 8 ? kHalfSmBytes : kMaxSmem)) continue;
                distill_prep_kernel<<<(unsigned)((a.T + 7) / 8), 256, 0, stream>>>(a);
                PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
                return pw == 8 ? launch_row_clusters<pods_distill_pipe_kernel<DT, 8>>(a, a.T, size, 11 * 32, smem, stream)
                               : launch_row_clusters<pods_distill_pipe_kernel<DT, 16>>(a, a.T, size, 19 * 32, smem, stream);
            }
    }
    // segments that let as many CTAs share an SM as registers allow: four, or two with long lists.  Four against two, bf16:
    // 16 MB of V = 1000 94 : 154 us, of 8000 25 : 33, 64 MB of 151936 54 : 60; V = 32000 57 : 62; fp32 51 : 54.
    constexpr size_t kSegmentBytes = (KP == 1 ? 55 : 80) * 1024;
    int cl = 1;
    while (cl < kMaxCluster && (size_t)segment_vectors(a.V, esize, cl) * 16 > kSegmentBytes) cl *= 2;
    // few rows: spread over idle SMs down to a vector a thread (3 bf16 rows of 151936 and 16 of 32000: 14.6 -> 12.6 us)
    while (cl < kMaxCluster && 2 * cl * a.T <= 128 && segment_vectors(a.V, esize, 2 * cl) >= kThreads) cl *= 2;
    a.seg = segment_vectors(a.V, esize, cl);
    const size_t smem = kCtrlBytes + (size_t)a.seg * 16;
    if (smem > kMaxSmem) return PODS_ERR_UNSUPPORTED;
    return launch_row_clusters<pods_distill_kernel<DT, KP>>(a, a.T, cl, kThreads, smem, stream);
}

}  // namespace

extern "C" size_t pods_distill_chunk_workspace_bytes(int64_t T) {
    return T < 0 ? 0 : align_up((size_t)T * sizeof(double), 256) + align_up((size_t)T * sizeof(RowPrep), 256) + 256;
}

extern "C" int pods_distill_chunk(const void* logits, int64_t ldl, int32_t dtype, const int32_t* ids,
                                  const float* values, int64_t ldk, int32_t K, const float* teacher_lse,
                                  const double* seq_weight, const int64_t* cu_seqlens, int64_t M, int64_t row0,
                                  const uint8_t* mask, int64_t T, int32_t V, float temperature, uint32_t flags,
                                  float grad_scale, double* loss_acc, float* kl, void* dlogits, int64_t ldd,
                                  void* workspace, size_t workspace_bytes, uint32_t* status, void* stream) {
    if (dtype != PODS_DTYPE_BF16 && dtype != PODS_DTYPE_F16 && dtype != PODS_DTYPE_F32) return PODS_ERR_UNSUPPORTED;
    const size_t esize = dtype == PODS_DTYPE_F32 ? 4 : 2;
    if (T < 0 || V < 1 || M < 1 || row0 < 0 || ldl < V || K < 1 || ldk < K) return PODS_ERR_INVALID_ARG;
    if (V > PODS_MAX_ROW_V || K > PODS_MAX_TOPK || (flags & ~PODS_DISTILL_REST) != 0) return PODS_ERR_UNSUPPORTED;
    if (!(temperature >= FLT_MIN && temperature < INFINITY) || grad_scale != grad_scale) return PODS_ERR_INVALID_ARG;
    if ((flags & PODS_DISTILL_REST) && teacher_lse == nullptr) return PODS_ERR_INVALID_ARG;
    if (dlogits != nullptr && (ldd < V || !pods_aligned(dlogits, esize) || (dlogits == logits && ldd != ldl)))
        return PODS_ERR_INVALID_ARG;
    if (T == 0) return PODS_OK;
    if (logits == nullptr || ids == nullptr || values == nullptr || seq_weight == nullptr || cu_seqlens == nullptr ||
        loss_acc == nullptr || kl == nullptr)
        return PODS_ERR_INVALID_ARG;
    if (!pods_aligned(logits, esize) || !pods_all_aligned(8, loss_acc, seq_weight, cu_seqlens) ||
        !pods_all_aligned(4, ids, values, teacher_lse, kl, status))
        return PODS_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < pods_distill_chunk_workspace_bytes(T) || !pods_aligned(workspace, 16))
        return PODS_ERR_WORKSPACE;
    DistillArgs a = {};
    a.logits = logits;
    a.ldl = ldl;
    a.ids = ids;
    a.values = values;
    a.ldk = ldk;
    a.K = K;
    a.teacher_lse = teacher_lse;
    a.seq_weight = seq_weight;
    a.cu_seqlens = cu_seqlens;
    a.M = M;
    a.row0 = row0;
    a.mask = mask;
    a.T = T;
    a.V = V;
    a.temperature = temperature;
    a.rest = (flags & PODS_DISTILL_REST) ? 1 : 0;
    a.grad_scale = grad_scale;
    a.kl = kl;
    a.dlogits = dlogits;
    a.ldd = ldd;
    a.row_loss = static_cast<double*>(workspace);
    a.prep = reinterpret_cast<RowPrep*>(static_cast<unsigned char*>(workspace) + align_up((size_t)T * sizeof(double), 256));
    a.status = status;
    cudaStream_t s = pods_stream(stream);
    constexpr int kMany = PODS_MAX_TOPK / kThreads;
    const bool few = K <= kThreads;
    const int rc = dtype == PODS_DTYPE_BF16  ? (few ? launch_distill<PODS_DTYPE_BF16, 1>(a, s) : launch_distill<PODS_DTYPE_BF16, kMany>(a, s))
                   : dtype == PODS_DTYPE_F16 ? (few ? launch_distill<PODS_DTYPE_F16, 1>(a, s) : launch_distill<PODS_DTYPE_F16, kMany>(a, s))
                                             : (few ? launch_distill<PODS_DTYPE_F32, 1>(a, s) : launch_distill<PODS_DTYPE_F32, kMany>(a, s));
    if (rc != PODS_OK) return rc;
    return pods_loss::launch_loss_reduce(a.row_loss, T, loss_acc, s);
}
