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

#include "pods_logp.cuh"

namespace {

using namespace pods_row;
using pods_logp::FwdArgs;
using pods_logp::GradArgs;

constexpr int kThreads = 256;
constexpr int kBlockVecs = 4;          // vectors a thread takes at once
constexpr float kSumLimit = 1024.0f;   // a block's sum above this moves the reference
constexpr int kNoRef = -(1 << 30);
constexpr int kFar = 1 << 22;          // references from here on leave fp32 too few fractional bits: the row is taken in fp64

// A part of a row: S and U relative to 2^R.  R == kNoRef: nothing but -inf so far.
struct Part {
    double s, u;
    int R;
    int bad;                           // 1: NaN or +inf, 2: far
};

__device__ __forceinline__ double pow2_int(int n) {    // n <= 0
    return n < -1000 ? 0.0 : __hiloint2double((1023 + n) << 20, 0);
}

__device__ __forceinline__ Part join(const Part& a, const Part& b) {
    Part r;
    r.R = max(a.R, b.R);
    r.bad = a.bad | b.bad;
    const int da = a.R - r.R, db = b.R - r.R;
    const double fa = pow2_int(da), fb = pow2_int(db);
    r.s = a.s * fa + b.s * fb;
    // 2^(y - R) (y - R) = 2^(y - Ra) 2^(Ra - R) (y - Ra + Ra - R); an empty part (s = 0) adds nothing however far its reference
    r.u = (a.u + (a.s != 0.0 ? a.s * (double)da : 0.0)) * fa + (b.u + (b.s != 0.0 ? b.s * (double)db : 0.0)) * fb;
    return r;
}

// What a thread holds while it goes through its elements.
template <int DT, bool ENT>
struct Sums {
    using El = Elem<DT>;
    static constexpr int E = El::E;
    float s = 0.0f, u = 0.0f;
    int R = kNoRef, bad = 0;

    // e = 2^(x c - R) of a vector, added up; with ENT also e (x c - R)
    __device__ __forceinline__ void add(const uint4& q, float c, float R_, float& bs, float& bu) const {
        float x[E];
        El::unpack(q, x);
        const unsigned long long c2 = pack2(c, c), off2 = pack2(-R_, -R_);
        unsigned long long acc = 0ull, accu = 0ull;
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const unsigned long long d2 = fma2(pack2(x[i], x[i + 1]), c2, off2);
            float d0, d1;
            unpack2(d2, d0, d1);
            const unsigned long long e2 = pack2(ex2_approx(d0), ex2_approx(d1));
            acc = add2(acc, e2);
            if (ENT) accu = fma2(e2, pack2(fmaxf(d0, -1e4f), fmaxf(d1, -1e4f)), accu);   // 2^-inf (-inf) counts 0
        }
        float a, b;
        unpack2(acc, a, b);
        bs += a + b;
        if (ENT) {
            unpack2(accu, a, b);
            bu += a + b;
        }
    }
    template <int N>
    __device__ __forceinline__ void take(const uint4 (&q)[N], float c) {
        float bs = 0.0f, bu = 0.0f;
        const float ref = (float)R;
#pragma unroll
        for (int k = 0; k < N; ++k) add(q[k], c, ref, bs, bu);
        if (!(bs < kSumLimit)) {                       // rare: the first block, a block far above all before it, NaN, +inf
            float m = -INFINITY;
#pragma unroll
            for (int k = 0; k < N; ++k) m = max_nan(m, El::vec_max(q[k]));
            bs = bu = 0.0f;
            if (!(m < INFINITY)) bad |= 1;
            else if (m > -INFINITY) {
                const float top = ceilf(m * c);
                if (!(fabsf(top) < (float)kFar)) bad |= 2;
                else {
                    const int to = (int)top;
                    if (to > R) {
                        const float f = R - to < -126 ? 0.0f : __uint_as_float((uint32_t)(127 + R - to) << 23);
                        if (ENT) u = f == 0.0f ? 0.0f : (u + s * (float)(R - to)) * f;
                        s *= f;
                        R = to;
                    }
                    const float now = (float)R;
#pragma unroll
                    for (int k = 0; k < N; ++k) add(q[k], c, now, bs, bu);
                }
            }
        }
        s += bs;
        if (ENT) u += bu;
    }
    __device__ __forceinline__ Part part() const { return {(double)s, (double)u, R, bad}; }
};

template <typename T, typename Op>
__device__ __forceinline__ T warp_reduce(T v, Op op) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(PODS_FULL_MASK, v, d));
    return v;
}

// the row in fp64, by one group of `n` threads: what is left where fp32 has no fractional bits for the exponents
template <int DT>
__device__ Part row_fp64(const typename Elem<DT>::raw* row, int V, double inv_tau, float top, int at, int n) {
    Part r = {0.0, 0.0, 0, 0};
    for (int v = at; v < V; v += n) {
        const double d = ((double)Elem<DT>::to_float(row[v]) - (double)top) * inv_tau, e = exp64(d);
        r.s += e;
        if (e != 0.0) r.u += e * d;
    }
    return r;
}

// G threads a row: a warp (eight rows a CTA), or the CTAs of a cluster.  Rows are cut at 16-byte boundaries of memory.
template <int DT, bool ENT, bool WARP>
__global__ void __launch_bounds__(kThreads) pods_logp_kernel(const FwdArgs a) {
    using El = Elem<DT>;
    using raw = typename El::raw;
    constexpr int E = El::E;
    __shared__ Part parts[kMaxCluster * (kThreads / 32)];
    __shared__ float tops[kThreads / 32];
    cg::cluster_group cl = cg::this_cluster();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int CL = WARP ? 1 : (int)cl.num_blocks(), rank = WARP ? 0 : (int)cl.block_rank();
    const int64_t t = WARP ? (int64_t)blockIdx.x * (kThreads / 32) + warp : (int64_t)(blockIdx.x / CL);
    if (WARP && t >= a.T) return;
    if (CL > 1) cl.barrier_arrive();                   // met before the first store into another CTA
    if ((a.mask != nullptr && a.mask[t] == 0) || (a.rows_end != nullptr && t >= *a.rows_end)) {    // the same for the whole cluster
        if (a.fill && (WARP ? lane : (int)threadIdx.x) == 0 && rank == 0) a.logp[t] = 0.0f;
        if (CL > 1) cl.barrier_wait();
        return;
    }
    const raw* const row = static_cast<const raw*>(a.logits) + t * a.ldl;
    const int lead = (int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(raw));
    const int head = min(lead, a.V), nvec = (a.V - head) / E, tail = head + nvec * E;
    const uint4* const vec = reinterpret_cast<const uint4*>(row + head);
    const int G = WARP ? 32 : kThreads, me = WARP ? lane : (int)threadIdx.x;
    const int share = (nvec + CL - 1) / CL, lo = min(nvec, rank * share), hi = min(nvec, lo + share);
    Sums<DT, ENT> sums;
    int v = lo + me;
    for (; v + (kBlockVecs - 1) * G < hi; v += kBlockVecs * G) {
        uint4 q[kBlockVecs];
#pragma unroll
        for (int k = 0; k < kBlockVecs; ++k) q[k] = __ldg(vec + v + k * G);
        sums.take(q, a.c);
    }
    for (; v < hi; v += G) {
        const uint4 q[1] = {__ldg(vec + v)};
        sums.take(q, a.c);
    }
    if (rank == 0) {                                   // the ends: less than 2 E elements
        const int i = me < head ? me : tail + me - head;
        if (me < head + a.V - tail && PODS_INDEX_OK(i, a.V, a.status)) {
            raw e[16 / sizeof(raw)];
#pragma unroll
            for (int k = 0; k < E; ++k) e[k] = k == 0 ? row[i] : El::kNegInf;
            const uint4 q[1] = {*reinterpret_cast<const uint4*>(e)};
            sums.take(q, a.c);
        }
    }
    Part p = sums.part();
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        Part o;
        o.s = __shfl_xor_sync(PODS_FULL_MASK, p.s, d);
        o.u = ENT ? __shfl_xor_sync(PODS_FULL_MASK, p.u, d) : 0.0;
        o.R = __shfl_xor_sync(PODS_FULL_MASK, p.R, d);
        o.bad = __shfl_xor_sync(PODS_FULL_MASK, p.bad, d);
        p = join(p, o);
    }
    if (!WARP) {
        if (CL == 1) {
            if (lane == 0) parts[warp] = p;
            __syncthreads();
        } else {
            cl.barrier_wait();
            if (lane == 0) *cl.map_shared_rank(&parts[rank * (kThreads / 32) + warp], 0) = p;
            cl.sync();
        }
        if (rank != 0) return;
        p = parts[0];
        for (int i = 1; i < CL * (kThreads / 32); ++i) p = join(p, parts[i]);
    }
    // far, or nothing above 2^kNoRef: fp64 tells huge negative logits from a row of -inf
    const bool far = p.bad == 2 || (p.bad == 0 && p.R == kNoRef);
    float top = 0.0f;
    if (far) {
        float m = -INFINITY;
        for (int i = me; i < a.V; i += G) m = max_nan(m, El::to_float(row[i]));
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(PODS_FULL_MASK, m, d));
        if (!WARP) {
            if (lane == 0) tops[warp] = m;
            __syncthreads();
            for (int w = 0; w < kThreads / 32; ++w) m = max_nan(m, tops[w]);
        }
        top = m;
        p = {0.0, 0.0, 0, top < INFINITY ? 0 : 1};
        if (fabsf(top) < INFINITY) {
            Part q = row_fp64<DT>(row, a.V, a.inv_tau, top, me, G);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                q.s += __shfl_xor_sync(PODS_FULL_MASK, q.s, d);
                q.u += __shfl_xor_sync(PODS_FULL_MASK, q.u, d);
            }
            if (!WARP) {
                __syncthreads();
                if (lane == 0) parts[warp] = q;
                __syncthreads();
                q = parts[0];
                for (int w = 1; w < kThreads / 32; ++w) {
                    q.s += parts[w].s;
                    q.u += parts[w].u;
                }
            }
            p.s = q.s;
            p.u = q.u;
        }
    }
    if (me != 0) return;
    int token = a.tokens[t];
    if ((unsigned)token >= (unsigned)a.V) {
        pods_raise(a.status, PODS_STATUS_TOKEN_RANGE);
        token = 0;
    }
    const double z = (double)El::to_float(row[token]);
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
        logp = (z - (double)top) * a.inv_tau - ls;
        H = ls - p.u / p.s;
    } else {
        const double ls = log2(p.s);
        lse = ((double)p.R + ls) * kLn2;
        logp = ((z * (double)a.c - (double)p.R) - ls) * kLn2;
        H = (ls - p.u / p.s) * kLn2;
    }
    a.logp[t] = (float)fmin(logp, 0.0);
    if (logp != logp) a.logp[t] = NAN;
    if (a.lse != nullptr) a.lse[t] = lse;
    if (ENT) a.entropy[t] = H == H ? (float)fmax(H, 0.0) : NAN;
}

// d objective / d logits.  A CTA takes a stretch of `seg` vectors of one row (WARP: a warp a whole row).
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
        const float d = fmaf(z, a.c, -n), p = ex2_approx(d);
        return ENT ? p * fmaf(B, fmaxf(d, -1e4f), A) : p * A;
    };
    auto vector = [&](const uint4& q, int v) {
        float x[E];
        El::unpack(q, x);
        const unsigned long long c2 = pack2(a.c, a.c), off2 = pack2(-n, -n);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            float d0, d1;
            unpack2(fma2(pack2(x[i], x[i + 1]), c2, off2), d0, d1);
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
    if (((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0) {
        const uint4* const src = reinterpret_cast<const uint4*>(row + head);
        int v = lo + me;
        for (; v + (kBlockVecs - 1) * G < hi; v += kBlockVecs * G) {
            uint4 q[kBlockVecs];
#pragma unroll
            for (int k = 0; k < kBlockVecs; ++k) q[k] = src[v + k * G];
#pragma unroll
            for (int k = 0; k < kBlockVecs; ++k) vector(q[k], v + k * G);
        }
        for (; v < hi; v += G) vector(src[v], v);
    } else {
        for (int v = lo + me; v < hi; v += G) {
            raw e[E];
#pragma unroll
            for (int i = 0; i < E; ++i) e[i] = row[head + v * E + i];
            uint4 q;
            memcpy(&q, e, sizeof q);
            vector(q, v);
        }
    }
    if (has_edge) {
        float x = one(El::to_float(row[edge]));
        if (edge == token) x += g;
        out[edge] = El::from_float(x);
    }
}

constexpr int kWarpVecs = 32 * 16;     // rows of up to this many vectors are taken a warp each

template <int DT, bool ENT>
int launch_fwd(const FwdArgs& a, cudaStream_t stream) {
    const int nvec = a.V / Elem<DT>::E;
    if (nvec <= kWarpVecs) {
        pods_logp_kernel<DT, ENT, true><<<(unsigned)((a.T + kThreads / 32 - 1) / (kThreads / 32)), kThreads, 0, stream>>>(a);
        PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
        return PODS_OK;
    }
    int cl = 1;                                        // few rows: spread over idle SMs
    while (cl < 8 && 2 * cl * a.T <= 4 * pods_sm_count() && nvec >= 2 * cl * kThreads) cl *= 2;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cl;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(a.T * cl));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    PODS_RETURN_IF_CUDA_ERROR(cudaLaunchKernelEx(&cfg, pods_logp_kernel<DT, ENT, false>, a));
    return PODS_OK;
}

template <int DT, bool ENT>
int launch_grad(GradArgs& a, cudaStream_t stream) {
    const int nvec = a.V / Elem<DT>::E;
    if (nvec <= kWarpVecs) {
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
    a.inv_tau = 1.0 / (double)temperature;
    a.c = pods_logp::exponent_scale(temperature);
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
    a.inv_tau = 1.0 / (double)temperature;
    a.c = pods_logp::exponent_scale(temperature);
    a.dlogits = dlogits;
    a.ldd = ldd;
    a.status = status;
    return pods_logp::launch_gradient(a, dtype, pods_stream(stream));
}
