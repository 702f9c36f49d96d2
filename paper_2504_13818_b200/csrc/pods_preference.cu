// pods_preference - losses of pairs of rollouts from their tokens' log-probabilities, with the derivative in every token's
// log-probability; pods_preference_fwd_bwd - the same from logits, with the gradient in the logits.
//
// A pair's slope is known only when both of its rollouts have been summed, and a token's coefficient only when every pair of
// its rollout has its slope: three phases with a barrier between them, which one thread-block cluster takes in one launch
// (a few MB at most are read: 8 bytes a token; latency bounds it).  Sums are fp64 in a fixed order.  A rollout's coefficient
// is summed over the stretch of the list that holds its first to its last pair, in the list's order: pairs that lie together cost little
// (65536 rollouts of 20 tokens, as many pairs in order 1.6 ms), shuffled ones the product of rollouts and pairs (69 ms).
#include <float.h>

#include "pods_logp.cuh"

namespace {

using namespace pods_row;

constexpr int kThreads = 1024;
constexpr int kCluster = 8;            // CTAs at most
constexpr int kAtOnce = 8;             // tokens a lane has on their way

struct PrefArgs {
    const float* logp;
    const double* logp64;              // used instead of logp where there is one
    const float* ref_logp;
    const uint8_t* mask;
    const int64_t* cu;
    int64_t M, T;
    const int32_t* pairs;
    const float* pair_weight;
    int64_t P;
    int kind, average;
    double beta, smoothing, margin, nll, grad_scale;
    const float* margin_pair;
    double* loss_acc;
    float* loss32;                     // the loss alone, written; used where loss_acc is NULL
    float* dlogp;
    float* reward;
    float* pair_loss;
    // workspace
    double* score;                     // [M] s_i
    double* like;                      // [M] mean -log-probability
    double* inv_n;                     // [M] 1 / |o_i|, 0 for an empty rollout
    double* slope;                     // [P] weight times d loss / d h
    double* weight;                    // [P]
    int2* span;                        // [M] first and last pair of the rollout
    double* parts;                     // [2 kCluster]
    uint32_t* status;
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(PODS_FULL_MASK, v, d);
    return v;
}

__device__ __forceinline__ double log1pexp(double x) {  // log(1 + e^x)
    return fmax(x, 0.0) + log1p(exp(-fabs(x)));
}

// loss of a pair and its slope in h
__device__ __forceinline__ void pair_terms(const PrefArgs& a, double h, double& loss, double& slope) {
    if (a.kind == PODS_PREFERENCE_SIGMOID) {
        const double e = a.smoothing;
        loss = (1.0 - e) * log1pexp(-h);
        slope = -(1.0 - e) / (1.0 + exp(h));
        if (e != 0.0) {
            loss += e * log1pexp(h);
            slope += e / (1.0 + exp(-h));
        }
    } else if (a.kind == PODS_PREFERENCE_HINGE) {
        loss = 1.0 - h > 0.0 ? 1.0 - h : h != h ? h : 0.0;
        slope = h < 1.0 ? -1.0 : h != h ? h : 0.0;
    } else {
        const double d = (h - 0.5) / a.beta;
        loss = d * d;
        slope = 2.0 * d / a.beta;
    }
}

__global__ void __launch_bounds__(kThreads) pods_preference_kernel(const PrefArgs a) {
    cg::cluster_group cl = cg::this_cluster();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int CL = (int)cl.num_blocks(), all = CL * kThreads;
    auto meet = [&] {                                  // after it everybody sees what anybody wrote
        if (CL == 1) __syncthreads();
        else cl.sync();
    };
    const int n_warps = CL * (kThreads / 32), gw = (int)cl.block_rank() * (kThreads / 32) + warp;
    const int64_t gt = (int64_t)cl.block_rank() * kThreads + threadIdx.x;
    __shared__ double scratch[2][kThreads / 32];

    // 1. every rollout's sums, a warp each
    for (int64_t i = gw; i < a.M; i += n_warps) {
        const int64_t lo = max((int64_t)0, min(a.T, a.cu[i])), hi = max(lo, min(a.T, a.cu[i + 1]));
        double sum = 0.0, like = 0.0;
        int64_t n = 0;
        for (int64_t t = lo + lane; t < hi; t += 32 * kAtOnce) {
            double lp[kAtOnce];
            float ref[kAtOnce];
            bool on[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int64_t at = t + 32 * k;
                on[k] = at < hi && (a.mask == nullptr || a.mask[at] != 0);
                lp[k] = at < hi ? (a.logp64 != nullptr ? a.logp64[at] : (double)a.logp[at]) : 0.0;
                ref[k] = at < hi && a.ref_logp != nullptr ? a.ref_logp[at] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (on[k]) {
                    sum += lp[k] - (double)ref[k];
                    like -= lp[k];
                    ++n;
                }
        }
        sum = warp_sum(sum);
        like = warp_sum(like);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) n += __shfl_xor_sync(PODS_FULL_MASK, n, d);
        if (lane == 0) {
            const double inv = n > 0 ? 1.0 / (double)n : 0.0;
            const double s = a.average ? (n > 0 ? sum * inv : 0.0) : sum;
            a.score[i] = s;
            a.like[i] = n > 0 ? like * inv : 0.0;
            a.inv_n[i] = inv;
            a.span[i] = make_int2(0x7fffffff, -1);
            if (a.reward != nullptr) a.reward[i] = (float)(a.beta * s);
        }
    }
    // the pairs in use, which share the weight where none is given
    auto used = [&](int64_t p, int& c, int& r) {
        c = a.pairs[2 * p];
        r = a.pairs[2 * p + 1];
        const bool c_ok = (uint32_t)c < (uint64_t)a.M, r_ok = (uint32_t)r < (uint64_t)a.M;
        if ((!c_ok && c != -1) || (!r_ok && r != -1)) pods_raise(a.status, PODS_STATUS_INDEX_RANGE);
        return c_ok && r_ok;
    };
    double count = 0.0;
    for (int64_t p = gt; p < a.P; p += all) {
        int c, r;
        count += used(p, c, r) ? 1.0 : 0.0;
    }
    count = warp_sum(count);
    if (lane == 0) scratch[0][warp] = count;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) count += scratch[0][w];
        a.parts[cl.block_rank()] = count;
    }
    meet();

    // 2. every pair's slope and loss
    count = 0.0;
    for (int b = 0; b < CL; ++b) count += a.parts[b];
    const double even = count > 0.0 ? 1.0 / count : 0.0;
    double total = 0.0;
    for (int64_t p = gt; p < a.P; p += all) {
        int c, r;
        double loss = 0.0, slope = 0.0, w = 0.0;
        if (used(p, c, r)) {
            w = a.pair_weight != nullptr ? (double)a.pair_weight[p] : even;
            const double margin = a.margin_pair != nullptr ? (double)a.margin_pair[p] : a.margin;
            pair_terms(a, a.beta * (a.score[c] - a.score[r]) - margin, loss, slope);
            if (a.nll != 0.0) loss += a.nll * a.like[c];
            if (w != 0.0) {                            // a pair of weight 0 leaves nothing behind, whatever its rollouts hold
                total += w * loss;
                atomicMin(&a.span[c].x, (int)p);
                atomicMax(&a.span[c].y, (int)p);
                atomicMin(&a.span[r].x, (int)p);
                atomicMax(&a.span[r].y, (int)p);
            }
        }
        a.slope[p] = w != 0.0 ? w * slope : 0.0;
        a.weight[p] = w;
        if (a.pair_loss != nullptr) a.pair_loss[p] = (float)loss;
    }
    total = warp_sum(total);
    if (lane == 0) scratch[1][warp] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) total += scratch[1][w];
        a.parts[kCluster + cl.block_rank()] = total;
    }
    meet();

    // 3. the loss, and every token's coefficient
    if (gt == 0) {
        total = 0.0;
        for (int b = 0; b < CL; ++b) total += a.parts[kCluster + b];
        if (a.loss_acc != nullptr) *a.loss_acc += total;
        else *a.loss32 = (float)total;
    }
    for (int64_t i = gw; i < a.M; i += n_warps) {
        const int2 span = a.span[i];
        const double inv = a.inv_n[i], per = a.average ? inv : 1.0;
        double coef = 0.0;
        for (int64_t p = (int64_t)span.x + lane; p <= span.y; p += 32) {
            const int c = a.pairs[2 * p], r = a.pairs[2 * p + 1];
            if (c == r || c < 0 || r < 0 || a.weight[p] == 0.0) {
                if (c == i && c == r && a.weight[p] != 0.0) coef -= a.weight[p] * a.nll * inv;
                continue;
            }
            if (c == i) coef += a.slope[p] * a.beta * per - a.weight[p] * a.nll * inv;
            if (r == i) coef -= a.slope[p] * a.beta * per;
        }
        coef = warp_sum(coef) * a.grad_scale;
        const int64_t lo = max((int64_t)0, min(a.T, a.cu[i])), hi = max(lo, min(a.T, a.cu[i + 1]));
        for (int64_t t = lo + lane; t < hi; t += 32) a.dlogp[t] = a.mask != nullptr && a.mask[t] == 0 ? 0.0f : (float)coef;
    }
    // rows ahead of the first and behind the last rollout
    const int64_t first = max((int64_t)0, min(a.T, a.cu[0])), last = max(first, min(a.T, a.cu[a.M]));
    for (int64_t t = gt; t < first; t += all) a.dlogp[t] = 0.0f;
    for (int64_t t = last + gt; t < a.T; t += all) a.dlogp[t] = 0.0f;
}

int launch_preference(const PrefArgs& a, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    // one CTA where it has warps and tokens enough for itself: its barriers cost less than a cluster's (32 rollouts of 188 tokens
    // 8.3 : 9.1 us; a cluster for 128 of 500 18.5 us, for 1024 of 500 and 4096 pairs 135)
    const int size = a.M <= 2 * kThreads / 32 && a.P <= kThreads && a.T <= 16384 ? 1 : kCluster;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)size);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    PODS_RETURN_IF_CUDA_ERROR(cudaLaunchKernelEx(&cfg, pods_preference_kernel, a));
    return PODS_OK;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// lays the kernel's arrays out in `base`; returns the bytes
size_t lay_out(PrefArgs* a, unsigned char* base, int64_t M, int64_t P) {
    size_t at = 0;
    auto take = [&](size_t bytes) {
        unsigned char* p = base == nullptr ? nullptr : base + at;
        at += up(bytes);
        return p;
    };
    unsigned char* const q[7] = {take((size_t)M * 8), take((size_t)M * 8), take((size_t)M * 8), take((size_t)P * 8),
                                 take((size_t)P * 8), take((size_t)M * 8), take(2 * kCluster * 8)};
    if (a != nullptr) {
        a->score = reinterpret_cast<double*>(q[0]);
        a->like = reinterpret_cast<double*>(q[1]);
        a->inv_n = reinterpret_cast<double*>(q[2]);
        a->slope = reinterpret_cast<double*>(q[3]);
        a->weight = reinterpret_cast<double*>(q[4]);
        a->span = reinterpret_cast<int2*>(q[5]);
        a->parts = reinterpret_cast<double*>(q[6]);
    }
    return at;
}

bool finite(float x) { return x - x == 0.0f; }

// what both calls check; fills the settings
int check_pairs(PrefArgs& a, const float* ref_logp, const uint8_t* mask, const int64_t* cu, int64_t M, int64_t T,
                const int32_t* pairs, const float* pair_weight, int64_t P, int32_t kind, uint32_t flags, float beta,
                float smoothing, const float* margin_pair, float margin, float nll, float grad_scale, float* reward,
                float* pair_loss, uint32_t* status) {
    if (M < 1 || P < 0 || T < 0) return PODS_ERR_INVALID_ARG;
    if (M > 0x7fffffff || P > 0x7fffffff || kind < PODS_PREFERENCE_SIGMOID || kind > PODS_PREFERENCE_SQUARED ||
        (flags & ~PODS_PREFERENCE_AVERAGE) != 0)
        return PODS_ERR_UNSUPPORTED;
    if (!(beta > 0.0f) || !finite(beta) || !(smoothing >= 0.0f && smoothing < 0.5f) || !finite(margin) || !(nll >= 0.0f) ||
        !finite(nll) || !finite(grad_scale))
        return PODS_ERR_INVALID_ARG;
    if (smoothing != 0.0f && kind != PODS_PREFERENCE_SIGMOID) return PODS_ERR_INVALID_ARG;
    if (cu == nullptr || (P > 0 && pairs == nullptr) || !pods_aligned(cu, 8) ||
        !pods_all_aligned(4, ref_logp, pairs, pair_weight, margin_pair, reward, pair_loss, status))
        return PODS_ERR_INVALID_ARG;
    a.ref_logp = ref_logp;
    a.mask = mask;
    a.cu = cu;
    a.M = M;
    a.T = T;
    a.pairs = pairs;
    a.pair_weight = pair_weight;
    a.P = P;
    a.kind = kind;
    a.average = (flags & PODS_PREFERENCE_AVERAGE) ? 1 : 0;
    a.beta = beta;
    a.smoothing = smoothing;
    a.margin = margin;
    a.nll = nll;
    a.grad_scale = grad_scale;
    a.margin_pair = margin_pair;
    a.reward = reward;
    a.pair_loss = pair_loss;
    a.status = status;
    return PODS_OK;
}

}  // namespace

extern "C" size_t pods_preference_workspace_bytes(int64_t M, int64_t P) {
    return M < 0 || P < 0 ? 0 : lay_out(nullptr, nullptr, M, P);
}

extern "C" int pods_preference(const float* logp, const float* ref_logp, const uint8_t* mask, const int64_t* cu_seqlens,
                               int64_t M, int64_t T, const int32_t* pairs, const float* pair_weight, int64_t P, int32_t kind,
                               uint32_t flags, float beta, float label_smoothing, const float* margin_pair, float margin,
                               float nll, float grad_scale, double* loss_acc, float* dlogp, float* reward, float* pair_loss,
                               void* workspace, size_t workspace_bytes, uint32_t* status, void* stream) {
    PrefArgs a = {};
    const int rc = check_pairs(a, ref_logp, mask, cu_seqlens, M, T, pairs, pair_weight, P, kind, flags, beta, label_smoothing,
                               margin_pair, margin, nll, grad_scale, reward, pair_loss, status);
    if (rc != PODS_OK) return rc;
    if (loss_acc == nullptr || !pods_aligned(loss_acc, 8) || !pods_all_aligned(4, logp, dlogp) ||
        (T > 0 && (logp == nullptr || dlogp == nullptr)))
        return PODS_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < lay_out(nullptr, nullptr, M, P) || !pods_aligned(workspace, 16))
        return PODS_ERR_WORKSPACE;
    lay_out(&a, static_cast<unsigned char*>(workspace), M, P);
    a.logp = logp;
    a.dlogp = dlogp;
    a.loss_acc = loss_acc;
    return launch_preference(a, pods_stream(stream));
}

extern "C" size_t pods_preference_fwd_bwd_workspace_bytes(int64_t T, int64_t M, int64_t P) {
    return T < 0 || M < 0 || P < 0 ? 0 : 2 * up((size_t)T * 8) + up((size_t)T * 4) + lay_out(nullptr, nullptr, M, P);
}

extern "C" int pods_preference_fwd_bwd(const void* logits, int64_t ldl, int32_t dtype, const int32_t* tokens,
                                       const float* ref_logp, const uint8_t* mask, const int64_t* cu_seqlens, int64_t M,
                                       int64_t T, int32_t V, float temperature, const int32_t* pairs,
                                       const float* pair_weight, int64_t P, int32_t kind, uint32_t flags, float beta,
                                       float label_smoothing, const float* margin_pair, float margin, float nll,
                                       float grad_scale, float* loss, float* logp, void* dlogits, int64_t ldd, float* reward,
                                       float* pair_loss, void* workspace, size_t workspace_bytes, uint32_t* status,
                                       void* stream) {
    int rc = pods_logp::check_rows(logits, ldl, dtype, T, V, temperature);
    if (rc != PODS_OK) return rc;
    PrefArgs a = {};
    rc = check_pairs(a, ref_logp, mask, cu_seqlens, M, T, pairs, pair_weight, P, kind, flags, beta, label_smoothing, margin_pair,
                     margin, nll, grad_scale, reward, pair_loss, status);
    if (rc != PODS_OK) return rc;
    const size_t esize = dtype == PODS_DTYPE_F32 ? 4 : 2;
    if (ldd < V || (dlogits == logits && ldd != ldl) || loss == nullptr || !pods_all_aligned(4, loss, logp, tokens) ||
        !pods_aligned(dlogits, esize) || (T > 0 && (tokens == nullptr || logp == nullptr || dlogits == nullptr)))
        return PODS_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < pods_preference_fwd_bwd_workspace_bytes(T, M, P) || !pods_aligned(workspace, 16))
        return PODS_ERR_WORKSPACE;
    unsigned char* const base = static_cast<unsigned char*>(workspace);
    double* const lse = reinterpret_cast<double*>(base);
    double* const logp64 = reinterpret_cast<double*>(base + up((size_t)T * 8));
    float* const dlogp = reinterpret_cast<float*>(base + 2 * up((size_t)T * 8));
    lay_out(&a, base + 2 * up((size_t)T * 8) + up((size_t)T * 4), M, P);
    cudaStream_t s = pods_stream(stream);
    if (T > 0) {
        pods_logp::FwdArgs f = {};
        f.logits = logits;
        f.ldl = ldl;
        f.tokens = tokens;
        f.mask = mask;
        f.rows_end = cu_seqlens + M;
        f.T = T;
        f.V = V;
        f.fill = 1;
        f.c64 = pods_logp::set_temperature(f, temperature);
        f.logp = logp;
        f.logp64 = logp64;
        f.lse = lse;
        f.status = status;
        rc = pods_logp::launch_forward(f, dtype, s);
        if (rc != PODS_OK) return rc;
    }
    a.logp = logp;
    a.logp64 = logp64;
    a.dlogp = dlogp;
    a.loss32 = loss;
    rc = launch_preference(a, s);
    if (rc != PODS_OK || T == 0) return rc;
    pods_logp::GradArgs g = {};
    g.logits = logits;
    g.ldl = ldl;
    g.tokens = tokens;
    g.lse = lse;
    g.dlogp = dlogp;
    g.T = T;
    g.V = V;
    pods_logp::set_temperature(g, temperature);
    g.dlogits = dlogits;
    g.ldd = ldd;
    g.status = status;
    return pods_logp::launch_gradient(g, dtype, s);
}
