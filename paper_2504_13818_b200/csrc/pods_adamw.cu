// pods_grad_norm - the 2-norm over many tensors; pods_adamw - a step of the optimiser over many tensors at once.
//
// One launch walks a table of tensors that travels as a kernel argument (no device table to keep in step with the tensors,
// nothing uploaded, the addresses are those of the call): tiles of kTile elements, numbered through the tensors.
//
// States in 8 bits: blocks of 32 elements under one power of two, the smallest that keeps the block within 448, each element an
// e4m3 number (4 significant bits, 2^-9 to 448).  Of the second moment its root is held, which halves the range of its
// exponents.  Rounding to a neighbour is decided by 16 random bits: to the nearest, an average that moves by 1 - beta a step
// (0.1 to 5 %, half a step of the format is 3 to 6 %) would stay where it is.  A root above 0 is never rounded to 0, which would
// let the element's next step be its first moment over eps.
//
// Bound: HBM, each tensor read and written once; 12.1 bytes an element for bf16 weights, fp32 gradients, 8-bit states, 28 for fp32
// weights with a bf16 copy, bf16 gradients, fp32 states.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <float.h>
#include <math.h>

#include "pods_common.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;
constexpr int kTile = kThreads * 4 * kUnroll;          // elements; a multiple of 32

struct Tensor {
    void* p;
    const void* g;
    void* m;
    void* v;
    uint8_t* m_scale;
    uint8_t* v_scale;
    void* copy;
    int64_t n, first;                  // elements; the number of the first one among all of the call
    uint32_t tile0;                    // tiles of this launch ahead of it
    uint8_t p_type, g_type, copy_type, bits, aligned;
    float decay, lr_scale;
};

template <int N>
struct Table {
    int count;
    uint32_t tiles;
    Tensor t[N];
};

// A kernel argument may hold 32764 bytes; most sets of tensors need few entries, and an argument costs its upload.
constexpr int kFew = 40, kMany = 320;
static_assert(sizeof(Table<kMany>) < 32000, "a kernel argument");

struct Step {
    float lr, beta1, beta2, eps, grad_scale, max_norm;
    double bias1, bias2;               // 1 - beta^step, where step_dev is NULL
    const float* lr_dev;
    const int64_t* step_dev;
    int64_t step;
    const float* norm;
    uint64_t seed;
    int stochastic;
    uint32_t* status;
};

// 32 bits to 32 bits, one to one: an input bit turns every output bit in half of the cases (measured over 2^17 inputs: mean
// square deviation 1.9e-6, that of coin tosses).
__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x888ec647u;
    x ^= x >> 15;
    x *= 0x246ce511u;
    return x ^ (x >> 16);
}

template <int N>
__device__ __forceinline__ const Tensor& tensor_of(const Table<N>& tab, uint32_t tile) {
    int lo = 0, hi = tab.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.t[mid].tile0 <= tile) lo = mid;
        else hi = mid - 1;
    }
    return tab.t[lo];
}

// Four elements as they lie in memory.
struct Raw4 {
    uint4 w;
};
__device__ __forceinline__ Raw4 load4(const void* base, int type, int64_t i) {
    Raw4 r;
    if (type == PODS_DTYPE_F32) {
        r.w = *reinterpret_cast<const uint4*>(static_cast<const float*>(base) + i);
    } else {
        const uint2 h = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + i);
        r.w = make_uint4(h.x, h.y, 0, 0);
    }
    return r;
}
__device__ __forceinline__ float one(uint32_t bits, int type) {
    return type == PODS_DTYPE_BF16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half((unsigned short)bits));
}
__device__ __forceinline__ void to_floats(const Raw4& r, int type, float (&x)[4]) {
    if (type == PODS_DTYPE_F32) {
        x[0] = __uint_as_float(r.w.x);
        x[1] = __uint_as_float(r.w.y);
        x[2] = __uint_as_float(r.w.z);
        x[3] = __uint_as_float(r.w.w);
    } else {
        x[0] = one(r.w.x & 0xffffu, type);
        x[1] = one(r.w.x >> 16, type);
        x[2] = one(r.w.y & 0xffffu, type);
        x[3] = one(r.w.y >> 16, type);
    }
}
// Element by element: ends of a tensor, and tensors that do not lie on the vectors' boundaries.
__device__ __forceinline__ Raw4 gather4(const void* base, int type, int64_t i, int64_t n) {
    uint32_t x[4] = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) x[k] = type == PODS_DTYPE_F32 ? static_cast<const uint32_t*>(base)[i + k] : static_cast<const uint16_t*>(base)[i + k];
    Raw4 r;
    r.w = type == PODS_DTYPE_F32 ? make_uint4(x[0], x[1], x[2], x[3]) : make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, 0, 0);
    return r;
}
__device__ __forceinline__ Raw4 from_floats(const float (&x)[4], int type) {
    Raw4 r;
    if (type == PODS_DTYPE_F32) {
        r.w = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    } else if (type == PODS_DTYPE_BF16) {
        uint32_t a, b;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(a) : "f"(x[1]), "f"(x[0]));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b) : "f"(x[3]), "f"(x[2]));
        r.w = make_uint4(a, b, 0, 0);
    } else {
        const __half2 a = __floats2half2_rn(x[0], x[1]), b = __floats2half2_rn(x[2], x[3]);
        r.w = make_uint4(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b), 0, 0);
    }
    return r;
}
__device__ __forceinline__ void store4(void* base, int type, int64_t i, int64_t n, bool whole, const Raw4& r) {
    if (whole) {
        if (type == PODS_DTYPE_F32) *reinterpret_cast<uint4*>(static_cast<float*>(base) + i) = r.w;
        else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + i) = make_uint2(r.w.x, r.w.y);
        return;
    }
    const uint32_t x[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) {
            if (type == PODS_DTYPE_F32) static_cast<uint32_t*>(base)[i + k] = x[k];
            else static_cast<uint16_t*>(base)[i + k] = (uint16_t)(x[k >> 1] >> (16 * (k & 1)));
        }
}

// ---- e4m3 blocks ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void codes_to_floats(uint32_t codes, uint32_t scale, float (&x)[4]) {
    const float s = __uint_as_float(scale << 23);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const __half2 h = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> (16 * k)), __NV_E4M3));
        const float2 f = __half22float2(h);
        x[2 * k] = f.x * s;
        x[2 * k + 1] = f.y * s;
    }
}
// The smallest power of two 2^(k - 127), k >= 1, with top / 2^(k - 127) <= 448 = 1.75 * 2^8; 255 where top is no number.
__device__ __forceinline__ uint32_t block_scale(float top) {
    if (!(top <= FLT_MAX)) return 255u;
    return (uint32_t)max(1, (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8);
}
// |x| / 2^(k - 127) on e4m3's grid: numbers below 2^-6 gain 2^-6, after which 20 bits lie below the grid for all.
__device__ __forceinline__ uint32_t round_code(float y, uint32_t word) {
    const bool low = y < 0.015625f;
    const uint32_t b = __float_as_uint(low ? y + 0.015625f : y);
    return ((b + (word << 4) + 8u) >> 20) - (low ? 968u : 960u);
}

struct Coefs {
    float g, beta1, beta2, keep1, keep2, lr, step, root, eps;
};

// One element: m, v (or its root r) and p move on.
__device__ __forceinline__ void advance(const Coefs& c, float decay, float g, float& m, float& v, float& r, float& p) {
    g *= c.g;
    m = c.beta1 * m + c.keep1 * g;
    v = c.beta2 * v + c.keep2 * (g * g);
    r = sqrtf(v);
    p = p * decay - c.step * (m / (r * c.root + c.eps));
}

template <int BITS>
__device__ __forceinline__ void adamw_tile(const Tensor& t, uint32_t tile, const Step& a, const Coefs& c0, uint32_t key) {
    const int64_t base = (int64_t)(tile - t.tile0) * kTile;
    Coefs c = c0;
    c.step *= t.lr_scale;
    const float decay = 1.0f - c.lr * t.lr_scale * t.decay;
    Raw4 p[kUnroll], g[kUnroll], m[kUnroll], v[kUnroll];
    uint32_t ms[kUnroll], vs[kUnroll];
    const bool fast = t.aligned && base + kTile <= t.n;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t i = base + (int64_t)(u * kThreads + threadIdx.x) * 4;
        if (fast) {
            g[u] = load4(t.g, t.g_type, i);
            p[u] = load4(t.p, t.p_type, i);
            if (BITS == 32) {
                m[u] = load4(t.m, PODS_DTYPE_F32, i);
                v[u] = load4(t.v, PODS_DTYPE_F32, i);
            } else {
                m[u].w.x = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.m) + i);
                v[u].w.x = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.v) + i);
                ms[u] = t.m_scale[i >> 5];
                vs[u] = t.v_scale[i >> 5];
            }
        } else {
            g[u] = gather4(t.g, t.g_type, i, t.n);
            p[u] = gather4(t.p, t.p_type, i, t.n);
            if (BITS == 32) {
                m[u] = gather4(t.m, PODS_DTYPE_F32, i, t.n);
                v[u] = gather4(t.v, PODS_DTYPE_F32, i, t.n);
            } else {
                m[u].w.x = v[u].w.x = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i + k < t.n) {
                        m[u].w.x |= (uint32_t) static_cast<const uint8_t*>(t.m)[i + k] << (8 * k);
                        v[u].w.x |= (uint32_t) static_cast<const uint8_t*>(t.v)[i + k] << (8 * k);
                    }
                ms[u] = i < t.n ? t.m_scale[i >> 5] : 0;
                vs[u] = i < t.n ? t.v_scale[i >> 5] : 0;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t i = base + (int64_t)(u * kThreads + threadIdx.x) * 4;
        float pf[4], gf[4], mf[4], vf[4], rf[4];
        to_floats(g[u], t.g_type, gf);
        to_floats(p[u], t.p_type, pf);
        if (BITS == 32) {
            to_floats(m[u], PODS_DTYPE_F32, mf);
            to_floats(v[u], PODS_DTYPE_F32, vf);
        } else {
            codes_to_floats(m[u].w.x, ms[u], mf);
            codes_to_floats(v[u].w.x, vs[u], vf);
#pragma unroll
            for (int k = 0; k < 4; ++k) vf[k] *= vf[k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) advance(c, decay, gf[k], mf[k], vf[k], rf[k], pf[k]);
        uint32_t word[4];
        if (BITS == 8 || a.stochastic) {
            const uint64_t number = (uint64_t)(t.first + i);   // a multiple of 4: the four share the high word
            const uint32_t k32 = (uint32_t)(number >> 32) == 0 ? mix(key) : mix(key + (uint32_t)(number >> 32));
#pragma unroll
            for (int k = 0; k < 4; ++k) word[k] = mix(((uint32_t)number + k) ^ k32);
        }
        if (t.copy != nullptr) store4(t.copy, t.copy_type, i, t.n, fast, from_floats(pf, t.copy_type));
        if (a.stochastic && t.p_type == PODS_DTYPE_BF16) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (fabsf(pf[k]) <= FLT_MAX) pf[k] = __uint_as_float((__float_as_uint(pf[k]) + (word[k] & 0xffffu)) & 0xffff0000u);
        }
        store4(t.p, t.p_type, i, t.n, fast, from_floats(pf, t.p_type));
        if (BITS == 32) {
            store4(t.m, PODS_DTYPE_F32, i, t.n, fast, from_floats(mf, PODS_DTYPE_F32));
            store4(t.v, PODS_DTYPE_F32, i, t.n, fast, from_floats(vf, PODS_DTYPE_F32));
        } else {
            // the block's largest, over the eight lanes that hold it; a NaN stays one
            float mt = 0.0f, rt = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bool in = i + k < t.n;
                mt = in ? (fabsf(mf[k]) > mt || mf[k] != mf[k] ? fabsf(mf[k]) : mt) : mt;
                rt = in ? (rf[k] > rt || rf[k] != rf[k] ? rf[k] : rt) : rt;
            }
            uint32_t mb = __float_as_uint(mt), rb = __float_as_uint(rt);        // of numbers >= 0 and NaN the order is that of the bits
#pragma unroll
            for (int d = 4; d > 0; d >>= 1) {
                mb = max(mb, __shfl_xor_sync(PODS_FULL_MASK, mb, d));
                rb = max(rb, __shfl_xor_sync(PODS_FULL_MASK, rb, d));
            }
            const uint32_t mk = block_scale(__uint_as_float(mb)), rk = block_scale(__uint_as_float(rb));
            const float mi = __uint_as_float((254u - min(mk, 253u)) << 23), ri = __uint_as_float((254u - min(rk, 253u)) << 23);
            uint32_t mc = 0, rc = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t sign = (__float_as_uint(mf[k]) >> 24) & 0x80u;
                const uint32_t a8 = mk == 255u ? 0x7fu : round_code(fabsf(mf[k]) * mi, word[k] >> 16);
                uint32_t b8 = rk == 255u ? 0x7fu : round_code(rf[k] * ri, (word[k] * 0x9e3779b1u) >> 16);
                if (b8 == 0 && rf[k] > 0.0f) b8 = 1;
                mc |= (a8 | sign) << (8 * k);
                rc |= b8 << (8 * k);
            }
            if (fast) {
                *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.m) + i) = mc;
                *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + i) = rc;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i + k < t.n) {
                        static_cast<uint8_t*>(t.m)[i + k] = (uint8_t)(mc >> (8 * k));
                        static_cast<uint8_t*>(t.v)[i + k] = (uint8_t)(rc >> (8 * k));
                    }
            }
            if ((i & 31) == 0 && i < t.n) {
                t.m_scale[i >> 5] = (uint8_t)mk;
                t.v_scale[i >> 5] = (uint8_t)rk;
            }
        }
    }
}

template <int N>
__global__ void __launch_bounds__(kThreads) pods_adamw_kernel(const __grid_constant__ Table<N> tab, const Step a) {
    __shared__ double bias[2];
    __shared__ int64_t step_now;
    float clip = a.grad_scale;
    if (a.norm != nullptr) {
        const float norm = *a.norm;
        if (!(norm <= FLT_MAX)) {                      // NaN or inf: everything stays as it was
            if (blockIdx.x == 0 && threadIdx.x == 0) pods_raise(a.status, PODS_STATUS_NONFINITE_GRAD);
            return;
        }
        if (a.max_norm > 0.0f && norm > a.max_norm) clip *= a.max_norm / norm;
    }
    double b1 = a.bias1, b2 = a.bias2;
    int64_t step = a.step;
    if (a.step_dev != nullptr) {
        if (threadIdx.x == 0) {
            const double n = (double)max(*a.step_dev, (int64_t)1);
            step_now = *a.step_dev;
            bias[0] = -expm1(n * log((double)a.beta1));
            bias[1] = -expm1(n * log((double)a.beta2));
        }
        __syncthreads();
        b1 = bias[0];
        b2 = bias[1];
        step = step_now;
    }
    Coefs c;
    c.g = clip;
    c.beta1 = a.beta1;
    c.beta2 = a.beta2;
    c.keep1 = (float)(1.0 - (double)a.beta1);
    c.keep2 = (float)(1.0 - (double)a.beta2);
    c.lr = a.lr_dev != nullptr ? *a.lr_dev : a.lr;
    c.step = (float)((double)c.lr / b1);
    c.root = (float)(1.0 / sqrt(b2));
    c.eps = a.eps;
    const uint32_t key = mix(mix(mix((uint32_t)a.seed + 0x9e3779b9u) ^ (uint32_t)(a.seed >> 32)) ^ (uint32_t)step);
    for (uint32_t tile = blockIdx.x; tile < tab.tiles; tile += gridDim.x) {
        const Tensor& t = tensor_of(tab, tile);
        if (t.bits == 32) adamw_tile<32>(t, tile, a, c, key);
        else adamw_tile<8>(t, tile, a, c, key);
    }
}

// ---- norm -------------------------------------------------------------------------------------------------------------
// Squares of four in fp32, everything beyond in fp64; where a sum of four leaves the middle of fp32's range its squares are
// taken again in fp64, so that neither large nor small gradients are lost.
template <int N>
__global__ void __launch_bounds__(kThreads) pods_grad_norm_kernel(const __grid_constant__ Table<N> tab, double* parts) {
    double sum = 0.0;
    for (uint32_t tile = blockIdx.x; tile < tab.tiles; tile += gridDim.x) {
        const Tensor& t = tensor_of(tab, tile);
        const int64_t base = (int64_t)(tile - t.tile0) * kTile;
        Raw4 g[kUnroll];
        const bool fast = t.aligned && base + kTile <= t.n;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t i = base + (int64_t)(u * kThreads + threadIdx.x) * 4;
            g[u] = fast ? load4(t.g, t.g_type, i) : gather4(t.g, t.g_type, i, t.n);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float x[4];
            to_floats(g[u], t.g_type, x);
            const float q = (x[0] * x[0] + x[1] * x[1]) + (x[2] * x[2] + x[3] * x[3]);
            if (q > 1e-24f && q < 1e38f) sum += (double)q;
            else
#pragma unroll
                for (int k = 0; k < 4; ++k) sum += (double)x[k] * (double)x[k];
        }
    }
    __shared__ double scratch[kThreads / 32];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(PODS_FULL_MASK, sum, d);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) sum += scratch[w];
        parts[blockIdx.x] = sum;
    }
}

__global__ void __launch_bounds__(1024) norm_finish_kernel(const double* parts, int n, float scale, float* norm, uint32_t* status) {
    __shared__ double scratch[32];
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += 1024) sum += parts[i];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(PODS_FULL_MASK, sum, d);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 32; ++w) sum += scratch[w];
        const float r = (float)(sqrt(sum) * fabs((double)scale));
        *norm = r;
        if (!(r <= FLT_MAX)) pods_raise(status, PODS_STATUS_NONFINITE_GRAD);
    }
}

size_t esize(int type) { return type == PODS_DTYPE_F32 ? 4 : 2; }
bool known(int type) { return type == PODS_DTYPE_BF16 || type == PODS_DTYPE_F16 || type == PODS_DTYPE_F32; }

constexpr int64_t kMostElements = (int64_t)1 << 42;   // of a call: 2^30 tiles

int check_table(const pods_adamw_tensor* t, int32_t n, bool all) {
    if (n < 0 || (n > 0 && t == nullptr)) return PODS_ERR_INVALID_ARG;
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
        const pods_adamw_tensor& x = t[i];
        if (!known(x.grad_type) || (all && !known(x.param_type))) return PODS_ERR_UNSUPPORTED;
        if (all && x.state_bits != 8 && x.state_bits != 32) return PODS_ERR_UNSUPPORTED;
        if (all && x.copy != nullptr && !known(x.copy_type)) return PODS_ERR_UNSUPPORTED;
        if (x.n < 0) return PODS_ERR_INVALID_ARG;
        if (x.n > kMostElements || (total += x.n) > kMostElements) return PODS_ERR_UNSUPPORTED;
        if (x.n == 0) continue;
        if (x.grad == nullptr || !pods_aligned(x.grad, esize(x.grad_type))) return PODS_ERR_INVALID_ARG;
        if (!all) continue;
        if (x.param == nullptr || x.m == nullptr || x.v == nullptr || !pods_aligned(x.param, esize(x.param_type)) ||
            (x.copy != nullptr && !pods_aligned(x.copy, esize(x.copy_type))))
            return PODS_ERR_INVALID_ARG;
        if (x.state_bits == 32 ? !pods_all_aligned(4, x.m, x.v) : x.m_scale == nullptr || x.v_scale == nullptr) return PODS_ERR_INVALID_ARG;
        if (!(x.weight_decay >= 0.0f && x.weight_decay <= FLT_MAX) || !(x.lr_scale >= 0.0f && x.lr_scale <= FLT_MAX)) return PODS_ERR_INVALID_ARG;
    }
    return PODS_OK;
}

// Tiles of tensors [from, ...) into the table until it is full; returns the first tensor left, and the element count ahead of it.
template <int N>
int fill(Table<N>& tab, const pods_adamw_tensor* t, int from, int n, int64_t& first) {
    tab.count = 0;
    uint64_t tiles = 0;
    int i = from;
    for (; i < n && tab.count < N; ++i) {
        const pods_adamw_tensor& x = t[i];
        if (x.n == 0) continue;
        const uint64_t mine = (uint64_t)((x.n + kTile - 1) / kTile);
        Tensor& d = tab.t[tab.count++];
        d = {x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.n, first, (uint32_t)tiles,
             (uint8_t)x.param_type, (uint8_t)x.grad_type, (uint8_t)x.copy_type, (uint8_t)x.state_bits, 0, x.weight_decay, x.lr_scale};
        const size_t state = x.state_bits == 32 ? 16 : 4;
        d.aligned = pods_aligned(x.grad, 4 * esize(x.grad_type)) &&
                    (x.param == nullptr || (pods_aligned(x.param, 4 * esize(x.param_type)) && pods_all_aligned(state, x.m, x.v) &&
                                            pods_aligned(x.copy, x.copy == nullptr ? 1 : 4 * esize(x.copy_type))));
        tiles += mine;
        first += (x.n + 31) / 32 * 32;
    }
    tab.tiles = (uint32_t)tiles;
    return i;
}

constexpr int kNormParts = 148 * 8;    // CTAs of the norm at most; their sums are joined by one

template <int N>
int norm_launches(const pods_adamw_tensor* t, int32_t n, double* parts, int& used, cudaStream_t s) {
    static Table<N> zero;                              // entries that stay unused are copied too
    int64_t first = 0;
    for (int from = 0; from < n;) {
        Table<N> tab = zero;
        from = fill(tab, t, from, n, first);
        if (tab.count == 0) continue;
        const unsigned grid = tab.tiles < (uint32_t)kNormParts ? tab.tiles : (uint32_t)kNormParts;
        pods_grad_norm_kernel<N><<<grid, kThreads, 0, s>>>(tab, parts + used);
        PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
        used += (int)grid;
    }
    return PODS_OK;
}

template <int N>
int adamw_launches(const pods_adamw_tensor* t, int32_t n, const Step& a, cudaStream_t s) {
    static Table<N> zero;
    int64_t first = 0;
    for (int from = 0; from < n;) {
        Table<N> tab = zero;
        from = fill(tab, t, from, n, first);
        if (tab.count == 0) continue;
        pods_adamw_kernel<N><<<tab.tiles, kThreads, 0, s>>>(tab, a);
        PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
    }
    return PODS_OK;
}

}  // namespace

extern "C" size_t pods_grad_norm_workspace_bytes(int32_t n) {
    return n < 0 ? 0 : (size_t)(n / kMany + 2) * kNormParts * sizeof(double);
}

extern "C" int pods_grad_norm(const pods_adamw_tensor* tensors, int32_t n, float scale, float* norm, void* workspace,
                              size_t workspace_bytes, uint32_t* status, void* stream) {
    const int rc = check_table(tensors, n, false);
    if (rc != PODS_OK) return rc;
    if (norm == nullptr || !pods_all_aligned(4, norm, status) || scale - scale != 0.0f) return PODS_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < pods_grad_norm_workspace_bytes(n) || !pods_aligned(workspace, 8)) return PODS_ERR_WORKSPACE;
    cudaStream_t s = pods_stream(stream);
    double* const parts = static_cast<double*>(workspace);
    int used = 0;
    const int e = n <= kFew ? norm_launches<kFew>(tensors, n, parts, used, s) : norm_launches<kMany>(tensors, n, parts, used, s);
    if (e != PODS_OK) return e;
    norm_finish_kernel<<<1, 1024, 0, s>>>(parts, used, scale, norm, status);
    PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
    return PODS_OK;
}

extern "C" int pods_adamw(const pods_adamw_tensor* tensors, int32_t n, int64_t step, const int64_t* step_dev, float lr,
                          const float* lr_dev, float beta1, float beta2, float eps, float grad_scale, const float* norm,
                          float max_norm, uint32_t flags, uint64_t seed, uint32_t* status, void* stream) {
    const int rc = check_table(tensors, n, true);
    if (rc != PODS_OK) return rc;
    if ((flags & ~PODS_ADAMW_STOCHASTIC) != 0) return PODS_ERR_UNSUPPORTED;
    if ((step_dev == nullptr && step < 1) || (lr_dev == nullptr && lr - lr != 0.0f) || !(beta1 >= 0.0f && beta1 < 1.0f) ||
        !(beta2 >= 0.0f && beta2 < 1.0f) || !(eps >= 0.0f && eps <= FLT_MAX) || grad_scale - grad_scale != 0.0f ||
        !(max_norm >= 0.0f) || (max_norm > 0.0f && norm == nullptr) || !pods_all_aligned(4, lr_dev, norm, status) ||
        !pods_aligned(step_dev, 8))
        return PODS_ERR_INVALID_ARG;
    Step a = {};
    a.lr = lr;
    a.beta1 = beta1;
    a.beta2 = beta2;
    a.eps = eps;
    a.grad_scale = grad_scale;
    a.max_norm = max_norm;
    a.step = step;
    a.step_dev = step_dev;
    a.lr_dev = lr_dev;
    if (step_dev == nullptr) {
        a.bias1 = -expm1((double)step * log((double)beta1));
        a.bias2 = -expm1((double)step * log((double)beta2));
    }
    a.norm = norm;
    a.seed = seed;
    a.stochastic = (flags & PODS_ADAMW_STOCHASTIC) ? 1 : 0;
    a.status = status;
    cudaStream_t s = pods_stream(stream);
    return n <= kFew ? adamw_launches<kFew>(tensors, n, a, s) : adamw_launches<kMany>(tensors, n, a, s);
}
