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
constexpr int kTile = kThreads * 8;                    // elements, eight a thread; a multiple of 32
constexpr int kMostCtas = 148 * 4;                     // of a launch; each takes one run of consecutive tiles
constexpr int kMostNormCtas = 148 * 6;

struct Tensor32 {
    void* p;
    const void* g;
    void* m;
    void* v;
    void* copy;
    int64_t n, first;                  // elements; the number of the first one among all of the call
    uint32_t tile0;                    // tiles of this launch ahead of it
    uint8_t copy_type;
    uint8_t vectors;                   // 2: eight elements of every buffer lie on their boundary (32 bytes of fp32), 1: 16 bytes, 0: neither
    float decay, lr_scale;
};
struct Tensor8 : Tensor32 {
    uint8_t* m_scale;
    uint8_t* v_scale;
};
struct TensorG {                       // of the norm
    const void* g;
    int64_t n;
    uint32_t tile0;
    uint8_t g_type, vectors;
};

// The launch's tensors, and the tensor in which each CTA's run of tiles begins: a search in a table of this size would cost a CTA
// several misses of the constant cache, one after the other (a norm over 217 tensors: 183 us with it).
template <typename E, int N, int CTAS>
struct Table {
    using Entry = E;
    static constexpr int most = N;
    int count;
    uint32_t tiles;
    uint16_t start[CTAS];
    E t[N];
};

// A kernel argument may hold 32764 bytes; most sets of tensors need few entries, and an argument costs its upload.
constexpr int kFew = 24;
using Few8 = Table<Tensor8, kFew, kMostCtas>;
using Many8 = Table<Tensor8, 352, kMostCtas>;
using Few32 = Table<Tensor32, kFew, kMostCtas>;
using Many32 = Table<Tensor32, 432, kMostCtas>;
using FewG = Table<TensorG, kFew, kMostNormCtas>;
using ManyG = Table<TensorG, 1248, kMostNormCtas>;
static_assert(sizeof(Many8) < 32500 && sizeof(Many32) < 32500 && sizeof(ManyG) < 32700, "a kernel argument");

struct Step {
    float lr, beta1, beta2, eps, grad_scale, max_norm;
    double bias1, bias2;               // 1 - beta^step, where step_dev is NULL
    const float* lr_dev;
    const int64_t* step_dev;
    int64_t step;
    const float* norm;
    uint64_t seed;
    int stochastic;
    uint32_t least_ms, least_vs, fold_vs;  // block scales that may go into the betas: from least_ms on; fold_vs from least_vs on
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

// Eight elements as they lie in memory; 16-bit types use the first half.
struct Raw8 {
    uint32_t w[8];
};
__device__ __forceinline__ Raw8 load8(const void* base, int type, uint32_t i, int vectors) {
    Raw8 r = {};
    if (type == PODS_DTYPE_F32) {
        const float* at = static_cast<const float*>(base) + i;
        if (vectors == 2) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7]) : "l"(at));
        } else {
            const uint4 a = reinterpret_cast<const uint4*>(at)[0], b = reinterpret_cast<const uint4*>(at)[1];
            r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
            r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
        }
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + i);
        r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
    }
    return r;
}
// Element by element, the first n of eight: ends of a tensor, and tensors that do not lie on the vectors' boundaries.
__device__ __forceinline__ Raw8 gather8(const void* base, int type, uint32_t i, int n) {
    Raw8 r = {};
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) {
            if (type == PODS_DTYPE_F32) r.w[k] = static_cast<const uint32_t*>(base)[i + k];
            else r.w[k >> 1] |= (uint32_t) static_cast<const uint16_t*>(base)[i + k] << (16 * (k & 1));
        }
    return r;
}
__device__ __forceinline__ void to_floats(const Raw8& r, int type, float (&x)[8]) {
    if (type == PODS_DTYPE_F32) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(r.w[k]);
    } else if (type == PODS_DTYPE_BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[2 * k] = __uint_as_float(r.w[k] << 16);
            x[2 * k + 1] = __uint_as_float(r.w[k] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r.w[k]));
            x[2 * k] = f.x;
            x[2 * k + 1] = f.y;
        }
    }
}
__device__ __forceinline__ Raw8 from_floats(const float (&x)[8], int type) {
    Raw8 r = {};
    if (type == PODS_DTYPE_F32) {
#pragma unroll
        for (int k = 0; k < 8; ++k) r.w[k] = __float_as_uint(x[k]);
    } else if (type == PODS_DTYPE_BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w[k]) : "f"(x[2 * k + 1]), "f"(x[2 * k]));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __half2 h = __floats2half2_rn(x[2 * k], x[2 * k + 1]);
            r.w[k] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return r;
}
__device__ __forceinline__ void store8(void* base, int type, uint32_t i, int n, int vectors, const Raw8& r) {
    if (vectors) {
        if (type == PODS_DTYPE_F32) {
            float* at = static_cast<float*>(base) + i;
            if (vectors == 2) {
                asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                             ::"r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]), "l"(at) : "memory");
            } else {
                reinterpret_cast<uint4*>(at)[0] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
                reinterpret_cast<uint4*>(at)[1] = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
            }
        } else {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + i) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) {
            if (type == PODS_DTYPE_F32) static_cast<uint32_t*>(base)[i + k] = r.w[k];
            else static_cast<uint16_t*>(base)[i + k] = (uint16_t)(r.w[k >> 1] >> (16 * (k & 1)));
        }
}

// ---- e4m3 blocks: a block of 32 is held by four lanes -----------------------------------------------------------------------
__device__ __forceinline__ uint2 gather_codes(const void* base, uint32_t i, int n) {
    const uint8_t* at = static_cast<const uint8_t*>(base) + i;
    uint2 r = make_uint2(0, 0);
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) (k < 4 ? r.x : r.y) |= (uint32_t)at[k] << (8 * (k & 3));
    return r;
}
__device__ __forceinline__ void store_codes(void* base, uint32_t i, int n, bool fast, uint2 c) {
    uint8_t* at = static_cast<uint8_t*>(base) + i;
    if (fast) {
        *reinterpret_cast<uint2*>(at) = c;
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) at[k] = (uint8_t)((k < 4 ? c.x : c.y) >> (8 * (k & 3)));
}
// Eight codes as numbers, without their block's scale.
__device__ __forceinline__ void codes_to_floats(uint2 codes, float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t two = (k < 2 ? codes.x : codes.y) >> (16 * (k & 1));
        const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3)));
        x[2 * k] = f.x;
        x[2 * k + 1] = f.y;
    }
}
// The largest |x| of eight, NaN if one of them is.
__device__ __forceinline__ float largest8(const float (&x)[8]) {
    float a, b;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(x[0]), "f"(x[1]), "f"(x[2]));
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(b) : "f"(x[3]), "f"(x[4]), "f"(x[5]));
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(a), "f"(x[6]), "f"(x[7]));
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(a), "f"(b), "f"(b));
    return a;
}
// The smallest k >= 1 with top / 2^(k - 127) <= 448 = 1.75 * 2^8; 255 where top is no number.
__device__ __forceinline__ uint32_t block_scale(float top) {
    const uint32_t b = __float_as_uint(top) & 0x7fffffffu;
    return b >= 0x7f800000u ? 255u : (uint32_t)max(1, (int)((b + 0x1fffffu) >> 23) - 8);
}
// Two fp32 numbers an instruction.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Codes of eight numbers in a block of scale k.  A number times 2^(127 - k) 2^-120 has e4m3's exponent where fp32 keeps its
// own, and e4m3's smallest numbers are fp32's: for all of them the code lies above the lowest 20 bits, and 16 random bits and a
// half (a number that is on the grid stays) added there carry into it with the probability that keeps the average.  Four bits
// further up the code is the highest byte: one multiply-add makes it, and bytes are picked, so that the integer pipe has little to
// do.  The 16 random bits go to bytes 1 and 2, the half to byte 0.
template <bool ROOT>
__device__ __forceinline__ uint2 to_codes(float (&x)[8], uint32_t k, const uint32_t (&word)[8]) {
    float f = __uint_as_float((134u - k) << 23);
    if (k > 133u) {                                    // 2^(7 - k) is no normal number: blocks above 28672, in two factors; NaN
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= 0x1p-120f;
        f = __uint_as_float((254u - min(k, 253u)) << 23);
    }
    uint32_t c[8];
    const uint64_t f2 = ROOT ? pair(-f, -f) : pair(f, f);                               // roots come with their sign turned
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float y[2];
        unpair(mul2(pair(x[i], x[i + 1]), f2), y[0], y[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (ROOT) y[h] = fmaxf(y[h], 0x1p-129f);   // the smallest code; a root of 0 is put right by the caller
            const uint32_t w = ROOT ? word[i + h] * 0x9e3779b1u : word[i + h];
            c[i + h] = __float_as_uint(y[h]) * 16u + __byte_perm(w, 0x80u, 0x7324);
            if (!ROOT) c[i + h] |= __float_as_uint(y[h]) & 0x80000000u;
        }
    }
    uint2 r;
    r.x = __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410);
    r.y = __byte_perm(__byte_perm(c[4], c[5], 0x0073), __byte_perm(c[6], c[7], 0x0073), 0x5410);
    if (k == 255u) r = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
    return r;
}

__device__ __forceinline__ float rsqrt_fast(float x) {
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// a + b, two numbers at a time but one by one: ptxas makes a fused product and sum of mul.rn.f32x2 and add.rn.f32x2, though both
// name their rounding (a quarter of the sums differed in the last bit).
__device__ __forceinline__ void sums(uint64_t a, uint64_t b, float& lo, float& hi) {
    float al, ah, bl, bh;
    unpair(a, al, ah);
    unpair(b, bl, bh);
    lo = __fadd_rn(al, bl);
    hi = __fadd_rn(ah, bh);
}
// off by 2^-23 at most; numbers below the normal ones are 0 to it, so that eps is 0 or one that leaves it none
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
struct Coefs {
    float g, beta1, beta2, keep1, keep2, lr, step, root, eps;
};

// A thread's eight elements of a tile, and what they are stored with.
template <int BITS>
struct Loaded {
    Raw8 g, p, m, v;
    uint2 mc, vc;
    uint32_t ms, vs;
};

// `off`: elements into the stretch; left: elements of the tensor from the tile's first on.  PT, GT: types of parameter and gradient.
// FAST: whole tiles of tensors on the vectors' boundaries (those with 8-bit states go through shared memory, see ask_tile).
template <int PT, int GT, int BITS, bool FAST>
__device__ __forceinline__ void load_tile(Loaded<BITS>& d, const Tensor8& at, int vectors, uint32_t off, int left) {
    static_assert(BITS == 32 || !FAST);
    const int n = FAST ? 8 : left - (int)threadIdx.x * 8;         // the thread's elements and those behind
    constexpr bool fast = FAST;
    if (fast) {
        d.g = load8(at.g, GT, off, vectors);
        d.p = load8(at.p, PT, off, vectors);
    } else {
        d.g = gather8(at.g, GT, off, n);
        d.p = gather8(at.p, PT, off, n);
    }
    if (BITS == 32) {
        d.m = fast ? load8(at.m, PODS_DTYPE_F32, off, vectors) : gather8(at.m, PODS_DTYPE_F32, off, n);
        d.v = fast ? load8(at.v, PODS_DTYPE_F32, off, vectors) : gather8(at.v, PODS_DTYPE_F32, off, n);
    } else {
        d.mc = gather_codes(at.m, off, n);
        d.vc = gather_codes(at.v, off, n);
        d.ms = n > 0 ? at.m_scale[off >> 5] : 0;
        d.vs = n > 0 ? at.v_scale[off >> 5] : 0;
    }
}

// What the threads of a CTA have on its way to shared memory for a whole tile; each thread reads only what it asked for itself.
template <int PT, int GT>
struct Ahead {
    static constexpr int gv = GT == PODS_DTYPE_F32 ? 2 : 1, pv = PT == PODS_DTYPE_F32 ? 2 : 1;
    uint4 g[gv][kThreads], p[pv][kThreads];
    uint2 m[kThreads], v[kThreads];
};
template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "n"(BYTES) : "memory");
}
template <int PT, int GT>
__device__ __forceinline__ void ask_tile(Ahead<PT, GT>& d, const Tensor8& at, uint32_t off) {
    const char* const g = static_cast<const char*>(at.g) + (size_t)off * (GT == PODS_DTYPE_F32 ? 4 : 2);
    const char* const p = static_cast<const char*>(at.p) + (size_t)off * (PT == PODS_DTYPE_F32 ? 4 : 2);
#pragma unroll
    for (int k = 0; k < Ahead<PT, GT>::gv; ++k) copy_async<16>(&d.g[k][threadIdx.x], g + 16 * k);
#pragma unroll
    for (int k = 0; k < Ahead<PT, GT>::pv; ++k) copy_async<16>(&d.p[k][threadIdx.x], p + 16 * k);
    copy_async<8>(&d.m[threadIdx.x], static_cast<const uint8_t*>(at.m) + off);
    copy_async<8>(&d.v[threadIdx.x], static_cast<const uint8_t*>(at.v) + off);
}
template <int PT, int GT>
__device__ __forceinline__ void take_tile(Loaded<8>& x, const Ahead<PT, GT>& d) {
#pragma unroll
    for (int k = 0; k < Ahead<PT, GT>::gv; ++k) {
        const uint4 q = d.g[k][threadIdx.x];
        x.g.w[4 * k] = q.x; x.g.w[4 * k + 1] = q.y; x.g.w[4 * k + 2] = q.z; x.g.w[4 * k + 3] = q.w;
    }
#pragma unroll
    for (int k = 0; k < Ahead<PT, GT>::pv; ++k) {
        const uint4 q = d.p[k][threadIdx.x];
        x.p.w[4 * k] = q.x; x.p.w[4 * k + 1] = q.y; x.p.w[4 * k + 2] = q.z; x.p.w[4 * k + 3] = q.w;
    }
    x.mc = d.m[threadIdx.x];
    x.vc = d.v[threadIdx.x];
}

template <int PT, int GT, int BITS, bool FAST>
__device__ __forceinline__ void adamw_tile(const Loaded<BITS>& d, const Tensor32& t, const Tensor8& at, uint32_t off, int left, const Step& a,
                                           const Coefs& c, float decay, float rate, uint64_t first, uint32_t key) {
    const int vectors = FAST ? t.vectors : 0;
    constexpr bool fast = FAST;
    const int n = FAST ? 8 : left - (int)threadIdx.x * 8;
    float pf[8], gf[8], mf[8], vf[8], rf[8];
    to_floats(d.g, GT, gf);
    to_floats(d.p, PT, pf);
    if (BITS == 32) {
        to_floats(d.m, PODS_DTYPE_F32, mf);
        to_floats(d.v, PODS_DTYPE_F32, vf);
    } else {
        codes_to_floats(d.mc, mf);
        codes_to_floats(d.vc, vf);
    }
    // the blocks' scales, powers of two, go into the betas: the same numbers as if they had gone into the codes, as long as the square
    // of the second and both products are normal numbers
    float b1 = c.beta1, b2 = c.beta2;
    if (BITS == 8) {
        const float s1 = __uint_as_float(d.ms << 23), s2 = __uint_as_float(d.vs << 23);
        if (d.ms >= a.least_ms && d.vs - a.least_vs < a.fold_vs) {
            b1 *= s1;
            b2 *= s2 * s2;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                mf[k] *= s1;
                vf[k] *= s2;
            }
        }
    }
    // The moments are those of fp32 products and sums, each rounded by itself: what an 8-bit state is rounded to then depends on
    // nothing but these, for a fused product would turn one code in a million, and with it the element's next step.  Their root by a
    // Newton step, r - (r^2 - v) / (2 r), from r = v rsqrt(v), whose error of 2^-22 goes to 2^-45: the nearest number, or, less than
    // once in a million, the one next to it, which turns a code once in a million of these; all of it with v's and r's signs turned,
    // which saves the negations.
    const uint64_t c_g = pair(c.g, c.g), beta1 = pair(b1, b1), keep1 = pair(c.keep1, c.keep1), minus_beta2 = pair(-b2, -b2),
                   minus_keep2 = pair(-c.keep2, -c.keep2), minus_root = pair(-c.root, -c.root), eps = pair(c.eps, c.eps), shrink = pair(decay, decay),
                   minus = pair(-rate, -rate), half = pair(0.5f, 0.5f);
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const uint64_t x = mul2(pair(gf[k], gf[k + 1]), c_g);
        uint64_t w = pair(vf[k], vf[k + 1]);
        if (BITS == 8) w = mul2(w, w);
        sums(mul2(beta1, pair(mf[k], mf[k + 1])), mul2(keep1, x), mf[k], mf[k + 1]);
        sums(mul2(minus_beta2, w), mul2(minus_keep2, mul2(x, x)), vf[k], vf[k + 1]);     // -v
        const uint64_t v2 = pair(vf[k], vf[k + 1]);
        const uint64_t y = pair(rsqrt_fast(-vf[k]), rsqrt_fast(-vf[k + 1])), r = mul2(v2, y);
        unpair(fma2(fma2(r, r, v2), mul2(half, y), r), rf[k], rf[k + 1]);               // -r
    }
    // no root came of a v of 0 (elements that never had a gradient, mostly), below the normal numbers, infinite or NaN.  311 M weights
    // with 8-bit states, fp32 gradients: 698 us without such elements, 876 with nine rows in ten of them; 32-bit states 1394 : 1400.
    float top = largest8(rf);
    const bool odd = !(top <= FLT_MAX);
    if (odd) {
#pragma unroll
        for (int k = 0; k < 8; ++k) rf[k] = -sqrtf(-vf[k]);
        top = largest8(rf);
    }
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        float d0, d1;
        unpair(fma2(pair(rf[k], rf[k + 1]), minus_root, eps), d0, d1);
        const uint64_t u = mul2(pair(mf[k], mf[k + 1]), pair(rcp_fast(d0), rcp_fast(d1)));
        unpair(fma2(minus, u, mul2(pair(pf[k], pf[k + 1]), shrink)), pf[k], pf[k + 1]);
    }
    // words = mix(number ^ k32), number a multiple of 8 for the first: the eight share the high word and the mix's first step
    uint32_t word[8];
    if (BITS == 8 || a.stochastic) {
        const uint64_t number = first + off;
        uint32_t x0 = (uint32_t)number ^ mix(key + (uint32_t)(number >> 32));
        x0 ^= x0 >> 16;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            uint32_t x = (x0 ^ k) * 0x888ec647u;
            x = (x ^ (x >> 15)) * 0x246ce511u;
            word[k] = x ^ (x >> 16);
        }
    }
    if (at.copy != nullptr) store8(at.copy, t.copy_type, off, n, vectors, from_floats(pf, t.copy_type));
    if (PT == PODS_DTYPE_BF16 && a.stochastic) {
        if (largest8(pf) <= FLT_MAX) {
            Raw8 r = {};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                r.w[k] = __byte_perm(__float_as_uint(pf[2 * k]) + (word[2 * k] & 0xffffu), __float_as_uint(pf[2 * k + 1]) + (word[2 * k + 1] & 0xffffu), 0x7632);
            store8(at.p, PODS_DTYPE_BF16, off, n, vectors, r);
        } else {                                       // what is no number stays none
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (fabsf(pf[k]) <= FLT_MAX) pf[k] = __uint_as_float((__float_as_uint(pf[k]) + (word[k] & 0xffffu)) & 0xffff0000u);
            store8(at.p, PODS_DTYPE_BF16, off, n, vectors, from_floats(pf, PODS_DTYPE_BF16));
        }
    } else {
        store8(at.p, PT, off, n, vectors, from_floats(pf, PT));
    }
    if (BITS == 32) {
        store8(at.m, PODS_DTYPE_F32, off, n, vectors, from_floats(mf, PODS_DTYPE_F32));
#pragma unroll
        for (int k = 0; k < 8; ++k) vf[k] = -vf[k];
        store8(at.v, PODS_DTYPE_F32, off, n, vectors, from_floats(vf, PODS_DTYPE_F32));
        return;
    }
    if (!fast) {                                       // what lies behind the tensor's end counts nothing
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k >= n) mf[k] = rf[k] = 0.0f;
        top = largest8(rf);
    }
    uint32_t scales = block_scale(largest8(mf)) | block_scale(top) << 16;     // larger numbers have larger scales
    scales = __vmaxu2(scales, __shfl_xor_sync(PODS_FULL_MASK, scales, 1));
    scales = __vmaxu2(scales, __shfl_xor_sync(PODS_FULL_MASK, scales, 2));
    const uint32_t mk = scales & 0xffffu, rk = scales >> 16;
    uint32_t zero_x = 0, zero_y = 0;                   // bytes of the roots that are 0
    if (odd || !fast) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            zero_x |= rf[k] == 0.0f ? 0xffu << (8 * k) : 0u;
            zero_y |= rf[k + 4] == 0.0f ? 0xffu << (8 * k) : 0u;
        }
    }
    store_codes(at.m, off, n, fast, to_codes<false>(mf, mk, word));
    uint2 rc = to_codes<true>(rf, rk, word);
    if (odd || !fast) {
        rc.x &= ~zero_x;
        rc.y &= ~zero_y;
    }
    store_codes(at.v, off, n, fast, rc);
    if ((threadIdx.x & 3) == 0 && n > 0) {
        at.m_scale[off >> 5] = (uint8_t)mk;
        at.v_scale[off >> 5] = (uint8_t)rk;
    }
}

// This CTA's run of tiles, a stretch of each tensor at a time: f(tensor, first element, tiles)
template <typename T, typename F>
__device__ __forceinline__ void each_stretch(const T& tab, uint32_t* status, F f) {
    const uint32_t lo = (uint32_t)((uint64_t)tab.tiles * blockIdx.x / gridDim.x);
    const uint32_t hi = (uint32_t)((uint64_t)tab.tiles * (blockIdx.x + 1) / gridDim.x);
    int i = tab.start[blockIdx.x];
    for (uint32_t tile = lo; tile < hi; ++i) {
        if (!PODS_INDEX_OK(i, tab.count, status)) return;
        const auto& t = tab.t[i];
        const uint32_t end = min(hi, i + 1 < tab.count ? tab.t[i + 1].tile0 : tab.tiles);
        if (PODS_INDEX_OK((int64_t)(end - 1 - t.tile0) * kTile, t.n, status)) f(t, (int64_t)(tile - t.tile0) * kTile, (int)(end - tile));
        tile = end;
    }
}

__device__ __forceinline__ size_t bytes_of(int type) { return type == PODS_DTYPE_F32 ? 4 : 2; }

constexpr int kCtas8 = 4, kCtas32 = 3;                 // an SM

// Eight consecutive elements a thread, since a block of 32 is then four lanes' (four: 2.1 ms), and a run of tiles a CTA, since the
// tensor is looked up once a stretch.  32-bit states: HBM bounds it, 1.42 ms of 303 M fp32 weights with bf16 copy and gradients
// (6.0 TB/s).  8-bit states: instruction issue (77 % of the cycles), 705 us of 311 M bf16 weights with fp32 gradients (5.35 TB/s), 658
// with bf16 gradients (4.8 TB/s); loads a tile ahead in registers took 731 where copies to shared memory took
// 701.
template <typename T, int PT, int GT, int BITS>
__global__ void __launch_bounds__(kThreads, BITS == 8 ? kCtas8 : kCtas32) pods_adamw_kernel(const __grid_constant__ T tab, const Step a) {
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
    each_stretch(tab, a.status, [&](const typename T::Entry& t, int64_t base, int tiles) {
        // the stretch's own addresses, so that offsets in it have 32 bits (at most 2^40 elements over the CTAs of a full grid)
        Tensor8 at;
        at.g = static_cast<const char*>(t.g) + base * bytes_of(GT);
        at.p = static_cast<char*>(t.p) + base * bytes_of(PT);
        at.m = static_cast<char*>(t.m) + base * (BITS == 32 ? 4 : 1);
        at.v = static_cast<char*>(t.v) + base * (BITS == 32 ? 4 : 1);
        if constexpr (BITS == 8) {
            at.m_scale = t.m_scale + (base >> 5);
            at.v_scale = t.v_scale + (base >> 5);
        }
        at.copy = t.copy == nullptr ? nullptr : static_cast<char*>(t.copy) + base * bytes_of(t.copy_type);
        const float decay = 1.0f - c.lr * t.lr_scale * t.decay, rate = c.step * t.lr_scale;
        // in registers: read from the table again for each tile they cost more than the arithmetic of an element
        if (BITS == 8) asm volatile("" : "+l"(at.g), "+l"(at.p), "+l"(at.m), "+l"(at.v));
        if (BITS == 8) asm volatile("" : "+l"(at.m_scale), "+l"(at.v_scale));
        const int64_t behind = t.n - base;
        const int whole = t.vectors ? (int)min((int64_t)tiles, behind / kTile) : 0;
        const uint64_t first = (uint64_t)(t.first + base);
        uint32_t off = threadIdx.x * 8;
        int k = 0;
        if constexpr (BITS == 8) {                     // the next tile is on its way while one is worked on
            extern __shared__ __align__(16) unsigned char smem[];
            Ahead<PT, GT>* const ahead = reinterpret_cast<Ahead<PT, GT>*>(smem);
            uint32_t ms = 0, vs = 0;
            if (whole > 0) {
                ask_tile(ahead[0], at, off);
                ms = at.m_scale[off >> 5];
                vs = at.v_scale[off >> 5];
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll 1
            for (; k < whole; ++k, off += kTile) {
                Loaded<8> x;
                x.ms = ms;
                x.vs = vs;
                if (k + 1 < whole) {
                    ask_tile(ahead[(k + 1) & 1], at, off + kTile);
                    ms = at.m_scale[(off + kTile) >> 5];
                    vs = at.v_scale[(off + kTile) >> 5];
                }
                asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 1;" ::: "memory");
                take_tile(x, ahead[k & 1]);
                adamw_tile<PT, GT, 8, true>(x, t, at, off, 0, a, c, decay, rate, first, key);
            }
        } else {
#pragma unroll 1
            for (; k < whole; ++k, off += kTile) {
                Loaded<BITS> x;
                load_tile<PT, GT, BITS, true>(x, at, t.vectors, off, 0);
                adamw_tile<PT, GT, BITS, true>(x, t, at, off, 0, a, c, decay, rate, first, key);
            }
        }
#pragma unroll 1
        for (; k < tiles; ++k, off += kTile) {
            const int left = (int)min((int64_t)kTile, behind - (int64_t)k * kTile);
            Loaded<BITS> x;
            load_tile<PT, GT, BITS, false>(x, at, 0, off, left);
            adamw_tile<PT, GT, BITS, false>(x, t, at, off, left, a, c, decay, rate, first, key);
        }
    });
}

// ---- norm -------------------------------------------------------------------------------------------------------------
// Squares and sums in fp64: exact but for 2^-53 a sum, whatever the gradients' size, so that the clipping factor does not depend on
// how they are grouped.  HBM bounds it: 1.24 GB of fp32 gradients in 189 us (6.6 TB/s); eight CTAs an SM instead of six 198 to 207 us.
template <typename T>
__global__ void __launch_bounds__(kThreads, 6) pods_grad_norm_kernel(const __grid_constant__ T tab, double* parts, uint32_t* status) {
    double s4[4] = {0.0, 0.0, 0.0, 0.0};
    auto add = [&](const Raw8& g, int type) {
        float x[8];
        to_floats(g, type, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) s4[k & 3] = fma((double)x[k], (double)x[k], s4[k & 3]);
    };
    each_stretch(tab, status, [&](const TensorG& t, int64_t base, int tiles) {
        const int type = t.g_type;
        const char* const at = static_cast<const char*>(t.g) + base * bytes_of(type);
        uint32_t i = threadIdx.x * 8;
        const int whole = t.vectors ? (int)min((int64_t)tiles, (t.n - base) / kTile) : 0;
        int k = 0;
        for (; k + 2 <= whole; k += 2, i += 2 * kTile) {
            Raw8 g[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) g[u] = load8(at, type, i + u * kTile, t.vectors);
#pragma unroll
            for (int u = 0; u < 2; ++u) add(g[u], type);
        }
        for (; k < whole; ++k, i += kTile) add(load8(at, type, i, t.vectors), type);
        for (; k < tiles; ++k, i += kTile) add(gather8(at, type, i, (int)max((int64_t)0, min((int64_t)8, t.n - base - i))), type);
    });
    double sum = (s4[0] + s4[1]) + (s4[2] + s4[3]);
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

constexpr int64_t kMostElements = (int64_t)1 << 40;   // of a call

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

// What a kernel is made for: the types of parameter and gradient, and the states' bits.
struct Kind {
    int p, g, bits;
    bool operator==(const Kind& o) const { return p == o.p && g == o.g && bits == o.bits; }
};
Kind kind_of(const pods_adamw_tensor& x) { return {x.param_type, x.grad_type, x.state_bits}; }

// The entry of a tensor but for its place in the table.
void enter(TensorG& d, const pods_adamw_tensor& x, int64_t) {
    d = {x.grad, x.n, 0, (uint8_t)x.grad_type, 0};
    for (int level = 1; level <= 2; ++level)
        if (pods_aligned(x.grad, x.grad_type == PODS_DTYPE_F32 ? 16 * level : 16)) d.vectors = (uint8_t)level;
}
void enter(Tensor32& d, const pods_adamw_tensor& x, int64_t first) {
    d = {x.param, x.grad, x.m, x.v, x.copy, x.n, first, 0, (uint8_t)x.copy_type, 0, x.weight_decay, x.lr_scale};
    for (int level = 1; level <= 2; ++level) {
        const size_t f = 16 * level;
        if (pods_aligned(x.grad, x.grad_type == PODS_DTYPE_F32 ? f : 16) && pods_aligned(x.param, x.param_type == PODS_DTYPE_F32 ? f : 16) &&
            pods_all_aligned(x.state_bits == 32 ? f : 8, x.m, x.v) &&
            (x.copy == nullptr || pods_aligned(x.copy, x.copy_type == PODS_DTYPE_F32 ? f : 16)))
            d.vectors = (uint8_t)level;
    }
}
void enter(Tensor8& d, const pods_adamw_tensor& x, int64_t first) {
    enter(static_cast<Tensor32&>(d), x, first);
    d.m_scale = x.m_scale;
    d.v_scale = x.v_scale;
}

// Tensors [from, ...) of a kind (of any, where none is given) into the table until it is full; returns the first tensor left.
// `first`: elements ahead of tensor `from` in the call.  The runs of tiles are for `grid` CTAs.
template <typename T>
int fill(T& tab, const pods_adamw_tensor* t, int from, int n, const Kind* kind, int most, int64_t& first, unsigned& grid) {
    tab.count = 0;
    uint32_t tiles = 0;
    int i = from;
    for (; i < n && tab.count < T::most; ++i) {
        const pods_adamw_tensor& x = t[i];
        if (x.n != 0 && (kind == nullptr || kind_of(x) == *kind)) {
            auto& d = tab.t[tab.count++];
            enter(d, x, first);
            d.tile0 = tiles;
            tiles += (uint32_t)((x.n + kTile - 1) / kTile);
        }
        first += (x.n + 31) / 32 * 32;
    }
    tab.tiles = tiles;
    grid = tiles < (uint32_t)most ? tiles : (unsigned)most;
    for (unsigned b = 0, at = 0; b < grid; ++b) {
        const uint32_t lo = (uint32_t)((uint64_t)tiles * b / grid);
        while ((int)at + 1 < tab.count && tab.t[at + 1].tile0 <= lo) ++at;
        tab.start[b] = (uint16_t)at;
    }
    return i;
}

int most_ctas(int per_sm, int most) {
    const int n = pods_sm_count() * per_sm;
    return n < most ? n : most;
}

template <typename T>
int norm_launches(const pods_adamw_tensor* t, int32_t n, double* parts, int& used, uint32_t* status, cudaStream_t s) {
    int64_t first = 0;
    for (int from = 0; from < n;) {
        T tab;
        unsigned grid;
        from = fill(tab, t, from, n, nullptr, most_ctas(6, kMostNormCtas), first, grid);
        if (tab.count == 0) continue;
        pods_grad_norm_kernel<<<grid, kThreads, 0, s>>>(tab, parts + used, status);
        PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
        used += (int)grid;
    }
    return PODS_OK;
}

template <typename T, int PT, int GT, int BITS>
void launch_kind(const T& tab, const Step& a, unsigned grid, cudaStream_t s) {
    pods_adamw_kernel<T, PT, GT, BITS><<<grid, kThreads, BITS == 8 ? 2 * sizeof(Ahead<PT, GT>) : 0, s>>>(tab, a);
}
template <typename T, int PT, int BITS>
void launch_kind(const T& tab, const Step& a, unsigned grid, cudaStream_t s, int g) {
    if (g == PODS_DTYPE_BF16) launch_kind<T, PT, PODS_DTYPE_BF16, BITS>(tab, a, grid, s);
    else if (g == PODS_DTYPE_F16) launch_kind<T, PT, PODS_DTYPE_F16, BITS>(tab, a, grid, s);
    else launch_kind<T, PT, PODS_DTYPE_F32, BITS>(tab, a, grid, s);
}

template <typename T, int BITS>
int adamw_launches(const pods_adamw_tensor* t, int32_t n, const Kind& k, const Step& a, cudaStream_t s) {
    int64_t first = 0;
    for (int from = 0; from < n;) {
        T tab;
        unsigned grid;
        from = fill(tab, t, from, n, &k, most_ctas(BITS == 8 ? kCtas8 : kCtas32, kMostCtas), first, grid);
        if (tab.count == 0) continue;
        if (k.p == PODS_DTYPE_BF16) launch_kind<T, PODS_DTYPE_BF16, BITS>(tab, a, grid, s, k.g);
        else if (k.p == PODS_DTYPE_F16) launch_kind<T, PODS_DTYPE_F16, BITS>(tab, a, grid, s, k.g);
        else launch_kind<T, PODS_DTYPE_F32, BITS>(tab, a, grid, s, k.g);
        PODS_RETURN_IF_CUDA_ERROR(cudaGetLastError());
    }
    return PODS_OK;
}

}  // namespace

extern "C" size_t pods_grad_norm_workspace_bytes(int32_t n) {
    return n < 0 ? 0 : (size_t)(n / ManyG::most + 2) * kMostNormCtas * sizeof(double);
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
    const int e = n <= kFew ? norm_launches<FewG>(tensors, n, parts, used, status, s) : norm_launches<ManyG>(tensors, n, parts, used, status, s);
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
        !(beta2 >= 0.0f && beta2 < 1.0f) || !(eps == 0.0f || (eps >= FLT_MIN && eps <= 0x1p126f)) || grad_scale - grad_scale != 0.0f ||
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
    // beta = f 2^e with f in [1/2, 1): its product with a power of two is normal from 2^(-125 - e) on
    int e1, e2;
    frexpf(beta1, &e1);
    frexpf(beta2, &e2);
    a.least_ms = (uint32_t)max(2 - e1, 1);
    a.least_vs = (uint32_t)max((130 - e2) / 2, 65);
    a.fold_vs = a.least_vs < 190u ? 190u - a.least_vs : 0u;
    a.status = status;
    cudaStream_t s = pods_stream(stream);
    // a launch for each kind of tensor; sets have one or two
    int e = PODS_OK;
    uint32_t done = 0;
    for (int i = 0; i < n && e == PODS_OK; ++i) {
        if (tensors[i].n == 0) continue;
        const Kind k = kind_of(tensors[i]);
        const uint32_t bit = 1u << (k.p * 6 + k.g * 2 + (k.bits == 8 ? 1 : 0));
        if (done & bit) continue;
        done |= bit;
        if (k.bits == 8) e = n <= kFew ? adamw_launches<Few8, 8>(tensors, n, k, a, s) : adamw_launches<Many8, 8>(tensors, n, k, a, s);
        else e = n <= kFew ? adamw_launches<Few32, 32>(tensors, n, k, a, s) : adamw_launches<Many32, 32>(tensors, n, k, a, s);
    }
    return e;
}
