// A row of logits held by a thread-block cluster: helpers shared by the sampler, the top-K lists and the distillation
// objective.
//
// CTA r of the cluster holds the r-th segment of the row in shared memory, so that the row crosses HBM once however often
// it is looked at.  Rows may start at any element: the row is cut at the 16-byte boundaries of global memory.  Whole
// vectors inside the row arrive by bulk asynchronous copies, the at most two vectors that the row covers only in part by
// element loads, and every slot that is no logit of the row holds -inf, which adds nothing to a maximum or a sum of
// exponentials.  Element i of CTA r's segment is the logit of id  r * seg * E + i - lead,  where E is the number of
// elements of a vector and lead the number of elements between the boundary and the row's start.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cooperative_groups.h>
#include <math.h>

#include "pods_common.cuh"

namespace pods_row {

namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kSpinLimit = 1u << 24;     // polls of the load barrier before giving up
constexpr uint32_t kSuspendNs = 1000;         // upper bound of one poll
constexpr int kMaxCluster = 16;

template <int DT> struct Elem;

template <> struct Elem<PODS_DTYPE_BF16> {
    using raw = uint16_t;
    static constexpr int E = 8;
    static constexpr raw kNegInf = 0xff80u;
    __device__ static __forceinline__ float to_float(raw r) { return __uint_as_float((uint32_t)r << 16); }
    __device__ static __forceinline__ raw from_float(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
    __device__ static __forceinline__ void unpack(const uint4& q, float (&x)[E]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[E]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // the largest element, NaN if one of them is
    __device__ static __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static __forceinline__ float vec_max(const uint4& q) {
        const uint32_t m = max2(max2(q.x, q.y), max2(q.z, q.w));
        return to_float((raw)max2(m, m >> 16));
    }
    // keys whose unsigned order is the order of the values (-0 == +0)
    __device__ static __forceinline__ uint32_t to_key(float v) {
        const uint32_t u = __float_as_uint(v + 0.0f) >> 16;
        return (u & 0x8000u) ? (~u & 0xffffu) : (u | 0x8000u);
    }
    __device__ static __forceinline__ float from_key(uint32_t k) {
        return __uint_as_float(((k & 0x8000u) ? (k & 0x7fffu) : (~k & 0xffffu)) << 16);
    }
};

template <> struct Elem<PODS_DTYPE_F16> {
    using raw = uint16_t;
    static constexpr int E = 8;
    static constexpr raw kNegInf = 0xfc00u;
    __device__ static __forceinline__ float to_float(raw r) { return __half2float(__ushort_as_half(r)); }
    __device__ static __forceinline__ raw from_float(float v) { return __half_as_ushort(__float2half_rn(v)); }
    __device__ static __forceinline__ void unpack(const uint4& q, float (&x)[E]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[E]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static __forceinline__ float vec_max(const uint4& q) {
        const uint32_t m = max2(max2(q.x, q.y), max2(q.z, q.w));
        return to_float((raw)max2(m, m >> 16));
    }
    __device__ static __forceinline__ uint32_t to_key(float v) {
        const uint32_t u = from_float(v + 0.0f);
        return (u & 0x8000u) ? (~u & 0xffffu) : (u | 0x8000u);
    }
    __device__ static __forceinline__ float from_key(uint32_t k) {
        return to_float((raw)((k & 0x8000u) ? (k & 0x7fffu) : (~k & 0xffffu)));
    }
};

template <> struct Elem<PODS_DTYPE_F32> {
    using raw = uint32_t;
    static constexpr int E = 4;
    static constexpr raw kNegInf = 0xff800000u;
    __device__ static __forceinline__ float to_float(raw r) { return __uint_as_float(r); }
    __device__ static __forceinline__ raw from_float(float v) { return __float_as_uint(v); }
    __device__ static __forceinline__ void unpack(const uint4& q, float (&x)[E]) {
        x[0] = __uint_as_float(q.x);
        x[1] = __uint_as_float(q.y);
        x[2] = __uint_as_float(q.z);
        x[3] = __uint_as_float(q.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[E]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ static __forceinline__ float max_nan(float a, float b) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
        return r;
    }
    __device__ static __forceinline__ float vec_max(const uint4& q) {
        return max_nan(max_nan(__uint_as_float(q.x), __uint_as_float(q.y)), max_nan(__uint_as_float(q.z), __uint_as_float(q.w)));
    }
    __device__ static __forceinline__ uint32_t to_key(float v) {
        const uint32_t u = __float_as_uint(v + 0.0f);
        return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    }
    __device__ static __forceinline__ float from_key(uint32_t k) {
        return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
    }
};

// value -> 32-bit key in value order, for entries that leave their row (lists)
__device__ __forceinline__ uint32_t order32(float v) { return Elem<PODS_DTYPE_F32>::to_key(v); }
__device__ __forceinline__ float unorder32(uint32_t k) { return Elem<PODS_DTYPE_F32>::from_key(k); }

__device__ __forceinline__ float max_nan(float a, float b) { return Elem<PODS_DTYPE_F32>::max_nan(a, b); }

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- exponentials of a vector -----------------------------------------------------------------------------------------
// Two lanes of fp32 an instruction (fma.rn.f32x2): 3 issue slots an element with the unpacking and the exponential.

__device__ __forceinline__ unsigned long long pack2(float lo, float hi) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(unsigned long long v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// What exponentials are taken relative to: e_i = 2^(x_i c - R) with R = fl(m c) for the reference value m, one fused
// rounding an element.  Where R is so large that its own rounding matters (cold temperatures, huge logits) the difference is
// taken first, e_i = 2^((x_i - m) c).  A reference of -inf (nothing in sight) makes every e 0.
struct ExpRef {
    float m, R;
    bool far;
    unsigned long long c2, off2;
    __device__ __forceinline__ ExpRef(float m_, float c) {
        m = fabsf(m_) < INFINITY ? m_ : 0.0f;
        R = m * c;
        far = !(fabsf(R) < 0x1p24f);
        c2 = pack2(c, c);
        off2 = far ? pack2(-m, -m) : pack2(-R, -R);
    }
    template <int E>
    __device__ __forceinline__ void exps(float (&x)[E]) const {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const unsigned long long v = pack2(x[i], x[i + 1]);
            float a, b;
            unpack2(far ? mul2(add2(v, off2), c2) : fma2(v, c2, off2), a, b);
            x[i] = ex2_approx(a);
            x[i + 1] = ex2_approx(b);
        }
    }
    __device__ __forceinline__ float exp1(float x, float c) const { return ex2_approx(far ? (x - m) * c : fmaf(x, c, -R)); }
    // a sum relative to this reference, times scale_to(z), is relative to z (fp64; z c and R are exact there)
    __device__ __forceinline__ double scale_to(float z, float c) const {
        return exp2(far ? ((double)m - (double)z) * (double)c : (double)R - (double)z * (double)c);
    }
};

template <int E>
__device__ __forceinline__ float vec_add(const float (&x)[E]) {
    unsigned long long s[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) s[i] = pack2(x[2 * i], x[2 * i + 1]);
#pragma unroll
    for (int d = E / 4; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < d; ++i) s[i] = add2(s[i], s[i + d]);
    float a, b;
    unpack2(s[0], a, b);
    return a + b;
}
// e^d for d <= 0 in fp64 without a branch, so that several run side by side: d log2 e = n + f with |f| <= 1/2, then the
// Taylor polynomial of 2^f (the first term left out is 6.3e-15 of the sum).  Below e^-700: 0.
template <int K> struct Exp2Term { static constexpr double value = Exp2Term<K - 1>::value * (0.69314718055994530942 / K); };
template <> struct Exp2Term<0> { static constexpr double value = 1.0; };
template <int K>
__device__ __forceinline__ double exp2_poly(double p, double f) {
    if constexpr (K < 0) return p;
    else return exp2_poly<K - 1>(fma(p, f, Exp2Term<K>::value), f);
}
__device__ __forceinline__ double exp64(double d) {
    const double y = d * 1.4426950408889634074;
    const double t = y + 6755399441055744.0;           // 1.5 * 2^52: the integer part is in the low word
    const double f = y - (t - 6755399441055744.0);
    const double p = exp2_poly<10>(Exp2Term<11>::value, f);
    const double e = __hiloint2double(__double2hiint(p) + (int)((unsigned)__double2loint(t) << 20), __double2loint(p));
    return d > -700.0 ? e : 0.0;
}
// Four at a time, step by step, which hides the latency of the fp64 pipe: d becomes e^d.
template <int K>
__device__ __forceinline__ void exp2_poly4(double (&p)[4], const double (&f)[4]) {
    if constexpr (K >= 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = fma(p[i], f[i], Exp2Term<K>::value);
        exp2_poly4<K - 1>(p, f);
    }
}
__device__ __forceinline__ void exp64x4(double (&d)[4]) {
    double f[4], p[4];
    int n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double y = d[i] * 1.4426950408889634074, t = y + 6755399441055744.0;
        f[i] = y - (t - 6755399441055744.0);
        n[i] = d[i] > -700.0 ? (int)((unsigned)__double2loint(t) << 20) : (int)0x80000000;
        p[i] = Exp2Term<11>::value;
    }
    exp2_poly4<10>(p, f);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        d[i] = n[i] != (int)0x80000000 ? __hiloint2double(__double2hiint(p[i]) + n[i], __double2loint(p[i])) : 0.0;
}

constexpr double kLn2 = 0.6931471805599453;

__device__ __forceinline__ double pow2(int n) {       // n <= 0; below the normal numbers: 0
    return n < -1000 ? 0.0 : __hiloint2double((1023 + n) << 20, 0);
}

__device__ __forceinline__ float pow2_any(float n) {  // n an integer; outside the normal numbers: 0 or +inf
    return n < -126.0f ? 0.0f : n > 127.0f ? INFINITY : __uint_as_float((uint32_t)(127 + (int)n) << 23);
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
    template <bool FAR, int E>
    __device__ __forceinline__ void exps(float (&x)[E]) const {
        const unsigned long long c2 = pack2(c, c), off2 = FAR ? pack2(-m, -m) : pack2(-R, -R);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const unsigned long long v = pack2(x[i], x[i + 1]);
            float p, q;
            unpack2(FAR ? mul2(add2(v, off2), c2) : fma2(v, c2, off2), p, q);
            x[i] = ex2_approx(p);
            x[i + 1] = ex2_approx(q);
        }
    }
    __device__ __forceinline__ double exp1(float x) const { return (double)ex2_approx(far ? (x - m) * c : fmaf(x, c, -R)); }
    // what sums relative to this reference are multiplied with to be relative to that of `top`, the row's
    __device__ __forceinline__ double scale_to(const PartRef& top) const {
        if (!top.far && !far) return pow2((int)fmaxf(R - top.R, -2000.0f));
        if (!top.far) return exp2((double)m * (double)c - (double)top.R);
        return exp2((far ? (double)m * (double)c : (double)R) - (double)top.m * (double)c);
    }
    // whether a part that counts beside this one may be far
    __device__ __forceinline__ bool near_far() const { return !(fabsf(R) < 0x1p22f); }
    // ln of this reference's own weight over e^(m / tau): what log sums relative to it lack
    __device__ __forceinline__ double log_offset() const { return far ? 0.0 : ((double)R - (double)m * (double)c) * kLn2; }
};

// Inclusive scan over a warp.
template <typename T>
__device__ __forceinline__ T warp_scan(T v, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T o = __shfl_up_sync(PODS_FULL_MASK, v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Of a warp_scan's results: the sum of the lanes ahead.
template <typename T>
__device__ __forceinline__ T scan_ahead(T incl, int lane) {
    const T o = __shfl_up_sync(PODS_FULL_MASK, incl, 1);
    return lane > 0 ? o : T(0);
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(unsigned long long* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(unsigned long long* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_wait(unsigned long long* bar, uint32_t parity, uint32_t limit) {
    for (uint32_t i = 0; i < limit; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(kSuspendNs) : "memory");
        if (ok) return true;
    }
    return false;
}
// A pipeline's place in its ring of stages: the stage, and the parity of its barriers' current use.
struct StageRing {
    int st = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int n) {
        if (++st == n) {
            st = 0;
            parity ^= 1u;
        }
    }
};

// ---- barriers and stores across the cluster -----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t mapa(const void* p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
// 16 bytes into a CTA of the cluster, counted on an mbarrier there.
__device__ __forceinline__ void store_async(uint32_t at, uint32_t bar, double a, unsigned long long b) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];"
                 ::"r"(at), "l"(__double_as_longlong(a)), "l"(b), "r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_remote(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_local(unsigned long long* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ bool wait_cluster(unsigned long long* bar, uint32_t parity, uint32_t limit) {
    for (uint32_t i = 0; i < limit; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(kSuspendNs) : "memory");
        if (ok) return true;
    }
    return false;
}

// Global -> this CTA's shared memory, completion counted on an mbarrier.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, unsigned long long* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// This CTA's segment of a row.
struct Segment {
    int cnt;          // vectors of the row in the segment
    int id0;          // id of the segment's element 0 (negative where the row starts inside the first vector)
    int full0, full1; // local vectors [full0, full1) lie in the row whole
    const uint4* src; // global address of local vector 0
};

template <int DT>
__device__ __forceinline__ Segment make_segment(const void* base, int64_t pitch, int64_t t, int V, int rank, int seg) {
    using El = Elem<DT>;
    const typename El::raw* row = static_cast<const typename El::raw*>(base) + t * pitch;
    const int lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(typename El::raw));
    const uint4* aligned = reinterpret_cast<const uint4*>(row - lead);
    const int nvec = (lead + V + El::E - 1) / El::E;
    const int j0 = rank * seg;
    Segment s;
    s.cnt = max(0, min(seg, nvec - j0));
    s.id0 = j0 * El::E - lead;
    s.full0 = min(s.cnt, max(0, (lead ? 1 : 0) - j0));
    s.full1 = max(s.full0, min(s.cnt, (lead + V) / El::E - j0));
    s.src = aligned + j0;
    return s;
}

// The vectors at the row's two ends (one thread: at most two of them).
template <int DT>
__device__ __forceinline__ void fill_edges(const Segment& s, int V, uint4* buf) {
    using El = Elem<DT>;
    for (int j = 0; j < s.cnt; ++j) {
        if (j == s.full0) j = s.full1;
        if (j >= s.cnt) break;
        typename El::raw* dst = reinterpret_cast<typename El::raw*>(buf + j);
        const typename El::raw* src = reinterpret_cast<const typename El::raw*>(s.src + j);
        for (int e = 0; e < El::E; ++e) {
            const int id = s.id0 + j * El::E + e;
            dst[e] = (id >= 0 && id < V) ? src[e] : El::kNegInf;
        }
    }
}
// Starts the copy of the others, counted on `bar` (one thread).
__device__ __forceinline__ void start_copy(const Segment& s, uint4* buf, unsigned long long* bar) {
    constexpr int kPiece = 512;
    const int n = s.full1 - s.full0;
    mbar_expect_tx(bar, (uint32_t)n * 16u);
    for (int v = 0; v < n; v += kPiece)
        bulk_load(buf + s.full0 + v, s.src + s.full0 + v, (uint32_t)min(kPiece, n - v) * 16u, bar);
}
// Both, the copy first: the waiters see the ends after mbar_wait on `bar` and a CTA barrier.
template <int DT>
__device__ __forceinline__ void start_load(const Segment& s, int V, uint4* buf, unsigned long long* bar) {
    start_copy(s, buf, bar);
    fill_edges<DT>(s, V, buf);
}

// ---- reductions over a CTA of W warps; `part` is scratch of W entries, every thread gets the result -------------------
template <int W, typename T, typename Op>
__device__ __forceinline__ T block_reduce(T v, T* part, Op op) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(PODS_FULL_MASK, v, d));
    __syncthreads();                                   // an earlier use of `part` is over
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    T r = part[0];
#pragma unroll
    for (int w = 1; w < W; ++w) r = op(r, part[w]);
    return r;
}

struct Plus {
    template <typename T> __device__ T operator()(T a, T b) const { return a + b; }
};
struct MaxNan {
    __device__ float operator()(float a, float b) const { return max_nan(a, b); }
};
struct Min {
    template <typename T> __device__ T operator()(T a, T b) const { return a < b ? a : b; }
};

// Host: vectors per CTA for rows of V elements of `esize` bytes over `cl` CTAs (whole 128-byte lines).
static inline int segment_vectors(int64_t V, int esize, int cl) {
    const int64_t e = 16 / esize, nvec = (V + 2 * (e - 1)) / e + 1;
    return (int)(((nvec + cl - 1) / cl + 7) & ~7ll);
}

// Host: launches KERNEL on clusters of cl CTAs that go round over T rows: as many clusters as are resident at once, since a
// cluster that started late would leave its rows for a second round.  The query is left out where every row has its SMs.
// The kernel's attributes are set once per device, and the last answer of the query is kept (both cost a small call more
// than its launch: 5 us together).
template <auto KERNEL, typename Args>
int launch_row_clusters(const Args& a, int64_t T, int cl, int threads, size_t smem, cudaStream_t stream) {
    static uint64_t prepared = 0, last = 0;            // devices as bits; device, cl, smem / 128 and the answer in 16 bits each
    int dev = 0;
    PODS_RETURN_IF_CUDA_ERROR(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return PODS_ERR_UNSUPPORTED;
    if (!(__atomic_load_n(&prepared, __ATOMIC_ACQUIRE) >> dev & 1)) {
        PODS_RETURN_IF_CUDA_ERROR(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024));
        PODS_RETURN_IF_CUDA_ERROR(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        __atomic_fetch_or(&prepared, 1ull << dev, __ATOMIC_RELEASE);
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cl;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)cl, 1, 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int64_t n = T;
    if (T * cl > 128) {
        const uint64_t key = (uint64_t)dev << 48 | (uint64_t)cl << 32 | (uint64_t)(smem / 128) << 16;
        const uint64_t kept = __atomic_load_n(&last, __ATOMIC_RELAXED);
        int resident = (int)(kept & 0xffff);
        if (kept >> 16 != key >> 16 || resident == 0) {
            PODS_RETURN_IF_CUDA_ERROR(cudaOccupancyMaxActiveClusters(&resident, KERNEL, &cfg));
            if (resident < 1) return PODS_ERR_UNSUPPORTED;
            __atomic_store_n(&last, key | (uint64_t)(resident & 0xffff), __ATOMIC_RELAXED);
        }
        if (n > resident) n = resident;
    }
    cfg.gridDim = dim3((unsigned)(n * cl), 1, 1);
    PODS_RETURN_IF_CUDA_ERROR(cudaLaunchKernelEx(&cfg, KERNEL, a));
    return PODS_OK;
}

}  // namespace pods_row
