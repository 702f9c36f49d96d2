// Arguments of the token log-probability kernels, for the calls that launch them between others.
#pragma once

#include "row_cluster.cuh"

namespace pods_logp {

constexpr int64_t kMaxRows = 1 << 24;  // rows of one call: with at most 64 stretches a row, block numbers stay within 31 bits

struct FwdArgs {
    const void* logits;
    int64_t ldl;
    const int32_t* tokens;
    const uint8_t* mask;
    const int64_t* rows_end;           // rows from *rows_end on are left out like masked ones; NULL: none
    int64_t T;
    int32_t V;
    int32_t fill;                      // rows left out get logp 0 (otherwise they stay as they were)
    double inv_tau, c64;               // c64 = log2 e / temperature, c + c_lo the same in two fp32 numbers
    float c, c_lo;
    float* logp;
    double* logp64;                    // the same before it is rounded; NULL: not wanted
    double* lse;
    float* entropy;
    uint32_t* status;
};

struct GradArgs {
    const void* logits;
    int64_t ldl;
    const int32_t* tokens;
    const double* lse;
    const float* dlogp;
    const float* entropy;
    const float* dentropy;
    int64_t T;
    int32_t V;
    int32_t n_seg, seg;
    double inv_tau;
    float c, c_lo;                     // their sum is log2 e / temperature
    void* dlogits;
    int64_t ldd;
    uint32_t* status;
};

// Sets the scales of a call; returns log2 e / temperature, which is at most 1.3e38 (temperatures are normal numbers).
template <typename Args>
double set_temperature(Args& a, float temperature) {
    a.inv_tau = 1.0 / (double)temperature;
    const double c = 1.4426950408889634074 / (double)temperature;
    a.c = (float)c;
    if ((double)a.c > c) a.c = nextafterf(a.c, 0.0f);
    // above 0, so that -inf times it is -inf as -inf times c is
    const float lo = (float)(c - (double)a.c), least = a.c * 0x1p-48f;
    a.c_lo = lo > least ? lo : least > 1e-45f ? least : 1e-45f;
    return c;
}

// The current device and its SMs (asked once a device).
inline int device_sms(int& dev) {
    static int known[64];
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        dev = -1;
        return 0;
    }
    int n = __atomic_load_n(&known[dev], __ATOMIC_RELAXED);
    if (n == 0) {
        n = pods_sm_count();
        __atomic_store_n(&known[dev], n, __ATOMIC_RELAXED);
    }
    return n;
}

int check_rows(const void* logits, int64_t ldl, int32_t dtype, int64_t T, int32_t V, float temperature);
int launch_forward(const FwdArgs& a, int dtype, cudaStream_t s);
int launch_gradient(GradArgs& a, int dtype, cudaStream_t s);

}  // namespace pods_logp
