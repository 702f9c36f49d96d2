// Which kernel takes the rows of a pods_logp_chunk call, by their number, their length and the device's SMs.  Host arithmetic on
// plain numbers.
#pragma once

#include <stdint.h>

namespace pods_logp {

// Log-probabilities of many rows: up to kRowsVecs vectors a warp each, beyond them the pipeline.  Measured, a warp each against
// the pipeline: bf16 V = 1000 51 : 390 us (100000 rows), V = 8000 63 : 90 us (20000), V = 16000 65.3 : 65.7 us (10000), fp16
// V = 32000 78 : 71 us (6007).
constexpr int kRowsVecs = 1024;
// The pipeline in groups of four warps for shares of up to this many vectors; sixteen warps a row against it: V = 16000 79 : 66 us,
// V = 32000 74 : 71 us, V = 50257 64 : 60 us (3000 rows), but 20 : 22 us of 700 rows, which leave a group one or two.
constexpr int kGroupVecs = 8192;
// Rows of up to kCtaVecs vectors, up to kFewRows of them an SM, get a CTA each.  Measured, a CTA each against what takes more of
// them: bf16 V = 1000 3.5 : 4.1 us (37 rows), 4.5 : 5.3 (1200), 20.8 : 17.2 (20000); V = 8000 3.7 : 7.7, 11.9 : 11.6, 116 : 64;
// V = 32000 5.4 : 6.2, 21.3 : 21.0, 67 : 59 (5000).
constexpr int kFewRows = 8, kCtaVecs = 4096;
constexpr int kBatch = 8;              // rows a warp takes one after the other and finishes together

enum RowKernel { kRowEach, kRowsWarp, kRowsPipe };

struct RowPlan {
    RowKernel kernel;
    int batch;                         // kRowsWarp: rows of a warp's batch
    int warps;                         // kRowsPipe: warps of a group
    int cluster;                       // kRowsPipe: CTAs of a cluster
};

// nvec: whole 16-byte vectors of a row; sms: of the device, 1 at least.
inline RowPlan plan_rows(int64_t T, int64_t nvec, int sms) {
    if (nvec <= kCtaVecs && T <= (int64_t)kFewRows * sms) return {kRowEach, 1, 0, 1};
    if (nvec <= kRowsVecs) {
        const int64_t per = T / ((int64_t)sms * 24);
        return {kRowsWarp, (int)(per < 1 ? 1 : per > kBatch ? kBatch : per), 0, 1};
    }
    // the cluster size with the shortest longest share: rounds of rows times the vectors of a share and what a row costs beside
    // (V = 151936, one CTA a row against what is chosen: 32.4 : 31.0 us of 512 rows, 12.3 : 10.6 of 64, 11.0 : 6.4 of one)
    int best = 1;
    int64_t least = INT64_MAX;
    for (int cl = 1; cl <= 8; cl *= 2) {
        const int64_t n = cl == 1 ? sms : cl == 2 ? sms / 2 : (sms - 16) / cl;         // clusters at once; larger ones leave SMs empty
        if (n < 1) break;                              // a device, or a part of one, too small for any
        const int64_t cost = (T + n - 1) / n * (nvec / cl + (cl == 1 ? 1000 : 1250));
        if (cost < least) {
            least = cost;
            best = cl;
        }
    }
    // groups of four warps want several rows each
    return {kRowsPipe, 1, nvec / best <= kGroupVecs && T * best >= 16 * (int64_t)sms ? 4 : 16, best};
}

}  // namespace pods_logp
