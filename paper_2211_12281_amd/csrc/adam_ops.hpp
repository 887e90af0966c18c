// Shared by the optimisers (sparse_adam.hip, adamw.hip).
#pragma once
#include "kge_internal.h"

// 1 / (1 - beta^step) by binary powering in fp64: products only, so the host (plain calls) and the device (steps read
// from a counter in device memory) arrive at the same bits.
__host__ __device__ inline float adam_inv_bias(float beta, uint64_t step) {
    double p = 1.0, b = (double)beta;
    for (; step; step >>= 1) {
        if (step & 1) p *= b;
        b *= b;
    }
    return (float)(1.0 / (1.0 - p));
}
