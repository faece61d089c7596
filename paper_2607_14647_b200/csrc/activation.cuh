// The activations of the linear layer's and the adapters' epilogues, in fp32.
#pragma once
#include <cuda_runtime.h>

#include "dcut.h"

namespace {

// (e^-x overflows to infinity: 0.  The fast quotient returns 0 for a divisor above 2^126, where the value is below 2^-126.)
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.0f, 1.0f + __expf(-x)); }
// A function of its own: inlined for every column of the epilogue, the five cases made a loop body larger than the
// instruction cache (gelu_tanh over 1088 x 12288, K = 4096: 108 us against 97).
__device__ __noinline__ float4 activate4(int act, float4 v) {
    float x[4] = {v.x, v.y, v.z, v.w};
    if (act == DCUT_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = x[j] < 0.0f ? 0.0f : x[j];                        // (a NaN stays)
    } else if (act == DCUT_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] *= 0.5f * erfcf(x[j] * -0.7071067811865476f);       // Phi(x) without cancellation
    } else if (act == DCUT_ACT_GELU_TANH) {
        // (1 + tanh u) / 2 = sigmoid(2 u), u = sqrt(2 / pi) (x + 0.044715 x^3)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] *= sigmoid(1.5957691216057308f * x[j] * fmaf(0.044715f * x[j], x[j], 1.0f));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] *= sigmoid(x[j]);
    }
    return make_float4(x[0], x[1], x[2], x[3]);
}

}  // namespace
