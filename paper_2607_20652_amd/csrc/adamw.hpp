// AdamW over many tensors: arguments of a launch.
#pragma once

#include "device_common.hpp"

namespace dpb {

constexpr int kAdamwBlock = 256;     // elements that share the scales of 8-bit states
constexpr int kAdamwChunk = 32;      // blocks a workgroup
constexpr int kAdamwTensors = 96;    // tensors a launch: their table travels in the kernel arguments (4 KB)

struct AdamwTensor {
    void* param;
    const void* grad;
    int64_t n;
    int32_t block;         // first block of its states
    float shrink;          // 1 - lr * weight decay
};

struct AdamwArgs {
    void *m, *v;           // [blocks * 256] fp32, or 8-bit floats (v: the square root)
    float *scales;         // [blocks][2], 8-bit states
    float *master;         // [blocks * 256], or null
    const float* grad_scale;
    float beta1, rest1, beta2, rest2, eps;
    float rate;            // lr / (1 - beta1^t)
    float unbias2;         // 1 / sqrt(1 - beta2^t)
    uint32_t seed;
    int count;
    int32_t first_chunk[kAdamwTensors];
    AdamwTensor tensor[kAdamwTensors];
};
static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");

hipError_t launch_adamw(const AdamwArgs& a, int chunks, bool param_bf16, bool grad_bf16, bool bits8, hipStream_t stream);

}  // namespace dpb
