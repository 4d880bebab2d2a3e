// The AdamW step over many tensors at once: kernel arguments and launch function (adamw.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bd {

constexpr int kAdamwTensors = 40;        // tensors of one launch
constexpr int kAdamwBlock = 256;         // elements that share a scale where states are held in 8 bits; a wavefront's step
constexpr int kAdamwChunk = 4096;        // elements of a workgroup

struct AdamwTensor {
    float* param;
    uint16_t* param_f16;                 // may be nullptr
    const void* grad;
    void *exp_avg, *exp_avg_sq;
    float *avg_scale, *sq_scale;         // 8-bit states
    int64_t numel;
};
struct AdamwArgs {
    const float* lr;
    const int64_t* step;
    const float* grad_scale;             // may be nullptr: 1
    const int32_t* skip;                 // may be nullptr: no
    double beta1, beta2;
    float beta1_f, beta2_f, rest1, rest2, eps, decay;   // rest = 1 - beta
    int32_t chunk_begin[kAdamwTensors];  // first workgroup of every tensor (unused ones: the largest int)
    AdamwTensor tensor[kAdamwTensors];
};

hipError_t launch_adamw(const AdamwArgs& a, int chunks, bool grad_f16, bool bits8, hipStream_t st);

}  // namespace bd
