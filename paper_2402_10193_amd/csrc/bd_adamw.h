// The AdamW step over many tensors at once: what a plan holds, and the launch functions (adamw.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bd {

constexpr int kAdamwBlock = 256;         // elements that share a scale where states are held in 8 bits; a wavefront's step
constexpr int kAdamwChunk = 2048;        // elements of a workgroup

struct AdamwTensor {
    float* param;
    uint16_t* param_f16;                 // may be nullptr
    const void* grad;
    void *exp_avg, *exp_avg_sq;
    float *avg_scale, *sq_scale;         // 8-bit states
    int64_t numel;
    int64_t chunk_begin;                 // its first chunk
};
struct AdamwArgs {
    const AdamwTensor* tensor;           // device
    const int32_t* tensor_of_chunk;      // device
    const float* lr;
    const int64_t* step;
    const float* grad_scale;             // may be nullptr: 1
    const int32_t* skip;                 // may be nullptr: no
    double beta1, beta2;
    int64_t chunk_first;
    float beta1_f, beta2_f, rest1, rest2, eps, decay;   // rest = 1 - beta
};

hipError_t launch_adamw(const AdamwArgs& a, int64_t chunks, bool grad_f16, bool bits8, hipStream_t st);
hipError_t launch_adamw_values(const uint8_t* codes, int64_t n, bool second, uint16_t* values, hipStream_t st);

}  // namespace bd
