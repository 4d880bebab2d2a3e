// AdamW over many tensors at once, for gfx950: one pass over parameters, gradients and states, which may be held in 8 bits.
//
//   g = grad * grad_scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g g
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps);   p16 = fp16(p)
//
// Bound: HBM.  An element costs 28 bytes with binary32 states and gradients (30 with the binary16 copy), 16.06 (18.06) with 8-bit states.
// The seven matrices of a layer, 4096 and 11008 wide, 202 million elements, fp16 gradients and copies (5.67 GB): 1060 us, 5.3 TB/s; 8-bit states,
// binary32 gradients (3.66 GB): 685 us, 5.3 TB/s; 16 tenants' adapters of rank 13, 224 tensors of 53248 and 143104 elements, 8-bit (293 MB):
// 62 us, 4.7 TB/s.  A plain copy of 1 GiB moves 5.2 TB/s.
//
// 8-bit states: 256 neighbours of a tensor, what a wavefront handles per step, share one binary32 scale each for m and v, found
// by a reduction across the wavefront, so that nothing is read twice.  A code is a small float without a bias, its value the
// integer V: 3 exponent bits e and F fraction bits f, V = f for e = 0, else (2^F + f) 2^(e - 1).
//   m  sign and F = 4:  m = +-scale V,        scale = max |m| / 1984          (steps of 3 to 6 %, range 1 : 1984)
//   v  F = 5:           sqrt(v) = scale V,    scale = sqrt(max v) / 4032      (steps of 1.6 to 3 %, range of v 1 : 1.6e7)
// m is rounded to nearest (even): beside gradients that do not change at all it stops within half a code step / (1 - b1) of them, some 16 to 31 % of m
// for b1 = 0.9; noise of a third of a gradient's size brings it to 1 % on average.  v moves by little: b2 = 0.999 changes sqrt(v) by 0.05 % a step, a thirtieth of a code step, and
// nearest rounding would hold it where it is (with gradients of constant size at a 25th of g^2, so steps five times too
// long).  It is rounded up with the probability of its fraction of a code step, from a hash of the element's index and the
// number of the step: right on average, and the same bits for the same inputs.  A v that is not zero does not become zero,
// which would leave eps alone under m.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "bd_adamw.h"
#include "bd_device.h"
#include "bd_host.h"
#include "bitdelta.h"

namespace bd {

namespace {

constexpr float kAvgTop = 1984.0f, kSqTop = 4032.0f;   // 31 * 2^6, 63 * 2^6; scales are products with their reciprocals

// value of a code without its sign; F fraction bits
template <int F>
__device__ __forceinline__ float code_value(uint32_t c) {
    return c < (1u << F) ? (float)c : __uint_as_float((c + ((127u + F - 1) << F)) << (23 - F));
}
// code of u in [0, top], rounded to nearest even
__device__ __forceinline__ uint32_t avg_code(float u) {
    const uint32_t bits = __float_as_uint(u);
    const uint32_t low = (uint32_t)__builtin_rintf(u), high = ((bits + 0x3FFFFu + ((bits >> 19) & 1u)) >> 19) - (130u << 4);
    return u < 16.0f ? low : min(high, 127u);
}
// code of u, rounded up where the fraction of a step and r / 2^18 together pass 1
__device__ __forceinline__ uint32_t sq_code(float u, uint32_t r) {
    const uint32_t low = (uint32_t)(u + (float)r * 0x1p-18f), high = ((__float_as_uint(u) + r) >> 18) - (131u << 5);
    return u < 32.0f ? low : min(high, 255u);
}
// 18 bits for element i of a tensor in this step: two rounds of shift and multiply behind a multiplication
__device__ __forceinline__ uint32_t dither(uint32_t i, uint32_t step) {
    uint32_t k = (i + step * 0x9E3779B9u) * 0xD1B54A33u;
    k = (k ^ (k >> 15)) * 0xB5297A4Du;
    k = (k ^ (k >> 16)) * 0x9E3779B9u;
    return k >> 14;
}

__device__ __forceinline__ double power(double b, int64_t t) {
    double p = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) p *= b;
    return p;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d, kWave));
    return v;
}

template <typename T>
__device__ __forceinline__ void load4(const T* p, int n, float (&out)[4]) {   // n = 4: one load
    if constexpr (sizeof(T) == 2) {
        if (n == 4) {
            const half4 v = *(const half4*)p;
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] = (float)v[k];
            return;
        }
    } else if (n == 4) {
        const float4v v = *(const float4v*)p;
#pragma unroll
        for (int k = 0; k < 4; ++k) out[k] = v[k];
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = k < n ? (float)p[k] : 0.0f;
}
__device__ __forceinline__ void store4(float* p, int n, const float (&v)[4]) {
    if (n == 4) {
        *(float4v*)p = float4v{v[0], v[1], v[2], v[3]};
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < n) p[k] = v[k];
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n) {
    if (n == 4) return *(const uint32_t*)p;
    uint32_t c = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < n) c |= (uint32_t)p[k] << (8 * k);
    return c;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int n, uint32_t c) {
    if (n == 4) {
        *(uint32_t*)p = c;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < n) p[k] = (uint8_t)(c >> (8 * k));
}

// a / b, correctly rounded, from y = 1 / b, which is: one step of Markstein's correction (b and a / b normal, as they are here)
__device__ __forceinline__ float quotient(float a, float b, float y) {
    const float q = a * y;
    return __builtin_fmaf(__builtin_fmaf(-b, q, a), y, q);
}

// All loads of a workgroup's 2048 elements, two blocks of 256 for each wavefront, come before the first store.
template <typename G, bool Q8>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwArgs a) {
    if (a.skip && *a.skip) return;
    const int64_t chunk = a.chunk_first + blockIdx.x;
    const AdamwTensor t = a.tensor[a.tensor_of_chunk[chunk]];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t base = (chunk - t.chunk_begin) * (kAdamwChunk / kAdamwBlock) + wave;   // the wavefront's first block
    constexpr int kSteps = kAdamwChunk / kAdamwBlock / 4;
    float p[kSteps][4], g[kSteps][4], m[kSteps][4], v[kSteps][4], ms[kSteps], vs[kSteps];
    uint32_t mc[kSteps], vc[kSteps];
    int n[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int64_t block = base + 4 * s, i = block * kAdamwBlock + 4 * lane;
        n[s] = (int)max((int64_t)0, min((int64_t)4, t.numel - i));
        if (block * kAdamwBlock >= t.numel) continue;
        load4((const G*)t.grad + i, n[s], g[s]);
        load4(t.param + i, n[s], p[s]);
        if constexpr (Q8) {
            mc[s] = load_codes((const uint8_t*)t.exp_avg + i, n[s]);
            vc[s] = load_codes((const uint8_t*)t.exp_avg_sq + i, n[s]);
            ms[s] = t.avg_scale[block];
            vs[s] = t.sq_scale[block];
        } else {
            load4((const float*)t.exp_avg + i, n[s], m[s]);
            load4((const float*)t.exp_avg_sq + i, n[s], v[s]);
        }
    }
    const float grad_scale = a.grad_scale ? *a.grad_scale : 1.0f, lr = *a.lr;
    const int64_t step = *a.step;
    const float rate = (float)((double)lr / (1.0 - power(a.beta1, step))), root = (float)(1.0 / sqrt(1.0 - power(a.beta2, step)));
    const float keep = 1.0f - lr * a.decay;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int64_t block = base + 4 * s, i = block * kAdamwBlock + 4 * lane;
        if (block * kAdamwBlock >= t.numel) return;
        if constexpr (Q8) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t c = (mc[s] >> (8 * k)) & 255u;
                const float size = code_value<4>(c & 127u) * ms[s], r = code_value<5>((vc[s] >> (8 * k)) & 255u) * vs[s];
                m[s][k] = c & 128u ? -size : size;
                v[s][k] = r * r;
            }
        }
        float r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float gk = g[s][k] * grad_scale;
            m[s][k] = m[s][k] * a.beta1_f + gk * a.rest1;
            v[s][k] = v[s][k] * a.beta2_f + gk * gk * a.rest2;
            r[k] = sqrtf(v[s][k]);
            p[s][k] = p[s][k] * keep - rate * (m[s][k] / (r[k] * root + a.eps));
        }
        store4(t.param + i, n[s], p[s]);
        if (t.param_f16) {
            if (n[s] == 4) {
                half4 h;
#pragma unroll
                for (int k = 0; k < 4; ++k) h[k] = (_Float16)p[s][k];
                *(half4*)(t.param_f16 + i) = h;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k < n[s]) t.param_f16[i + k] = f2h_rne(p[s][k]);
            }
        }
        if constexpr (Q8) {
            // as integers: a NaN is larger than an infinity, that larger than any number, and none is lost in the maximum
            uint32_t mt = 0, rt = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k >= n[s]) continue;
                mt = max(mt, __float_as_uint(m[s][k]) & 0x7fffffffu);
                rt = max(rt, __float_as_uint(r[k]) & 0x7fffffffu);
            }
            mt = wave_max(mt);
            rt = wave_max(rt);
            // a block with an infinity or a NaN is NaN; one whose largest |m| is below 2^-100 is zero
            const bool m_ok = mt < 0x7f800000u, r_ok = rt < 0x7f800000u, m_any = m_ok && mt >= (27u << 23), r_any = r_ok && rt > 0;
            const float m_scale = !m_ok ? __builtin_nanf("") : m_any ? __uint_as_float(mt) * (1.0f / kAvgTop) : 0.0f;
            const float v_scale = !r_ok ? __builtin_nanf("") : r_any ? __uint_as_float(rt) * (1.0f / kSqTop) : 0.0f;
            const float my = m_any ? 1.0f / m_scale : 0.0f, vy = r_any ? 1.0f / v_scale : 0.0f;
            uint32_t mo = 0, vo = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t cm = m_any ? avg_code(quotient(__builtin_fabsf(m[s][k]), m_scale, my)) | (m[s][k] < 0.0f ? 128u : 0u) : 0u;
                const uint32_t cv = r_any && r[k] > 0.0f ? max(sq_code(quotient(r[k], v_scale, vy), dither((uint32_t)(i + k), (uint32_t)step)), 1u) : 0u;
                mo |= cm << (8 * k);
                vo |= cv << (8 * k);
            }
            store_codes((uint8_t*)t.exp_avg + i, n[s], mo);
            store_codes((uint8_t*)t.exp_avg_sq + i, n[s], vo);
            if (lane == 0) {
                t.avg_scale[block] = m_scale;
                t.sq_scale[block] = v_scale;
            }
        } else {
            store4((float*)t.exp_avg + i, n[s], m[s]);
            store4((float*)t.exp_avg_sq + i, n[s], v[s]);
        }
    }
}

// the values V of 8-bit states, 8 at a time; binary16 holds them exactly
template <bool SECOND>
__global__ __launch_bounds__(256) void adamw_values_kernel(const uint8_t* __restrict__ codes, const int64_t n, _Float16* __restrict__ values) {
    auto value = [](uint32_t c) {
        const float v = SECOND ? code_value<5>(c) : code_value<4>(c & 127u);
        return (_Float16)(!SECOND && (c & 128u) ? -v : v);
    };
    for (int64_t i = 8 * ((int64_t)blockIdx.x * 256 + threadIdx.x); i < n; i += (int64_t)gridDim.x * 256 * 8) {
        if (i + 8 <= n) {
            const u32x2 c = *(const u32x2*)(codes + i);
            half8 v;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = value((c[k >> 2] >> (8 * (k & 3))) & 255u);
            *(half8*)(values + i) = v;
        } else {
            for (int64_t k = i; k < n; ++k) values[k] = value(codes[k]);
        }
    }
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, int64_t chunks, bool grad_f16, bool bits8, hipStream_t st) {
    if (chunks < 1 || chunks > (1 << 23)) return hipErrorInvalidValue;   // (threads of a launch: below 2^32)
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)chunks), dim3(256), 0, st, a);
        return hipGetLastError();
    };
    if (grad_f16) return bits8 ? go(adamw_kernel<_Float16, true>) : go(adamw_kernel<_Float16, false>);
    return bits8 ? go(adamw_kernel<float, true>) : go(adamw_kernel<float, false>);
}

hipError_t launch_adamw_values(const uint8_t* codes, int64_t n, bool second, uint16_t* values, hipStream_t st) {
    const int64_t blocks = std::min<int64_t>((n + 2047) / 2048, 256 * 32);
    if (second)
        hipLaunchKernelGGL(adamw_values_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, st, codes, n, (_Float16*)values);
    else
        hipLaunchKernelGGL(adamw_values_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, codes, n, (_Float16*)values);
    return hipGetLastError();
}

}  // namespace bd

// ---- C ABI ---------------------------------------------------------------------------------

namespace {

constexpr uint64_t kPlanMagic = 0x31304d4144414c50ull;
struct PlanHeader {
    uint64_t magic, bytes;
    int64_t chunks;
    int32_t n, grad_f16, bits8, unused;
};
// behind the header: the tensors that have elements, then the tensor of every chunk
size_t tensors_at() { return sizeof(PlanHeader); }
size_t chunks_at(int32_t n) { return tensors_at() + (size_t)n * sizeof(bd::AdamwTensor); }
int64_t chunks_of(int64_t numel) { return (numel + bd::kAdamwChunk - 1) / bd::kAdamwChunk; }

bd_status make_plan(void* plan, size_t plan_bytes, int32_t n, float* const* param, uint16_t* const* param_f16, const void* const* grad,
                    int32_t grad_f16, void* const* exp_avg, void* const* exp_avg_sq, float* const* avg_scale, float* const* sq_scale,
                    const int64_t* numel) {
    using bd::misaligned;
    if (n < 0 || n > BD_ADAMW_MAX_TENSORS) return BD_ERR_SHAPE;
    if (!plan) return BD_ERR_NULL;
    if (misaligned(plan, 8)) return BD_ERR_ALIGN;
    if (n > 0 && !numel) return BD_ERR_NULL;
    for (int32_t i = 0; i < n; ++i)
        if (numel[i] < 0 || numel[i] > BD_ADAMW_MAX_ELEMENTS) return BD_ERR_SHAPE;
    const size_t need = bd_adamw_plan_bytes(n, numel);
    if (need == 0) return BD_ERR_SHAPE;   // more elements than a plan takes
    if (plan_bytes < need) return BD_ERR_WORKSPACE;
    if (n > 0 && (!param || !grad || !exp_avg || !exp_avg_sq || (avg_scale == nullptr) != (sq_scale == nullptr))) return BD_ERR_NULL;
    const bool bits8 = avg_scale != nullptr;
    PlanHeader head{kPlanMagic, 0, 0, 0, grad_f16 ? 1 : 0, bits8 ? 1 : 0, 0};
    std::vector<bd::AdamwTensor> tensors;
    std::vector<bd::Range> ranges;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        bd::AdamwTensor t{param[i], param_f16 ? param_f16[i] : nullptr, grad[i], exp_avg[i], exp_avg_sq[i],
                          bits8 ? avg_scale[i] : nullptr, bits8 ? sq_scale[i] : nullptr, numel[i], head.chunks};
        head.chunks += chunks_of(numel[i]);
        if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq || (bits8 && (!t.avg_scale || !t.sq_scale))) return BD_ERR_NULL;
        if (misaligned(t.param, 16) || misaligned(t.param_f16, 16) || misaligned(t.grad, 16) || misaligned(t.exp_avg, 16) || misaligned(t.exp_avg_sq, 16) ||
            misaligned(t.avg_scale, 4) || misaligned(t.sq_scale, 4))
            return BD_ERR_ALIGN;
        const size_t count = (size_t)numel[i], state = count * (bits8 ? 1 : 4), scales = (count + bd::kAdamwBlock - 1) / bd::kAdamwBlock * 4;
        auto range = [&](const void* p, size_t bytes, bool written) { bd::add_range(ranges, p, bytes, written); };
        range(t.param, count * 4, true);
        range(t.param_f16, count * 2, true);
        range(t.grad, count * (grad_f16 ? 2 : 4), false);
        range(t.exp_avg, state, true);
        range(t.exp_avg_sq, state, true);
        range(t.avg_scale, scales, true);
        range(t.sq_scale, scales, true);
        tensors.push_back(t);
    }
    if (bd::any_alias(ranges)) return BD_ERR_ALIAS;
    head.n = (int32_t)tensors.size();
    head.bytes = chunks_at(head.n) + (size_t)head.chunks * sizeof(int32_t);
    std::memcpy(plan, &head, sizeof(head));
    if (head.n > 0) std::memcpy((char*)plan + tensors_at(), tensors.data(), tensors.size() * sizeof(bd::AdamwTensor));
    int32_t* to = (int32_t*)((char*)plan + chunks_at(head.n));
    for (int32_t i = 0; i < head.n; ++i) to = std::fill_n(to, chunks_of(tensors[(size_t)i].numel), i);
    return BD_OK;
}

}  // namespace

extern "C" {

size_t bd_adamw_plan_bytes(int32_t n, const int64_t* numel) {
    if (n < 0 || n > BD_ADAMW_MAX_TENSORS || (n > 0 && !numel)) return 0;
    int64_t chunks = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] < 0 || numel[i] > BD_ADAMW_MAX_ELEMENTS) return 0;
        chunks += chunks_of(numel[i]);
    }
    if (chunks > INT32_MAX) return 0;
    return (chunks_at(n) + (size_t)chunks * sizeof(int32_t) + 7) & ~(size_t)7;
}

bd_status bd_adamw_plan(void* plan, size_t plan_bytes, int32_t n, float* const* param, uint16_t* const* param_f16, const void* const* grad,
                        int32_t grad_f16, void* const* exp_avg, void* const* exp_avg_sq, float* const* exp_avg_scale,
                        float* const* exp_avg_sq_scale, const int64_t* numel) {
    try {
        return make_plan(plan, plan_bytes, n, param, param_f16, grad, grad_f16, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale, numel);
    } catch (...) {   // no host memory
        return BD_ERR_DEVICE;
    }
}

bd_status bd_adamw(const void* plan, size_t plan_bytes, const void* plan_device, const float* lr, const int64_t* step, const float* grad_scale,
                   const int32_t* skip, double beta1, double beta2, double eps, double weight_decay, void* stream) {
    if (!plan) return BD_ERR_NULL;
    PlanHeader head;
    if (bd::misaligned(plan, 8)) return BD_ERR_ALIGN;
    if (plan_bytes < sizeof(head)) return BD_ERR_FORMAT;
    std::memcpy(&head, plan, sizeof(head));
    if (head.magic != kPlanMagic || head.n < 0 || head.chunks < 0 || plan_bytes < head.bytes || head.bytes != chunks_at(head.n) + (size_t)head.chunks * sizeof(int32_t))
        return BD_ERR_FORMAT;
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0 && eps >= 0.0 && weight_decay >= 0.0)) return BD_ERR_UNSUPPORTED;
    if (head.n == 0) return BD_OK;
    if (!plan_device || !lr || !step) return BD_ERR_NULL;
    if (bd::misaligned(plan_device, 16) || bd::misaligned(lr, 4) || bd::misaligned(step, 8) || bd::misaligned(grad_scale, 4) || bd::misaligned(skip, 4)) return BD_ERR_ALIGN;
    bd::AdamwArgs a;
    std::memset(&a, 0, sizeof(a));
    a.tensor = (const bd::AdamwTensor*)((const char*)plan_device + tensors_at());
    a.tensor_of_chunk = (const int32_t*)((const char*)plan_device + chunks_at(head.n));
    a.lr = lr;
    a.step = step;
    a.grad_scale = grad_scale;
    a.skip = skip;
    a.beta1 = beta1;
    a.beta2 = beta2;
    a.beta1_f = (float)beta1;
    a.beta2_f = (float)beta2;
    a.rest1 = (float)(1.0 - beta1);
    a.rest2 = (float)(1.0 - beta2);
    a.eps = (float)eps;
    a.decay = (float)weight_decay;
    constexpr int64_t kMost = 1 << 23;   // chunks of a launch
    for (a.chunk_first = 0; a.chunk_first < head.chunks; a.chunk_first += kMost)
        if (bd::launch_adamw(a, std::min(kMost, head.chunks - a.chunk_first), head.grad_f16, head.bits8, (hipStream_t)stream) != hipSuccess) return BD_ERR_DEVICE;
    return BD_OK;
}

bd_status bd_adamw_values(const uint8_t* codes, int64_t n, int32_t second, uint16_t* values_f16, void* stream) {
    if (n < 0 || n > BD_ADAMW_MAX_ELEMENTS) return BD_ERR_SHAPE;
    if (n == 0) return BD_OK;
    if (!codes || !values_f16) return BD_ERR_NULL;
    if (bd::misaligned(codes, 16) || bd::misaligned(values_f16, 16)) return BD_ERR_ALIGN;
    if (bd::overlaps(codes, (size_t)n, values_f16, (size_t)n * 2)) return BD_ERR_ALIAS;
    return bd::launch_adamw_values(codes, n, second != 0, values_f16, (hipStream_t)stream) == hipSuccess ? BD_OK : BD_ERR_DEVICE;
}

}  // extern "C"
