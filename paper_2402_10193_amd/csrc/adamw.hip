// AdamW over many tensors at once, for gfx950: one pass over parameters, gradients and states, which may be held in 8 bits.
//
//   g = grad * grad_scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g g
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps);   p16 = fp16(p)
//
// Bound: HBM.  An element costs 28 bytes with binary32 states and gradients (30 with the binary16 copy), 18.06 with 8-bit ones.
//
// 8-bit states: 256 neighbours of a tensor, what a wavefront handles per step, share one binary32 scale each for m and v, found
// by a reduction across the wavefront, so that nothing is read twice.  A code is a small float without a bias, its value the
// integer V: 3 exponent bits e and F fraction bits f, V = f for e = 0, else (2^F + f) 2^(e - 1).
//   m  sign and F = 4:  m = +-scale V,        scale = max |m| / 1984          (steps of 3 to 6 %, range 1 : 1984)
//   v  F = 5:           sqrt(v) = scale V,    scale = sqrt(max v) / 4032      (steps of 1.6 to 3 %, range of v 1 : 1.6e7)
// m is rounded to nearest (even).  v moves by little: b2 = 0.999 changes sqrt(v) by 0.05 % a step, a thirtieth of a code step, and
// nearest rounding would hold it where it is (with gradients of constant size at a 25th of g^2, so steps five times too
// long).  It is rounded up with the probability of its fraction of a code step, from a hash of the element's index and the
// number of the step: right on average, and the same bits for the same inputs.  A v that is not zero does not become zero,
// which would leave eps alone under m.
#include <climits>
#include <cmath>
#include <cstring>

#include "bd_adamw.h"
#include "bd_device.h"
#include "bd_host.h"
#include "bitdelta.h"

namespace bd {

namespace {

constexpr float kAvgTop = 1984.0f, kSqTop = 4032.0f;   // 31 * 2^6, 63 * 2^6

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

template <typename G, bool Q8>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwArgs a) {
    if (a.skip && *a.skip) return;
    int which = 0;
#pragma unroll
    for (int k = 1; k < kAdamwTensors; ++k) which += (int)blockIdx.x >= a.chunk_begin[k] ? 1 : 0;
    const AdamwTensor& t = a.tensor[which];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t base = (int64_t)((int)blockIdx.x - a.chunk_begin[which]) * kAdamwChunk, numel = t.numel;
    const float grad_scale = a.grad_scale ? *a.grad_scale : 1.0f, lr = *a.lr;
    const int64_t step = *a.step;
    const float rate = (float)((double)lr / (1.0 - power(a.beta1, step))), root = (float)(1.0 / sqrt(1.0 - power(a.beta2, step)));
    const float keep = 1.0f - lr * a.decay;
    constexpr int kSteps = kAdamwChunk / kAdamwBlock / 4;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int64_t block = base / kAdamwBlock + 4 * s + wave, first = block * kAdamwBlock;
        if (first >= numel) return;
        const int64_t i = first + 4 * lane;
        const int n = (int)max((int64_t)0, min((int64_t)4, numel - i));
        float p[4], g[4], m[4], v[4];
        load4((const G*)t.grad + i, n, g);
        load4(t.param + i, n, p);
        if constexpr (Q8) {
            const uint32_t mc = load_codes((const uint8_t*)t.exp_avg + i, n), vc = load_codes((const uint8_t*)t.exp_avg_sq + i, n);
            const float ms = t.avg_scale[block], vs = t.sq_scale[block];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t c = (mc >> (8 * k)) & 255u;
                const float size = code_value<4>(c & 127u) * ms, r = code_value<5>((vc >> (8 * k)) & 255u) * vs;
                m[k] = c & 128u ? -size : size;
                v[k] = r * r;
            }
        } else {
            load4((const float*)t.exp_avg + i, n, m);
            load4((const float*)t.exp_avg_sq + i, n, v);
        }
        float r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float gk = g[k] * grad_scale;
            m[k] = m[k] * a.beta1_f + gk * a.rest1;
            v[k] = v[k] * a.beta2_f + gk * gk * a.rest2;
            r[k] = sqrtf(v[k]);
            p[k] = p[k] * keep - rate * (m[k] / (r[k] * root + a.eps));
        }
        store4(t.param + i, n, p);
        if (t.param_f16) {
            half4 h;
#pragma unroll
            for (int k = 0; k < 4; ++k) h[k] = (_Float16)p[k];
            if (n == 4) {
                *(half4*)(t.param_f16 + i) = h;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k < n) t.param_f16[i + k] = f2h_rne(p[k]);
            }
        }
        if constexpr (Q8) {
            // as integers: a NaN is larger than an infinity, that larger than any number, and none is lost in the maximum
            uint32_t mt = 0, rt = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k >= n) continue;
                mt = max(mt, __float_as_uint(m[k]) & 0x7fffffffu);
                rt = max(rt, __float_as_uint(r[k]) & 0x7fffffffu);
            }
            mt = wave_max(mt);
            rt = wave_max(rt);
            // a block with an infinity or a NaN is NaN; one whose largest |m| is below 2^-100 is zero
            const bool m_ok = mt < 0x7f800000u, r_ok = rt < 0x7f800000u, m_any = m_ok && mt >= (27u << 23), r_any = r_ok && rt > 0;
            const float ms = !m_ok ? __builtin_nanf("") : m_any ? __uint_as_float(mt) / kAvgTop : 0.0f;
            const float vs = !r_ok ? __builtin_nanf("") : r_any ? __uint_as_float(rt) / kSqTop : 0.0f;
            const float mi = m_any ? 1.0f / ms : 0.0f, vi = r_any ? 1.0f / vs : 0.0f;
            uint32_t mc = 0, vc = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t cm = m_any ? avg_code(__builtin_fabsf(m[k]) * mi) | (m[k] < 0.0f ? 128u : 0u) : 0u;
                const uint32_t cv = r_any && r[k] > 0.0f ? max(sq_code(r[k] * vi, dither((uint32_t)(i + k), (uint32_t)step)), 1u) : 0u;
                mc |= cm << (8 * k);
                vc |= cv << (8 * k);
            }
            store_codes((uint8_t*)t.exp_avg + i, n, mc);
            store_codes((uint8_t*)t.exp_avg_sq + i, n, vc);
            if (lane == 0) {
                t.avg_scale[block] = ms;
                t.sq_scale[block] = vs;
            }
        } else {
            store4((float*)t.exp_avg + i, n, m);
            store4((float*)t.exp_avg_sq + i, n, v);
        }
    }
}

}  // namespace

static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");

hipError_t launch_adamw(const AdamwArgs& a, int chunks, bool grad_f16, bool bits8, hipStream_t st) {
    if (chunks < 1) return hipErrorInvalidValue;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)chunks), dim3(256), 0, st, a);
        return hipGetLastError();
    };
    if (grad_f16) return bits8 ? go(adamw_kernel<_Float16, true>) : go(adamw_kernel<_Float16, false>);
    return bits8 ? go(adamw_kernel<float, true>) : go(adamw_kernel<float, false>);
}

}  // namespace bd

// ---- C ABI ---------------------------------------------------------------------------------

namespace {

constexpr int64_t kMostChunks = BD_ADAMW_MAX_ELEMENTS / bd::kAdamwChunk;   // workgroups of a launch: 2^23, below 2^32 threads
constexpr uint64_t kPlanMagic = 0x31304d4144414c50ull;
struct PlanHeader {
    uint64_t magic;
    int32_t n, grad_f16, bits8, unused;
};
// the tensors that have elements, behind the header
const bd::AdamwTensor* plan_tensors(const void* plan) { return (const bd::AdamwTensor*)((const char*)plan + sizeof(PlanHeader)); }

bd_status make_plan(void* plan, size_t plan_bytes, int32_t n, float* const* param, uint16_t* const* param_f16, const void* const* grad,
                    int32_t grad_f16, void* const* exp_avg, void* const* exp_avg_sq, float* const* avg_scale, float* const* sq_scale,
                    const int64_t* numel) {
    using bd::misaligned;
    if (n < 0 || n > BD_ADAMW_MAX_TENSORS) return BD_ERR_SHAPE;
    if (!plan) return BD_ERR_NULL;
    if (plan_bytes < bd_adamw_plan_bytes(n)) return BD_ERR_WORKSPACE;
    if (misaligned(plan, 8)) return BD_ERR_ALIGN;
    if (n > 0 && (!param || !grad || !exp_avg || !exp_avg_sq || !numel || (avg_scale == nullptr) != (sq_scale == nullptr))) return BD_ERR_NULL;
    const bool bits8 = avg_scale != nullptr;
    PlanHeader head{kPlanMagic, 0, grad_f16 ? 1 : 0, bits8 ? 1 : 0, 0};
    std::vector<bd::AdamwTensor> tensors;
    std::vector<bd::Range> ranges;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] < 0 || numel[i] > BD_ADAMW_MAX_ELEMENTS) return BD_ERR_SHAPE;
        if (numel[i] == 0) continue;
        bd::AdamwTensor t{param[i], param_f16 ? param_f16[i] : nullptr, grad[i], exp_avg[i], exp_avg_sq[i],
                          bits8 ? avg_scale[i] : nullptr, bits8 ? sq_scale[i] : nullptr, numel[i]};
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
    std::memcpy(plan, &head, sizeof(head));
    if (head.n > 0) std::memcpy((char*)plan + sizeof(head), tensors.data(), tensors.size() * sizeof(bd::AdamwTensor));
    return BD_OK;
}

}  // namespace

extern "C" {

size_t bd_adamw_plan_bytes(int32_t n) {
    return n < 0 || n > BD_ADAMW_MAX_TENSORS ? 0 : sizeof(PlanHeader) + (size_t)n * sizeof(bd::AdamwTensor);
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

bd_status bd_adamw(const void* plan, size_t plan_bytes, const float* lr, const int64_t* step, const float* grad_scale, const int32_t* skip,
                   double beta1, double beta2, double eps, double weight_decay, void* stream) {
    if (!plan) return BD_ERR_NULL;
    PlanHeader head;
    if (bd::misaligned(plan, 8)) return BD_ERR_ALIGN;
    if (plan_bytes < sizeof(head)) return BD_ERR_FORMAT;
    std::memcpy(&head, plan, sizeof(head));
    if (head.magic != kPlanMagic || head.n < 0 || plan_bytes < bd_adamw_plan_bytes(head.n)) return BD_ERR_FORMAT;
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0 && eps >= 0.0 && weight_decay >= 0.0)) return BD_ERR_UNSUPPORTED;
    if (head.n == 0) return BD_OK;
    if (!lr || !step) return BD_ERR_NULL;
    if (bd::misaligned(lr, 4) || bd::misaligned(step, 8) || bd::misaligned(grad_scale, 4) || bd::misaligned(skip, 4)) return BD_ERR_ALIGN;
    const bd::AdamwTensor* const tensors = plan_tensors(plan);
    bd::AdamwArgs a;
    std::memset(&a, 0, sizeof(a));
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
    for (int32_t at = 0; at < head.n;) {
        int k = 0;
        int64_t chunks = 0;
        for (; at < head.n && k < bd::kAdamwTensors; ++at, ++k) {
            const int64_t more = (tensors[at].numel + bd::kAdamwChunk - 1) / bd::kAdamwChunk;
            if (k > 0 && chunks + more > kMostChunks) break;
            a.tensor[k] = tensors[at];
            a.chunk_begin[k] = (int32_t)chunks;
            chunks += more;
        }
        for (int j = k; j < bd::kAdamwTensors; ++j) a.chunk_begin[j] = INT_MAX;
        if (bd::launch_adamw(a, (int)chunks, head.grad_f16, head.bits8, (hipStream_t)stream) != hipSuccess) return BD_ERR_DEVICE;
    }
    return BD_OK;
}

}  // extern "C"
