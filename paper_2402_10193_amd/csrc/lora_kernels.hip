// Low-rank adapters of many tenants at once, forward and backward, for gfx950.
//
//   forward    h = A_e x      (shrink)     y = y0 + s_e B_e h        (expand)
//   backward   g = s_e B_e^T dy (shrink)   dx = dx0 + A_e^T g        (expand)
//              dA_e = sum_t g x^T          dB_e = s_e sum_t dy h^T   (grad)
//
// The ranks are a few to a few dozen, so that every product here is bound by the activations it streams (x, dy, y0, y) or, in
// a decode step, by latency; the matrix cores have room to spare.  That room buys precision: h and g are held in binary32 and
// enter the matrix cores as two binary16 numbers each, hi = fp16(v 2^-e) and lo = fp16(v 2^-e - hi), some 22 bits together.  e
// brings the largest of a token's values (grad: of a wavefront's values) to 2^14 .. 2^15, so that neither part leaves the
// range of binary16 whatever the scale of the activations or of the loss.  x, dy, A and B are binary16 as they are, the sums
// binary32.
//
// v_mfma_f32_16x16x32_f16: lane l = (r, g) = (l % 16, l / 16) supplies row r, elements 8 g .. 8 g + 7 of either operand; result
// register i of lane (n, q) is element (4 q + i, n).
#include "bd_device.h"
#include "bd_lora.h"

namespace bd {

namespace {

__device__ __forceinline__ half8 load8(const uint16_t* p) {   // any 2-byte alignment: rows of odd length
    half8 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
__device__ __forceinline__ half8 load8_first(const uint16_t* p, int64_t n) {   // the first n elements (n < 8), zeros behind them
    half8 v = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) v[i] = __builtin_bit_cast(_Float16, p[i]);
    return v;
}
__device__ __forceinline__ half8 load8_upto(const uint16_t* p, int64_t n) { return n >= 8 ? load8(p) : load8_first(p, n); }

// Rows of 8 halves -> columns: element i of out[j] = element j of in[i].  32 byte permutes.
__device__ __forceinline__ void transpose8(const half8 (&in)[8], half8 (&out)[8]) {
    u32x4 r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __builtin_bit_cast(u32x4, in[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        u32x4 c;
#pragma unroll
        for (int p = 0; p < 4; ++p)
            c[p] = __builtin_amdgcn_perm(r[2 * p + 1][j >> 1], r[2 * p][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
        out[j] = __builtin_bit_cast(half8, c);
    }
}

__device__ __forceinline__ float4v mfma(const half8 a, const half8 b, const float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ float finite_abs(float v) { return finite(v) ? __builtin_fabsf(v) : 0.0f; }

// The exponent e of a group of values whose largest finite one is m: m 2^-e lies in [2^14, 2^15).  Bounded so that 2^-e is a
// normal number: groups below 2^-86 keep fewer bits.
__device__ __forceinline__ int group_exponent(float m) {
    const int e = (int)(__float_as_uint(m) >> 23) - 127 - 14;
    return e < -100 ? -100 : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// hi and lo of v 2^-e (scale = 2^-e); an infinity or NaN goes through in hi alone
__device__ __forceinline__ void split_half(float v, float scale, _Float16* hi, _Float16* lo) {
    const float s = v * scale;
    *hi = (_Float16)s;
    *lo = finite(s) ? (_Float16)(s - (float)*hi) : (_Float16)0.0f;
}

// What a workgroup works on.
struct Where {
    const uint16_t* w;
    int32_t hrow, tenant, count, rank, mat;   // hrow: of the tile's first token; count: tokens of the tile
    int32_t first;                            // many tokens: sorted position of the tile's first token
    int32_t record;
};

template <int NT, typename Args>
__device__ __forceinline__ Where find_tile(const Args& a, int t) {
    Where u;
    if constexpr (NT == 1) {
        const LoraTile& k = a.tile[t];
        u = Where{k.w, k.hrow, k.tenant, k.count, k.rank, k.mat, 0, t};
    } else {
        int j = 0;
        while (j + 1 < a.n_records && a.job[j + 1].tile_begin <= t) ++j;
        const LoraJob& k = a.job[j];
        const int skip = (t - k.tile_begin) * 16 * NT;
        u = Where{k.w, k.hrow + skip, k.tenant, min(k.count - skip, 16 * NT), k.rank, k.mat, k.first + skip, j};
    }
    return u;
}
template <int NT, typename Args>
__device__ __forceinline__ int token_of(const Args& a, const Where& u, int column) {
    if constexpr (NT == 1) return a.tile[u.record].col[column];
    const int p = u.first + column;
    return a.order ? a.order[p] : p;
}

constexpr int kShrinkThreads = kLoraShrinkWaves * kWave;

// h = A x or g = s B^T dy of one tile, 16 RT ranks and one part of the sum.  The wavefronts divide the part among them; each
// reads its operands straight into matrix-core order (a row's 64 bytes per instruction), the eight sums meet in LDS.
// Rows of A beyond the rank and columns without a token repeat the first: rows and columns do not mix, and what they give is
// not kept.
template <bool TR, int NT, int RT>
__global__ __launch_bounds__(kShrinkThreads) void lora_shrink_kernel(const LoraShrinkArgs a) {
    const Where u = find_tile<NT>(a, blockIdx.x);
    const int rt0 = blockIdx.z * RT;
    if (16 * rt0 >= u.rank) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const uint16_t* row[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = 16 * n + m;
        row[n] = a.src + (int64_t)token_of<NT>(a, u, c < u.count ? c : 0) * a.K + 8 * g;
    }
    const uint16_t* wrow[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int rank = 16 * (rt0 + r) + m < u.rank ? 16 * (rt0 + r) + m : 0;
        wrow[r] = TR ? u.w + (int64_t)8 * g * u.rank + rank : u.w + (int64_t)rank * a.K + 8 * g;
    }
    float4v acc[RT][NT] = {};
    const int64_t steps = (a.K + 31) / 32, parts = (int64_t)a.splits * kLoraShrinkWaves, part = (int64_t)blockIdx.y * kLoraShrinkWaves + wave;
    const int64_t s0 = steps * part / parts, s1 = steps * (part + 1) / parts;
    const int64_t whole = a.K / 32 < s1 ? a.K / 32 : s1;   // steps of 32 elements; a last one of fewer is the backward pass's only
    auto steps_at = [&](auto count, int64_t s) {   // `count` steps: all their loads, then their products
        constexpr int C = decltype(count)::value;
        half8 xv[C][NT], wv[C][RT];
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int n = 0; n < NT; ++n) xv[c][n] = load8(row[n] + 32 * (s + c));
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if constexpr (TR) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) wv[c][r][i] = __builtin_bit_cast(_Float16, wrow[r][(32 * (s + c) + i) * u.rank]);
                } else {
                    wv[c][r] = load8(wrow[r] + 32 * (s + c));
                }
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[r][n] = mfma(wv[c][r], xv[c][n], acc[r][n]);
    };
    constexpr int kAtOnce = NT * RT == 1 ? 8 : NT + RT <= 5 ? 4 : 2;   // what the registers hold
    int64_t s = s0;
    for (; s + kAtOnce <= whole; s += kAtOnce) steps_at(std::integral_constant<int, kAtOnce>{}, s);
    for (; s < whole; ++s) steps_at(std::integral_constant<int, 1>{}, s);
    if (TR && whole < s1 && s0 < s1) {
        s = s1 - 1;
        const int64_t left = a.K - 32 * s - 8 * g;
        half8 xv[NT], wv[RT];
#pragma unroll
        for (int n = 0; n < NT; ++n) xv[n] = load8_upto(row[n] + 32 * s, left);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            wv[r] = half8{};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) wv[r][i] = __builtin_bit_cast(_Float16, wrow[r][(32 * s + i) * u.rank]);
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[r][n] = mfma(wv[r], xv[n], acc[r][n]);
    }
    __shared__ float4v part_sum[kLoraShrinkWaves][NT][kWave];
    const float scale = TR ? a.scale[u.tenant] : 1.0f;
    float* const dst = a.h + (int64_t)blockIdx.y * a.split_stride;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (16 * (rt0 + r) >= u.rank) continue;   // (of the whole workgroup)
        if (r > 0) __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n) part_sum[wave][n][lane] = acc[r][n];
        __syncthreads();
        for (int t = threadIdx.x; t < NT * kWave; t += kShrinkThreads) {
            const int n = t / kWave, l = t & (kWave - 1), c = 16 * n + (l & 15), rank = 16 * (rt0 + r) + 4 * (l >> 4);
            if (c >= u.count) continue;
            float4v v = part_sum[0][n][l];
#pragma unroll
            for (int w = 1; w < kLoraShrinkWaves; ++w) v += part_sum[w][n][l];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = rank + i < u.rank ? v[i] * scale : 0.0f;
            *(float4v*)(dst + (int64_t)(u.hrow + c) * a.ld + rank) = v;
        }
    }
}

constexpr int kExpandThreads = kLoraExpandWaves * kWave;
constexpr int kExpandRanks = 128;   // ranks whose hi and lo are in LDS at a time

// y = y0 + s B h, or dx = dx0 + A^T g, of one tile by 512 features.  h comes in as `splits` partial sums.  Feature 8 m + j of a
// wavefront's 128 is row m of its MFMA j, so that a lane ends up with 8 neighbours of a token's row in the 8 accumulators: one
// 16-byte load of y0 and one such store for each.  The 32 elements of an MFMA's sum are 16 ranks, hi in lane groups 0 and 1 and
// lo in 2 and 3, both with the same weights.
template <bool TR, int NT>
__global__ __launch_bounds__(kExpandThreads) void lora_expand_kernel(const LoraExpandArgs a) {
    constexpr int kTokens = 16 * NT, kPer = kExpandThreads / kTokens;   // threads per token while h is prepared
    constexpr int kPitch = kExpandRanks + 8;
    __shared__ __align__(16) _Float16 hi[kTokens][kPitch], lo[kTokens][kPitch];
    __shared__ int exponent[kTokens];
    const Where u = find_tile<NT>(a, blockIdx.x);
    const int64_t F = a.F[u.mat];
    if (blockIdx.y > 0 && (int64_t)blockIdx.y * kLoraExpandWaves * kLoraFeatures >= F) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const int padded = (u.rank + 15) & ~15;

    const int c = threadIdx.x / kPer, sub = threadIdx.x % kPer;   // the token whose h this thread prepares
    const bool real = c < u.count;
    const float* const src = a.h + (int64_t)(u.hrow + (real ? c : 0)) * a.ld;
    auto sum4 = [&](int r) {
        float4v v = *(const float4v*)(src + r);
        for (int s = 1; s < a.splits; ++s) v += *(const float4v*)(src + s * a.split_stride + r);
        return v;
    };
    float top = 0.0f;
    float* const kept = !TR && a.h_out[u.mat] && blockIdx.y == 0 && real ? a.h_out[u.mat] + (int64_t)token_of<NT>(a, u, c) * a.h_ld : nullptr;
    for (int r = 4 * sub; r < padded; r += 4 * kPer) {
        const float4v v = sum4(r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top = fmaxf(top, finite_abs(v[i]));
            if (kept && r + i < u.rank) kept[r + i] = v[i];
        }
    }
#pragma unroll
    for (int d = kPer / 2; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
    const int e = group_exponent(top);
    if (sub == 0) exponent[c] = e;
    const float down = power_of_two(-e);

    const int64_t f0 = ((int64_t)blockIdx.y * kLoraExpandWaves + wave) * kLoraFeatures;
    const bool active = f0 < F;
    float4v acc[8][NT] = {};
    for (int r0 = 0; r0 < padded; r0 += kExpandRanks) {
        const int ranks = min(kExpandRanks, padded - r0);
        if (r0 > 0) __syncthreads();
        for (int r = 4 * sub; r < ranks; r += 4 * kPer) {
            const float4v v = sum4(r0 + r);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                _Float16 h = (_Float16)0.0f, l = (_Float16)0.0f;
                if (real) split_half(v[i], down, &h, &l);
                hi[c][r + i] = h;
                lo[c][r + i] = l;
            }
        }
        __syncthreads();
        if (!active) continue;
        for (int rc = 0; rc < ranks; rc += 16) {
            half8 wv[8];
            const int rank = r0 + rc + 8 * (g & 1), left = u.rank - rank;
            if constexpr (TR) {
                half8 rows[8];
                const int64_t f = f0 + 8 * m <= F - 8 ? f0 + 8 * m : F - 8;   // (F = in, a multiple of 32)
#pragma unroll
                for (int i = 0; i < 8; ++i) rows[i] = i < left ? load8(u.w + (int64_t)(rank + i) * F + f) : half8{};
                transpose8(rows, wv);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int64_t f = f0 + 8 * m + j < F ? f0 + 8 * m + j : F - 1;
                    wv[j] = load8_upto(u.w + f * u.rank + rank, left);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const half8 hv = *(const half8*)(g < 2 ? &hi[16 * n + m][rc + 8 * g] : &lo[16 * n + m][rc + 8 * (g - 2)]);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j][n] = mfma(wv[j], hv, acc[j][n]);
            }
        }
    }
    if (padded == 0) __syncthreads();   // `exponent`
    if (!active) return;
    const float scale = TR || u.rank == 0 ? 1.0f : a.scale[u.mat][u.tenant];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int col = 16 * n + m;
        if (col >= u.count) continue;
        const int64_t at = (int64_t)token_of<NT>(a, u, col) * F;
        const uint16_t* const y0 = a.y0[u.mat] ? a.y0[u.mat] + at : nullptr;
        uint16_t* const y = a.y[u.mat] + at;
        const float up = power_of_two(exponent[col]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t f = f0 + 32 * g + 8 * i;
            if (f >= F) continue;
            const half8 before = y0 ? load8_upto(y0 + f, F - f) : half8{};
            half8 v;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (_Float16)((float)before[j] + scale * (acc[j][n][i] * up));
            if (F - f >= 8) {
                __builtin_memcpy(y + f, &v, 16);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < F - f) *(_Float16*)(y + f + j) = v[j];
            }
        }
    }
}

constexpr int kGradThreads = kLoraGradWaves * kWave;

// dA or dB of one job: 128 features by 16 RT ranks, summed over one part of the job's tokens.  The tokens are the sum's index, so
// both operands want 8 tokens of one feature (rank) in a lane: a lane loads 16 bytes of 8 tokens' rows (256 bytes of a row per
// instruction) and turns the 8 x 8 block in its registers.  The wavefronts divide the tokens and meet in LDS.
template <int RT>
__global__ __launch_bounds__(kGradThreads) void lora_grad_kernel(const LoraGradArgs a) {
    const LoraGradJob& job = a.job[blockIdx.y / a.token_splits];
    const int split = blockIdx.y % a.token_splits, rt0 = blockIdx.z * RT, rank_all = job.rank, count = job.count, first = job.first;
    if (16 * rt0 >= rank_all) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const int64_t F = a.F, f0 = (int64_t)blockIdx.x * kLoraFeatures, fl = f0 + 8 * m;
    const int steps = (count + 31) / 32, parts = a.token_splits * kLoraGradWaves, part = split * kLoraGradWaves + wave;
    const int s0 = (int)((int64_t)steps * part / parts), s1 = (int)((int64_t)steps * (part + 1) / parts);
    auto token_at = [&](int i) { return a.order ? a.order[first + i] : first + i; };
    auto weight = [&](int i, int rank) {   // w of the job's token i; 0 where there is none
        if (i >= count || rank >= rank_all) return 0.0f;
        if (a.w_by_token) return a.w[(int64_t)token_at(i) * a.w_ld + rank];
        const float* const p = a.w + (int64_t)(first + i) * a.w_ld + rank;
        float v = p[0];
        for (int s = 1; s < a.w_splits; ++s) v += p[s * a.w_split_stride];
        return v;
    };
    float top = 0.0f;
    for (int s = s0; s < s1; ++s)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(weight(32 * s + 8 * g + i, 16 * (rt0 + r) + m)));
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
    const int e = group_exponent(top);
    const float down = power_of_two(-e), up = power_of_two(e);

    float4v acc[8][RT] = {};
    for (int s = s0; s < s1; ++s) {
        half8 rows[8], dv[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = 32 * s + 8 * g + i;
            rows[i] = t < count && fl < F ? load8_upto(a.d + (int64_t)token_at(t) * F + fl, F - fl) : half8{};
        }
        transpose8(rows, dv);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            half8 hi, lo;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                _Float16 h, l;
                split_half(weight(32 * s + 8 * g + i, 16 * (rt0 + r) + m), down, &h, &l);
                hi[i] = h;
                lo[i] = l;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j][r] = mfma(dv[j], hi, acc[j][r]);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j][r] = mfma(dv[j], lo, acc[j][r]);
        }
    }
    __shared__ float sum[kLoraGradWaves][8][4][kWave];   // [wave][j][i][lane (n, q)] = feature 8 (4 q + i) + j, rank n
    const float scale = a.scale ? a.scale[job.tenant] : 1.0f;
    float* const out = a.token_splits > 1 ? a.partial + split * a.part_stride + job.part : job.out;
    const bool add = a.accumulate && a.token_splits == 1;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (16 * (rt0 + r) >= rank_all) continue;   // (of the whole workgroup)
        if (r > 0) __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[wave][j][i][lane] = acc[j][r][i] * up;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = threadIdx.x + k * kGradThreads;   // of 16 x 128
            const int n = a.rank_major ? at / kLoraFeatures : at & 15, f = a.rank_major ? at % kLoraFeatures : at >> 4;
            const int row = f >> 3, j = f & 7, rank = 16 * (rt0 + r) + n;
            if (rank >= rank_all || f0 + f >= F) continue;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kLoraGradWaves; ++w) v += sum[w][j][row & 3][16 * (row >> 2) + n];
            v *= scale;
            float* const p = out + (a.rank_major ? (int64_t)rank * F + f0 + f : (f0 + f) * rank_all + rank);
            *p = add ? *p + v : v;
        }
    }
}

// out (+)= the sum of the parts, in their order; zeros where there are none
__global__ __launch_bounds__(256) void lora_reduce_kernel(const LoraReduceArgs a) {
    const auto& job = a.job[blockIdx.y];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < job.n; i += (int64_t)gridDim.x * 256) {
        float v = 0.0f;
        for (int s = 0; a.partial && s < a.token_splits; ++s) v += a.partial[s * a.part_stride + job.part + i];
        job.out[i] = a.accumulate ? job.out[i] + v : v;
    }
}

}  // namespace

static_assert(sizeof(LoraShrinkArgs) <= 4096 && sizeof(LoraExpandArgs) <= 4096 && sizeof(LoraGradArgs) <= 4096 && sizeof(LoraReduceArgs) <= 4096,
              "kernel arguments");

hipError_t launch_lora_shrink(const LoraShrinkArgs& a, int columns, bool transposed, int max_rank, hipStream_t st) {
    const int rank_tiles = (max_rank + 15) / 16;
    if (a.n_tiles < 1 || rank_tiles < 1 || a.splits < 1) return hipErrorInvalidValue;
    auto go = [&](auto kernel, int RT) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_tiles, (unsigned)a.splits, (unsigned)((rank_tiles + RT - 1) / RT)), dim3(kShrinkThreads), 0, st, a);
        return hipGetLastError();
    };
    if (columns == 16) return transposed ? go(lora_shrink_kernel<true, 1, 1>, 1) : go(lora_shrink_kernel<false, 1, 1>, 1);
    if (rank_tiles == 1) return transposed ? go(lora_shrink_kernel<true, 4, 1>, 1) : go(lora_shrink_kernel<false, 4, 1>, 1);
    return transposed ? go(lora_shrink_kernel<true, 4, 4>, 4) : go(lora_shrink_kernel<false, 4, 4>, 4);
}

hipError_t launch_lora_expand(const LoraExpandArgs& a, int columns, bool transposed, int64_t max_F, hipStream_t st) {
    constexpr int64_t per_group = kLoraExpandWaves * kLoraFeatures;
    const int64_t groups = max_F > 0 ? (max_F + per_group - 1) / per_group : 1;   // (F = 0: h alone)
    if (a.n_tiles < 1 || groups > 65535) return hipErrorInvalidValue;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_tiles, (unsigned)groups), dim3(kExpandThreads), 0, st, a);
        return hipGetLastError();
    };
    if (columns == 16) return transposed ? go(lora_expand_kernel<true, 1>) : go(lora_expand_kernel<false, 1>);
    return transposed ? go(lora_expand_kernel<true, 4>) : go(lora_expand_kernel<false, 4>);
}

hipError_t launch_lora_grad(const LoraGradArgs& a, int max_rank, hipStream_t st) {
    const int rank_tiles = (max_rank + 15) / 16;
    const int64_t groups = (a.F + kLoraFeatures - 1) / kLoraFeatures;
    if (a.n_jobs < 1 || rank_tiles < 1 || groups < 1 || a.token_splits < 1) return hipErrorInvalidValue;
    auto go = [&](auto kernel, int RT) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (unsigned)(a.n_jobs * a.token_splits), (unsigned)((rank_tiles + RT - 1) / RT)), dim3(kGradThreads), 0, st, a);
        return hipGetLastError();
    };
    return rank_tiles == 1 ? go(lora_grad_kernel<1>, 1) : rank_tiles == 2 ? go(lora_grad_kernel<2>, 2) : go(lora_grad_kernel<4>, 4);
}

hipError_t launch_lora_reduce(const LoraReduceArgs& a, int64_t max_n, hipStream_t st) {
    if (a.n_jobs < 1) return hipErrorInvalidValue;
    const int64_t blocks = (max_n + 1023) / 1024;
    hipLaunchKernelGGL(lora_reduce_kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks > 1024 ? 1024 : blocks), (unsigned)a.n_jobs), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace bd
