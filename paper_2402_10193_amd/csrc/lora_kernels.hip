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
#include <algorithm>

#include "bd_device.h"
#include "bd_lora.h"

namespace bd {

namespace {

__device__ __forceinline__ half8 load8(const uint16_t* p) {   // any 2-byte alignment: rows of odd length
    half8 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
// 8 elements one by one, those behind element `last` repeat it: short rows, rows of odd length
__device__ __forceinline__ half8 load8_each(const uint16_t* p, int64_t last) {
    half8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = *(const _Float16*)(p + (i < last ? i : last));
    return v;
}
// v with zeros where element i is not in [first, end)
__device__ __forceinline__ half8 only(half8 v, int first, int end) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i >= first && i < end ? v[i] : (_Float16)0.0f;
    return v;
}

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
#pragma unroll
        for (int k = 1; k < kLoraRecords; ++k) j += t >= a.jobs.tile_begin[k] ? 1 : 0;
        const LoraJob& k = a.jobs.job[j];
        const int skip = (t - a.jobs.tile_begin[j]) * 16 * NT;
        u = Where{k.w, k.hrow + skip, k.tenant, min(k.count - skip, 16 * NT), k.rank, k.mat, k.first + skip, j};
    }
    return u;
}
template <int NT, typename Args>
__device__ __forceinline__ int token_of(const Args& a, const Where& u, int column) {
    if constexpr (NT == 1) {   // a choice among words that came by a scalar load: no vector load of a kernel argument
        const LoraTile& t = a.tile[u.record];
        uint32_t w = t.col[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) w = (column >> 1) == k ? t.col[k] : w;
        return (column & 1) ? w >> 16 : w & 0xFFFFu;
    }
    const int p = u.first + column;
    return a.order ? a.order[p] : p;
}

// The tokens of N columns, the loads of the order all at once.
template <int NT, int N, typename Args>
__device__ __forceinline__ void tokens_of(const Args& a, const Where& u, const int (&column)[N], int (&token)[N]) {
    if constexpr (NT == 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) token[k] = token_of<NT>(a, u, column[k]);
    } else if (a.order) {
#pragma unroll
        for (int k = 0; k < N; ++k) token[k] = a.order[u.first + column[k]];
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) token[k] = u.first + column[k];
    }
}

constexpr int kShrinkThreads = kLoraShrinkWaves * kWave;

// A wavefront's own piece of LDS, 32 rows of 16 RT ranks of B (B [K, rank] has the sum's index outside): stored as rows, read back
// as matrix-core operands by the transposing read, which gives lane c of 16 the column c of the 4 x 16 block that the 16 lanes'
// addresses cover.  The pitch of 8 more keeps rows on different banks.
template <int RT>
struct Stage {
    static constexpr int kPitch = 16 * RT + 8;
    _Float16 row[32][kPitch];

    __device__ __forceinline__ half8 operand(int r, int lane) const {
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4 lds4;
        const int g = lane >> 4, c = lane & 15;
        const _Float16* const p = &row[8 * g + (c >> 2)][16 * r + 4 * (c & 3)];
        const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + 4 * kPitch));
        half8 v;
        __builtin_memcpy(&v, &lo, 8);
        __builtin_memcpy((char*)&v + 8, &hi, 8);
        return v;
    }
};

// h = A x or g = s B^T dy of one tile, 16 RT ranks and one part of the sum.  The wavefronts divide the part among them; each
// reads x (and A) straight into matrix-core order (a row's 64 bytes per instruction), the eight sums meet in LDS.
// Ranks and columns beyond the last repeat others or hold anything: rows and columns do not mix, and what they give is not kept.
template <bool TR, int NT, int RT, bool ODD>
__global__ __launch_bounds__(kShrinkThreads) void lora_shrink_kernel(const LoraShrinkArgs a) {
    const Where u = find_tile<NT>(a, blockIdx.x);
    const int rt0 = blockIdx.z * RT;
    if (16 * rt0 >= u.rank) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const uint16_t* row[NT];
    int column[NT], token[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) column[n] = 16 * n + m < u.count ? 16 * n + m : 0;
    tokens_of<NT>(a, u, column, token);
#pragma unroll
    for (int n = 0; n < NT; ++n) row[n] = a.src + (int64_t)token[n] * a.K + 8 * g;
    constexpr size_t kSums = sizeof(float4v) * kLoraShrinkWaves * NT * kWave, kStages = TR ? sizeof(Stage<RT>) * kLoraShrinkWaves : 0;
    __shared__ __align__(16) char lds[kSums > kStages ? kSums : kStages];
    Stage<RT>& stage = ((Stage<RT>*)lds)[wave];
    // backward: the lane's 16-byte pieces of 32 rows of B, where rows are whole pieces; else element by element
    const int width = min(16 * RT, u.rank - 16 * rt0);
    const bool pieces = !ODD || u.rank % 8 == 0;
    int piece_row[RT], piece_col[RT];
    const uint16_t* wrow[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if constexpr (TR) {
            const int at = lane + kWave * r, per_row = width / 8;
            piece_row[r] = pieces ? at / per_row : 32;   // 32 and more: none
            piece_col[r] = pieces ? 8 * (at % per_row) : 0;
            wrow[r] = u.w + 16 * rt0 + piece_col[r];
        } else {
            const int rank = 16 * (rt0 + r) + m < u.rank ? 16 * (rt0 + r) + m : 0;
            wrow[r] = u.w + (int64_t)rank * a.K + 8 * g;
        }
    }
    float4v acc[RT][NT] = {};
    // Steps of 32 elements.  A last one of fewer (the backward pass's only: K is then `out`) is the last 32 elements, those zero that
    // an earlier step has had; a K below 32 is read element by element.
    const int64_t steps = (a.K + 31) / 32, parts = (int64_t)a.splits * kLoraShrinkWaves, part = (int64_t)blockIdx.y * kLoraShrinkWaves + wave;
    const int64_t s0 = steps * part / parts, s1 = steps * (part + 1) / parts;
    const int64_t whole = a.K / 32 < s1 ? a.K / 32 : s1;
    auto steps_at = [&](auto count, auto ragged, int64_t s) {   // `count` steps: all their loads, then their products
        constexpr int C = decltype(count)::value;
        constexpr bool kRagged = decltype(ragged)::value;
        const int64_t k0 = kRagged ? (!ODD || a.K >= 32 ? a.K - 32 : 0) : 32 * s;
        const int had = kRagged ? (int)(32 * s - k0) : 0, end = ODD && kRagged && a.K < 32 ? (int)a.K : 32;   // rows that count: had .. end - 1
        half8 xv[C][NT], wv[C][RT];
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (ODD && kRagged && a.K < 32)
                    xv[c][n] = load8_each(row[n] - 8 * g + min(8 * g, end - 1), max(end - 1 - 8 * g, 0));
                else
                    xv[c][n] = load8(row[n] + k0 + 32 * c);
                if constexpr (kRagged) xv[c][n] = only(xv[c][n], had - 8 * g, end - 8 * g);
            }
            if constexpr (!TR) {
#pragma unroll
                for (int r = 0; r < RT; ++r) wv[c][r] = load8(wrow[r] + k0 + 32 * c);
            } else if (pieces) {   // a lane without a piece reads another's: loads without branches
#pragma unroll
                for (int r = 0; r < RT; ++r) wv[c][r] = load8(wrow[r] + (k0 + 32 * c + min(piece_row[r], end - 1)) * u.rank);
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (TR) {
                if (pieces) {
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        if (piece_row[r] < 32) *(half8*)&stage.row[piece_row[r]][piece_col[r]] = piece_row[r] >= had && piece_row[r] < end ? wv[c][r] : half8{};
                } else if constexpr (ODD) {
                    _Float16 v[8 * RT];
#pragma unroll
                    for (int k = 0; k < 8 * RT; ++k) {
                        const int at = lane + kWave * k, r = at / (16 * RT), rank = 16 * rt0 + at % (16 * RT);
                        v[k] = *(const _Float16*)(u.w + (k0 + 32 * c + min(r, end - 1)) * u.rank + min(rank, u.rank - 1));
                    }
#pragma unroll
                    for (int k = 0; k < 8 * RT; ++k) {
                        const int at = lane + kWave * k, r = at / (16 * RT);
                        stage.row[r][at % (16 * RT)] = r >= had && r < end ? v[k] : (_Float16)0.0f;
                    }
                }
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const half8 w = TR ? stage.operand(r, lane) : wv[c][r];
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[r][n] = mfma(w, xv[c][n], acc[r][n]);
            }
            if constexpr (TR) __builtin_amdgcn_wave_barrier();
        }
    };
    constexpr int kAtOnce = ODD ? 1 : NT * RT == 1 ? 8 : NT + RT <= 5 ? 4 : 2;   // what the registers hold
    int64_t s = s0;
    for (; s + kAtOnce <= whole; s += kAtOnce) steps_at(std::integral_constant<int, kAtOnce>{}, std::false_type{}, s);
    for (; s < whole; ++s) steps_at(std::integral_constant<int, 1>{}, std::false_type{}, s);
    if constexpr (TR)
        if (s < s1) steps_at(std::integral_constant<int, 1>{}, std::true_type{}, s);
    const float scale = TR ? a.scale[u.tenant] : 1.0f;
    float* const dst = a.h + (int64_t)blockIdx.y * a.split_stride;
    auto* const sum = (float4v(*)[NT][kWave])lds;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (16 * (rt0 + r) >= u.rank) continue;   // (of the whole workgroup)
        if (TR || r > 0) __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n) sum[wave][n][lane] = acc[r][n];
        __syncthreads();
        for (int t = threadIdx.x; t < NT * kWave; t += kShrinkThreads) {
            const int n = t / kWave, l = t & (kWave - 1), c = 16 * n + (l & 15), rank = 16 * (rt0 + r) + 4 * (l >> 4);
            if (c >= u.count) continue;
            float4v v = sum[0][n][l];
#pragma unroll
            for (int w = 1; w < kLoraShrinkWaves; ++w) v += sum[w][n][l];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = rank + i < u.rank ? v[i] * scale : 0.0f;
            *(float4v*)(dst + (int64_t)(u.hrow + c) * a.ld + rank) = v;
        }
    }
}

constexpr int kExpandThreads = kLoraExpandWaves * kWave;
constexpr int kExpandRanks = 128;   // ranks whose hi and lo are in LDS at a time

// y = y0 + s B h, or dx = dx0 + A^T g, of one tile by 512 features.  h comes in as `splits` partial sums.  Rows of a result are
// tokens, columns features: feature 8 n + j of a wavefront's 128 is column n of its MFMA j, so that a lane ends up with 8
// neighbours of a token's row in its 8 accumulators, and 16 lanes with 256 bytes of the row: one load of y0 and one store for
// each.  The 32 elements of an MFMA's sum are 16 ranks, hi in lane groups 0 and 1 and lo in 2 and 3, both with the same weights.
// y0 and the first weights are asked for before h is prepared: three waits for memory become one.
template <bool TR, int NT, bool ODD>
__global__ __launch_bounds__(kExpandThreads) void lora_expand_kernel(const LoraExpandArgs a) {
    constexpr int kTokens = 16 * NT, kPer = kExpandThreads / kTokens;   // threads per token while h is prepared
    constexpr int kPitch = kExpandRanks + 8;
    __shared__ __align__(16) _Float16 hi[kTokens][kPitch], lo[kTokens][kPitch];
    __shared__ float unit[kTokens];
    const Where u = find_tile<NT>(a, blockIdx.x);
    const int64_t F = a.F[u.mat];
    if (blockIdx.y > 0 && (int64_t)blockIdx.y * kLoraExpandWaves * kLoraFeatures >= F) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const int padded = (u.rank + 15) & ~15;
    // the wavefront's features, f0 .. f0 + 127; the last one's 128 end with the row and it keeps what is its own; a row below 128 is
    // read element by element
    const int64_t f0 = ((int64_t)blockIdx.y * kLoraExpandWaves + wave) * kLoraFeatures, f = min(f0, max(F - kLoraFeatures, (int64_t)0)) + 8 * m;
    const bool active = f0 < F, vectors = !ODD || F >= kLoraFeatures;

    int64_t at[NT][4];   // the rows of y that the lane's results belong to: token 16 n + 4 g + i
    half8 before[NT][4];
    int column[4 * NT], token[4 * NT];
#pragma unroll
    for (int k = 0; k < 4 * NT; ++k) {
        const int c = 16 * (k >> 2) + 4 * g + (k & 3);
        column[k] = c < u.count ? c : 0;
    }
    tokens_of<NT>(a, u, column, token);
#pragma unroll
    for (int k = 0; k < 4 * NT; ++k) at[k >> 2][k & 3] = (int64_t)token[k] * F + f;
    const uint16_t* const y0 = active ? a.y0[u.mat] : nullptr;
    if (y0 && vectors) {
#pragma unroll
        for (int k = 0; k < 4 * NT; ++k) before[k >> 2][k & 3] = load8(y0 + at[k >> 2][k & 3]);
    } else if (ODD && y0) {
        const int64_t back = f < F ? 0 : f - (F - 1);   // a lane behind the row reads its last element
#pragma unroll
        for (int k = 0; k < 4 * NT; ++k) before[k >> 2][k & 3] = load8_each(y0 + at[k >> 2][k & 3] - back, F - 1 - f + back);
    } else {
#pragma unroll
        for (int k = 0; k < 4 * NT; ++k) before[k >> 2][k & 3] = half8{};
    }
    half8 wv[8];   // forward: the weights of 16 ranks; backward: 8 ranks' rows of A, still to be turned
    auto load_weights = [&](int r) {
        const int rank = r + 8 * (g & 1), left = u.rank - rank;
        if constexpr (TR) {
            const uint16_t* const w = u.w + (f <= F - 8 ? f : F - 8);   // (F = in, a multiple of 32)
#pragma unroll
            for (int i = 0; i < 8; ++i) wv[i] = load8(w + (int64_t)(i < left ? rank + i : u.rank - 1) * F);
            if (u.rank - r < 16) {   // rows beyond the rank repeat the last one: they do not count
#pragma unroll
                for (int i = 0; i < 8; ++i) wv[i] = i < left ? wv[i] : half8{};
            }
        } else {
            const uint16_t* w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = u.w + (f + j < F ? f + j : F - 1) * u.rank;
            if (!ODD || u.rank % 8 == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) wv[j] = load8(w[j] + (left > 0 ? rank : r));
                if (u.rank - r < 16) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) wv[j] = left > 0 ? wv[j] : half8{};
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) wv[j] = only(load8_each(w[j] + (left > 0 ? rank : r), left > 0 ? left - 1 : 0), 0, left);
            }
        }
    };
    if (active && padded > 0) load_weights(0);

    const int c = threadIdx.x / kPer, sub = threadIdx.x % kPer;   // the token whose h this thread prepares
    const bool real = c < u.count;
    const float* const src = a.h + (int64_t)(u.hrow + (real ? c : 0)) * a.ld;
    auto sum4 = [&](int r) {
        float4v part[kLoraMaxSplits];   // all loads before the first addition
#pragma unroll
        for (int s = 0; s < kLoraMaxSplits; ++s) part[s] = s < a.splits ? *(const float4v*)(src + s * a.split_stride + r) : float4v{};
        float4v v = part[0];
#pragma unroll
        for (int s = 1; s < kLoraMaxSplits; ++s) v += part[s];
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
    if (sub == 0) unit[c] = power_of_two(e);
    const float down = power_of_two(-e);

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
            half8 cols[8];
            if constexpr (TR) {
                transpose8(wv, cols);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) cols[j] = wv[j];
            }
            if (r0 + rc + 16 < padded) load_weights(r0 + rc + 16);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const half8 hv = *(const half8*)(g < 2 ? &hi[16 * n + m][rc + 8 * g] : &lo[16 * n + m][rc + 8 * (g - 2)]);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j][n] = mfma(hv, cols[j], acc[j][n]);
            }
        }
    }
    if (padded == 0) __syncthreads();   // `unit`
    if (!active) return;
    const float scale = TR || u.rank == 0 ? 1.0f : a.scale[u.mat][u.tenant];
    uint16_t* const y = a.y[u.mat];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = 16 * n + 4 * g + i;
            if (col >= u.count || f >= F) continue;
            const float up = unit[col];
            half8 v;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (_Float16)((float)before[n][i][j] + scale * (acc[j][n][i] * up));
            if (f >= f0 && F - f >= 8) {
                __builtin_memcpy(y + at[n][i], &v, 16);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (f + j >= f0 && f + j < F) *(_Float16*)(y + at[n][i] + j) = v[j];
            }
        }
}

constexpr int kPrepThreads = 256;

// The second operand of the gradients, once for all their workgroups: 32 tokens' g (or h) as hi and lo in matrix-core order, one
// exponent for the 32.  Lane (n, q) holds rank n of its 16, tokens 8 q .. 8 q + 7, in 16 bytes.  Where g came in parts their sum
// takes the first part's place.
__global__ __launch_bounds__(kPrepThreads) void lora_prep_kernel(const LoraPrepArgs a) {
    int j = 0;
    while (j + 1 < a.n_jobs && a.job[j + 1].chunk_begin <= (int)blockIdx.x + a.chunk_first) ++j;
    const LoraPrepJob& job = a.job[j];
    const bool of_h = blockIdx.y + a.side_first == 1;
    const int chunk = blockIdx.x + a.chunk_first, t0 = (chunk - job.chunk_begin) * 32, rank_all = job.rank, tiles = (rank_all + 15) / 16;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, n = lane & 15, q = lane >> 4;
    constexpr int kMine = kLoraMaxRank / 16 / (kPrepThreads / kWave);   // rank tiles of a wavefront
    // tokens and ranks beyond the last repeat it: loads without branches; what they bring is replaced by zeros
    int64_t at[8];
    const float* const src = of_h ? a.h : a.g;
    {
        int p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = job.first + min(t0 + 8 * q + i, job.count - 1);
        if (of_h && a.order) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = a.order[p[i]];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) at[i] = (int64_t)p[i] * (of_h ? a.h_ld : a.ld);
    }
    const int splits = of_h ? 1 : a.splits;
    float v[kMine][8];
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const int rt = wave + k * (kPrepThreads / kWave), rank = 16 * rt + n, column = min(rank, rank_all - 1);
        if (rt >= tiles) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = src[at[i] + column];
        for (int s = 1; s < splits; ++s) {
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = src[s * a.split_stride + at[i] + column];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] += w[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool real = t0 + 8 * q + i < job.count && rank < rank_all;
            if (splits > 1 && real) a.g[at[i] + column] = v[k][i];
            v[k][i] = real ? v[k][i] : 0.0f;
            top = fmaxf(top, finite_abs(v[k][i]));
        }
    }
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
    __shared__ float tops[kPrepThreads / kWave];
    if (lane == 0) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPrepThreads / kWave; ++w) top = fmaxf(top, tops[w]);
    const int e = group_exponent(top);
    if (threadIdx.x == 0) a.exponent[of_h][chunk] = e;
    const float down = power_of_two(-e);
    half8* const out = a.operand[of_h] + (int64_t)chunk * (a.ld / 16) * 2 * kWave;
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const int rt = wave + k * (kPrepThreads / kWave);
        if (rt >= tiles) continue;
        half8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            _Float16 h, l;
            split_half(v[k][i], down, &h, &l);
            hi[i] = h;
            lo[i] = l;
        }
        out[(2 * rt) * kWave + lane] = hi;
        out[(2 * rt + 1) * kWave + lane] = lo;
    }
}

constexpr int kGradThreads = kLoraGradWaves * kWave;

// dA or dB of one job: 128 features by 16 RT ranks, summed over one part of the job's tokens.  The tokens are the sum's index, so
// both operands want 8 tokens of one feature (rank) in a lane: the second comes prepared, of x (dy) a lane loads 16 bytes of 8
// tokens' rows (256 bytes of a row per instruction) and turns the 8 x 8 block in its registers.  The wavefronts divide the tokens
// and meet in LDS.  The sums are kept in units of the present 32 tokens' exponent; tokens whose largest value is 2^-64 of the
// largest so far are below what binary32 would keep of them.
template <int RT, bool ODD>
__global__ __launch_bounds__(kGradThreads) void lora_grad_kernel(const LoraGradArgs a) {
    const int which = (int)blockIdx.z / a.rank_groups, rt0 = (int)blockIdx.z % a.rank_groups * RT;
    const LoraGradSide& side = a.side[which];
    const LoraGradJob& job = a.job[blockIdx.y / a.token_splits];
    const int split = blockIdx.y % a.token_splits, rank_all = job.rank, count = job.count, first = job.first;
    float* const result = job.out[which];
    const int64_t F = side.F, f0 = (int64_t)blockIdx.x * kLoraFeatures;
    if (!result || 16 * rt0 >= rank_all || f0 >= F) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const int64_t base = min(f0, max(F - kLoraFeatures, (int64_t)0)), fl = base + 8 * m;   // the last 128 features end with the row
    const int steps = (count + 31) / 32, parts = a.token_splits * kLoraGradWaves, part = split * kLoraGradWaves + wave;
    const int s0 = (int)((int64_t)steps * part / parts), s1 = (int)((int64_t)steps * (part + 1) / parts);
    const bool vectors = !ODD || F >= kLoraFeatures;
    const int64_t back = fl < F ? 0 : fl - (F - 1);
    half8 rows[8];
    auto load_rows = [&](int s) {   // tokens beyond the last repeat it: loads without branches
        int64_t at[8];
        int p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = first + min(32 * s + 8 * g + i, count - 1);
        if (a.order) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = a.order[p[i]];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) at[i] = p[i] * F + fl;
        if (vectors) {
#pragma unroll
            for (int i = 0; i < 8; ++i) rows[i] = load8(side.d + at[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) rows[i] = load8_each(side.d + at[i] - back, F - 1 - fl + back);
        }
    };
    float4v acc[8][RT] = {};
    int e = -200, largest = -200;   // none yet
    if (s0 < s1) load_rows(s0);
    for (int s = s0; s < s1; ++s) {
        const int chunk = job.chunk_begin + s, now = side.exponent[chunk];
        const half8* const op = side.operand + ((int64_t)chunk * (a.ld / 16) + rt0) * 2 * kWave + lane;
        half8 hi[RT], lo[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r)
            if (16 * (rt0 + r) < rank_all) {
                hi[r] = op[2 * r * kWave];
                lo[r] = op[(2 * r + 1) * kWave];
            }
        if (32 * s + 32 > count) {
#pragma unroll
            for (int i = 0; i < 8; ++i) rows[i] = 32 * s + 8 * g + i < count ? rows[i] : half8{};
        }
        half8 dv[8];
        transpose8(rows, dv);
        if (s + 1 < s1) load_rows(s + 1);
        if (now < largest - 64) continue;
        largest = max(largest, now);
        if (now != e) {
            if (e > -200) {
                const float f = e - now < -126 ? 0.0f : power_of_two(e - now);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int r = 0; r < RT; ++r) acc[j][r] *= f;
            }
            e = now;
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
            if (16 * (rt0 + r) < rank_all) {
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j][r] = mfma(dv[j], hi[r], acc[j][r]);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j][r] = mfma(dv[j], lo[r], acc[j][r]);
            }
    }
    const float up = e > -200 ? power_of_two(e) : 0.0f;
    __shared__ float sum[kLoraGradWaves][8][4][kWave];   // [wave][j][i][lane (n, q)] = feature 8 (4 q + i) + j, rank n
    const float scale = side.scale ? side.scale[job.tenant] : 1.0f;
    float* const out = a.token_splits > 1 ? side.partial + split * side.part_stride + job.part * F : result;
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
        for (int k = 0; k < 16 * kLoraFeatures / kGradThreads; ++k) {
            const int at = threadIdx.x + k * kGradThreads;   // of 16 x 128
            const int n = which == 0 ? at / kLoraFeatures : at & 15, f = which == 0 ? at % kLoraFeatures : at >> 4;
            const int row = f >> 3, j = f & 7, rank = 16 * (rt0 + r) + n;
            if (rank >= rank_all || base + f < f0 || base + f >= F) continue;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kLoraGradWaves; ++w) v += sum[w][j][row & 3][16 * (row >> 2) + n];
            v *= scale;
            float* const p = out + (which == 0 ? (int64_t)rank * F + base + f : (base + f) * rank_all + rank);
            *p = add ? *p + v : v;
        }
    }
}

// out (+)= the sum of the parts, in their order; zeros where there are none
__global__ __launch_bounds__(256) void lora_reduce_kernel(const LoraReduceArgs a) {
    const auto& job = a.job[blockIdx.y];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < job.n; i += (int64_t)gridDim.x * 256) {
        float v = 0.0f;
        for (int s = 0; s < a.token_splits; ++s) v += job.partial[s * job.part_stride + i];
        job.out[i] = a.accumulate ? job.out[i] + v : v;
    }
}

}  // namespace

static_assert(sizeof(LoraShrinkArgs) <= 4096 && sizeof(LoraExpandArgs) <= 4096 && sizeof(LoraGradArgs) <= 4096 && sizeof(LoraReduceArgs) <= 4096 && sizeof(LoraPrepArgs) <= 4096,
              "kernel arguments");

hipError_t launch_lora_shrink(const LoraShrinkArgs& a, int columns, bool transposed, int max_rank, bool odd, hipStream_t st) {
    const int rank_tiles = (max_rank + 15) / 16;
    if (a.n_tiles < 1 || rank_tiles < 1 || a.splits < 1 || a.splits > kLoraMaxSplits) return hipErrorInvalidValue;
    auto go = [&](auto kernel, int RT) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_tiles, (unsigned)a.splits, (unsigned)((rank_tiles + RT - 1) / RT)), dim3(kShrinkThreads), 0, st, a);
        return hipGetLastError();
    };
    odd |= a.K < 32;
    if (columns == 16) return !transposed ? go(lora_shrink_kernel<false, 1, 1, false>, 1) : odd ? go(lora_shrink_kernel<true, 1, 1, true>, 1) : go(lora_shrink_kernel<true, 1, 1, false>, 1);
    if (rank_tiles == 1) return !transposed ? go(lora_shrink_kernel<false, 4, 1, false>, 1) : odd ? go(lora_shrink_kernel<true, 4, 1, true>, 1) : go(lora_shrink_kernel<true, 4, 1, false>, 1);
    return !transposed ? go(lora_shrink_kernel<false, 4, 4, false>, 4) : odd ? go(lora_shrink_kernel<true, 4, 4, true>, 4) : go(lora_shrink_kernel<true, 4, 4, false>, 4);
}

hipError_t launch_lora_expand(const LoraExpandArgs& a, int columns, bool transposed, int64_t min_F, int64_t max_F, bool odd, hipStream_t st) {
    constexpr int64_t per_group = kLoraExpandWaves * kLoraFeatures;
    const int64_t groups = max_F > 0 ? (max_F + per_group - 1) / per_group : 1;   // (F = 0: h alone)
    if (a.n_tiles < 1 || groups > 65535 || a.splits > kLoraMaxSplits) return hipErrorInvalidValue;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_tiles, (unsigned)groups), dim3(kExpandThreads), 0, st, a);
        return hipGetLastError();
    };
    odd = (odd && !transposed) || min_F < kLoraFeatures;
    if (columns == 16) return transposed ? (odd ? go(lora_expand_kernel<true, 1, true>) : go(lora_expand_kernel<true, 1, false>)) : odd ? go(lora_expand_kernel<false, 1, true>) : go(lora_expand_kernel<false, 1, false>);
    return transposed ? (odd ? go(lora_expand_kernel<true, 2, true>) : go(lora_expand_kernel<true, 2, false>)) : odd ? go(lora_expand_kernel<false, 2, true>) : go(lora_expand_kernel<false, 2, false>);
}

hipError_t launch_lora_prep(const LoraPrepArgs& a, int chunks, int sides, hipStream_t st) {
    if (a.n_jobs < 1 || chunks < 1 || sides < 1) return hipErrorInvalidValue;
    hipLaunchKernelGGL(lora_prep_kernel, dim3((unsigned)chunks, (unsigned)sides), dim3(kPrepThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_lora_grad(const LoraGradArgs& a, int max_rank, hipStream_t st) {
    const int rank_tiles = (max_rank + 15) / 16, RT = rank_tiles >= 3 ? 4 : rank_tiles;
    const int64_t F = std::max(a.side[0].F, a.side[1].F), groups = (F + kLoraFeatures - 1) / kLoraFeatures;
    if (a.n_jobs < 1 || rank_tiles < 1 || groups < 1 || a.token_splits < 1) return hipErrorInvalidValue;
    LoraGradArgs b = a;
    b.rank_groups = (rank_tiles + RT - 1) / RT;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (unsigned)(b.n_jobs * b.token_splits), (unsigned)(2 * b.rank_groups)), dim3(kGradThreads), 0, st, b);
        return hipGetLastError();
    };
    // rows below 128 elements (a side that is not wanted has none)
    const bool odd = (a.side[0].F > 0 && a.side[0].F < kLoraFeatures) || (a.side[1].F > 0 && a.side[1].F < kLoraFeatures);
    if (odd) return RT == 1 ? go(lora_grad_kernel<1, true>) : RT == 2 ? go(lora_grad_kernel<2, true>) : go(lora_grad_kernel<4, true>);
    return RT == 1 ? go(lora_grad_kernel<1, false>) : RT == 2 ? go(lora_grad_kernel<2, false>) : go(lora_grad_kernel<4, false>);
}

hipError_t launch_lora_reduce(const LoraReduceArgs& a, int64_t max_n, hipStream_t st) {
    if (a.n_jobs < 1) return hipErrorInvalidValue;
    const int64_t blocks = (max_n + 1023) / 1024;
    hipLaunchKernelGGL(lora_reduce_kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks > 1024 ? 1024 : blocks), (unsigned)a.n_jobs), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace bd
