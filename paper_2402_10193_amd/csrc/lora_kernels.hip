// Low-rank adapters of many tenants at once, forward and backward, for gfx950.
//
//   forward    h = A_e x      (shrink)     y = y0 + s_e B_e h        (expand)
//   backward   g = s_e B_e^T dy (shrink)   dx = dx0 + A_e^T g        (expand)
//              dA_e = sum_t g x^T          dB_e = s_e sum_t dy h^T   (grad)
//
// The ranks are a few to a few dozen, so that every product here is bound by the activations it streams (x, dy, y0, y) or, in
// a decode step, by latency; the matrix cores have room to spare.  That room buys precision: h and g are held in binary32 and
// enter the matrix cores as two binary16 numbers each, hi = fp16(v 2^-e), toward zero, and lo = fp16(v 2^-e - hi), 22 bits together.  e
// brings the largest of a token's values (grad: of a rank's values in 32 tokens) to 2^14 .. 2^15, so that neither part leaves the
// range of binary16 whatever the scale of the activations or of the loss: a value keeps 22 bits, or what lies above 2^-39 of the
// largest of those it is added up with.  x, dy, A and B are binary16 as they are, the sums binary32.
//
// v_mfma_f32_16x16x32_f16: lane l = (r, g) = (l % 16, l / 16) supplies row r, elements 8 g .. 8 g + 7 of either operand; result
// register i of lane (n, q) is element (4 q + i, n).
#include <algorithm>

#include "bd_device.h"
#include "bd_launch.h"
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
// Elements at .. at + 7 of an array of n, those behind its end anything: the last 8, moved.  Rows that do not begin at 16 bytes, read past
// their ends.
template <bool SHORT>   // n may be below 8
__device__ __forceinline__ half8 load8_of(const uint16_t* p, int64_t at, int64_t n) {
    if (SHORT && n < 8) return load8_each(p + min(at, n - 1), max(n - 1 - at, (int64_t)0));
    const int64_t from = min(at, n - 8);
    const half8 v = load8(p + from);
    return __builtin_bit_cast(half8, __builtin_bit_cast(unsigned __int128, v) >> (16 * (int)min(at - from, (int64_t)7)));
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

// hi and lo of v 2^-e (scale = 2^-e), both of v's sign and neither zero (down to 2^-37 of the group's largest), so that times an infinity
// they add up to one; of what is not finite both are v.
__device__ __forceinline__ void split_half(float v, float scale, _Float16* hi, _Float16* lo) {
    const float s = v * scale;
    const uint16_t toward_zero = (uint16_t)__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(s, 0.0f));
    _Float16 h = __builtin_bit_cast(_Float16, toward_zero), l = (_Float16)(s - (float)h);
    if (l == (_Float16)0.0f) {   // (s is as good as a binary16 number: the one before it, and the step between them)
        h = __builtin_bit_cast(_Float16, (uint16_t)(toward_zero - ((toward_zero & 0x7fffu) > 0 ? 1 : 0)));
        l = (_Float16)(s - (float)h);
    }
    *hi = h;
    *lo = finite(s) ? l : h;
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
        // a lane looks at a record: few instructions (a kernel's code, too, comes out of memory when it begins)
        const int j = __builtin_amdgcn_readfirstlane(__popcll(__ballot(t >= a.jobs.tile_begin[threadIdx.x & (kWave - 1)])) - 1);
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

constexpr int kOrderThreads = 1024;

// The stable sort of tokens by job, one workgroup: a wavefront counts its run of tokens by job, the counts become places, and it goes through the
// run again, 64 tokens at a time: a token's place among the 64 from one vote per bit of the job.  4756 tokens of 5 jobs: 5 us, where their
// order itself, 960 tokens to a launch's arguments, takes 5 launches of 3 us.
__global__ __launch_bounds__(kOrderThreads) void lora_order_kernel(const LoraOrderArgs a) {
    constexpr int kWaves = kOrderThreads / kWave;
    __shared__ int place[kWaves][kLoraOrderJobs];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int each = (a.count + kOrderThreads - 1) / kOrderThreads * kWave, begin = min(wave * each, a.count), end = min(begin + each, a.count);
    auto job_of = [&](int i) { return (a.job[i * a.bits >> 3] >> (i * a.bits & 7)) & ((1 << a.bits) - 1); };
    for (int j = threadIdx.x; j < kWaves * kLoraOrderJobs; j += kOrderThreads) (&place[0][0])[j] = 0;
    __syncthreads();
    for (int i = begin + lane; i < end; i += kWave) atomicAdd(&place[wave][job_of(i)], 1);
    __syncthreads();
    if ((int)threadIdx.x < a.n_jobs) {
        int at = a.begin[threadIdx.x];
        for (int w = 0; w < kWaves; ++w) {
            const int n = place[w][threadIdx.x];
            place[w][threadIdx.x] = at;
            at += n;
        }
    }
    __syncthreads();
    for (int i0 = begin; i0 < end; i0 += kWave) {
        const int i = i0 + lane;
        const bool real = i < end;
        const int job = real ? job_of(i) : 0;
        uint64_t same = __ballot(real);
        for (int k = 0; k < a.bits; ++k) {
            const uint64_t set = __ballot((job >> k) & 1);
            same &= (job >> k) & 1 ? set : ~set;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        const int at = place[wave][job];
        __builtin_amdgcn_wave_barrier();
        if (real) {
            a.order[at + before] = a.first + i;
            if (before == 0) place[wave][job] = at + __popcll(same);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

constexpr int kDecodeThreads = 512;

// A decode step: up to 2 tokens of a tenant, up to 16 ranks, both products in one launch, bound by latency.  Every workgroup of 1024
// features forms all of h (A comes out of the cache again for the next one): a launch and the way of h through memory would take longer.
// Vector arithmetic: a wavefront reads rows of A as they are, 1 KB of a row per instruction, and a lane the rows of B of its two features;
// the matrix cores' order would take the address unit four times as long.  y0 and B are asked for before h is formed.
// 4096 x 4096, rank 16, a call in a graph: one token 4.6 us, q, k and v for 16 tenants (13.5 MB) 5.0 us, 2.7 TB/s; two launches 7.8 and 9 us.
template <int TOK, bool ODD>
__global__ __launch_bounds__(kDecodeThreads) void lora_decode_kernel(const LoraDecodeArgs a) {
    constexpr int kWaves = kDecodeThreads / kWave, kOctets = kLoraDecodeRank / 8, kRows = kLoraDecodeRank / kWaves, kSegments = 8, kFeatures = kLoraDecodeFeatures / kDecodeThreads;
    __shared__ __align__(16) float h[TOK][kLoraDecodeRank];
    const LoraDecodeTile& k = a.tile[blockIdx.x];
    const int rank = k.rank, count = k.count, mat = k.mat;
    const int64_t F = a.F[mat], base = (int64_t)blockIdx.y * kLoraDecodeFeatures;
    if (blockIdx.y > 0 && base >= F) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    int64_t token[TOK];
#pragma unroll
    for (int t = 0; t < TOK; ++t) token[t] = k.col[t < count ? t : 0];
    const uint16_t* const y0 = a.y0[mat];
    const bool work = base < F;   // (not for a matrix without outputs, whose h alone is asked for)

    _Float16 before[kFeatures][TOK];
    half8 b[kFeatures][kOctets];
    if (work) {
#pragma unroll
        for (int i = 0; i < kFeatures; ++i) {
            const int64_t f = min(base + i * kDecodeThreads + (int)threadIdx.x, F - 1);
#pragma unroll
            for (int t = 0; t < TOK; ++t) before[i][t] = y0 ? *(const _Float16*)(y0 + token[t] * F + f) : (_Float16)0.0f;
            const uint16_t* const row = k.wb + f * rank;
#pragma unroll
            for (int o = 0; o < kOctets; ++o)
                if (8 * o < rank) {
                    if (!ODD || 8 * o + 8 <= rank)
                        b[i][o] = load8(row + 8 * o);
                    else
                        b[i][o] = load8_each(row + 8 * o, rank - 1 - 8 * o);
                }
        }
    }

    // h: row by row of A, rows wave, wave + 8, ...; two rows at a time
#pragma unroll
    for (int i0 = 0; i0 < kRows; i0 += 2) {
        if (wave + kWaves * i0 >= rank) continue;   // (of the whole wavefront)
        float sum[2][TOK] = {};
        const uint16_t* row[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) row[i] = k.wa + (int64_t)min(wave + kWaves * (i0 + i), rank - 1) * a.in;
        for (int64_t k0 = 8 * lane; k0 < a.in + 8 * lane; k0 += 512 * kSegments) {
            half8 av[2][kSegments], xv[TOK][kSegments];
#pragma unroll
            for (int g = 0; g < kSegments; ++g) {   // (behind the row: its last elements, which count as zeros)
                const int64_t at = min(k0 + 512 * g, a.in - 8);
#pragma unroll
                for (int i = 0; i < 2; ++i) av[i][g] = load8(row[i] + at);
#pragma unroll
                for (int t = 0; t < TOK; ++t) xv[t][g] = load8(a.x + token[t] * a.in + at);
            }
#pragma unroll
            for (int g = 0; g < kSegments; ++g) {
                const bool real = k0 + 512 * g < a.in;
#pragma unroll
                for (int t = 0; t < TOK; ++t)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float s = 0.0f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) s = __builtin_fmaf((float)av[i][g][e], (float)xv[t][g][e], s);
                        sum[i][t] += real ? s : 0.0f;
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int t = 0; t < TOK; ++t) {
                const float v = wave_sum(sum[i][t]);
                const int r = wave + kWaves * (i0 + i);
                if (lane == 0 && r < rank) h[t][r] = v;
            }
    }
    __syncthreads();
    if (a.h_out[mat] && blockIdx.y == 0) {
        const int t = threadIdx.x / kLoraDecodeRank, r = threadIdx.x % kLoraDecodeRank;
        if (t < count && r < rank) a.h_out[mat][(int64_t)k.col[t] * a.h_ld + r] = h[t][r];
    }
    if (!work) return;
    const float scale = rank > 0 ? a.scale[mat][k.tenant] : 0.0f;
    float sum[kFeatures][TOK] = {};
#pragma unroll
    for (int o = 0; o < kOctets; ++o)
        if (8 * o < rank) {
#pragma unroll
            for (int t = 0; t < TOK; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!ODD || 8 * o + e < rank) {
                        const float v = h[t][8 * o + e];
#pragma unroll
                        for (int i = 0; i < kFeatures; ++i) sum[i][t] = __builtin_fmaf((float)b[i][o][e], v, sum[i][t]);
                    }
        }
#pragma unroll
    for (int i = 0; i < kFeatures; ++i) {
        const int64_t f = base + i * kDecodeThreads + threadIdx.x;
#pragma unroll
        for (int t = 0; t < TOK; ++t)
            if (f < F && t < count)   // (without an adapter every bit of y0, of zeros and NaN too)
                *(_Float16*)(a.y[mat] + token[t] * F + f) = rank > 0 ? (_Float16)__builtin_fmaf(sum[i][t], scale, (float)before[i][t]) : before[i][t];
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

// 16 N rows of 64 bytes: lane 4 r + p has loaded bytes 16 p of row r of each 16 (neighbouring lanes neighbouring bytes; the other way
// round an instruction takes the address unit four times as long).  Through a piece of LDS of the wavefront's own they come to lane
// 16 p + r.  The pitch of 80 keeps both accesses free of bank conflicts.
template <int N>
struct Turn {
    char row[16 * N][80];

    __device__ __forceinline__ void operator()(const half8 (&v)[N], half8 (&o)[N], int lane) {
#pragma unroll
        for (int n = 0; n < N; ++n) *(half8*)&row[16 * n + (lane >> 2)][16 * (lane & 3)] = v[n];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int n = 0; n < N; ++n) o[n] = *(const half8*)&row[16 * n + (lane & 15)][16 * (lane >> 4)];
        __builtin_amdgcn_wave_barrier();
    }
};

// h = A x or g = s B^T dy of one tile of 16 NT tokens, 16 RT ranks and one part of the sum.  The wavefronts divide the part among them,
// step by step of 32 elements, and their sums meet in LDS.  A and x go through a wavefront's own piece of LDS on their way (Turn), B too
// (Stage): in matrix-core order a load would take the address unit four times as long.  B is B [K, rank]: the sum's index outside.
// Ranks and columns beyond the last repeat others or hold anything: rows and columns do not mix, and what they give is not kept.
// Bound by the stream of x (dy), up to its start of some 4 us: 4096 tokens of 8 tenants by 4096, rank 16 (33.5 MB) 11 us, 3.0 TB/s; 8192 of 2 by
// 11008, rank 64 (180 MB) 60 us, 3.0 TB/s: there B comes out of L2 once for 64 tokens, and registers allow 8 wavefronts on a compute unit.
template <bool TR, int NT, int RT, bool ODD>
__global__ __launch_bounds__(kShrinkThreads) void lora_shrink_kernel(const LoraShrinkArgs a) {
    const Where u = find_tile<NT>(a, blockIdx.x);
    const int rt0 = blockIdx.z * RT;
    if (16 * rt0 >= u.rank) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const int mr = lane >> 2, mp = lane & 3;   // the row and the 16 bytes of 64 that the lane loads
    const uint16_t* row[NT];
    int column[NT], token[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) column[n] = 16 * n + mr < u.count ? 16 * n + mr : 0;
    tokens_of<NT>(a, u, column, token);
#pragma unroll
    for (int n = 0; n < NT; ++n) row[n] = a.src + (int64_t)token[n] * a.K + 8 * mp;
    // a wavefront's piece of LDS takes B, then (A, then) x; at the end all of it takes the sums
    constexpr size_t kTurn = sizeof(Turn<(NT > RT ? NT : RT)>), kStage = TR ? sizeof(Stage<RT>) : 0, kMine = kTurn > kStage ? kTurn : kStage;
    constexpr size_t kSums = sizeof(float4v) * kLoraShrinkWaves * RT * NT * kWave;
    __shared__ __align__(16) char lds[kSums > kLoraShrinkWaves * kMine ? kSums : kLoraShrinkWaves * kMine];
    Stage<RT>& stage = *(Stage<RT>*)(lds + wave * kMine);
    // backward: the lane's 16-byte pieces of 32 rows of B, where rows are whole pieces; else element by element
    const int width = min(16 * RT, u.rank - 16 * rt0);
    const bool pieces = !ODD || u.rank % 8 == 0;
    int piece_row[RT], piece_col[RT];
    const uint16_t* wrow[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if constexpr (TR) {
            const int at = lane + kWave * r, per_row = max(width / 8, 1);   // (below 8 ranks there are no whole pieces: not used)
            // (a lane without a piece of its own reads and stores one of the last row's once more: no branches)
            const int over = (int)(((unsigned)at * (65536u / (unsigned)per_row + 1)) >> 16);   // at / per_row
            piece_row[r] = pieces ? min(over, 31) : 0;
            piece_col[r] = pieces ? 8 * (at - over * per_row) : 0;
            wrow[r] = u.w + 16 * rt0 + piece_col[r];
        } else {
            const int rank = 16 * (rt0 + r) + mr < u.rank ? 16 * (rt0 + r) + mr : 0;
            wrow[r] = u.w + (int64_t)rank * a.K + 8 * mp;
        }
    }
    const float scale = TR ? a.scale[u.tenant] : 1.0f;
    float4v acc[RT][NT] = {};
    // Steps of 32 elements.  A last one of fewer (the backward pass's only: K is then `out`) is the last 32 elements, those zero that
    // an earlier step has had; a K below 32 is read element by element.
    // The wavefronts of a workgroup take neighbouring steps, so that what it reads of a row at a time is a run of 256 bytes.
    const int parts = a.splits * kLoraShrinkWaves, part = (int)blockIdx.y * kLoraShrinkWaves + wave;
    const int whole = (int)(a.K / 32), mine = part < whole ? (int)((unsigned)(whole - part + parts - 1) / (unsigned)parts) : 0;   // steps part, part + parts, ...
    constexpr int C = ODD ? 1 : NT * RT == 1 ? 4 : NT + RT <= 5 ? 2 : 1;   // steps of one of two buffers: what the registers hold
    half8 xv[2][C][NT], wv[2][C][RT];
    auto load = [&](int buffer, int s) {   // (a step beyond the last repeats it)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t k0 = 32 * (part + (int64_t)parts * min(s + c, mine - 1));
#pragma unroll
            for (int n = 0; n < NT; ++n) xv[buffer][c][n] = load8(row[n] + k0);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if constexpr (!TR)
                    wv[buffer][c][r] = load8(wrow[r] + k0);
                else if (pieces)
                    wv[buffer][c][r] = load8(wrow[r] + (k0 + piece_row[r]) * u.rank);
            }
        }
    };
    // One step: B goes through LDS, rows outside [had, end) as zeros
    auto product = [&](const half8 (&x)[NT], const half8 (&w)[RT], int64_t k0, int had, int end) {
        if constexpr (TR) {
            if (pieces) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    *(half8*)&stage.row[piece_row[r]][piece_col[r]] = piece_row[r] >= had && piece_row[r] < end ? w[r] : half8{};
            } else if constexpr (ODD) {
                _Float16 v[8 * RT];
#pragma unroll
                for (int k = 0; k < 8 * RT; ++k) {
                    const int at = lane + kWave * k, r = at / (16 * RT), rank = 16 * rt0 + at % (16 * RT);
                    v[k] = *(const _Float16*)(u.w + (k0 + min(r, end - 1)) * u.rank + min(rank, u.rank - 1));
                }
#pragma unroll
                for (int k = 0; k < 8 * RT; ++k) {
                    const int at = lane + kWave * k, r = at / (16 * RT);
                    stage.row[r][at % (16 * RT)] = r >= had && r < end ? v[k] : (_Float16)0.0f;
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        half8 xo[NT], wo[RT];
        if constexpr (TR) {
#pragma unroll
            for (int r = 0; r < RT; ++r) wo[r] = stage.operand(r, lane);
            __builtin_amdgcn_wave_barrier();
        } else {
            (*(Turn<RT>*)(lds + wave * kMine))(w, wo, lane);
        }
        (*(Turn<NT>*)(lds + wave * kMine))(x, xo, lane);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[r][n] = mfma(wo[r], xo[n], acc[r][n]);
    };
    // Two buffers; loads are never under a condition (past the end they repeat the last step's), or the wait for them would be for all.
    if (mine > 0) {
        load(0, 0);
        int s = 0;
        for (; s + 2 * C <= mine; s += 2 * C) {
            load(1, s + C);
#pragma unroll
            for (int c = 0; c < C; ++c) product(xv[0][c], wv[0][c], 32 * (part + (int64_t)parts * (s + c)), 0, 32);
            load(0, s + 2 * C);
#pragma unroll
            for (int c = 0; c < C; ++c) product(xv[1][c], wv[1][c], 32 * (part + (int64_t)parts * (s + C + c)), 0, 32);
        }
        if (C > 1) load(1, s + C);
#pragma unroll
        for (int c = 0; c < 2 * C - 1; ++c)
            if (s + c < mine) product(xv[c / C][c % C], wv[c / C][c % C], 32 * (part + (int64_t)parts * (s + c)), 0, 32);
    }
    if constexpr (TR) {
        if (a.K % 32 != 0 && whole % parts == part) {   // the last step, of fewer than 32
            const int64_t k0 = !ODD || a.K >= 32 ? a.K - 32 : 0;
            const int had = (int)(32 * whole - k0), end = ODD && a.K < 32 ? (int)a.K : 32;
            half8 x[NT], w[RT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (ODD && a.K < 32)
                    x[n] = load8_each(row[n] - 8 * mp + min(8 * mp, end - 1), max(end - 1 - 8 * mp, 0));
                else
                    x[n] = load8(row[n] + k0);
                x[n] = only(x[n], had - 8 * mp, end - 8 * mp);
            }
#pragma unroll
            for (int r = 0; r < RT; ++r)
                if (pieces) w[r] = load8(wrow[r] + (k0 + min(piece_row[r], end - 1)) * u.rank);   // (rows beyond `end` are stored as zeros)
            product(x, w, k0, had, end);
        }
    }
    float* const dst = a.h + (int64_t)blockIdx.y * a.split_stride;
    auto* const sum = (float4v(*)[RT * NT][kWave])lds;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) sum[wave][r * NT + n][lane] = acc[r][n];
    __syncthreads();
#pragma unroll
    for (int t = wave; t < RT * NT; t += kLoraShrinkWaves) {
        const int c = 16 * (t % NT) + m, rank = 16 * (rt0 + t / NT) + 4 * g;
        if (c >= u.count || 16 * (rt0 + t / NT) >= u.rank) continue;
        float4v v = sum[0][t][lane];
#pragma unroll
        for (int w = 1; w < kLoraShrinkWaves; ++w) v += sum[w][t][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = rank + i < u.rank ? v[i] * scale : 0.0f;
        *(float4v*)(dst + (int64_t)(u.hrow + c) * a.ld + rank) = v;
    }
}

constexpr int kExpandThreads = kLoraExpandWaves * kWave;
// Kernels of their own for the rows of the weights and results: 16-byte pieces, ranks that are no multiple of 8, fewer than 128 features
enum { kEvenRanks, kOddRanks, kShortRows };

// Few tokens: y = y0 + s B h, or dx = dx0 + A^T g, of one tile of 16 tokens by 512 features, 128 for each wavefront.  h comes in as
// `splits` partial sums.  Rows of a result are tokens, columns features: feature 8 n + j of a wavefront's 128 is column n of its MFMA
// j, so that a lane ends up with 8 neighbours of a token's row in its 8 accumulators, and 16 lanes with 256 bytes of the row: one
// load of y0 and one store for each.  The 32 elements of an MFMA's sum are 16 ranks, hi in lane groups 0 and 1 and lo in 2 and 3, both
// with the same weights.  Forward a wavefront's weights, 32 ranks of 128 features at a time, are read in runs of neighbouring bytes and
// come into that order through a piece of LDS of its own (64 bytes a feature, 16 more behind 8 features: no bank conflicts); backward
// 8 ranks' rows of A are turned in registers.
// y0 and the first weights are asked for before h is prepared: three waits for memory become one.
// Bound by latency and issue: 96 tokens of 3 tenants, 4096 features, rank 8: 5 us; 200 of 40 tenants, 5003 features, ranks to 64 (18 MB): 13 us.
constexpr int kFewStage = 128 * 64 + 16 * 16;   // bytes
template <bool TR, int ROWS>
__global__ __launch_bounds__(kExpandThreads) void lora_expand_few_kernel(const LoraExpandArgs a) {
    constexpr int kTokens = 16, kPer = kExpandThreads / kTokens;   // threads per token while h is prepared
    extern __shared__ __align__(16) char lds[];
    __shared__ float unit[kTokens];
    const Where u = find_tile<1>(a, blockIdx.x);
    const int64_t F = a.F[u.mat];
    if (blockIdx.y > 0 && (int64_t)blockIdx.y * kLoraExpandWaves * kLoraFeatures >= F) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const int padded = (u.rank + 15) & ~15, pitch = padded + 8;
    char* const stage = lds + wave * kFewStage;   // (forward)
    _Float16* const hi = (_Float16*)(lds + (TR ? 0 : kLoraExpandWaves * kFewStage));
    _Float16* const lo = hi + kTokens * pitch;
    // the wavefront's features, f0 .. f0 + 127; the last one's 128 end with the row and it keeps what is its own; a row below 128 is
    // read element by element
    const int64_t f0 = ((int64_t)blockIdx.y * kLoraExpandWaves + wave) * kLoraFeatures, base = min(f0, max(F - kLoraFeatures, (int64_t)0)), f = base + 8 * m;
    const bool active = f0 < F, vectors = ROWS != kShortRows || F >= kLoraFeatures;
    const float scale = TR || u.rank == 0 || F == 0 ? 1.0f : a.scale[u.mat][u.tenant];   // (a matrix whose h alone is asked for may have none)

    int64_t at[4];   // where the lane's results belong: token 4 g + i
    half8 before[4];
    {
        int column[4], token[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) column[i] = 4 * g + i < u.count ? 4 * g + i : 0;
        tokens_of<1>(a, u, column, token);
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = (int64_t)token[i] * F + f;
    }
    const uint16_t* const y0 = active ? a.y0[u.mat] : nullptr;
    if (y0 && vectors) {
#pragma unroll
        for (int i = 0; i < 4; ++i) before[i] = load8(y0 + at[i]);
    } else if (ROWS == kShortRows && y0) {
        const int64_t back = f < F ? 0 : f - (F - 1);   // a lane behind the row reads its last element
#pragma unroll
        for (int i = 0; i < 4; ++i) before[i] = load8_each(y0 + at[i] - back, F - 1 - f + back);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) before[i] = half8{};
    }
    // Forward: lane and instruction i have piece q = 64 i + lane, 8 ranks of feature q / per_row (and the next feature's first ones, where the
    // rank is no multiple of 8).  Backward: 8 ranks' rows of A.
    half8 wv[8];
    auto per_row = [&](int r) { return (min(32, u.rank - r) + 7) / 8; };
    auto piece_row = [&](int i, int n) { return (int)(((unsigned)(kWave * i + lane) * (65536u / (unsigned)n + 1)) >> 16); };
    auto piece_rank = [&](int i, int n, int r) { return r + 8 * (kWave * i + lane - piece_row(i, n) * n); };
    auto load_weights = [&](int r) {
        if constexpr (TR) {
            const int rank = r + 8 * (g & 1), left = u.rank - rank;
            const uint16_t* const w = u.w + (f <= F - 8 ? f : F - 8);   // (F = in, a multiple of 32)
#pragma unroll
            for (int i = 0; i < 8; ++i) wv[i] = load8(w + (int64_t)(i < left ? rank + i : u.rank - 1) * F);
        } else {
            const int n = per_row(r);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < 2 * n) {
                    const int64_t at = min(base + piece_row(i, n), F - 1) * u.rank + piece_rank(i, n, r);
                    wv[i] = ROWS != kEvenRanks ? load8_of<ROWS == kShortRows>(u.w, at, F * u.rank) : load8(u.w + at);
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
    float* const kept = !TR && a.h_out[u.mat] && blockIdx.y == 0 && real ? a.h_out[u.mat] + (int64_t)token_of<1>(a, u, c) * a.h_ld : nullptr;
    float top = 0.0f;
    float4v first = {};   // of the thread's first four ranks: all there are up to 64
    for (int r = 4 * sub; r < padded; r += 4 * kPer) {
        const float4v v = sum4(r);
        if (r == 4 * sub) first = v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top = fmaxf(top, finite_abs(v[i]));
            if (kept && r + i < u.rank) kept[r + i] = v[i];
        }
    }
#pragma unroll
    for (int d = kPer / 2; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
    const int e = group_exponent(top);
    if (sub == 0) unit[c] = power_of_two(e) * scale;
    const float down = power_of_two(-e);
    for (int r = 4 * sub; r < padded; r += 4 * kPer) {
        const float4v v = r == 4 * sub ? first : sum4(r);
        half4 h, l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            _Float16 p, q;
            split_half(v[i], down, &p, &q);
            h[i] = real ? p : (_Float16)0.0f;
            l[i] = real ? q : (_Float16)0.0f;
        }
        *(half4*)(hi + c * pitch + r) = h;
        *(half4*)(lo + c * pitch + r) = l;
    }
    __syncthreads();
    if (!active) return;

    const _Float16* const mine = (g < 2 ? hi : lo) + m * pitch + 8 * (g & 1);
    float4v acc[8] = {};
    auto product = [&](const half8 (&cols)[8], int r) {
        const half8 hv = *(const half8*)(mine + r);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = mfma(hv, cols[j], acc[j]);
    };
    for (int r0 = 0; r0 < padded; r0 += TR ? 16 : 32) {
        if constexpr (TR) {
            half8 cols[8];
            if (u.rank - r0 < 16) {   // rows beyond the rank repeat the last one: they do not count
#pragma unroll
                for (int i = 0; i < 8; ++i) wv[i] = i < u.rank - r0 - 8 * (g & 1) ? wv[i] : half8{};
            }
            transpose8(wv, cols);
            if (r0 + 16 < padded) load_weights(r0 + 16);
            product(cols, r0);
        } else {
            const int n = per_row(r0);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < 2 * n) {
                    const int row = piece_row(i, n), rank = piece_rank(i, n, r0) - r0;
                    *(half8*)(stage + row * 64 + (row >> 3) * 16 + 2 * rank) = wv[i];
                }
            __builtin_amdgcn_wave_barrier();
            if (r0 + 32 < padded) load_weights(r0 + 32);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int r = r0 + 16 * half, left = u.rank - r - 8 * (g & 1);
                if (r >= padded) continue;
                half8 cols[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) cols[j] = *(const half8*)(stage + m * (8 * 64 + 16) + j * 64 + half * 32 + (g & 1) * 16);
                if (u.rank - r < 16) {   // what lies beyond the rank does not count
#pragma unroll
                    for (int j = 0; j < 8; ++j) cols[j] = ROWS != kEvenRanks ? only(cols[j], 0, left) : left > 0 ? cols[j] : half8{};
                }
                product(cols, r);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    uint16_t* const y = a.y[u.mat];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = 4 * g + i;
        if (col >= u.count || f >= F) continue;
        const float up = unit[col];
        half8 v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (_Float16)__builtin_fmaf(acc[j][i], up, (float)before[i][j]);
        if (u.rank == 0) v = before[i];   // every bit of y0, of zeros and NaN too
        if (f >= f0 && F - f >= 8) {
            __builtin_memcpy(y + at[i], &v, 16);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (f + j >= f0 && f + j < F) *(_Float16*)(y + at[i] + j) = v[j];
        }
    }
}

// Many tokens: the same of one tile of 64 tokens, 16 for each wavefront, which take 128 features at a time together, gridDim.y of
// them in turn.  The weights of 128 features by 16 RS ranks, 16 RS bytes of them from each thread, go through one of two buffers in LDS
// (kPieces: [feature][16 ranks] forward, with 16 bytes more behind 8 features; [16 ranks][128 features] backward, with 16 bytes more
// behind a row), where every wavefront reads them into matrix-core order without bank conflicts: read from memory in that order,
// neighbouring lanes would be rows apart and an instruction would take the address unit four times as long.  While a piece is used the
// next but one is on its way, and the next features' y0.
// Bound by y0 and y: 4096 tokens by 11008, rank 16 (180 MB) 42 us, 4.3 TB/s; 8192 by 4096, rank 64 (134 MB) 39 us, 3.4 TB/s (a barrier for every
// 16 ranks instead of 32: 42.9 us).  Features in turn, not next to each other, for a workgroup: 43 us, else 47.
constexpr int kPieces = 128 * 32 + 16 * 16;
template <bool TR, int ROWS, int RS>   // RS: times 16 ranks at a time
__global__ __launch_bounds__(kExpandThreads, ROWS == kShortRows ? 2 : 3) void lora_expand_many_kernel(const LoraExpandArgs a) {
    constexpr int kTokens = kLoraExpandTokens, kPer = kExpandThreads / kTokens;   // threads per token while h is prepared
    extern __shared__ __align__(16) char lds[];
    __shared__ float unit[kTokens];
    const Where u = find_tile<kTokens / 16>(a, blockIdx.x);
    const int64_t F = a.F[u.mat];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, m = lane & 15, g = lane >> 4;
    const int padded = (u.rank + 15) & ~15, pitch = padded + 8;
    char* const pieces = lds;
    _Float16* const hi = (_Float16*)(lds + 2 * RS * kPieces);
    _Float16* const lo = hi + kTokens * pitch;
    const int64_t stride = (int64_t)gridDim.y * kLoraFeatures;
    // Features f0 .. f0 + 127; a row's last 128 end with it, and of them only those from f0 on are kept.  A row below 128 is read element
    // by element.
    int64_t f0 = (int64_t)blockIdx.y * kLoraFeatures;
    const float scale = TR || F == 0 ? 1.0f : a.scale[u.mat][u.tenant];   // (a matrix whose h alone is asked for may have none)
    const bool vectors = ROWS != kShortRows || F >= kLoraFeatures;
    auto begin_of = [&](int64_t first) { return min(first, max(F - kLoraFeatures, (int64_t)0)); };

    int64_t row[4];   // the rows of y that the lane's results belong to: token 16 wave + 4 g + i
    {
        int column[4], token[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 16 * wave + 4 * g + i;
            column[i] = c < u.count ? c : 0;
        }
        tokens_of<kTokens / 16>(a, u, column, token);
#pragma unroll
        for (int i = 0; i < 4; ++i) row[i] = (int64_t)token[i] * F + 8 * m;
    }
    const uint16_t* const y0 = a.y0[u.mat];
    half8 before[4];
    auto load_y0 = [&](half8 (&to)[4], int64_t f) {
        if (vectors) {   // (without y0 something that is in the cache: no branch)
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = load8(y0 ? y0 + row[i] + f : a.y[u.mat] + 8 * m);
        } else if (ROWS == kShortRows && y0) {
            const int64_t at = 8 * m < F ? 0 : F - 1 - 8 * m;   // a lane behind the row reads its last element
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = load8_each(y0 + row[i] + at, max(F - 1 - 8 * m, (int64_t)0));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = half8{};
        }
    };
    uint16_t* const y = a.y[u.mat];
    auto store_y = [&](const half8 (&v)[4], int64_t f) {   // at the features f .. f + 127, those before f0 left out
        const int64_t fl = f + 8 * m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (16 * wave + 4 * g + i >= u.count) continue;
            if (fl >= f0 && F - fl >= 8) {
                __builtin_memcpy(y + row[i] + f, &v[i], 16);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (fl + j >= f0 && fl + j < F) *(_Float16*)(y + row[i] + f + j) = v[i][j];
            }
        }
    };
    if (u.rank == 0) {   // every bit of y0, of zeros and NaN too
        for (; f0 < F; f0 += stride) {
            load_y0(before, begin_of(f0));
#pragma unroll
            for (int i = 0; i < 4; ++i) before[i] = y0 ? before[i] : half8{};
            store_y(before, begin_of(f0));
        }
        return;
    }
    // the thread's 16 bytes of the weights
    const int piece_row = TR ? (int)threadIdx.x >> 4 : (int)threadIdx.x >> 1, piece_col = TR ? 8 * ((int)threadIdx.x & 15) : 8 * ((int)threadIdx.x & 1);
    char* const piece_at = pieces + (TR ? piece_row * 272 + piece_col * 2 : piece_row * 32 + piece_col * 2 + (piece_row >> 3) * 16);
    half8 piece[RS];
    int piece_left[RS] = {};   // ranks of it that count (backward: whether it does); looked at when it goes to LDS, so that nothing waits for the load
    auto load_piece = [&](int64_t f, int r0) {
#pragma unroll
        for (int k = 0; k < RS; ++k) {
            const int r = r0 + 16 * k;
            if constexpr (TR) {   // (F = in, a multiple of 32)
                piece_left[k] = u.rank - r - piece_row;
                piece[k] = load8(u.w + (int64_t)min(r + piece_row, u.rank - 1) * F + min(f + piece_col, F - 8));
            } else {
                piece_left[k] = u.rank - r - piece_col;
                const int64_t at = min(f + piece_row, F - 1) * u.rank + (piece_left[k] > 0 ? r + piece_col : r < u.rank ? r : 0);
                piece[k] = ROWS != kEvenRanks ? load8_of<ROWS == kShortRows>(u.w, at, F * u.rank) : load8(u.w + at);
            }
        }
    };
    auto put_piece = [&](int buffer, const half8 (&v)[RS], const int (&left)[RS]) {
#pragma unroll
        for (int k = 0; k < RS; ++k)
            *(half8*)(piece_at + (RS * buffer + k) * kPieces) = !TR && ROWS != kEvenRanks ? only(v[k], 0, left[k]) : left[k] > 0 ? v[k] : half8{};
    };
    // the pieces come in the order of their use: ranks after ranks, then the next features; past the end the last once more
    int64_t piece_f0 = f0;
    int piece_r = 0;
    auto next_piece = [&] {
        load_piece(begin_of(piece_f0), piece_r);
        if (piece_r + 16 * RS < padded) {
            piece_r += 16 * RS;
        } else if (piece_f0 + stride < F) {
            piece_r = 0;
            piece_f0 += stride;
        }
    };
    const bool work = f0 < F;   // (not for a matrix without outputs, whose h alone is asked for)
    half8 piece0[RS] = {};
    int left0[RS] = {};
    if (work) {
        next_piece();   // two pieces before h: nothing is in flight when the turns begin
#pragma unroll
        for (int k = 0; k < RS; ++k) piece0[k] = piece[k], left0[k] = piece_left[k];
        next_piece();
        load_y0(before, begin_of(f0));
    }

    // h of the tile's tokens: the parts added up, the exponent, hi and lo into LDS
    const int c = threadIdx.x / kPer, sub = threadIdx.x % kPer;
    const bool real = c < u.count;
    const float* const src = a.h + (int64_t)(u.hrow + (real ? c : 0)) * a.ld;
    // HELD times four ranks of the thread at a time, 4 sub + 16 k behind r, two parts of each: all their loads before the first addition
    constexpr int kHeld = RS == 1 ? 1 : 4;
    auto sums = [&](int r, float4v (&v)[kHeld]) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k) v[k] = float4v{};
        constexpr int kAtOnce = RS == 1 ? 4 : 2;
        for (int s = 0; s < a.splits; s += kAtOnce) {
            float4v part[kAtOnce][kHeld];
#pragma unroll
            for (int c = 0; c < kAtOnce; ++c)
#pragma unroll
                for (int k = 0; k < kHeld; ++k) part[c][k] = *(const float4v*)(src + min(s + c, a.splits - 1) * a.split_stride + min(r + 16 * k, padded - 16) + 4 * sub);
#pragma unroll
            for (int c = 0; c < kAtOnce; ++c)
#pragma unroll
                for (int k = 0; k < kHeld; ++k) v[k] += s + c < a.splits ? part[c][k] : float4v{};
        }
    };
    float* const kept = !TR && a.h_out[u.mat] && blockIdx.y == 0 && real ? a.h_out[u.mat] + (int64_t)token_of<kTokens / 16>(a, u, c) * a.h_ld : nullptr;
    float top = 0.0f;
    float4v first[kHeld];   // of the thread's first ranks: all there are up to 16 (RS = 1) or 64
    for (int r = 0; r < padded; r += 16 * kHeld) {
        float4v v[kHeld];
        sums(r, v);
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            if (r == 0) first[k] = v[k];
            if (r + 16 * k >= padded) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                top = fmaxf(top, finite_abs(v[k][i]));
                if (kept && r + 16 * k + 4 * sub + i < u.rank) kept[r + 16 * k + 4 * sub + i] = v[k][i];
            }
        }
    }
#pragma unroll
    for (int d = kPer / 2; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
    const int e = group_exponent(top);
    if (sub == 0) unit[c] = power_of_two(e) * scale;
    const float down = power_of_two(-e);
    for (int r = 0; r < padded; r += 16 * kHeld) {
        float4v v[kHeld];
        if (r == 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) v[k] = first[k];
        } else {
            sums(r, v);
        }
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            if (r + 16 * k >= padded) continue;
            half4 h, l;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                _Float16 p, q;
                split_half(v[k][i], down, &p, &q);
                h[i] = real ? p : (_Float16)0.0f;
                l[i] = real ? q : (_Float16)0.0f;
            }
            *(half4*)(hi + c * pitch + r + 16 * k + 4 * sub) = h;
            *(half4*)(lo + c * pitch + r + 16 * k + 4 * sub) = l;
        }
    }
    if (!work) return;   // (of the whole workgroup)
    put_piece(0, piece0, left0);
    __syncthreads();

    const _Float16* const mine = (g < 2 ? hi : lo) + (16 * wave + m) * pitch + 8 * (g & 1);
    float up[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) up[i] = unit[16 * wave + 4 * g + i];
    int buffer = 0;
    for (; f0 < F; f0 += stride) {
        const int64_t f = begin_of(f0);
        float4v acc[8] = {};
        auto step = [&](int r) {
            put_piece(buffer ^ 1, piece, piece_left);   // of the next ranks or features
            next_piece();
#pragma unroll
            for (int k = 0; k < RS; ++k) {
                if (k > 0 && r + 16 * k >= padded) continue;
                const char* const at = pieces + (RS * buffer + k) * kPieces + (TR ? 8 * (g & 1) * 272 + m * 16 : m * (8 * 32 + 16) + (g & 1) * 16);
                half8 wv[8], cols[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) wv[j] = *(const half8*)(at + j * (TR ? 272 : 32));
                if constexpr (TR) {
                    transpose8(wv, cols);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) cols[j] = wv[j];
                }
                const half8 hv = *(const half8*)(mine + r + 16 * k);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = mfma(hv, cols[j], acc[j]);
            }
            buffer ^= 1;
            __syncthreads();
        };
        step(0);   // (not in the loop: what is in flight is known at each of its waits)
        for (int r = 16 * RS; r < padded; r += 16 * RS) step(r);
        half8 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = (_Float16)__builtin_fmaf(acc[j][i], up[i], y0 ? (float)before[i][j] : 0.0f);
        // the next y0 is asked for before the stores: no wait for it has to wait for them (past the end: the last features' once more)
        load_y0(before, begin_of(min(f0 + stride, F - 1)));
        store_y(v, f);
    }
}

constexpr int kPrepThreads = 256;

// The second operand of the gradients, once for all their workgroups: 32 tokens' g (or h) as hi and lo in matrix-core order, with an
// exponent for each rank (ranks share no sum: the weakest is held as well as the strongest).  Lane (n, q) holds rank n of its 16,
// tokens 8 q .. 8 q + 7, in 16 bytes.  Where g came in parts their sum takes the first part's place.  Once for 8192 tokens of rank 64: 6 us; in the workgroups of the sums, each for itself: 3 us less for 32
// tokens per tenant, up to twice the sums' time for 64 tenants or 512 tokens.
__global__ __launch_bounds__(kPrepThreads) void lora_prep_kernel(const LoraPrepArgs a) {
    const int record = threadIdx.x & (kWave - 1);
    const int j = __builtin_amdgcn_readfirstlane(__popcll(__ballot(record < a.n_jobs && a.job[min(record, a.n_jobs - 1)].chunk_begin <= (int)blockIdx.x + a.chunk_first)) - 1);
    const LoraPrepJob& job = a.job[j];
    const bool of_h = blockIdx.y + a.side_first == 1;
    if (!(job.sides >> (int)of_h & 1)) return;   // (nobody has written this tenant's g, or nobody reads what h would become)
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
    half8* const out = a.operand[of_h] + (int64_t)chunk * (a.ld / 16) * 2 * kWave;
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const int rt = wave + k * (kPrepThreads / kWave), rank = 16 * rt + n, column = min(rank, rank_all - 1);
        if (rt >= tiles) continue;
        float v[8], top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = src[at[i] + column];
        for (int s = 1; s < splits; s += 4) {   // the loads of four parts at a time
            float w[4][8];
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) w[c][i] = src[min(s + c, splits - 1) * a.split_stride + at[i] + column];
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += s + c < splits ? w[c][i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool real = t0 + 8 * q + i < job.count && rank < rank_all;
            if (splits > 1 && real) a.g[at[i] + column] = v[i];
            v[i] = real ? v[i] : 0.0f;
            top = fmaxf(top, finite_abs(v[i]));
        }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));   // of the rank's 32 tokens
        const int e = group_exponent(top);
        if (q == 0) a.exponent[of_h][(int64_t)chunk * a.ld + rank] = (uint8_t)(127 + e);
        const float down = power_of_two(-e);
        half8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            _Float16 h, l;
            split_half(v[i], down, &h, &l);
            hi[i] = h;
            lo[i] = l;
        }
        out[(2 * rt) * kWave + lane] = hi;
        out[(2 * rt + 1) * kWave + lane] = lo;
    }
}

constexpr int kGradThreads = kLoraGradWaves * kWave;
constexpr int kGradPitch = 128 + 16;   // halves: 4 rows apart on banks of their own for the transposing read

// dA or dB of one job: 128 features by 16 RW ranks, summed over one part of the job's tokens.  RW wavefronts with 16 ranks each share a
// tile of 32 tokens' x (dy); 4 / RW such groups take the tiles in turn and meet in LDS at the end.  The tokens are the sum's index, so
// both operands want 8 tokens of one feature (rank) in a lane: the second comes prepared, the tile goes through LDS as it is (256 bytes
// of a row from 16 lanes) and is read transposed.  A tile's products are added up in the matrix cores in units of their rank's 2^e
// and then go into the sum, whatever the sizes of the tiles before.
// Loads are never under a condition (past the end they repeat the last tile's), or the wait for them would be for all.
// Bound by the streams of x and dy: 4096 tokens of 8 tenants, 4096 -> 4096, rank 16 (67 MB) 22 us, 3.0 TB/s; 8192 of 2, 4096 -> 11008, rank 64
// (247 MB) 68 us, 3.6 TB/s.
template <int RW, bool ODD>
__global__ __launch_bounds__(kGradThreads) __attribute__((amdgpu_waves_per_eu(ODD ? 2 : 3, 3))) void lora_grad_kernel(const LoraGradArgs a) {
    constexpr int TW = kLoraGradWaves / RW, N = 8 / RW, kBuffers = RW > 1 ? 2 : 1;   // groups; rows of 4 per wavefront and tile
    typedef _Float16 Tile[32][kGradPitch];
    constexpr size_t kTiles = sizeof(Tile) * TW * kBuffers, kSums = sizeof(float) * kLoraGradWaves * 8 * 4 * kWave;
    __shared__ __align__(16) char lds[kTiles > kSums ? kTiles : kSums];
    __shared__ uint16_t ids[kLoraPartTokens];
    const int which = (int)blockIdx.z >= a.rank_groups ? 1 : 0, rt0 = ((int)blockIdx.z - which * a.rank_groups) * RW;
    const LoraGradSide& side = a.side[which];
    const int record = threadIdx.x & (kWave - 1);
    const int which_job = __builtin_amdgcn_readfirstlane(__popcll(__ballot(record < kLoraGradJobs && (int)blockIdx.y >= a.part_begin[min(record, kLoraGradJobs - 1)])) - 1);
    const LoraGradJob& job = a.job[which_job];
    const int split = blockIdx.y - a.part_begin[which_job], rank_all = job.rank;
    float* const result = job.out[which];
    const int64_t F = side.F, f0 = (int64_t)blockIdx.x * kLoraFeatures;
    if (!result || 16 * rt0 >= rank_all || f0 >= F) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, group = wave / RW, rank_wave = wave % RW;
    const int n = lane & 15, q = lane >> 4;
    // the part's tokens, t0 .. t0 + count - 1 of the job; whole tiles of 32 but for the job's last
    const int c0 = split * job.part_chunks, t0 = 32 * c0, count = min(32 * job.part_chunks, job.count - t0), chunks = (count + 31) / 32;
    const float scale = side.scale ? side.scale[job.tenant] : 1.0f;
    for (int i = threadIdx.x; i < 32 * chunks; i += kGradThreads) {   // (behind the last token: the first once more)
        const int p = job.first + t0 + (i < count ? i : 0);
        ids[i] = (uint16_t)(a.order ? a.order[p] : p);
    }
    __syncthreads();

    const int64_t base = min(f0, max(F - kLoraFeatures, (int64_t)0)), fl = base + 8 * n;   // the last 128 features end with the row
    const uint16_t* const d = side.d + (ODD && fl >= F ? F - 1 : fl);
    const int64_t last = ODD ? max(F - 1 - fl, (int64_t)0) : 7;
    half8 rows[2][N], op[2][2];
    uint8_t exponent[2];   // 127 + e of the lane's rank
    const int mine = rank_wave * 4 * N + q;   // the lane's rows of a tile: mine, mine + 4, ...
    auto chunk_at = [&](int k) { return min(TW * k + group, chunks - 1); };
    auto load_rows = [&](int buffer, int k) {
        const uint16_t* const id = ids + 32 * chunk_at(k) + mine;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint16_t* const p = d + (int64_t)id[4 * i] * F;
            rows[buffer][i] = !ODD || F >= kLoraFeatures ? load8(p) : load8_each(p, last);
        }
    };
    auto load_operand = [&](int buffer, int k) {   // (a wavefront without ranks takes the last's)
        const int chunk = job.chunk_begin + c0 + chunk_at(k), rt = min(rt0 + rank_wave, (rank_all - 1) / 16);
        exponent[buffer] = side.exponent[(int64_t)chunk * a.ld + 16 * rt + n];
        const half8* const p = side.operand + ((int64_t)chunk * (a.ld / 16) + rt) * 2 * kWave + lane;
        op[buffer][0] = p[0];
        op[buffer][1] = p[kWave];
    };
    float4v acc[8] = {};
    auto step = [&](auto which_buffer, int k) {
        constexpr int b = decltype(which_buffer)::value;
        Tile& tile = ((Tile*)lds)[(RW > 1 ? b : 0) * TW + group];
        const int chunk = TW * k + group;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = mine + 4 * i;
            *(half8*)&tile[row][8 * n] = 32 * chunk + row < count ? rows[b][i] : half8{};
        }
        load_rows(b, k + 2);
        load_operand(1 - b, k + 1);
        if constexpr (RW > 1)
            __syncthreads();
        else
            __builtin_amdgcn_wave_barrier();
        if (chunk >= chunks) return;   // (of the whole group: rows of zeros times an infinity of the last tile's operand would be NaN)
        const float unit = __uint_as_float((uint32_t)exponent[b] << 23);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4 lds4;
            const _Float16* const p = &tile[8 * q + (n >> 2)][16 * j + 4 * (n & 3)];
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + 4 * kGradPitch));
            half8 v;
            __builtin_memcpy(&v, &lo, 8);
            __builtin_memcpy((char*)&v + 8, &hi, 8);
            const float4v part = mfma(v, op[b][1], mfma(v, op[b][0], float4v{}));
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] = __builtin_fmaf(part[i], unit, acc[j][i]);
        }
    };
    load_operand(0, 0);
    load_rows(0, 0);
    load_rows(1, 1);
    for (int k = 0; TW * k < chunks; k += 2) {   // (of the whole workgroup; steps beyond the last bring nothing)
        step(std::integral_constant<int, 0>{}, k);
        step(std::integral_constant<int, 1>{}, k + 1);
    }
    __syncthreads();
    auto* const sum = (float(*)[8][4][kWave])lds;   // [wave][j][i][lane (n, q)] = feature 16 j + 4 q + i, rank n
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[wave][j][i][lane] = acc[j][i];
    __syncthreads();
    float* const out = job.parts > 1 ? side.partial + (job.partial + (int64_t)split * rank_all) * F : result;
    const bool add = a.accumulate && job.parts == 1;
    constexpr int kRanks = 16 * RW;
#pragma unroll 4
    for (int k = 0; k < kRanks * kLoraFeatures / kGradThreads; ++k) {
        const int at = threadIdx.x + k * kGradThreads;
        const int r = which == 0 ? at / kLoraFeatures : at % kRanks, f = which == 0 ? at % kLoraFeatures : at / kRanks;
        const int rank = 16 * rt0 + r;
        if (rank >= rank_all || base + f < f0 || base + f >= F) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < TW; ++w) v += sum[w * RW + (r >> 4)][f >> 4][f & 3][16 * ((f >> 2) & 3) + (r & 15)];
        v *= scale;
        float* const p = out + (which == 0 ? (int64_t)rank * F + base + f : (base + f) * rank_all + rank);
        *p = add ? *p + v : v;
    }
}

// out (+)= the sum of the parts, in their order; zeros where there are none.  3 parts of 2 tenants' gradients of 64 x (4096 + 11008): 7 us
__global__ __launch_bounds__(256) void lora_reduce_kernel(const LoraReduceArgs a) {
    const auto& job = a.job[blockIdx.y];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < job.n; i += (int64_t)gridDim.x * 256) {
        float v = 0.0f;
        for (int s = 0; s < job.parts; ++s) v += job.partial[s * job.n + i];
        job.out[i] = a.accumulate ? job.out[i] + v : v;
    }
}

}  // namespace

static_assert(sizeof(LoraOrderArgs) <= 4096 && sizeof(LoraDecodeArgs) <= 4096 && sizeof(LoraShrinkArgs) <= 4096 && sizeof(LoraExpandArgs) <= 4096 && sizeof(LoraGradArgs) <= 4096 && sizeof(LoraReduceArgs) <= 4096 && sizeof(LoraPrepArgs) <= 4096,
              "kernel arguments");

hipError_t launch_lora_order(const LoraOrderArgs& a, hipStream_t st) {
    if (a.count < 1 || a.n_jobs < 1 || a.n_jobs > kLoraOrderJobs || (a.bits != 1 && a.bits != 2 && a.bits != 4 && a.bits != 8) || a.n_jobs > 1 << a.bits || a.count > kLoraOrderBytes * 8 / a.bits)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(lora_order_kernel, dim3(1), dim3(kOrderThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_lora_decode(const LoraDecodeArgs& a, int max_tokens, int64_t max_F, bool odd, hipStream_t st) {
    const int64_t groups = max_F > 0 ? (max_F + kLoraDecodeFeatures - 1) / kLoraDecodeFeatures : 1;   // (F = 0: h alone)
    if (a.n_tiles < 1 || groups > 65535 || max_tokens > kLoraDecodeTokens || a.in < 8) return hipErrorInvalidValue;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_tiles, (unsigned)groups), dim3(kDecodeThreads), 0, st, a);
        return hipGetLastError();
    };
    if (odd) return max_tokens == 1 ? go(lora_decode_kernel<1, true>) : go(lora_decode_kernel<2, true>);
    return max_tokens == 1 ? go(lora_decode_kernel<1, false>) : go(lora_decode_kernel<2, false>);
}

hipError_t launch_lora_shrink(const LoraShrinkArgs& a, int columns, bool transposed, int max_rank, bool odd, hipStream_t st) {
    const int rank_tiles = (max_rank + 15) / 16;
    if (a.n_tiles < 1 || rank_tiles < 1 || a.splits < 1 || a.splits > kLoraMaxSplits) return hipErrorInvalidValue;
    auto go = [&](auto kernel, int RT) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_tiles, (unsigned)a.splits, (unsigned)((rank_tiles + RT - 1) / RT)), dim3(kShrinkThreads), 0, st, a);
        return hipGetLastError();
    };
    odd |= a.K < 32;
    if (columns == 16) return !transposed ? go(lora_shrink_kernel<false, 1, 1, false>, 1) : odd ? go(lora_shrink_kernel<true, 1, 1, true>, 1) : go(lora_shrink_kernel<true, 1, 1, false>, 1);
    if (transposed && odd) return go(lora_shrink_kernel<true, 4, 1, true>, 1);
    if (rank_tiles == 1) return transposed ? go(lora_shrink_kernel<true, 4, 1, false>, 1) : go(lora_shrink_kernel<false, 4, 1, false>, 1);
    return transposed ? go(lora_shrink_kernel<true, 4, 4, false>, 4) : go(lora_shrink_kernel<false, 4, 4, false>, 4);
}

hipError_t launch_lora_expand(const LoraExpandArgs& a, int columns, bool transposed, int max_rank, int64_t min_F, int64_t max_F, bool odd, hipStream_t st) {
    if (a.n_tiles < 1 || max_rank > kLoraMaxRank || a.splits > kLoraMaxSplits) return hipErrorInvalidValue;
    const int rows = min_F < kLoraFeatures ? kShortRows : odd && !transposed ? kOddRanks : kEvenRanks;
    const int64_t wide = std::max<int64_t>(1, (max_F + kLoraFeatures - 1) / kLoraFeatures);   // (F = 0: h alone)
    if (columns == 16) {
        const int64_t groups = (wide + kLoraExpandWaves - 1) / kLoraExpandWaves;
        if (groups > 65535) return hipErrorInvalidValue;
        const unsigned lds = (unsigned)((transposed ? 0 : kLoraExpandWaves * kFewStage) + 2 * 16 * (((max_rank + 15) & ~15) + 8) * 2);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_tiles, (unsigned)groups), dim3(kExpandThreads), lds, st, a);
            return hipGetLastError();
        };
        if (transposed) return rows == kShortRows ? go(lora_expand_few_kernel<true, kShortRows>) : go(lora_expand_few_kernel<true, kEvenRanks>);
        return rows == kShortRows ? go(lora_expand_few_kernel<false, kShortRows>) : rows == kOddRanks ? go(lora_expand_few_kernel<false, kOddRanks>) : go(lora_expand_few_kernel<false, kEvenRanks>);
    }
    int cus = 256;
    if (const hipError_t e = device_cu_count(&cus); e != hipSuccess) return e;
    // Up to 3 workgroups to a compute unit, each taking the same number of turns.  1 / 2 / 3 / 4 of them, us: 1172 tokens by 5504, rank 64:
    // 14.9 / 13.7 / 13.6 / 16.6; 4096 by 11008, rank 16: 57 / 47 / 46.6 / 45.8, rank 64: 83 / 56 / 54 / 59; backward, 8192 by 4096, rank 64: 83 / 43 / 39 / 42
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(wide, (int64_t)3 * cus / a.n_tiles));
    const int64_t each = (wide + most - 1) / most, turns = (wide + each - 1) / each;
    const int RS = max_rank <= 16 ? 1 : 2;
    const unsigned lds = (unsigned)(2 * RS * kPieces + 2 * kLoraExpandTokens * (((max_rank + 15) & ~15) + 8) * 2);
    static PerDeviceOnce once[10];
    auto go = [&](auto kernel, int which) {
        const hipError_t e = once[which].run([&] { return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * 2 * kPieces + 2 * kLoraExpandTokens * (kLoraMaxRank + 8) * 2); });
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_tiles, (unsigned)turns), dim3(kExpandThreads), lds, st, a);
        return hipGetLastError();
    };
    auto of = [&](auto ranks_at_once, int first) {
        constexpr int R = decltype(ranks_at_once)::value;
        if (transposed) return rows == kShortRows ? go(lora_expand_many_kernel<true, kShortRows, R>, first) : go(lora_expand_many_kernel<true, kEvenRanks, R>, first + 1);
        return rows == kShortRows ? go(lora_expand_many_kernel<false, kShortRows, R>, first + 2) : rows == kOddRanks ? go(lora_expand_many_kernel<false, kOddRanks, R>, first + 3) : go(lora_expand_many_kernel<false, kEvenRanks, R>, first + 4);
    };
    return RS == 1 ? of(std::integral_constant<int, 1>{}, 0) : of(std::integral_constant<int, 2>{}, 5);
}

hipError_t launch_lora_prep(const LoraPrepArgs& a, int chunks, int sides, hipStream_t st) {
    if (a.n_jobs < 1 || chunks < 1 || sides < 1) return hipErrorInvalidValue;
    hipLaunchKernelGGL(lora_prep_kernel, dim3((unsigned)chunks, (unsigned)sides), dim3(kPrepThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_lora_grad(const LoraGradArgs& a, int max_rank, hipStream_t st) {
    const int rank_tiles = (max_rank + 15) / 16, RW = lora_grad_rank_waves(max_rank);
    const int64_t F = std::max(a.side[0].F, a.side[1].F), groups = (F + kLoraFeatures - 1) / kLoraFeatures;
    if (a.n_jobs < 1 || rank_tiles < 1 || groups < 1 || a.n_parts < 1) return hipErrorInvalidValue;
    LoraGradArgs b = a;
    b.rank_groups = (rank_tiles + RW - 1) / RW;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (unsigned)b.n_parts, (unsigned)(2 * b.rank_groups)), dim3(kGradThreads), 0, st, b);
        return hipGetLastError();
    };
    // rows below 128 elements (a side that is not wanted has none)
    const bool odd = (a.side[0].F > 0 && a.side[0].F < kLoraFeatures) || (a.side[1].F > 0 && a.side[1].F < kLoraFeatures);
    if (odd) return RW == 1 ? go(lora_grad_kernel<1, true>) : RW == 2 ? go(lora_grad_kernel<2, true>) : go(lora_grad_kernel<4, true>);
    return RW == 1 ? go(lora_grad_kernel<1, false>) : RW == 2 ? go(lora_grad_kernel<2, false>) : go(lora_grad_kernel<4, false>);
}

hipError_t launch_lora_reduce(const LoraReduceArgs& a, int64_t max_n, hipStream_t st) {
    if (a.n_jobs < 1) return hipErrorInvalidValue;
    const int64_t blocks = (max_n + 1023) / 1024;
    hipLaunchKernelGGL(lora_reduce_kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks > 1024 ? 1024 : blocks), (unsigned)a.n_jobs), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace bd
