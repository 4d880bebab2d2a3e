// Kernel arguments and launch functions of the low-rank adapters (lora_kernels.hip), called by lora_api.hip.
//
// A call's tokens are sorted by tenant; a tenant's tokens are a JOB, its tokens in runs of 16 NT columns are TILES.  Two ways to
// tell a workgroup what its tile is, both by value in the kernel arguments (no table that another launch must write first, and
// nothing that two calls could share):
//   few tokens    one record per (tile of 16 tokens, matrix), the tokens' ids in the record: one scalar load per workgroup
//   many tokens   one record per (job, matrix); the workgroup searches its tile among the records' first tiles
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bd {

constexpr int kLoraMaxRank = 256;
constexpr int kLoraMaxMats = 3;
constexpr int kLoraRecords = 64;        // records of one launch
constexpr int kLoraFeatures = 128;      // output features of one wavefront's step: 8 MFMA rows of 16
constexpr int kLoraShrinkWaves = 8;
constexpr int kLoraExpandWaves = 4;
constexpr int kLoraGradWaves = 8;

struct LoraTile {                       // few tokens
    const uint16_t* w;                  // the launch's weight: A or B of this tenant and matrix
    int32_t hrow;                       // row of its first token in the workspace's h (or g)
    int32_t tenant;
    uint16_t rank, count, mat, unused;
    uint16_t col[16];                   // the tokens
};
struct LoraJob {                        // many tokens
    const uint16_t* w;
    int32_t hrow, tenant, count, tile_begin;
    int32_t first;                      // sorted position of the first token
    uint16_t rank, mat;
};

// h[p][j] = sum_k w_j[k] src[token(p)][k], split over `splits` parts of the sum: A x (forward) or B^T dy (backward, w is then
// [K, rank] and the result is multiplied by the tenant's scale)
struct LoraShrinkArgs {
    const uint16_t* src;                // [T, K]
    const float* scale;                 // backward: the tenants' scales (device)
    const int32_t* order;               // sorted position -> token, nullptr: the same (many tokens only)
    float* h;                           // [splits][rows][ld]
    int64_t K, split_stride;            // split_stride = rows * ld
    int32_t ld, splits, n_records, n_tiles;
    union {
        LoraTile tile[kLoraRecords];
        LoraJob job[kLoraRecords];
    };
};

// y[token][f] = fp16(y0[token][f] + scale * sum_j w_j[f] h[p][j]): B h (forward, w is [F, rank]) or A^T g (backward, w is
// [rank, F], no scale)
struct LoraExpandArgs {
    const float* h;
    float* h_out[kLoraMaxMats];         // forward, may be nullptr: h in token order, [T, h_ld]
    const uint16_t* y0[kLoraMaxMats];   // may be nullptr
    uint16_t* y[kLoraMaxMats];
    const float* scale[kLoraMaxMats];   // forward: device, by tenant
    const int32_t* order;
    int64_t F[kLoraMaxMats], split_stride;
    int32_t ld, splits, n_records, n_tiles, h_ld;
    union {
        LoraTile tile[kLoraRecords];
        LoraJob job[kLoraRecords];
    };
};

// out[r][f] (dA) or out[f][r] (dB) = scale * sum over a job's tokens of w[token][r] d[token][f]
struct LoraGradJob {
    float* out;
    int64_t part;                       // where the job's partial sums begin in `partial` (floats)
    int32_t tenant, count, first;       // first: sorted position, also the row of w in position order
    int32_t rank;
};
struct LoraGradArgs {
    const uint16_t* d;                  // [T, F]
    const float* w;                     // dA: g [splits][rows][w_ld] by sorted position; dB: h [T, w_ld] by token
    const float* scale;                 // dB: device, by tenant; dA: nullptr (g has it)
    const int32_t* order;
    float* partial;                     // [token_splits][part_stride], used where token_splits > 1
    int64_t F, w_split_stride, part_stride;
    int32_t w_ld, w_splits, token_splits, n_jobs, accumulate, w_by_token, rank_major;   // rank_major: out is [rank][F]
    LoraGradJob job[kLoraRecords];
};
// out (+)= sum over the splits of the partial sums; or zeros for gradients of tenants without a token
struct LoraReduceArgs {
    const float* partial;               // nullptr: zeros
    int64_t part_stride;
    int32_t token_splits, n_jobs, accumulate;
    struct { float* out; int64_t part, n; } job[kLoraRecords];
};

// `columns`: tokens of a tile (16: records are tiles; 64: records are jobs).  max_rank: the largest rank of the records.
hipError_t launch_lora_shrink(const LoraShrinkArgs& a, int columns, bool transposed, int max_rank, hipStream_t st);
hipError_t launch_lora_expand(const LoraExpandArgs& a, int columns, bool transposed, int64_t max_F, hipStream_t st);
hipError_t launch_lora_grad(const LoraGradArgs& a, int max_rank, hipStream_t st);
hipError_t launch_lora_reduce(const LoraReduceArgs& a, int64_t max_n, hipStream_t st);

}  // namespace bd
