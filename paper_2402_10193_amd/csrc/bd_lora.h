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
constexpr int kLoraMaxSplits = 8;       // parts that the shrink's sum may be cut into
constexpr int kLoraFeatures = 128;      // output features of one wavefront's step: 8 MFMA rows of 16
constexpr int kLoraExpandTokens = 64;   // tokens of a tile where there are many
constexpr int kLoraShrinkWaves = 4;
constexpr int kLoraExpandWaves = 4;
constexpr int kLoraGradWaves = 4;

struct LoraTile {                       // few tokens
    const uint16_t* w;                  // the launch's weight: A or B of this tenant and matrix
    int32_t hrow;                       // row of its first token in the workspace's h (or g)
    int32_t tenant;
    uint16_t rank, count, mat, unused;
    uint32_t col[8];                    // the tokens, two per word
};
struct LoraDecodeTile {                 // one or two tokens of a tenant, low ranks: both products in one launch
    const uint16_t *wa, *wb;
    int32_t tenant;
    uint16_t rank, count, mat, unused;
    uint16_t col[2];
};
constexpr int kLoraDecodeTokens = 2, kLoraDecodeRank = 16;   // at most, of such a tile
constexpr int kLoraDecodeRecords = 112;                      // of a launch: with the rest below the 4 KB of a kernel's arguments
constexpr int kLoraDecodeFeatures = 1024;                    // of a workgroup

struct LoraJob {                        // many tokens
    const uint16_t* w;
    int32_t hrow, tenant, count;
    int32_t first;                      // sorted position of the first token
    uint16_t rank, mat;
};

struct LoraJobs {
    int32_t tile_begin[kLoraRecords];   // first tile of every record; behind the last one the largest int
    LoraJob job[kLoraRecords];
};

// h[p][j] = sum_k w_j[k] src[token(p)][k], split over `splits` parts of the sum: A x (forward) or B^T dy (backward, w is then
// [K, rank] and the result is multiplied by the tenant's scale)
struct LoraShrinkArgs {
    const uint16_t* src;                // [T, K]
    const float* scale;                 // backward: the tenants' scales (device)
    const int32_t* order;               // sorted position -> token, nullptr: the same (many tokens only)
    float* h;                           // [splits][rows][ld]
    int64_t K, split_stride;            // split_stride = rows * ld
    int32_t ld, splits, n_tiles;
    union {
        LoraTile tile[kLoraRecords];
        LoraJobs jobs;
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
    int32_t ld, splits, n_tiles, h_ld;
    union {
        LoraTile tile[kLoraRecords];
        LoraJobs jobs;
    };
};

// order[position among the tokens sorted by job] = token, for `count` tokens from `first` on: their jobs, `bits` each, and where the next token of
// every job goes
constexpr int kLoraOrderJobs = 256, kLoraOrderBytes = 2944;
struct LoraOrderArgs {
    int32_t* order;
    int32_t first, count, bits, n_jobs;
    int32_t begin[kLoraOrderJobs];
    uint8_t job[kLoraOrderBytes];
};

struct LoraDecodeArgs {
    const uint16_t* x;                  // [T, in]
    const uint16_t* y0[kLoraMaxMats];   // may be nullptr
    uint16_t* y[kLoraMaxMats];
    const float* scale[kLoraMaxMats];
    float* h_out[kLoraMaxMats];         // may be nullptr
    int64_t F[kLoraMaxMats];
    int64_t in;
    int32_t n_tiles, h_ld;
    LoraDecodeTile tile[kLoraDecodeRecords];
};

typedef _Float16 half8 __attribute__((ext_vector_type(8)));

// g and h as operands of the gradients' sums over tokens, in chunks of 32 tokens of a job
struct LoraPrepJob {
    int32_t first, count, rank, chunk_begin, sides;   // sides: bit 0 where g is wanted, bit 1 where h is
};
struct LoraPrepArgs {
    float* g;                           // [splits][rows][ld] by sorted position; part 0 receives the sum
    const float* h;                     // [T, h_ld] by token
    const int32_t* order;
    half8* operand[2];                  // of g, of h: [chunk][ld / 16][hi, lo][64 lanes]
    uint8_t* exponent[2];               // [chunk][ld]: 127 + e, by rank
    int64_t split_stride;
    int32_t ld, splits, h_ld, n_jobs, chunk_first, side_first;   // side_first = 1: only h
    LoraPrepJob job[kLoraRecords];
};

// side 0: dA [r][F] = sum over a job's tokens of g[token][r] x[token][f];  side 1: dB [F][r] = scale * sum of dy[token][f] h[token][r]
constexpr int kLoraGradJobs = 48;
constexpr int kLoraPartTokens = 4096;   // most tokens of a part
constexpr int lora_grad_rank_waves(int max_rank) { return max_rank <= 16 ? 1 : max_rank <= 32 ? 2 : 4; }   // wavefronts that share a tile
struct LoraGradJob {
    float* out[2];                      // nullptr: not wanted
    int32_t partial;                    // where its parts begin in `partial`, in rows of F
    int32_t tenant, count, first, rank, chunk_begin, parts, part_chunks;   // part_chunks: chunks of 32 tokens of each part but the last
};
struct LoraGradSide {
    const uint16_t* d;                  // [T, F]
    const half8* operand;
    const uint8_t* exponent;
    const float* scale;                 // dB: device, by tenant; dA: nullptr (g has it)
    float* partial;                     // the sums of jobs whose tokens are in several parts: [part][rank * F]
    int64_t F;
};
struct LoraGradArgs {
    const int32_t* order;
    LoraGradSide side[2];
    int32_t ld, n_jobs, n_parts, accumulate, rank_groups;
    int32_t part_begin[kLoraGradJobs];  // first part of every job; behind the last one the largest int
    LoraGradJob job[kLoraGradJobs];
};
// out (+)= sum over the parts; or zeros (parts = 0) for gradients of tenants without a token
struct LoraReduceArgs {
    int32_t n_jobs, accumulate;
    struct { float* out; const float* partial; int64_t n; int32_t parts; } job[kLoraRecords];
};

// Workgroups of the shrink for one tile and part of the sum.  (The backward kernel of ranks that are no multiple of 8 takes 16 ranks each; how its sum
// is cut goes by this all the same.)
constexpr int lora_shrink_groups(int rank, int columns) { return (rank + 15) / 16 <= 1 || columns == 16 ? (rank + 15) / 16 : (rank + 63) / 64; }

// `columns`: tokens of a tile (16: records are tiles; else records are jobs, 64).  max_rank: the largest rank of the records;
// odd: some rank is not a multiple of 8 (B's rows are then no whole 16-byte pieces).
hipError_t launch_lora_order(const LoraOrderArgs& a, hipStream_t st);
hipError_t launch_lora_decode(const LoraDecodeArgs& a, int max_tokens, int64_t max_F, bool odd, hipStream_t st);
hipError_t launch_lora_shrink(const LoraShrinkArgs& a, int columns, bool transposed, int max_rank, bool odd, hipStream_t st);
hipError_t launch_lora_expand(const LoraExpandArgs& a, int columns, bool transposed, int max_rank, int64_t min_F, int64_t max_F, bool odd, hipStream_t st);
// prepares `chunks` chunks from a.chunk_first on, of `sides` sides from a.side_first on
hipError_t launch_lora_prep(const LoraPrepArgs& a, int chunks, int sides, hipStream_t st);
hipError_t launch_lora_grad(const LoraGradArgs& a, int max_rank, hipStream_t st);
hipError_t launch_lora_reduce(const LoraReduceArgs& a, int64_t max_n, hipStream_t st);

}  // namespace bd
