// C ABI of the low-rank adapters (include/bitdelta.h): argument checks, token grouping, launches.  Everything here runs on the
// host; nothing is enqueued before the arguments have passed.
#include "bitdelta.h"

#include <cstring>
#include <memory>
#include <vector>

#include "bd_host.h"
#include "bd_lora.h"

namespace {

using bd::misaligned;
using bd::overlaps;

constexpr int kFewColumns = 16, kManyColumns = bd::kLoraExpandTokens;   // tokens of a tile: records are tiles, or jobs
// The largest batch whose records are tiles of 16 tokens; more tokens: tiles of 64.  4096 -> 4096, us, tiles of 16 / 64: rank 16, 8 tenants: 512
// tokens 9.4 / 9.6, backward 23.1 / 23.4; 1024 tokens 13.3 / 10.8, 27.2 / 28.3; 2048 tokens 24.1 / 18.2, 40.6 / 34.1; rank 64: 512 tokens
// 16.7 / 18.0, 33.2 / 33.3; 1024 tokens 26.2 / 22.0, 42.0 / 37.8.
constexpr int64_t kFewTokens = 512;
constexpr int64_t kDecodeIn = 12288, kDecodeWeight = (int64_t)1 << 28;   // most of in x tokens, of in x out, of a decode launch
constexpr int kGradParts = 32;                       // parts of jobs whose tokens are in more than one, of all jobs together

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

int compute_units() {
    int cus = 256;
    return bd::device_cu_count(&cus) == hipSuccess && cus > 0 ? cus : 256;
}

// Parts that the shrink's sum is cut into, where `groups` workgroups take a part each.  Two run on a compute unit at a time: some 4 us, and
// for each workgroup of the compute unit and step of its wavefronts 0.25 us (64 tokens; 0.9 with more than 16 ranks at once), or for every two
// of them 0.2 us (a tile of 16 tokens: they wait more than they work).  A part costs the next kernel, which adds it up, 0.3 to 0.4 us and
// its bytes, and `again` rows out of the caches where all of its workgroups read their tile's.  Measured, us of the two kernels (backward: of all), parts 1 / 2 / 3 / 4 / 8, * the rule's: 512 tokens of 8 tenants, 4096 -> 4096,
// rank 16: 11.4 / 10.1 / 9.7 / 9.5* / 9.2; 4096 tokens 29.0 / 25.1 / 24.1 / 24.3* / 26.1, backward 49.6 / 46.3 / 45.5 / 45.7* / 47.1; 8192 tokens of 2,
// rank 64, backward of 4096 -> 11008, 128 tiles: 178 / 157* / 165 / 161.
int max_splits(int64_t T) { return T <= 4096 ? bd::kLoraMaxSplits : T <= 16384 ? 4 : T <= 32768 ? 2 : 1; }
int sum_splits(int64_t groups, int64_t K, int64_t T, int64_t rows, int64_t ld, bool few, int64_t again) {
    const int64_t steps = (K + 31) / 32, cus = compute_units();
    const double part = (few ? 0.3 : 0.4 + (double)(rows * ld * 8) / 4e6) + (double)(again * ld * 4) / 1e7;
    int best = 1;
    double least = 1e30;
    for (int n = 1; n <= max_splits(T) && (n == 1 || n * bd::kLoraShrinkWaves <= steps); ++n) {
        const int64_t layers = (groups * n + cus - 1) / cus, rounds = (layers + 1) / 2, per_wave = (steps + n * bd::kLoraShrinkWaves - 1) / (n * bd::kLoraShrinkWaves);
        const double work = few ? 0.2 * (double)rounds : (ld > 16 ? 0.9 : 0.25) * (double)layers;
        const double us = 4.0 * (double)rounds + work * (double)per_wave + part * n;
        if (us < least) least = us, best = n;
    }
    return best;
}

struct Job {
    int32_t tenant, first, count;   // first: position in the sorted order
};

// The batch by tenant.
struct Batch {
    std::vector<int32_t> order;   // empty: the tokens are sorted as they come
    std::vector<Job> jobs;
    int32_t token(int64_t p) const { return order.empty() ? (int32_t)p : order[(size_t)p]; }
};
Batch group(const int32_t* tenant_of_token, int64_t T, int32_t n_tenants) {
    Batch b;
    if (!std::is_sorted(tenant_of_token, tenant_of_token + T)) b.order = bd::order_by_tenant(tenant_of_token, T, n_tenants);
    for (int64_t p = 0; p < T; ++p) {
        const int32_t tenant = tenant_of_token[b.token(p)];
        if (b.jobs.empty() || b.jobs.back().tenant != tenant) b.jobs.push_back(Job{tenant, (int32_t)p, 0});
        ++b.jobs.back().count;
    }
    return b;
}

// Rows of h that the workgroups of the second product read: their tile's each (3 to a compute unit at most).
int64_t rows_again(const Batch& b, int64_t F, int columns) {
    int64_t tiles = 0;
    for (const Job& j : b.jobs) tiles += (j.count + columns - 1) / columns;
    const int64_t wide = (F + bd::kLoraFeatures - 1) / bd::kLoraFeatures;
    return columns == kFewColumns ? tiles * (wide + 3) / 4 * columns : std::min<int64_t>(3 * compute_units(), tiles * wide) * columns;
}

// The order of the tokens into device memory: by the tokens' jobs, which the device sorts, where that takes fewer launches than the order itself
// (bd::write_int_table: a few runs, or 960 tokens a launch).
hipError_t write_order(const Batch& b, int64_t T, int32_t* dst, hipStream_t st) {
    const int n = (int)std::min<size_t>(b.jobs.size(), bd::kLoraOrderJobs + 1);
    const int bits = n <= 2 ? 1 : n <= 4 ? 2 : n <= 16 ? 4 : 8;
    const int64_t each = bd::kLoraOrderBytes * 8 / bits;
    int64_t runs = 1;
    for (size_t i = 1; i < b.order.size(); ++i) runs += b.order[i] != b.order[i - 1] + 1;
    const int64_t launches = std::min((runs + 319) / 320, (T + 959) / 960);
    if (n > bd::kLoraOrderJobs || (T + each - 1) / each >= launches) return bd::write_int_table(b.order, dst, st);
    std::vector<uint8_t> job((size_t)T);
    auto a = std::make_unique<bd::LoraOrderArgs>();
    for (int j = 0; j < n; ++j) {
        a->begin[j] = b.jobs[(size_t)j].first;
        for (int32_t i = 0; i < b.jobs[(size_t)j].count; ++i) job[(size_t)b.order[(size_t)(b.jobs[(size_t)j].first + i)]] = (uint8_t)j;
    }
    a->order = dst;
    a->bits = bits;
    a->n_jobs = n;
    for (int64_t first = 0; first < T; first += each) {
        a->first = (int32_t)first;
        a->count = (int32_t)std::min(each, T - first);
        std::memset(a->job, 0, sizeof(a->job));
        for (int32_t i = 0; i < a->count; ++i) a->job[i * bits >> 3] |= (uint8_t)(job[(size_t)(first + i)] << (i * bits & 7));
        if (const hipError_t e = bd::launch_lora_order(*a, st); e != hipSuccess) return e;
        for (int32_t i = 0; i < a->count; ++i) ++a->begin[job[(size_t)(first + i)]];
    }
    return hipSuccess;
}

// Fills the records of one kernel's launches and runs them: `per_record` says whether a (job, matrix) takes part, with which
// weight and rank.
template <typename Args, typename Weight, typename Launch>
hipError_t for_records(Args& a, const Batch& b, int64_t T, int n_mats, int columns, Weight weight, Launch launch) {
    const bool few = columns == kFewColumns;
    int n = 0, tiles = 0, max_rank = 0;
    bool odd = false;
    auto flush = [&]() -> hipError_t {
        if (n == 0) return hipSuccess;
        a.n_tiles = tiles;
        for (int k = n; k < bd::kLoraRecords && !few; ++k) a.jobs.tile_begin[k] = INT32_MAX;
        const hipError_t e = launch(max_rank, odd);
        n = tiles = max_rank = 0;
        odd = false;
        return e;
    };
    for (const Job& j : b.jobs)
        for (int m = 0; m < n_mats; ++m) {
            const uint16_t* w = nullptr;
            int rank = 0;
            if (!weight(m, j.tenant, &w, &rank)) continue;
            const bool odd_rank = rank % 8 != 0;
            if (few) {
                for (int32_t at = 0; at < j.count; at += kFewColumns) {
                    bd::LoraTile& t = a.tile[n];
                    t = bd::LoraTile{};
                    t.w = w;
                    t.hrow = (int32_t)(m * T + j.first + at);
                    t.tenant = j.tenant;
                    t.rank = (uint16_t)rank;
                    t.count = (uint16_t)std::min(kFewColumns, j.count - at);
                    t.mat = (uint16_t)m;
                    for (int c = 0; c < t.count; ++c) t.col[c >> 1] |= (uint32_t)b.token(j.first + at + c) << (16 * (c & 1));
                    ++n, ++tiles;
                    max_rank = std::max(max_rank, rank);
                    odd |= odd_rank;
                    if (n == bd::kLoraRecords)
                        if (const hipError_t e = flush(); e != hipSuccess) return e;
                }
            } else {
                bd::LoraJob& t = a.jobs.job[n];
                t = bd::LoraJob{};
                t.w = w;
                t.hrow = (int32_t)(m * T + j.first);
                t.tenant = j.tenant;
                t.count = j.count;
                a.jobs.tile_begin[n] = tiles;
                t.first = j.first;
                t.rank = (uint16_t)rank;
                t.mat = (uint16_t)m;
                ++n;
                tiles += (j.count + columns - 1) / columns;
                max_rank = std::max(max_rank, rank);
                odd |= odd_rank;
                if (n == bd::kLoraRecords)
                    if (const hipError_t e = flush(); e != hipSuccess) return e;
            }
        }
    return flush();
}

// The workspace: the order of the tokens, then h (or g) as partial sums, then what the gradients need.
size_t order_bytes(int64_t T) { return (size_t)round_up(T * 4, 256); }
size_t h_bytes(int64_t T, int32_t n_mats, int32_t max_rank) {
    return (size_t)round_up((int64_t)max_splits(T) * n_mats * T * round_up(max_rank, 16) * 4, 256);
}
// operands of the gradients: 32 tokens of a job by 16 ranks as hi and lo, for g and for h, and an exponent for every rank of the 32
int64_t most_chunks(int64_t T, int32_t n_tenants) { return T / 32 + std::min<int64_t>(T, n_tenants); }
size_t operand_bytes(int64_t chunks, int32_t max_rank) { return (size_t)(chunks * (round_up(max_rank, 16) / 16) * 2 * 64 * 16); }
size_t exponent_bytes(int64_t chunks, int32_t max_rank) { return (size_t)round_up(chunks * round_up(max_rank, 16), 256); }
int64_t most_parts(int64_t T) { return std::min<int64_t>(kGradParts, T / 32); }
size_t grad_part_bytes(int64_t T, int64_t out, int64_t in, int32_t max_rank) {
    return (size_t)round_up(most_parts(T) * round_up(max_rank, 16) * (in + out) * 4, 256);
}

bool sizes_ok(int64_t T, int64_t out, int64_t in, int32_t n_tenants) {
    return T >= 0 && T <= 65535 && out >= 0 && in >= 0 && n_tenants >= 0 && in % 32 == 0 && out <= (int64_t)1 << 24 && in <= (int64_t)1 << 24;
}

// Both products in one launch (lora_decode_kernel), where it is quicker than two.  Every workgroup reads all of A and multiplies it with
// each of its tenant's tokens, so its time grows with in x tokens, and with in x out where many tenants' workgroups share the caches.
// Rank 16, out = 4096, 16 tenants, one launch against two: in = 4096: 5.0 / 7.9 us, 2 tokens each 7.0 / 7.8, 4 each 10.7 / 8.1;
// in = 11008: 7.8 / 8.2, 2 each 11.8 / 8.1; in = 28672: 13.3 / 9.6.  64 tenants, out = 32000: in = 4096: 25.1 / 34.7, 8192: 35.6 / 37.0,
// 11008: 47.8 / 37.9.  Rank 32 has each of its wavefronts read twice as many rows: in = 4096, 64 tenants: 12.8 / 11.3.
bool decode_fits(const Batch& b, int max_rank, int64_t in, int64_t max_out) {
    if (max_rank > bd::kLoraDecodeRank || in < 8 || in * max_out > kDecodeWeight) return false;
    for (const Job& j : b.jobs)
        if (j.count > bd::kLoraDecodeTokens || in * j.count > kDecodeIn) return false;
    return true;
}

bd_status forward(int32_t n_mats, const uint16_t* x, const uint16_t* const* a_by, const uint16_t* const* b_by, const int32_t* rank_by,
                  const float* const* scale, const int32_t* tenant_of_token, const uint16_t* const* y0, uint16_t* const* y,
                  float* const* h, int32_t h_ld, int64_t T, const int64_t* out, int64_t in, int32_t n_tenants, void* workspace,
                  size_t workspace_bytes, hipStream_t st) {
    if (n_mats < 1 || n_mats > bd::kLoraMaxMats) return BD_ERR_SHAPE;
    if (!out) return BD_ERR_NULL;
    for (int m = 0; m < n_mats; ++m)
        if (!sizes_ok(T, out[m], in, n_tenants)) return BD_ERR_SHAPE;
    if (T == 0) return BD_OK;
    if (!a_by || !b_by || !rank_by || !scale || !tenant_of_token || !y) return BD_ERR_NULL;
    for (int64_t t = 0; t < T; ++t)
        if (tenant_of_token[t] < 0 || tenant_of_token[t] >= n_tenants) return BD_ERR_TENANT;
    const Batch batch = group(tenant_of_token, T, n_tenants);
    int max_rank = 0;
    int64_t max_out = 0, min_out = out[0];
    for (int m = 0; m < n_mats; ++m) max_out = std::max(max_out, out[m]), min_out = std::min(min_out, out[m]);
    for (const Job& j : batch.jobs)
        for (int m = 0; m < n_mats; ++m) {
            const int32_t rank = rank_by[(size_t)m * n_tenants + j.tenant];
            if (rank < 0 || rank > bd::kLoraMaxRank) return BD_ERR_SHAPE;
            max_rank = std::max(max_rank, (int)rank);
        }
    if (max_rank > 0 && in > 0 && !x) return BD_ERR_NULL;
    if (misaligned(x, 16)) return BD_ERR_ALIGN;
    const size_t xbytes = (size_t)T * in * 2;
    for (int m = 0; m < n_mats; ++m) {
        const size_t ybytes = (size_t)T * out[m] * 2;
        if (out[m] > 0 && !y[m]) return BD_ERR_NULL;
        if (misaligned(y[m], 16) || (y0 && misaligned(y0[m], 16)) || misaligned(scale[m], 4) || (h && misaligned(h[m], 4))) return BD_ERR_ALIGN;
        if (max_rank > 0 && out[m] > 0 && !scale[m]) return BD_ERR_NULL;
        if (h && h[m] && (h_ld < 0 || h_ld < max_rank)) return BD_ERR_SHAPE;
        const size_t hbytes = h && h[m] ? (size_t)T * h_ld * 4 : 0;
        if (overlaps(y[m], ybytes, x, xbytes) || (hbytes && (overlaps(h[m], hbytes, x, xbytes) || overlaps(h[m], hbytes, y[m], ybytes)))) return BD_ERR_ALIAS;
        for (int o = 0; o < n_mats; ++o) {
            const size_t obytes = (size_t)T * out[o] * 2;
            if (max_rank > 0 && scale[o] && (overlaps(y[m], ybytes, scale[o], (size_t)n_tenants * 4) || (hbytes && overlaps(h[m], hbytes, scale[o], (size_t)n_tenants * 4)))) return BD_ERR_ALIAS;
            if (o != m && overlaps(y[m], ybytes, y[o], obytes)) return BD_ERR_ALIAS;
            if (o != m && hbytes && (overlaps(h[m], hbytes, y[o], obytes) || (h[o] && overlaps(h[m], hbytes, h[o], (size_t)T * h_ld * 4)))) return BD_ERR_ALIAS;
            if (y0 && y0[o] && !(o == m && y0[m] == y[m]) && overlaps(y[m], ybytes, y0[o], obytes)) return BD_ERR_ALIAS;
            if (y0 && y0[o] && hbytes && overlaps(h[m], hbytes, y0[o], obytes)) return BD_ERR_ALIAS;
        }
    }
    for (const Job& j : batch.jobs)
        for (int m = 0; m < n_mats; ++m) {
            const size_t at = (size_t)m * n_tenants + j.tenant;
            const size_t rank = (size_t)rank_by[at], abytes = rank * in * 2, bbytes = rank * out[m] * 2;
            if (rank == 0) continue;
            if ((abytes && !a_by[at]) || (bbytes && !b_by[at])) return BD_ERR_NULL;
            if (misaligned(a_by[at], 16) || misaligned(b_by[at], 16)) return BD_ERR_ALIGN;
            for (int o = 0; o < n_mats; ++o) {
                const size_t ybytes = (size_t)T * out[o] * 2, hbytes = h && h[o] ? (size_t)T * h_ld * 4 : 0;
                if (overlaps(y[o], ybytes, a_by[at], abytes) || overlaps(y[o], ybytes, b_by[at], bbytes)) return BD_ERR_ALIAS;
                if (hbytes && (overlaps(h[o], hbytes, a_by[at], abytes) || overlaps(h[o], hbytes, b_by[at], bbytes))) return BD_ERR_ALIAS;
            }
        }
    if (max_rank > 0 && (!workspace || workspace_bytes < order_bytes(T) + h_bytes(T, n_mats, max_rank) || misaligned(workspace, 256)))
        return BD_ERR_WORKSPACE;
    // without an adapter there is nothing to do where y is y0
    auto takes_part = [&](int m, int32_t rank) { return (out[m] > 0 || (h && h[m])) && (rank > 0 || !(y0 && y0[m] == y[m])); };
    // ---- checked: launches from here on ----
    if (decode_fits(batch, max_rank, in, max_out)) {
        auto d = std::make_unique<bd::LoraDecodeArgs>();
        for (int m = 0; m < n_mats; ++m) {
            d->y0[m] = y0 ? y0[m] : nullptr;
            d->y[m] = y[m];
            d->scale[m] = scale[m];
            d->F[m] = out[m];
            d->h_out[m] = h ? h[m] : nullptr;
        }
        d->x = x;
        d->in = in;
        d->h_ld = h_ld;
        int tokens = 1;
        bool odd = false;
        auto flush = [&]() {
            const bool ok = d->n_tiles == 0 || bd::launch_lora_decode(*d, tokens, max_out, odd, st) == hipSuccess;
            d->n_tiles = 0;
            tokens = 1;
            odd = false;
            return ok;
        };
        for (const Job& j : batch.jobs)
            for (int m = 0; m < n_mats; ++m) {
                const size_t at = (size_t)m * n_tenants + j.tenant;
                if (!takes_part(m, rank_by[at])) continue;
                bd::LoraDecodeTile& t = d->tile[d->n_tiles++];
                t = bd::LoraDecodeTile{a_by[at], b_by[at], j.tenant, (uint16_t)rank_by[at], (uint16_t)j.count, (uint16_t)m, 0, {0, 0}};
                for (int c = 0; c < j.count; ++c) t.col[c] = (uint16_t)batch.token(j.first + c);
                tokens = std::max(tokens, (int)j.count);
                odd |= rank_by[at] % 8 != 0;
                if (d->n_tiles == bd::kLoraDecodeRecords && !flush()) return BD_ERR_DEVICE;
            }
        return flush() ? BD_OK : BD_ERR_DEVICE;
    }
    const bool few = T <= kFewTokens;
    const int columns = few ? kFewColumns : kManyColumns;
    const int32_t* order = nullptr;
    if (!few && !batch.order.empty() && max_rank > 0) {
        if (write_order(batch, T, (int32_t*)workspace, st) != hipSuccess) return BD_ERR_DEVICE;
        order = (const int32_t*)workspace;
    }
    float* const hw = (float*)((char*)workspace + order_bytes(T));
    const int64_t ld = round_up(max_rank, 16);
    int64_t groups = 0;
    for (const Job& j : batch.jobs)
        for (int m = 0; m < n_mats; ++m)
            groups += (int64_t)(j.count + columns - 1) / columns * bd::lora_shrink_groups(rank_by[(size_t)m * n_tenants + j.tenant], columns);
    const int splits = sum_splits(groups, in, T, n_mats * T, ld, few, rows_again(batch, max_out, columns) * n_mats);
    if (max_rank > 0) {
        auto s = std::make_unique<bd::LoraShrinkArgs>();
        s->src = x;
        s->order = order;
        s->h = hw;
        s->K = in;
        s->ld = (int32_t)ld;
        s->splits = splits;
        s->split_stride = n_mats * T * ld;
        const hipError_t e = for_records(
            *s, batch, T, n_mats, columns,
            [&](int m, int32_t tenant, const uint16_t** w, int* rank) {
                const size_t at = (size_t)m * n_tenants + tenant;
                *w = a_by[at];
                *rank = rank_by[at];
                return rank_by[at] > 0;
            },
            [&](int rank, bool odd) { return bd::launch_lora_shrink(*s, columns, false, rank, odd, st); });
        if (e != hipSuccess) return BD_ERR_DEVICE;
    }
    auto x2 = std::make_unique<bd::LoraExpandArgs>();
    for (int m = 0; m < n_mats; ++m) {
        x2->y0[m] = y0 ? y0[m] : nullptr;
        x2->y[m] = y[m];
        x2->scale[m] = scale[m];
        x2->F[m] = out[m];
        x2->h_out[m] = h ? h[m] : nullptr;
    }
    x2->h = hw;
    x2->order = order;
    x2->ld = (int32_t)ld;
    x2->h_ld = h_ld;
    x2->splits = splits;
    x2->split_stride = n_mats * T * ld;
    const hipError_t e = for_records(
        *x2, batch, T, n_mats, columns,
        [&](int m, int32_t tenant, const uint16_t** w, int* rank) {
            const size_t at = (size_t)m * n_tenants + tenant;
            *w = b_by[at];
            *rank = rank_by[at];
            return takes_part(m, rank_by[at]);
        },
        [&](int rank, bool odd) { return bd::launch_lora_expand(*x2, columns, false, rank, min_out, max_out, odd, st); });
    return e == hipSuccess ? BD_OK : BD_ERR_DEVICE;
}

// Parts of every job's tokens in the gradients' sums: one, or more where that fills the compute units better (the parts must then be
// added up).  A workgroup of RW wavefronts to a tile takes some 5 us and 0.35 us for every tile of 32 tokens that each of its 4 / RW groups
// takes; 3 run on a compute unit at a time.  Backward, us, 1 / 2 / 3 / 4 / 8 parts of the longest job, * the rule's: 512 tokens of 8 tenants, rank 16,
// 4096 -> 4096: 22* / 35; 4096 tokens: 47* / 54 / 58 / 64; 8192 tokens of 2, rank 64, 4096 -> 11008: 188 / 170 / 160* / 178 / 195.
void cut_into_parts(bd::LoraGradJob* job, int n, int64_t wide, int rank, int64_t most) {
    int longest = 1;
    for (int i = 0; i < n; ++i) longest = std::max(longest, (int)job[i].count);
    const int RW = bd::lora_grad_rank_waves(rank), TW = bd::kLoraGradWaves / RW;
    const int64_t slots = (int64_t)compute_units() * 3;
    int best = std::min(longest, bd::kLoraPartTokens);
    double least = 1e30;
    for (int cut = 1; cut <= kGradParts; ++cut) {
        const int tokens = std::min((int)round_up((longest + cut - 1) / cut, 32), bd::kLoraPartTokens);
        int64_t parts = 0, partial = 0;
        for (int i = 0; i < n; ++i) {
            const int64_t p = (job[i].count + tokens - 1) / tokens;
            parts += p;
            if (p > 1) partial += p;
        }
        if (partial > most) continue;
        const int64_t rounds = (parts * wide + slots - 1) / slots;
        const double us = (double)rounds * (5.0 + 0.35 * (double)((tokens + 32 * TW - 1) / (32 * TW))) + (partial ? 4.0 + (double)partial * rank * wide * 128 * 8 / 3e6 : 0.0);
        if (us < least) least = us, best = tokens;
    }
    for (int i = 0; i < n; ++i) {
        job[i].parts = (job[i].count + best - 1) / best;
        job[i].part_chunks = ((job[i].count + 31) / 32 + job[i].parts - 1) / job[i].parts;
        job[i].parts = ((job[i].count + 31) / 32 + job[i].part_chunks - 1) / job[i].part_chunks;   // (no part without tokens)
    }
}

bd_status backward(const uint16_t* dy, const uint16_t* x, const float* h, int32_t h_ld, const uint16_t* const* a_by, const uint16_t* const* b_by,
                   const int32_t* rank_by, const float* scale, const int32_t* tenant_of_token, const uint16_t* dx0, uint16_t* dx,
                   float* const* da_by, float* const* db_by, int32_t accumulate, int64_t T, int64_t out, int64_t in, int32_t n_tenants,
                   void* workspace, size_t workspace_bytes, hipStream_t st) {
    if (!sizes_ok(T, out, in, n_tenants)) return BD_ERR_SHAPE;
    if (n_tenants > 0 && !rank_by) return BD_ERR_NULL;
    if (T > 0 && !tenant_of_token) return BD_ERR_NULL;
    for (int64_t t = 0; t < T; ++t)
        if (tenant_of_token[t] < 0 || tenant_of_token[t] >= n_tenants) return BD_ERR_TENANT;
    const Batch batch = group(tenant_of_token, T, n_tenants);
    std::vector<bd::Range> ranges;
    auto range = [&](const void* p, size_t bytes, bool written) { bd::add_range(ranges, p, bytes, written); };
    int max_rank = 0;
    bool any_da = false, any_db = false;
    std::vector<char> has_tokens((size_t)n_tenants, 0);
    for (const Job& j : batch.jobs) {
        const int32_t e = j.tenant, rank = rank_by[e];
        has_tokens[(size_t)e] = 1;
        if (rank < 0 || rank > bd::kLoraMaxRank) return BD_ERR_SHAPE;
        max_rank = std::max(max_rank, (int)rank);
        if (rank == 0) continue;
        const size_t abytes = (size_t)rank * in * 2, bbytes = (size_t)rank * out * 2;
        const bool da = da_by && da_by[e], db = db_by && db_by[e];
        any_da |= da;
        any_db |= db;
        if (dx && abytes && (!a_by || !a_by[e])) return BD_ERR_NULL;
        if ((dx || da) && bbytes && (!b_by || !b_by[e])) return BD_ERR_NULL;
        if ((a_by && misaligned(a_by[e], 16)) || (b_by && misaligned(b_by[e], 16))) return BD_ERR_ALIGN;
        if (dx && a_by) range(a_by[e], abytes, false);
        if ((dx || da) && b_by) range(b_by[e], bbytes, false);
    }
    for (int32_t e = 0; e < n_tenants; ++e) {
        const bool da = da_by && da_by[e], db = db_by && db_by[e];
        if (!da && !db) continue;
        if (rank_by[e] < 0 || rank_by[e] > bd::kLoraMaxRank) return BD_ERR_SHAPE;
        if ((da && misaligned(da_by[e], 4)) || (db && misaligned(db_by[e], 4))) return BD_ERR_ALIGN;
        if (!has_tokens[(size_t)e] && accumulate) continue;
        if (da) range(da_by[e], (size_t)rank_by[e] * in * 4, true);
        if (db) range(db_by[e], (size_t)rank_by[e] * out * 4, true);
    }
    any_da &= in > 0;
    any_db &= out > 0;
    const bool work = T > 0 && max_rank > 0, want_dx = dx && T > 0 && in > 0;
    if (work) {
        if (out > 0 && (dx || any_da || any_db) && !dy) return BD_ERR_NULL;
        if (in > 0 && any_da && !x) return BD_ERR_NULL;
        if (out > 0 && any_db && !h) return BD_ERR_NULL;
        if ((dx || any_da || any_db) && !scale) return BD_ERR_NULL;
        if (any_db && h_ld < max_rank) return BD_ERR_SHAPE;
    }
    if (misaligned(dy, 16) || misaligned(x, 16) || misaligned(h, 4) || misaligned(scale, 4) || misaligned(dx0, 16) || misaligned(dx, 16)) return BD_ERR_ALIGN;
    range(dy, (size_t)T * out * 2, false);
    range(x, (size_t)T * in * 2, false);
    if (any_db) range(h, (size_t)T * h_ld * 4, false);
    if (work) range(scale, (size_t)n_tenants * 4, false);
    if (want_dx) {
        range(dx, (size_t)T * in * 2, true);
        if (dx0 != dx) range(dx0, (size_t)T * in * 2, false);
    }
    if (bd::any_alias(ranges)) return BD_ERR_ALIAS;
    if (work && (!workspace || misaligned(workspace, 256) || workspace_bytes < bd_lora_backward_workspace_bytes(T, out, in, n_tenants, max_rank)))
        return BD_ERR_WORKSPACE;
    // ---- checked: launches from here on ----
    const bool few = T <= kFewTokens;
    const int columns = few ? kFewColumns : kManyColumns;
    const int64_t ld = round_up(max_rank, 16);
    const int32_t* order = nullptr;
    if (work && !batch.order.empty()) {   // (the gradients' sums run over a job's tokens, for few tokens too)
        if (write_order(batch, T, (int32_t*)workspace, st) != hipSuccess) return BD_ERR_DEVICE;
        order = (const int32_t*)workspace;
    }
    float* const g = work ? (float*)((char*)workspace + order_bytes(T)) : nullptr;
    int64_t groups = 0;
    for (const Job& j : batch.jobs) groups += (int64_t)(j.count + columns - 1) / columns * bd::lora_shrink_groups(rank_by[j.tenant], columns);
    int splits = sum_splits(groups, out, T, T, ld, few, any_da || any_db ? 0 : rows_again(batch, in, columns));
    // A tenant's g (and B) where dx or its own dA is wanted.  (The sum is cut as if all were: what else is wanted does not change its bits.)
    auto wants_da = [&](int32_t tenant) { return any_da && da_by && da_by[tenant]; };
    auto wants_db = [&](int32_t tenant) { return any_db && db_by && db_by[tenant]; };
    auto wants_g = [&](int32_t tenant) { return want_dx || wants_da(tenant); };
    auto weights_of = [&](const uint16_t* const* by, int32_t tenant, const uint16_t** w, int* rank) {
        *rank = rank_by[tenant];
        *w = by && *rank > 0 ? by[tenant] : nullptr;
    };
    if (work && (want_dx || any_da)) {
        auto s = std::make_unique<bd::LoraShrinkArgs>();
        s->src = dy;
        s->scale = scale;
        s->order = order;
        s->h = g;
        s->K = out;
        s->ld = (int32_t)ld;
        s->splits = splits;
        s->split_stride = T * ld;
        const hipError_t e = for_records(
            *s, batch, T, 1, columns,
            [&](int, int32_t tenant, const uint16_t** w, int* rank) {
                weights_of(b_by, tenant, w, rank);
                return *rank > 0 && wants_g(tenant);
            },
            [&](int rank, bool odd) { return bd::launch_lora_shrink(*s, columns, true, rank, odd, st); });
        if (e != hipSuccess) return BD_ERR_DEVICE;
    }
    // ---- g (parts added up) and h as operands of the gradients ----
    const int64_t chunks_most = most_chunks(T, n_tenants);
    bd::half8* operand[2] = {nullptr, nullptr};
    uint8_t* exponent[2] = {nullptr, nullptr};
    float* partial = nullptr;
    if (work) {
        char* p = (char*)g + h_bytes(T, 1, max_rank);
        for (int side = 0; side < 2; ++side, p += operand_bytes(chunks_most, max_rank)) operand[side] = (bd::half8*)p;
        for (int side = 0; side < 2; ++side, p += exponent_bytes(chunks_most, max_rank)) exponent[side] = (uint8_t*)p;
        partial = (float*)p;
    }
    if (work && (any_da || any_db)) {
        auto prep = std::make_unique<bd::LoraPrepArgs>();
        auto args = std::make_unique<bd::LoraGradArgs>();
        prep->g = g;
        prep->h = h;
        prep->order = args->order = order;
        for (int side = 0; side < 2; ++side) {
            prep->operand[side] = operand[side];
            prep->exponent[side] = exponent[side];
            bd::LoraGradSide& v = args->side[side];
            v.d = side ? dy : x;
            v.operand = operand[side];
            v.exponent = exponent[side];
            v.scale = side ? scale : nullptr;
            v.F = side ? (any_db ? out : 0) : (any_da ? in : 0);
            v.partial = partial + (side ? most_parts(T) * ld * in : 0);
        }
        prep->split_stride = T * ld;
        prep->ld = args->ld = (int32_t)ld;
        prep->splits = splits;
        prep->h_ld = h_ld;
        prep->side_first = any_da ? 0 : 1;
        args->accumulate = accumulate ? 1 : 0;
        std::vector<Job> wanted;   // (all with a rank: the sum of g's parts is the expand's input too, and what else is wanted cuts no sum otherwise)
        for (const Job& j : batch.jobs)
            if (rank_by[j.tenant] > 0) wanted.push_back(j);
        int32_t chunk = 0;
        for (size_t first = 0; first < wanted.size(); first += bd::kLoraGradJobs) {
            const int n = (int)std::min<size_t>(bd::kLoraGradJobs, wanted.size() - first);
            int most = 0;
            prep->chunk_first = chunk;
            for (int i = 0; i < n; ++i) {
                const Job& j = wanted[first + (size_t)i];
                const int rank = rank_by[j.tenant];
                prep->job[i] = bd::LoraPrepJob{j.first, j.count, rank, chunk, (any_da && wants_g(j.tenant) ? 1 : 0) | (wants_db(j.tenant) ? 2 : 0)};
                args->job[i] = bd::LoraGradJob{{da_by && in > 0 ? da_by[j.tenant] : nullptr, db_by && out > 0 ? db_by[j.tenant] : nullptr},
                                               0, j.tenant, j.count, j.first, rank, chunk, 1, 0};
                chunk += (j.count + 31) / 32;
                most = std::max(most, rank);
            }
            prep->n_jobs = args->n_jobs = n;
            if (bd::launch_lora_prep(*prep, chunk - prep->chunk_first, (any_da ? 1 : 0) + (any_db ? 1 : 0), st) != hipSuccess) return BD_ERR_DEVICE;
            const int64_t wide = (args->side[0].F + bd::kLoraFeatures - 1) / bd::kLoraFeatures + (args->side[1].F + bd::kLoraFeatures - 1) / bd::kLoraFeatures;
            if (wide == 0) continue;
            cut_into_parts(args->job, n, wide * ((most + 63) / 64), most, most_parts(T));
            auto sum = std::make_unique<bd::LoraReduceArgs>();
            sum->accumulate = args->accumulate;
            int64_t max_n = 0;
            int32_t rows = 0;
            args->n_parts = 0;
            for (int i = 0; i < bd::kLoraGradJobs; ++i) {
                if (i >= n) {
                    args->part_begin[i] = INT32_MAX;
                    continue;
                }
                bd::LoraGradJob& j = args->job[i];
                args->part_begin[i] = args->n_parts;
                args->n_parts += j.parts;
                if (j.parts == 1) continue;
                j.partial = rows;
                for (int side = 0; side < 2; ++side) {
                    if (!j.out[side]) continue;
                    auto& r = sum->job[sum->n_jobs++];
                    r.out = j.out[side];
                    r.partial = args->side[side].partial + (int64_t)rows * args->side[side].F;
                    r.n = j.rank * args->side[side].F;
                    r.parts = j.parts;
                    max_n = std::max(max_n, r.n);
                }
                rows += j.parts * j.rank;
            }
            if (bd::launch_lora_grad(*args, most, st) != hipSuccess) return BD_ERR_DEVICE;
            if (sum->n_jobs > 0 && bd::launch_lora_reduce(*sum, max_n, st) != hipSuccess) return BD_ERR_DEVICE;
        }
        if (any_da) splits = 1;   // g is whole
    }
    if (want_dx) {
        auto x2 = std::make_unique<bd::LoraExpandArgs>();
        x2->y0[0] = dx0;
        x2->y[0] = dx;
        x2->F[0] = in;
        x2->h = g;
        x2->order = order;
        x2->ld = (int32_t)ld;
        x2->splits = splits;
        x2->split_stride = T * ld;
        const hipError_t e = for_records(
            *x2, batch, T, 1, columns,
            [&](int, int32_t tenant, const uint16_t** w, int* rank) {
                weights_of(a_by, tenant, w, rank);
                return *rank > 0 || dx0 != dx;
            },
            [&](int rank, bool odd) { return bd::launch_lora_expand(*x2, columns, true, rank, in, in, odd, st); });
        if (e != hipSuccess) return BD_ERR_DEVICE;
    }
    if (!accumulate) {   // gradients of adapters that no token used
        auto zero = std::make_unique<bd::LoraReduceArgs>();
        int n = 0;
        int64_t max_n = 0;
        auto flush = [&]() {
            zero->n_jobs = n;   // (no parts: the sum of nothing)
            const bool ok = n == 0 || bd::launch_lora_reduce(*zero, max_n, st) == hipSuccess;
            n = 0;
            max_n = 0;
            return ok;
        };
        for (int32_t e = 0; e < n_tenants; ++e) {
            if (has_tokens[(size_t)e]) continue;
            for (int which = 0; which < 2; ++which) {
                float* const p = which ? (db_by ? db_by[e] : nullptr) : (da_by ? da_by[e] : nullptr);
                const int64_t count = rank_by[e] * (which ? out : in);
                if (!p || count == 0) continue;
                zero->job[n].out = p;
                zero->job[n].n = count;
                max_n = std::max(max_n, count);
                if (++n == bd::kLoraRecords && !flush()) return BD_ERR_DEVICE;
            }
        }
        if (!flush()) return BD_ERR_DEVICE;
    }
    return BD_OK;
}

}  // namespace

extern "C" {

size_t bd_lora_workspace_bytes(int64_t T, int32_t n_mats, int32_t max_rank) {
    if (T < 1 || T > 65535 || n_mats < 1 || n_mats > bd::kLoraMaxMats || max_rank < 1 || max_rank > bd::kLoraMaxRank) return 0;
    return order_bytes(T) + h_bytes(T, n_mats, max_rank);
}

size_t bd_lora_backward_workspace_bytes(int64_t T, int64_t out, int64_t in, int32_t n_tenants, int32_t max_rank) {
    if (T < 1 || !sizes_ok(T, out, in, n_tenants) || n_tenants < 1 || max_rank < 1 || max_rank > bd::kLoraMaxRank) return 0;
    const int64_t chunks = most_chunks(T, n_tenants);
    return order_bytes(T) + h_bytes(T, 1, max_rank) + 2 * (operand_bytes(chunks, max_rank) + exponent_bytes(chunks, max_rank)) + grad_part_bytes(T, out, in, max_rank);
}

// (what the standard library throws here is a lack of host memory)
bd_status bd_lora_multitenant_group(int32_t n_mats, const uint16_t* x_f16, const uint16_t* const* a_by_mat_tenant,
                                    const uint16_t* const* b_by_mat_tenant, const int32_t* rank_by_mat_tenant,
                                    const float* const* scale_by_mat, const int32_t* tenant_of_token, const uint16_t* const* y0_f16,
                                    uint16_t* const* y_f16, float* const* h, int32_t h_ld, int64_t T, const int64_t* out, int64_t in,
                                    int32_t n_tenants, void* workspace, size_t workspace_bytes, void* stream) {
    try {
        return forward(n_mats, x_f16, a_by_mat_tenant, b_by_mat_tenant, rank_by_mat_tenant, scale_by_mat, tenant_of_token, y0_f16, y_f16, h,
                       h_ld, T, out, in, n_tenants, workspace, workspace_bytes, (hipStream_t)stream);
    } catch (...) {
        return BD_ERR_DEVICE;
    }
}

bd_status bd_lora_multitenant(const uint16_t* x_f16, const uint16_t* const* a_by_tenant, const uint16_t* const* b_by_tenant,
                              const int32_t* rank_by_tenant, const float* scale_by_tenant, const int32_t* tenant_of_token,
                              const uint16_t* y0_f16, uint16_t* y_f16, float* h, int32_t h_ld, int64_t T, int64_t out, int64_t in,
                              int32_t n_tenants, void* workspace, size_t workspace_bytes, void* stream) {
    return bd_lora_multitenant_group(1, x_f16, a_by_tenant, b_by_tenant, rank_by_tenant, &scale_by_tenant, tenant_of_token, &y0_f16, &y_f16,
                                     &h, h_ld, T, &out, in, n_tenants, workspace, workspace_bytes, stream);
}

bd_status bd_lora_multitenant_backward(const uint16_t* dy_f16, const uint16_t* x_f16, const float* h, int32_t h_ld,
                                       const uint16_t* const* a_by_tenant, const uint16_t* const* b_by_tenant,
                                       const int32_t* rank_by_tenant, const float* scale_by_tenant, const int32_t* tenant_of_token,
                                       const uint16_t* dx0_f16, uint16_t* dx_f16, float* const* da_by_tenant, float* const* db_by_tenant,
                                       int32_t accumulate, int64_t T, int64_t out, int64_t in, int32_t n_tenants, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    try {
        return backward(dy_f16, x_f16, h, h_ld, a_by_tenant, b_by_tenant, rank_by_tenant, scale_by_tenant, tenant_of_token, dx0_f16, dx_f16,
                        da_by_tenant, db_by_tenant, accumulate, T, out, in, n_tenants, workspace, workspace_bytes, (hipStream_t)stream);
    } catch (...) {
        return BD_ERR_DEVICE;
    }
}

}  // extern "C"
