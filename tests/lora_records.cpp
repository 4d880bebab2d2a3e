// The host side of the low-rank adapters with stand-ins for its kernels' launches: what every launch would have read is written down, so
// that a test can look at it without a GPU.  Built by the test that uses it.
#include "lora_api.hip"

namespace {

struct Record {
    int64_t kind, tenant, rank, weight, sides, out0, out1;   // kind: 1 shrink, 2 expand, 3 operands, 4 gradients, 5 decode
};
std::vector<Record> records;

template <typename Args>
void of_tiles(const Args& a, int kind, int columns) {
    if (columns == 16) {
        for (int i = 0; i < a.n_tiles; ++i) records.push_back(Record{kind, a.tile[i].tenant, a.tile[i].rank, (int64_t)a.tile[i].w, 0, 0, 0});
    } else {
        for (int i = 0; i < bd::kLoraRecords && a.jobs.tile_begin[i] != INT32_MAX; ++i)
            records.push_back(Record{kind, a.jobs.job[i].tenant, a.jobs.job[i].rank, (int64_t)a.jobs.job[i].w, 0, 0, 0});
    }
}

}  // namespace

namespace bd {

hipError_t launch_prefill_meta(const PrefillMetaChunk&, int32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_prefill_meta_runs(const PrefillMetaChunk&, int32_t*, int, hipStream_t) { return hipSuccess; }
hipError_t launch_lora_order(const LoraOrderArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_lora_decode(const LoraDecodeArgs& a, int, int64_t, bool, hipStream_t) {
    for (int i = 0; i < a.n_tiles; ++i) records.push_back(Record{5, a.tile[i].tenant, a.tile[i].rank, (int64_t)a.tile[i].wa, 0, 0, 0});
    return hipSuccess;
}
hipError_t launch_lora_shrink(const LoraShrinkArgs& a, int columns, bool, int, bool, hipStream_t) {
    of_tiles(a, 1, columns);
    return hipSuccess;
}
hipError_t launch_lora_expand(const LoraExpandArgs& a, int columns, bool, int, int64_t, int64_t, bool, hipStream_t) {
    of_tiles(a, 2, columns);
    return hipSuccess;
}
// (its jobs are the gradients' of the launch behind it: `sides` has bit 0 where a launch prepares g, bit 1 where it prepares h)
hipError_t launch_lora_prep(const LoraPrepArgs& a, int, int sides, hipStream_t) {
    for (int i = 0; i < a.n_jobs; ++i)
        records.push_back(Record{3, a.job[i].first, a.job[i].rank, 0, (sides == 2 ? 3 : 1 << a.side_first) & a.job[i].sides, 0, 0});
    return hipSuccess;
}
hipError_t launch_lora_grad(const LoraGradArgs& a, int, hipStream_t) {
    for (int i = 0; i < a.n_jobs; ++i)
        records.push_back(Record{4, a.job[i].tenant, a.job[i].rank, 0, 0, (int64_t)a.job[i].out[0], (int64_t)a.job[i].out[1]});
    return hipSuccess;
}
hipError_t launch_lora_reduce(const LoraReduceArgs&, int64_t, hipStream_t) { return hipSuccess; }

}  // namespace bd

// copies the records of the calls since the last one, 7 numbers each, and forgets them
extern "C" int64_t lora_records(int64_t* to, int64_t room) {
    const int64_t n = (int64_t)records.size();
    for (int64_t i = 0; i < n && i < room; ++i) std::memcpy(to + 7 * i, &records[(size_t)i], sizeof(Record));
    records.clear();
    return n;
}
