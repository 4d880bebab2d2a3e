// Host-side helpers that the C entry points share: checks of addresses and the order of a batch's tokens.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cstring>
#include <vector>

#include "bd_launch.h"

namespace bd {

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

inline bool overlaps(const void* a, size_t abytes, const void* b, size_t bbytes) {
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a0 < b0 + bbytes && b0 < a0 + abytes;
}

// The tensors of a call: whether one that is written lies over any other.
struct Range {
    uintptr_t begin, end;
    bool written;
};
inline void add_range(std::vector<Range>& to, const void* p, size_t bytes, bool written) {
    if (p && bytes) to.push_back(Range{(uintptr_t)p, (uintptr_t)p + bytes, written});
}
inline bool any_alias(std::vector<Range>& r) {
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t end_written = 0, end_any = 0;
    for (const Range& v : r) {
        if (v.begin < end_written || (v.written && v.begin < end_any)) return true;
        end_any = std::max(end_any, v.end);
        if (v.written) end_written = std::max(end_written, v.end);
    }
    return false;
}

// Token ids by tenant, tokens of one tenant in their order.  (Tenant ids have been checked.)
inline std::vector<int32_t> order_by_tenant(const int32_t* tenant_of_token, int64_t T, int32_t n_tenants) {
    std::vector<int32_t> order((size_t)T);
    if (std::is_sorted(tenant_of_token, tenant_of_token + T)) {
        for (int64_t i = 0; i < T; ++i) order[(size_t)i] = (int32_t)i;
    } else if (n_tenants <= 8 * T) {
        std::vector<int32_t> next((size_t)n_tenants + 1, 0);
        for (int64_t i = 0; i < T; ++i) ++next[(size_t)tenant_of_token[i] + 1];
        for (int32_t t = 0; t < n_tenants; ++t) next[(size_t)t + 1] += next[(size_t)t];
        for (int64_t i = 0; i < T; ++i) order[(size_t)next[(size_t)tenant_of_token[i]]++] = (int32_t)i;
    } else {   // a table of counts would be larger than the batch
        for (int64_t i = 0; i < T; ++i) order[(size_t)i] = (int32_t)i;
        std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return tenant_of_token[a] < tenant_of_token[b]; });
    }
    return order;
}

// Writes a table of ints into device memory through kernel arguments (no host-to-device copy call): as runs of values that count
// up or repeat (tokens that arrive grouped by tenant: a few runs for the whole batch), where that takes fewer launches than the
// values themselves.
inline hipError_t write_int_table(const std::vector<int32_t>& all, int32_t* dst, hipStream_t st) {
    std::vector<int32_t> runs;   // triples: first index, first value, n (> 0 counting up, < 0 repeated)
    for (size_t i = 0; i < all.size();) {
        size_t e = i + 1;
        const int32_t step = e < all.size() ? all[e] - all[i] : 0;
        if (step == 0 || step == 1)
            while (e < all.size() && all[e] - all[e - 1] == step) ++e;
        runs.insert(runs.end(), {(int32_t)i, all[i], step == 1 ? (int32_t)(e - i) : -(int32_t)(e - i)});
        i = e;
    }
    const bool by_runs = (runs.size() / 3 + 319) / 320 < (all.size() + 959) / 960;
    const std::vector<int32_t>& from = by_runs ? runs : all;
    for (size_t off = 0; off < from.size(); off += 960) {
        PrefillMetaChunk c;
        const int n = (int)std::min<size_t>(960, from.size() - off);
        std::memcpy(c.v, from.data() + off, (size_t)n * sizeof(int32_t));
        const hipError_t e = by_runs ? launch_prefill_meta_runs(c, dst, n / 3, st) : launch_prefill_meta(c, dst + off, n, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace bd
