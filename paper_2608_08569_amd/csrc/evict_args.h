// What the eviction kernels share (evict.hip, and q4_evict.hip for a 4-bit cache).
#pragma once

#include "select.h"

namespace vz_evict {

constexpr int kSel = 1024;
constexpr int kLdsSlots = 16384;    // slots whose keys fit in LDS
static_assert(kLdsSlots % (2 * kSel) == 0, "one load round of the LDS keys");

template <bool LK>
using SelSh = vz_sel::SelShared<kSel, LK ? kLdsSlots : 0>;

// Status of sequence s for an eviction (VZ_OK when it can be served, VZ_IDLE
// for an idle slot).
__device__ __forceinline__ int ragged_evict_status(const VzRagged& r, int s, int n_sink, int n_recent, bool kept) {
    const int64_t b = r.base[s];
    const int c = r.cap[s], n = r.len[s], B = r.budget[s], p = r.next_pos[s];
    if (c == 0) return VZ_IDLE;
    if (n < 0 || c < 1 || b < 0 || b > r.total - c) return VZ_ERR_INVALID;
    if (n > c) return VZ_ERR_CAPACITY;
    const int M = n_recent < 0 ? B / 5 : n_recent;
    if (B < 1 || static_cast<int64_t>(n_sink) + M > B || p < n) return VZ_ERR_INVALID;
    if (kept && p > (1 << 18)) return VZ_ERR_UNSUPPORTED;
    return VZ_OK;
}

// Workspace: move counts [jobs rounded up to 64], then source and destination
// lists [L][plane] each.
struct EvictWs {
    int32_t* n;
    int32_t* src;
    int32_t* dst;
    EvictWs(void* ws, int64_t jobs, int32_t L, int64_t plane) {
        n = static_cast<int32_t*>(ws);
        src = n + 64 * ((jobs + 63) / 64);
        dst = src + static_cast<size_t>(L) * plane;
    }
};

}  // namespace vz_evict
