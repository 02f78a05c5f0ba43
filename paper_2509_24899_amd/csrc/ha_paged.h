// Building blocks of paged caches (gfx950): the problem as the kernels see it, which rows and slots belong together, tiles of slots.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hybrid_attn_paged.h"
#include "ha_rows.h"

namespace ha {

struct Paged {
  int B, H, Hkv, G, T, n_pages, page, page_log2, max_pages, max_new, causal;
  const int32_t *table, *key_len, *q_offset;
  __device__ __forceinline__ int capacity() const { return max_pages << page_log2; }
  __device__ __forceinline__ int held(int b) const { return min(max(key_len[b], 0), capacity()); }
  __device__ __forceinline__ int offset(int b) const { return q_offset ? min(max(q_offset[b], 0), T) : b * max_new; }
  // The page that holds a slot of sequence b, or -1.
  __device__ __forceinline__ int page_of(int b, int slot) const {
    const int id = table[(int64_t)b * max_pages + (slot >> page_log2)];
    return (unsigned)id < (unsigned)n_pages ? id : -1;
  }
};

// A sequence's new tokens: `first` of the T rows, `all` of them (which says where they stand), `n` that are computed.
struct NewRows {
  int first, all, n;
  __device__ __forceinline__ NewRows(const Paged &p, int b) : first(p.offset(b)), all(max(p.offset(b + 1) - first, 0)), n(min(all, p.max_new)) {}
};

// The last sequence b with at(b) <= x, at rising, at(0) <= x; 64 sequences at a time.
template <typename At>
static __device__ __forceinline__ int last_not_above(int B, int x, int lane, At at) {
  int lo = 0, hi = B;         // at(lo) <= x, at(hi) > x
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, b = lo + lane * step;
    const int below = __popcll(__ballot(b < hi && at(b) <= x));      // (lane 0 is one of them)
    lo = lo + max(below - 1, 0) * step;
    hi = min(lo + step, hi);
  }
  return lo;
}

// Numbers of a sequence's pages, 64 at a time in the lanes of a wave.
struct PageWalk {
  const int32_t *list;
  int n, n_pages, from, entry, lane;
  __device__ __forceinline__ PageWalk(const Paged &p, int b, int lane_) : list(p.table + (int64_t)b * p.max_pages), n(p.max_pages), n_pages(p.n_pages), from(-64), entry(-1), lane(lane_) {}
  // index: wave-uniform, below n
  __device__ __forceinline__ int at(int index) {
    if (index < from || index >= from + 64) {
      from = index;
      entry = from + lane < n ? list[from + lane] : -1;
    }
    const int id = __builtin_amdgcn_readlane(entry, index - from);
    return (unsigned)id < (unsigned)n_pages ? id : -1;
  }
};

// ---- host ----------------------------------------------------------------------------------------------------------
ha_status check_paged(const ha_paged_problem *p);
Paged paged_of(const ha_paged_problem &p);
static inline ha_status check_packed(const ha_paged_problem &p, const ha_view *v, int heads, bool written, View &out) {
  return check_rows(1, heads, p.T, p.d_head, p.dtype, v, written, out);
}
ha_status check_pool(const ha_paged_problem &p, const ha_view *v, bool written, View &out);
static inline ha_status check_workspace(const void *ws, size_t bytes, size_t need) {
  return need > 0 && (!ws || reinterpret_cast<uintptr_t>(ws) & 255u || bytes < need) ? HA_ERR_WORKSPACE : HA_OK;
}

}  // namespace ha
