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

// Sum over the lanes up to this one (all of a wave call it), by DPP moves within rows of 16 lanes and then of the last sum of a row to those behind it.
template <int CTRL, int ROWS>
static __device__ __forceinline__ int dpp_add_rows(int x) { return (int)((unsigned)x + (unsigned)__builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false)); }
static __device__ __forceinline__ int sum_upto(int x) {
  x = dpp_add_rows<0x111, 0xf>(x);      // lane - 1, - 2, - 4, - 8
  x = dpp_add_rows<0x112, 0xf>(x);
  x = dpp_add_rows<0x114, 0xf>(x);
  x = dpp_add_rows<0x118, 0xf>(x);
  x = dpp_add_rows<0x142, 0xa>(x);      // lanes 15 and 47 to the rows behind them
  return dpp_add_rows<0x143, 0xc>(x);   // lane 31 to the upper half
}
// A sum of many positive terms, each a sum over a step of rows or slots, with what the roundings have left out: its error does not grow with their number.  (Of nearly equal terms the same part
// is lost again and again: 32768 one behind the other are off by 2e-4, and the weights of 2^20 rows were.)
struct LongSum {
  float sum = 0.f, rest = 0.f;
  __device__ __forceinline__ void add(float x) {
    const float s = sum + x;
    rest += x - (s - sum);
    sum = s;
  }
  __device__ __forceinline__ void scale(float f) {
    sum *= f;
    rest *= f;
  }
  // (an infinity leaves no rest, but NaN)
  __device__ __forceinline__ float value() const { return rest == rest ? sum + rest : sum; }
};

// Three bf16 pieces of eight fp32 values.  The first is cut off, so that the largest finite values do not become infinite, the second is the rounding of what that leaves, and the
// third holds the rest exactly: 8 + 8 + 8 bits.  An infinity becomes NaN (infinity less infinity).  Five and a half instructions a value, which is what a kernel that splits many spends
// its time on (ten, with tests for infinities and the second piece widened from another conversion: one token of 12 128-wide heads over 447 slots 19.2 us for 17.1).  Of the nine products of two splits the three
// that are left out are 2^-23, 2^-23 and 2^-32 of theirs.
static __device__ __forceinline__ void split8_cut(f32x4 lo, f32x4 hi, bf16x8 (&out)[3]) {
  f32x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), first;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    first[i] = __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
    x[i] -= first[i];
  }
  out[0] = __builtin_convertvector(first, bf16x8);
  out[1] = __builtin_convertvector(x, bf16x8);
  const i32x4 second = __builtin_bit_cast(i32x4, out[1]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] -= __int_as_float(second[i] << 16);
    x[2 * i + 1] -= __int_as_float(second[i] & (int)0xffff0000);
  }
  out[2] = __builtin_convertvector(x, bf16x8);
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
