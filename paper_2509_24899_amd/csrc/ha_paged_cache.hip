// Paged caches, gfx950: storing new tokens (normed and rotated on the way), and eviction of the slots that have had the least weight.
//
// Storing is one pass over the new rows, bound by memory, or by a few dependent loads where they are few (one token 4.1 us, 1560 of 12 + 12 + 12 heads 10.7).  Eviction finds, for each sequence and key head, the
// weight of the last slot that stays, and lists the slots that stay in order; then a second kernel copies their rows, which is what takes long.
#include <cmath>

#include "ha_paged.h"

#include <algorithm>

namespace ha {
namespace {

// ---- storing ---------------------------------------------------------------------------------------------------------
struct AppendArgs {
  Paged p;
  int Hq;                     // query heads (0: no queries); the key heads follow, then those of the values
  View q, k, v, qo, ko, vo;
  const float *wq, *wk;
  Rotary rot;
  float eps;
};


// U: heads whose rows are asked for at once: four where there are many tokens, one where there are few (one token: 4.2 us for 5.6).
template <int D, bool F32, bool NEXT, bool NORM, int U>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
  constexpr int TPR = D / 8;
  const Paged &p = a.p;
  const int t = threadIdx.x % TPR, n = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, nc = min(n, p.T - 1);
  int lo = 0, hi = p.B;       // the last sequence that begins at this row or before it
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (p.offset(mid) <= nc) lo = mid;
    else hi = mid;
  }
  const NewRows rows(p, lo);
  const int i = nc - rows.first, slot = p.held(lo) - rows.all + i;
  const bool there = n < p.T && i >= 0 && i < rows.n;
  const int id = there && slot >= 0 ? p.page_of(lo, slot) : -1;
  int ca, cb;
  own_channels<NEXT>(t, a.rot.rot, ca, cb);
  f32x4 c, s;
  pair_angles(a.rot, a.rot.positions + (int64_t)nc * a.rot.n_axes, t, c, s);
  const int pairs = a.rot.rot / 2 - 4 * t, heads = a.Hq + 2 * p.Hkv;
  Row8 wq, wk;
  if constexpr (NORM) {
    wq = weight8(a.wq, ca, cb);
    wk = weight8(a.wk, ca, cb);
  }
  for (int h0 = blockIdx.y * U; h0 < heads; h0 += gridDim.y * U) {
    Row8 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int hh = min(h0 + u, heads - 1);
      const int64_t h = hh < a.Hq ? hh : hh < a.Hq + p.Hkv ? hh - a.Hq : hh - a.Hq - p.Hkv;
      const View &v = hh < a.Hq ? a.q : hh < a.Hq + p.Hkv ? a.k : a.v;
      x[u] = load_row8<F32, NEXT>(v.p, h * v.sh + nc * v.sn, ca, cb);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int hh = h0 + u;
      if (hh >= heads) break;
      Row8 y = x[u];
      if (hh < a.Hq + p.Hkv) {
        if constexpr (NORM) y = times(times(y, inverse_rms<D>(y, a.eps)), hh < a.Hq ? wq : wk);
        y = turn<NEXT>(y, c, s, pairs);
      }
      if (hh < a.Hq) {
        if (there) store_row8<F32, NEXT>(a.qo.p, hh * a.qo.sh + nc * a.qo.sn, ca, cb, y);
      } else if (id >= 0) {
        const bool key = hh < a.Hq + p.Hkv;
        const int64_t h = hh - a.Hq - (key ? 0 : p.Hkv);
        const View &v = key ? a.ko : a.vo;
        store_row8<F32, NEXT>(v.p, id * v.sb + h * v.sh + (slot & (p.page - 1)) * v.sn, ca, cb, y);
      }
    }
  }
}

// ---- eviction --------------------------------------------------------------------------------------------------------
struct EvictArgs {
  Paged p;
  View k, v;
  const float *weights;
  const int32_t *out_table;
  int out_pages, keep, first, last;
  int32_t *len_out, *kept;
  float *weights_out;
  int row_blocks, chunks;     // workgroups of a sequence and head: copying, choosing
  unsigned *hist, *counts, *last_weight;      // [B H_kv][3][kBins], [B H_kv][chunks][2], [B H_kv][2]
};

// Order of weights as that of unsigned integers: a NaN above all.
static __device__ __forceinline__ unsigned ordered(float x) {
  if (x != x) return ~0u;
  const unsigned u = __float_as_uint(x + 0.f);      // (-0 as 0)
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// The order of the last weight that stays is found eleven, eleven and ten bits at a time: how many of the candidates have each digit, counted from the top.
constexpr int kBins = 2048;
static __device__ __forceinline__ int shift_of(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
static __device__ __forceinline__ unsigned digit_of(unsigned u, int pass) { return (u >> shift_of(pass)) & (pass == 2 ? 1023 : 2047); }
static __device__ __forceinline__ unsigned known_bits(int pass) { return pass == 0 ? 0 : ~0u << (pass == 1 ? 21 : 10); }      // ahead of a pass

// The sum over the threads ahead of this one of a workgroup, and over all; `sums` holds one number for each wave.
template <int THREADS>
static __device__ __forceinline__ unsigned prefix_sum(unsigned n, unsigned *sums, unsigned &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const unsigned upto = (unsigned)sum_upto((int)n);
  __syncthreads();
  if (lane == 63) sums[w] = upto;
  __syncthreads();
  unsigned before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) {
    before += i < w ? sums[i] : 0;
    total += sums[i];
  }
  return before + upto - n;
}
// The digit at which the count from the top reaches `need`, and how many are still needed of it.  All threads, `found` and `sums` in LDS.
template <int THREADS>
static __device__ __forceinline__ void find_digit(const unsigned *hist, int pass, unsigned &prefix, unsigned &need, unsigned *found, unsigned *sums) {
  constexpr int PER = kBins / THREADS;
  unsigned n[PER], mine = 0, total;
#pragma unroll
  for (int i = 0; i < PER; ++i) mine += n[i] = hist[kBins - 1 - (PER * threadIdx.x + i)];
  unsigned above = prefix_sum<THREADS>(mine, sums, total);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (above < need && need <= above + n[i]) {
      found[0] = kBins - 1 - (PER * threadIdx.x + i);
      found[1] = need - above;
    }
    above += n[i];
  }
  __syncthreads();
  prefix |= found[0] << shift_of(pass);
  need = found[1];
  __syncthreads();
}
// Counts a digit.  (Equal weights, of slots that nothing has looked at yet for instance, would queue up at one place.)
static __device__ __forceinline__ void count_digit(unsigned *hist, bool counts, unsigned digit) {
  const uint64_t who = __ballot(counts);
  if (who == 0) return;
  const int first = __ffsll((long long)who) - 1;
  if (__ballot(counts && digit == (unsigned)__builtin_amdgcn_readlane((int)digit, first)) == who) {
    if ((int)(threadIdx.x & 63) == first) atomicAdd(&hist[digit], (unsigned)__popcll(who));
  } else if (counts) {
    atomicAdd(&hist[digit], 1u);
  }
}

// Caches of 8192 slots at most: one sequence and key head to a workgroup of 1024, which holds its weights in registers, slot 1024 i + t in register i of thread t.
__global__ __launch_bounds__(1024) void evict_choose_kernel(EvictArgs a) {
  constexpr int PER = 8;
  __shared__ unsigned hist[kBins], sums[16], found[2], stays[PER * 16], ties[PER * 16];      // [register][wave]: how many; then how many ahead of them
  const Paged &p = a.p;
  const int bh = blockIdx.x, b = bh / p.Hkv, lane = threadIdx.x & 63, w = threadIdx.x >> 6, held = p.held(b);
  const float *x = a.weights + (int64_t)bh * p.capacity();
  int32_t *kept = a.kept + (int64_t)bh * a.keep;
  if (bh % p.Hkv == 0 && threadIdx.x == 0) a.len_out[b] = min(held, a.keep);
  for (int j = held + threadIdx.x; j < a.keep; j += 1024) kept[j] = -1;
  if (held <= a.keep) {
    for (int j = threadIdx.x; j < held; j += 1024) kept[j] = j;
    return;
  }
  const int lo = a.first, hi = held - a.last, wanted = a.keep - a.first - a.last;      // candidates lo .. hi - 1, how many of them stay
  unsigned u[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) u[i] = 1024 * i + (int)threadIdx.x < held ? ordered(x[1024 * i + threadIdx.x]) : 0;
  unsigned prefix = 0, need = wanted;         // the leading digits of the last weight that stays, and how many stay of those that share them
  for (int pass = 0; pass < 3 && wanted > 0; ++pass) {
    hist[2 * threadIdx.x] = hist[2 * threadIdx.x + 1] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int j = 1024 * i + threadIdx.x;
      if (1024 * i < held) count_digit(hist, j >= lo && j < hi && (u[i] & known_bits(pass)) == prefix, digit_of(u[i], pass));
    }
    __syncthreads();
    find_digit<1024>(hist, pass, prefix, need, found, sums);
  }
  // slots that stay, in order: outside of the candidates, above the last weight, and the first `need` of those that equal it
  auto kind = [&](int i) {                    // 0: goes, 1: stays, 2: a tie
    const int j = 1024 * i + threadIdx.x;
    return j >= held ? 0 : j < lo || j >= hi ? 1 : wanted == 0 || u[i] < prefix ? 0 : u[i] > prefix ? 1 : 2;
  };
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = kind(i);
    const unsigned s = __popcll(__ballot(k == 1)), t = __popcll(__ballot(k == 2));
    if (lane == 0) {
      stays[16 * i + w] = s;
      ties[16 * i + w] = t;
    }
  }
  __syncthreads();
  const bool entry = threadIdx.x < PER * 16;
  unsigned total;
  const unsigned my_ties = entry ? ties[threadIdx.x] : 0, ties_before = prefix_sum<1024>(my_ties, sums, total);
  const unsigned mine = entry ? stays[threadIdx.x] + min(ties_before < need ? need - ties_before : 0u, my_ties) : 0, before = prefix_sum<1024>(mine, sums, total);
  if (entry) {
    ties[threadIdx.x] = ties_before;
    stays[threadIdx.x] = before;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = kind(i);
    const uint64_t below = ((uint64_t)1 << lane) - 1, tied = __ballot(k == 2);
    const bool stay = k == 1 || (k == 2 && ties[16 * i + w] + __popcll(tied & below) < need);
    const uint64_t all = __ballot(stay);
    const unsigned to = stays[16 * i + w] + __popcll(all & below);
    if (stay && to < (unsigned)a.keep) kept[to] = 1024 * i + threadIdx.x;
  }
}

// Longer caches: 2048 slots to a workgroup, a launch for every step.  The counts of all slots of a sequence and key head meet in the workspace.  (Four sequences of up to 60000 slots, 4 heads:
// 36 us in six launches; one workgroup to a sequence and head 129.)
constexpr int kChunk = 2048;
__global__ __launch_bounds__(256) void evict_clear_kernel(unsigned *hist, int n) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) hist[i] = 0;
}
// A workgroup's slots: of thread t those from first + 8 t on.
struct Chunk {
  int bh, chunk, b, held, first, lo, hi, wanted;
  bool all;
  unsigned u[8];
  __device__ __forceinline__ Chunk(const EvictArgs &a) {
    const Paged &p = a.p;
    bh = blockIdx.x / a.chunks;
    chunk = blockIdx.x % a.chunks;
    b = bh / p.Hkv;
    held = p.held(b);
    first = chunk * kChunk + 8 * threadIdx.x;
    lo = a.first;
    hi = held - a.last;
    wanted = a.keep - a.first - a.last;
    all = held <= a.keep;
  }
  __device__ __forceinline__ void load(const EvictArgs &a) {
    const float *x = a.weights + (int64_t)bh * a.p.capacity() + first;
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = first + i < held ? ordered(x[i]) : 0;
  }
  __device__ __forceinline__ bool candidate(int i) const { return first + i >= lo && first + i < hi; }
  // 0: goes, 1: stays, 2: a tie
  __device__ __forceinline__ int kind(int i, unsigned prefix) const {
    return first + i >= held ? 0 : all || !candidate(i) ? 1 : wanted == 0 || u[i] < prefix ? 0 : u[i] > prefix ? 1 : 2;
  }
};
__global__ __launch_bounds__(256) void evict_count_kernel(EvictArgs a, int pass) {
  __shared__ unsigned hist[kBins], sums[4], found[2];
  Chunk c(a);
  if (c.all || c.wanted == 0 || c.chunk * kChunk >= c.hi || (c.chunk + 1) * kChunk <= c.lo) return;
  unsigned prefix = 0, need = c.wanted;
  c.load(a);
  for (int q = 0; q < pass; ++q) find_digit<256>(a.hist + ((int64_t)c.bh * 3 + q) * kBins, q, prefix, need, found, sums);
#pragma unroll
  for (int i = 0; i < kBins / 256; ++i) hist[threadIdx.x + 256 * i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) count_digit(hist, c.candidate(i) && (c.u[i] & known_bits(pass)) == prefix, digit_of(c.u[i], pass));
  __syncthreads();
  unsigned *to = a.hist + ((int64_t)c.bh * 3 + pass) * kBins;
#pragma unroll
  for (int i = 0; i < kBins / 256; ++i) {
    const unsigned n = hist[threadIdx.x + 256 * i];
    if (n) atomicAdd(&to[threadIdx.x + 256 * i], n);
  }
}
// LIST = false: how many slots of the chunk stay and how many are ties, and the last weight that stays.  LIST = true: the slots that stay.
template <bool LIST>
__global__ __launch_bounds__(256) void evict_list_kernel(EvictArgs a) {
  __shared__ unsigned sums[4], found[2];
  Chunk c(a);
  int32_t *kept = a.kept + (int64_t)c.bh * a.keep;
  unsigned *counts = a.counts + (int64_t)c.bh * a.chunks * 2, *last = a.last_weight + (int64_t)c.bh * 2, prefix = 0, need = c.wanted, total;
  c.load(a);
  if constexpr (LIST) {
    prefix = last[0];
    need = last[1];
  } else if (!c.all && c.wanted > 0) {
    for (int q = 0; q < 3; ++q) find_digit<256>(a.hist + ((int64_t)c.bh * 3 + q) * kBins, q, prefix, need, found, sums);
  }
  unsigned n_stay = 0, n_tie = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int k = c.kind(i, prefix);
    n_stay += k == 1;
    n_tie += k == 2;
  }
  const unsigned ties_here = prefix_sum<256>(n_tie, sums, total), all_ties = total, stays_here = prefix_sum<256>(n_stay, sums, total), all_stays = total;
  if constexpr (!LIST) {
    if (threadIdx.x == 0) {
      counts[2 * c.chunk] = all_stays;
      counts[2 * c.chunk + 1] = all_ties;
      if (c.chunk == 0) {
        last[0] = prefix;
        last[1] = need;
        if (c.bh % a.p.Hkv == 0) a.len_out[c.b] = min(c.held, a.keep);
      }
    }
  } else {
    // of the chunks ahead
    unsigned stays = 0, ties = 0;
    for (int i = threadIdx.x; i < c.chunk; i += 256) {
      stays += counts[2 * i];
      ties += counts[2 * i + 1];
    }
    prefix_sum<256>(ties, sums, total);
    unsigned tie = total + ties_here;
    prefix_sum<256>(stays, sums, total);
    unsigned at = total + stays_here + min(tie, need);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = c.kind(i, prefix);
      if (k == 1 || (k == 2 && tie < need)) {
        if (at < (unsigned)a.keep) kept[at] = c.first + i;      // (always, unless the weights changed from one launch to the next)
        ++at;
      }
      tie += k == 2;
    }
    // (all chunks share what is behind the last slot that stays)
    for (int j = c.held + c.chunk * 256 + threadIdx.x; j < a.keep; j += a.chunks * 256) kept[j] = -1;
  }
}

// Copies the rows and weights of the slots that stay, 64 of them to a workgroup, 16 bytes of a row to a thread (668 MB in 134 us, 5.0 TB/s).  The workgroups behind them clear the weights behind.
template <int ROW, bool ONCE>      // bytes of a row
__global__ __launch_bounds__(256) void evict_copy_kernel(EvictArgs a, int esz) {
  constexpr int TPR = ROW / 16, RPP = 256 / TPR, U = RPP >= 16 ? 64 / RPP : 4;
  const Paged &p = a.p;
  const int bh = blockIdx.x / a.row_blocks, b = bh / p.Hkv, hk = bh % p.Hkv, i0 = (blockIdx.x % a.row_blocks) * 64, capacity = p.capacity();
  const int stay = min(p.held(b), a.keep);
  if (threadIdx.x < 64) {
    const int i = i0 + threadIdx.x;
    if (i < capacity) a.weights_out[(int64_t)bh * capacity + i] = i < stay ? a.weights[(int64_t)bh * capacity + min(max(a.kept[(int64_t)bh * a.keep + i], 0), capacity - 1)] : 0.f;
  }
  if (i0 >= stay) return;
  const int c = threadIdx.x % TPR * 16;
#pragma unroll 1
  for (int i1 = i0 + threadIdx.x / TPR; i1 < min(i0 + 64, stay); i1 += U * RPP) {
    f32x4 k[U], v[U];
    int to[U];                // page that the row goes to, or -1
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i1 + u * RPP;
      to[u] = -1;
      k[u] = v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (i < stay) {
        const int slot = a.kept[(int64_t)bh * a.keep + i];
        const int id = (unsigned)slot < (unsigned)capacity ? p.page_of(b, slot) : -1, out = a.out_table[(int64_t)b * a.out_pages + (i >> p.page_log2)];
        if ((unsigned)out < (unsigned)p.n_pages) to[u] = out;
        if (id >= 0) {
          const int64_t row = slot & (p.page - 1);
          k[u] = *reinterpret_cast<const f32x4 *>(a.k.p + (id * a.k.sb + hk * a.k.sh + row * a.k.sn) * esz + c);
          v[u] = *reinterpret_cast<const f32x4 *>(a.v.p + (id * a.v.sb + hk * a.v.sh + row * a.v.sn) * esz + c);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = (i1 + u * RPP) & (p.page - 1);
      if (to[u] >= 0) {
        store_as<ONCE>(a.k.p + (to[u] * a.k.sb + hk * a.k.sh + row * a.k.sn) * esz + c, k[u]);
        store_as<ONCE>(a.v.p + (to[u] * a.v.sb + hk * a.v.sh + row * a.v.sn) * esz + c, v[u]);
      }
    }
  }
}

template <int D, bool F32, int U>
hipError_t launch_append(const AppendArgs &a, dim3 grid, bool next, bool norm, hipStream_t st) {
  if (next) { if (norm) paged_append_kernel<D, F32, true, true, U><<<grid, 256, 0, st>>>(a); else paged_append_kernel<D, F32, true, false, U><<<grid, 256, 0, st>>>(a); }
  else { if (norm) paged_append_kernel<D, F32, false, true, U><<<grid, 256, 0, st>>>(a); else paged_append_kernel<D, F32, false, false, U><<<grid, 256, 0, st>>>(a); }
  return hipGetLastError();
}
template <int D, bool F32>
hipError_t launch_append(const AppendArgs &a, bool next, bool norm, hipStream_t st) {
  const unsigned rows = 256 / (D / 8), groups = (a.p.T + rows - 1) / rows, heads = a.Hq + 2 * a.p.Hkv;
  if (groups >= 512) return launch_append<D, F32, 4>(a, dim3(groups), next, norm, st);
  const unsigned each = groups >= 64 ? 4 : 1;
  const dim3 grid(groups, std::min((heads + each - 1) / each, (1024 + groups - 1) / groups));
  return each == 4 ? launch_append<D, F32, 4>(a, grid, next, norm, st) : launch_append<D, F32, 1>(a, grid, next, norm, st);
}

// Whether two lists of n numbers of 32 bits share memory.
bool overlap(const void *a, const void *b, int64_t n) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return (x > y ? x - y : y - x) < (uintptr_t)n * 4;
}

// One workgroup chooses of 8192 slots at most; more are counted by many, in six launches.
struct EvictPlan {
  int chunks;                 // 0: one workgroup
  size_t off_counts, off_last, total;
};
EvictPlan evict_plan(const ha_paged_problem &p) {
  EvictPlan f{};
  const int64_t slots = (int64_t)p.max_pages * p.page, groups = (int64_t)p.B * p.H_kv;
  if (slots <= 8192) return f;
  f.chunks = (int)((slots + kChunk - 1) / kChunk);
  f.off_counts = round256((size_t)groups * 3 * kBins * 4);
  f.off_last = f.off_counts + round256((size_t)groups * f.chunks * 8);
  f.total = f.off_last + round256((size_t)groups * 8);
  return f;
}
hipError_t launch_choice(EvictArgs a, const EvictPlan &f, char *ws, hipStream_t st) {
  const unsigned groups = (unsigned)a.p.B * a.p.Hkv;
  if (f.chunks == 0) {
    evict_choose_kernel<<<groups, 1024, 0, st>>>(a);
    return hipGetLastError();
  }
  a.chunks = f.chunks;
  a.hist = reinterpret_cast<unsigned *>(ws);
  a.counts = reinterpret_cast<unsigned *>(ws + f.off_counts);
  a.last_weight = reinterpret_cast<unsigned *>(ws + f.off_last);
  const unsigned grid = groups * f.chunks;
  hipError_t e;
  evict_clear_kernel<<<std::min(groups * 3 * kBins / 256, 1024u), 256, 0, st>>>(a.hist, (int)(groups * 3 * kBins));
  if ((e = hipGetLastError()) != hipSuccess) return e;
  for (int pass = 0; pass < 3; ++pass) {
    evict_count_kernel<<<grid, 256, 0, st>>>(a, pass);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  evict_list_kernel<false><<<grid, 256, 0, st>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  evict_list_kernel<true><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" ha_status hybrid_attn_paged_append(const ha_paged_problem *p, const ha_rotary *r, int32_t norm, float eps, const ha_view *q, const ha_view *k, const ha_view *v,
                                              const float *w_q, const float *w_k, const ha_view *k_pages, const ha_view *v_pages, const ha_view *q_out, void *hip_stream) {
  ha_status st = check_paged(p);
  if (st != HA_OK) return st;
  AppendArgs a{};
  if (norm != 0 && norm != 1) return HA_ERR_SHAPE;
  if (norm && (!(eps >= 0.f) || !std::isfinite(eps))) return HA_ERR_SHAPE;
  if (r && (st = check_rotary(r, p->d_head, p->T, true, a.rot)) != HA_OK) return st;
  if ((q == nullptr) != (q_out == nullptr)) return HA_ERR_NULL;
  if (q && ((st = check_packed(*p, q, p->H, false, a.q)) != HA_OK || (st = check_packed(*p, q_out, p->H, true, a.qo)) != HA_OK)) return st;
  if ((st = check_packed(*p, k, p->H_kv, false, a.k)) != HA_OK || (st = check_packed(*p, v, p->H_kv, false, a.v)) != HA_OK ||
      (st = check_pool(*p, k_pages, true, a.ko)) != HA_OK || (st = check_pool(*p, v_pages, true, a.vo)) != HA_OK)
    return st;
  if (norm && ((reinterpret_cast<uintptr_t>(w_q) | reinterpret_cast<uintptr_t>(w_k)) & 15u)) return HA_ERR_ALIGN;
  if (p->T == 0) return HA_OK;
  a.p = paged_of(*p);
  a.Hq = q ? p->H : 0;
  a.wq = w_q;
  a.wk = w_k;
  a.eps = eps;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool f32 = p->dtype == HA_F32, next = !r || r->interleaved;
  const hipError_t e = p->d_head == 128 ? (f32 ? launch_append<128, true>(a, next, norm, stream) : launch_append<128, false>(a, next, norm, stream))
                                        : (f32 ? launch_append<64, true>(a, next, norm, stream) : launch_append<64, false>(a, next, norm, stream));
  return e == hipSuccess ? HA_OK : device_error(e);
}

extern "C" size_t hybrid_attn_paged_evict_workspace_bytes(const ha_paged_problem *p, int32_t keep) {
  if (check_paged(p) != HA_OK || keep < 1) return 0;
  return evict_plan(*p).total;
}

extern "C" ha_status hybrid_attn_paged_evict(const ha_paged_problem *p, int32_t keep, int32_t keep_first, int32_t keep_last, const float *weights, const int32_t *out_table,
                                             int32_t out_pages, const ha_view *k_pages, const ha_view *v_pages, int32_t *len_out, float *weights_out, int32_t *kept,
                                             void *workspace, size_t workspace_bytes, void *hip_stream) {
  ha_status st = check_paged(p);
  if (st != HA_OK) return st;
  EvictArgs a{};
  if (keep < 1 || keep_first < 0 || keep_last < 0 || (int64_t)keep_first + keep_last > keep || out_pages < 0) return HA_ERR_SHAPE;
  const int64_t slots = (int64_t)p->max_pages * p->page, row_blocks = (slots + 63) / 64;      // (of all slots: the weights behind those that stay are cleared)
  if ((int64_t)out_pages * p->page < keep) return HA_ERR_SHAPE;
  if (keep > (1 << 30) || (int64_t)p->B * p->H_kv * row_blocks > (1 << 23)) return HA_ERR_UNSUPPORTED;
  if ((st = check_pool(*p, k_pages, true, a.k)) != HA_OK || (st = check_pool(*p, v_pages, true, a.v)) != HA_OK) return st;
  if (!out_table || !len_out || !kept || (slots > 0 && (!weights || !weights_out))) return HA_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(out_table) | reinterpret_cast<uintptr_t>(len_out) | reinterpret_cast<uintptr_t>(kept) | reinterpret_cast<uintptr_t>(weights) |
       reinterpret_cast<uintptr_t>(weights_out)) & 3u)
    return HA_ERR_ALIGN;
  // (the choice and the copy read lengths and weights after the first of them has been written)
  if (overlap(len_out, p->key_len, p->B) || overlap(weights_out, weights, (int64_t)p->B * p->H_kv * slots)) return HA_ERR_SHAPE;
  const EvictPlan f = evict_plan(*p);
  if ((st = check_workspace(workspace, workspace_bytes, f.total)) != HA_OK) return st;
  a.p = paged_of(*p);
  a.weights = weights;
  a.out_table = out_table;
  a.out_pages = out_pages;
  a.keep = keep;
  a.first = keep_first;
  a.last = keep_last;
  a.len_out = len_out;
  a.kept = kept;
  a.weights_out = weights_out;
  a.row_blocks = (int)row_blocks;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  hipError_t e = launch_choice(a, f, static_cast<char *>(workspace), stream);
  if (e != hipSuccess) return device_error(e);
  if (slots == 0) return HA_OK;
  const unsigned grid = (unsigned)(p->B * p->H_kv * row_blocks);
  const int esz = p->dtype == HA_F32 ? 4 : 2, row = p->d_head * esz;
  const bool once = stream_once((int64_t)4 * p->B * p->H_kv * std::min<int64_t>(keep, slots) * row);
  if (row == 128) { if (once) evict_copy_kernel<128, true><<<grid, 256, 0, stream>>>(a, esz); else evict_copy_kernel<128, false><<<grid, 256, 0, stream>>>(a, esz); }
  else if (row == 256) { if (once) evict_copy_kernel<256, true><<<grid, 256, 0, stream>>>(a, esz); else evict_copy_kernel<256, false><<<grid, 256, 0, stream>>>(a, esz); }
  else { if (once) evict_copy_kernel<512, true><<<grid, 256, 0, stream>>>(a, esz); else evict_copy_kernel<512, false><<<grid, 256, 0, stream>>>(a, esz); }
  e = hipGetLastError();
  return e == hipSuccess ? HA_OK : device_error(e);
}
