// Paged caches, gfx950: storing new tokens (normed and rotated on the way), and eviction of the slots that have had the least weight.
//
// Storing is one pass over the new rows, bound by memory, or by a few dependent loads where they are few.  Eviction finds, for each sequence and key head, the
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

static __device__ __forceinline__ Row8 times(const Row8 &x, float f) { return Row8{x.a * f, x.b * f}; }
static __device__ __forceinline__ Row8 times(const Row8 &x, const Row8 &w) { return Row8{x.a * w.a, x.b * w.b}; }
static __device__ __forceinline__ Row8 weight8(const float *w, int ca, int cb) {
  if (!w) return Row8{f32x4{1.f, 1.f, 1.f, 1.f}, f32x4{1.f, 1.f, 1.f, 1.f}};
  return Row8{*reinterpret_cast<const f32x4 *>(w + ca), *reinterpret_cast<const f32x4 *>(w + cb)};
}

template <int D, bool F32, bool NEXT, bool NORM>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
  constexpr int U = 4, TPR = D / 8;
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
  int row_blocks;             // copying: workgroups of a sequence and head
};

// Order of weights as that of unsigned integers: a NaN above all.
static __device__ __forceinline__ unsigned ordered(float x) {
  if (x != x) return ~0u;
  const unsigned u = __float_as_uint(x + 0.f);      // (-0 as 0)
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// The slots that stay, of one sequence and key head to a workgroup of 1024.  The weights of 65536 slots are held in registers (more are read anew in every pass), slot
// j0 + 1024 i + t in register i of thread t.  Three passes over 11, 11 and 10 bits of their order count how many have each digit, from the top, until the last weight that
// stays is known; its ties stay from the lowest slot on.
__global__ __launch_bounds__(1024) void evict_choose_kernel(EvictArgs a) {
  constexpr int PER = 64, BINS = 2048, CHUNK = PER * 1024;
  __shared__ unsigned hist[BINS];
  __shared__ unsigned wave_sums[16];
  __shared__ unsigned found[2];               // the digit, what is still to be taken of it
  __shared__ unsigned stays[PER][16], ties[PER][16];      // [register][wave]: how many; then how many ahead of them
  const Paged &p = a.p;
  const int bh = blockIdx.x, b = bh / p.Hkv, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int held = p.held(b);
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
  auto load = [&](int j0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (j0 + 1024 * i >= held) break;
      const int j = j0 + 1024 * i + threadIdx.x;
      u[i] = j < held ? ordered(x[j]) : 0;
    }
  };
  const bool once = held <= CHUNK;
  if (once) load(0);
  // the sum over the threads ahead of this one, and over all
  auto prefix_sum = [&](unsigned n, unsigned &total) {
    unsigned upto = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    if (lane == 63) wave_sums[w] = upto;
    __syncthreads();
    unsigned before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      before += i < w ? wave_sums[i] : 0;
      total += wave_sums[i];
    }
    __syncthreads();
    return before + upto - n;
  };
  unsigned prefix = 0, need = wanted;         // the leading digits of the last weight that stays, and how many stay of those that share them
  if (wanted > 0) {
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
      const unsigned above = pass == 0 ? 0 : ~0u << (shift + bits);      // digits that are known
      hist[2 * threadIdx.x] = hist[2 * threadIdx.x + 1] = 0;
      __syncthreads();
      for (int j0 = 0; j0 < held; j0 += CHUNK) {
        if (!once) load(j0);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (j0 + 1024 * i >= held) break;
          const int j = j0 + 1024 * i + threadIdx.x;
          const bool counts = j >= lo && j < hi && (u[i] & above) == prefix;
          const unsigned digit = (u[i] >> shift) & ((1u << bits) - 1);
          const uint64_t who = __ballot(counts);
          if (who == 0) continue;
          // (equal weights, of slots that nothing has looked at yet for instance, would queue up at one place)
          const int first = __ffsll((long long)who) - 1;
          if (__ballot(counts && digit == __builtin_amdgcn_readlane(digit, first)) == who) {
            if (lane == first) atomicAdd(&hist[digit], (unsigned)__popcll(who));
          } else if (counts) {
            atomicAdd(&hist[digit], 1u);
          }
        }
      }
      __syncthreads();
      // from the largest digit down: thread t has digits 2047 - 2 t and 2046 - 2 t
      const unsigned n0 = hist[BINS - 1 - 2 * threadIdx.x], n1 = hist[BINS - 2 - 2 * threadIdx.x];
      unsigned total;
      const unsigned before = prefix_sum(n0 + n1, total);
      if (before < need && need <= before + n0 + n1) {
        const bool second = need > before + n0;
        found[0] = BINS - 1 - 2 * threadIdx.x - second;
        found[1] = need - before - (second ? n0 : 0);
      }
      __syncthreads();
      prefix |= found[0] << shift;
      need = found[1];
    }
  }
  // slots that stay, in order: outside of the candidates, above the last weight, and the first `need` of those that equal it
  unsigned base = 0, tie_base = 0;
  for (int j0 = 0; j0 < held; j0 += CHUNK) {
    if (!once) load(j0);
    // 0: goes, 1: stays, 2: a tie
    auto kind = [&](int i) {
      const int j = j0 + 1024 * i + threadIdx.x;
      if (j >= held) return 0;
      if (j < lo || j >= hi) return 1;
      return wanted == 0 || u[i] < prefix ? 0 : u[i] > prefix ? 1 : 2;
    };
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      unsigned s = 0, t = 0;
      if (j0 + 1024 * i < held) {
        const int k = kind(i);
        s = __popcll(__ballot(k == 1));
        t = __popcll(__ballot(k == 2));
      }
      if (lane == 0) {
        stays[i][w] = s;
        ties[i][w] = t;
      }
    }
    __syncthreads();
    // entry t of the register-major list: ties ahead of it say how many of its own stay
    unsigned *all_stay = &stays[0][0], *all_ties = &ties[0][0], total_ties, total;
    const unsigned my_ties = all_ties[threadIdx.x], ties_before = tie_base + prefix_sum(my_ties, total_ties);
    const unsigned mine = all_stay[threadIdx.x] + min(ties_before < need ? need - ties_before : 0u, my_ties);
    const unsigned before = base + prefix_sum(mine, total);
    all_ties[threadIdx.x] = ties_before;
    all_stay[threadIdx.x] = before;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (j0 + 1024 * i >= held) break;
      const int k = kind(i);
      const uint64_t below = ((uint64_t)1 << lane) - 1, tied = __ballot(k == 2);
      const bool stay = k == 1 || (k == 2 && ties[i][w] + __popcll(tied & below) < need);
      const uint64_t all = __ballot(stay);
      if (stay) kept[stays[i][w] + __popcll(all & below)] = j0 + 1024 * i + threadIdx.x;
    }
    base += total;
    tie_base += total_ties;
  }
}

// Copies the rows and weights of the slots that stay, 64 of them to a workgroup, 16 bytes of a row to a thread.  The workgroups behind them clear the weights behind.
template <int ROW>            // bytes of a row
__global__ __launch_bounds__(256) void evict_copy_kernel(EvictArgs a, int esz) {
  constexpr int TPR = ROW / 16, RPP = 256 / TPR, U = RPP >= 16 ? 64 / RPP : 4;
  const Paged &p = a.p;
  const int bh = blockIdx.x / a.row_blocks, b = bh / p.Hkv, hk = bh % p.Hkv, i0 = (blockIdx.x % a.row_blocks) * 64, capacity = p.capacity();
  const int stay = min(p.held(b), a.keep);
  if (threadIdx.x < 64) {
    const int i = i0 + threadIdx.x;
    if (i < capacity) a.weights_out[(int64_t)bh * capacity + i] = i < stay ? a.weights[(int64_t)bh * capacity + a.kept[(int64_t)bh * a.keep + i]] : 0.f;
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
        const int id = p.page_of(b, slot), out = a.out_table[(int64_t)b * a.out_pages + (i >> p.page_log2)];
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
        *reinterpret_cast<f32x4 *>(a.k.p + (to[u] * a.k.sb + hk * a.k.sh + row * a.k.sn) * esz + c) = k[u];
        *reinterpret_cast<f32x4 *>(a.v.p + (to[u] * a.v.sb + hk * a.v.sh + row * a.v.sn) * esz + c) = v[u];
      }
    }
  }
}

template <int D, bool F32>
hipError_t launch_append(const AppendArgs &a, bool next, bool norm, hipStream_t st) {
  const unsigned rows = 256 / (D / 8), groups = (a.p.T + rows - 1) / rows, heads = a.Hq + 2 * a.p.Hkv;
  const dim3 grid(groups, groups < 512 ? std::min<unsigned>((heads + 3) / 4, (512 + groups - 1) / groups) : 1);
  if (next) { if (norm) paged_append_kernel<D, F32, true, true><<<grid, 256, 0, st>>>(a); else paged_append_kernel<D, F32, true, false><<<grid, 256, 0, st>>>(a); }
  else { if (norm) paged_append_kernel<D, F32, false, true><<<grid, 256, 0, st>>>(a); else paged_append_kernel<D, F32, false, false><<<grid, 256, 0, st>>>(a); }
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
  (void)p;
  (void)keep;
  return 0;
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
  if (slots > 0 && weights_out == weights) return HA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(out_table) | reinterpret_cast<uintptr_t>(len_out) | reinterpret_cast<uintptr_t>(kept) | reinterpret_cast<uintptr_t>(weights) |
       reinterpret_cast<uintptr_t>(weights_out)) & 3u)
    return HA_ERR_ALIGN;
  if ((st = check_workspace(workspace, workspace_bytes, hybrid_attn_paged_evict_workspace_bytes(p, keep))) != HA_OK) return st;
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
  evict_choose_kernel<<<p->B * p->H_kv, 1024, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return device_error(e);
  if (slots == 0) return HA_OK;
  const unsigned grid = (unsigned)(p->B * p->H_kv * row_blocks);
  const int esz = p->dtype == HA_F32 ? 4 : 2, row = p->d_head * esz;
  if (row == 128) evict_copy_kernel<128><<<grid, 256, 0, stream>>>(a, esz);
  else if (row == 256) evict_copy_kernel<256><<<grid, 256, 0, stream>>>(a, esz);
  else evict_copy_kernel<512><<<grid, 256, 0, stream>>>(a, esz);
  e = hipGetLastError();
  return e == hipSuccess ? HA_OK : device_error(e);
}
