// The weight that every slot of a paged cache gets from new tokens, gfx950.
//
//   w_j += sum over rows R that see slot j of exp(scale q_R . k_j - lse_R)
//
// A wave owns 32 slots at a time, S = Q K^T with the slot as the lane's column, so that a slot's sum over the rows is a lane's own (and its other half's).
//   few   32 rows at most: bound by reading the keys (188 MB in 32 us, 5.8 TB/s).  The rows stay in registers, the wave walks slots.
//   tile  more rows: an exponential for every row and slot next to 2 d operations of the matrix cores, which take about as long.  The keys stay in registers, the
//         four waves of a workgroup walk the rows, which they share in LDS.
#include "ha_paged.h"

#include <algorithm>

namespace ha {
namespace {

struct WeightArgs {
  Paged p;
  View q, k;
  const float *lse, *weights;
  float *out;
  float scale_log2e;
  int parts, few_parts;       // workgroups of a sequence and key head
  int few;                    // tile: sequences of 32 rows or fewer are another launch's
  int row_parts;              // tile: parts of the rows, whose sums are joined where there are several
  float *sums;                // [row_parts][B H_kv][slots]
  float inv_G;
};

// Row R of a sequence: its query, - lse log2 e (- infinity where it sees nothing or is none), and how many slots it sees.
struct WeightRow {
  int64_t query;              // in elements
  float shift;
  int see;
  __device__ __forceinline__ WeightRow(const WeightArgs &a, const NewRows &n, int held, int hk, int R) {
    const Paged &p = a.p;
    const int n_rows = n.n * p.G, Rc = min(R, n_rows - 1);
    const int i = (int)((Rc + 0.5f) * a.inv_G), h = hk * p.G + Rc - i * p.G;      // (Rc / G: the quotient is 0.5 / G from a whole number, and off by 2^-22 of itself, Rc < 2^20)
    const int64_t token = n.first + i;
    const float x = a.lse[token * p.H + h];
    query = h * a.q.sh + token * a.q.sn;
    shift = R < n_rows && x != -INFINITY ? -x * kLog2e : -INFINITY;
    see = p.causal ? min(held, held - n.all + i + 1) : held;
  }
};

static __device__ __forceinline__ void add_weight(const WeightArgs &a, int64_t at, float sum) { a.out[at] = (a.weights ? a.weights[at] : 0.f) + sum; }

// Sum over 32 rows of the weights of this lane's slot; shift and see of the rows in LDS.  ALL: every row sees the slot, and none that there is has a shift of - infinity.
template <bool ALL>
static __device__ __forceinline__ float sum_rows(const f32x16 &sc, const float *shift, const int *see, int slot, float c, int g) {
  float sum = 0.f;
#pragma unroll
  for (int y4 = 0; y4 < 4; ++y4) {
    const f32x4 t = *reinterpret_cast<const f32x4 *>(shift + 8 * y4 + 4 * g);
    const i32x4 s = ALL ? i32x4{} : *reinterpret_cast<const i32x4 *>(see + 8 * y4 + 4 * g);
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float e = fast_exp2(__builtin_fmaf(sc[4 * y4 + y], c, t[y]));
      sum += ALL || (slot < s[y] && t[y] != -INFINITY) ? e : 0.f;
    }
  }
  return sum;
}

template <int D, bool F32>
static constexpr int few_weight_bytes() { return F32 ? 16 : 4 * Tile<D>::bytes(32); }
template <int D, bool F32>
__device__ __forceinline__ void weights_of_few(const WeightArgs &a, unsigned block, char *lds, float *shift, int *see) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, NS = F32 ? 3 : 1, ESZ = F32 ? 4 : 2;
  const Paged &p = a.p;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int bh = block / a.few_parts, part = block % a.few_parts, b = bh / p.Hkv, hk = bh % p.Hkv, capacity = p.capacity();
  const NewRows n(p, b);
  const int held = p.held(b), n_rows = n.n * p.G;
  if (n_rows > 32) return;
  bf16x8 qf[KS][NS];
  if (n_rows > 0) {
    const WeightRow row(a, n, held, hk, r);
    const char *qp = a.q.p + (row.query + 8 * g) * ESZ;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (F32) split8_cut(*reinterpret_cast<const f32x4 *>(qp + 64 * ks), *reinterpret_cast<const f32x4 *>(qp + 64 * ks + 16), qf[ks]);
      else qf[ks][0] = *reinterpret_cast<const bf16x8 *>(qp + 32 * ks);
    }
    if (threadIdx.x < 32) {
      shift[r] = row.shift;
      see[r] = row.see;
    }
  }
  __syncthreads();
  // (the logits of a row that does not count may be NaN)
  const int first_sees = __any(r < n_rows && shift[r] == -INFINITY) ? 0 : p.causal ? min(held, held - n.all + 1) : held;
  char *mine = lds + w * T::bytes(32);
  const unsigned rows0 = F32 ? 0 : T::rows_base(mine, lane);
  const char *kbase = a.k.p + hk * a.k.sh * ESZ;
  for (int slot0 = (part * 4 + w) * 32; slot0 < capacity; slot0 += a.few_parts * 128) {
    const int slot = slot0 + r;
    float sum = 0.f;
    if (slot0 < held && n_rows > 0) {
      const int id0 = __builtin_amdgcn_readfirstlane(p.page_of(b, slot0)), id1 = p.page > 16 || slot0 + 16 >= capacity ? id0 : __builtin_amdgcn_readfirstlane(p.page_of(b, slot0 + 16));
      f32x16 sc;
#pragma unroll
      for (int x = 0; x < 16; ++x) sc[x] = 0.f;
      if constexpr (F32) {
        const int id = r < 16 ? id0 : id1;
        const bool there = id >= 0 && slot < held;
        const char *kp = kbase + ((there ? id * a.k.sb + (int64_t)(slot & (p.page - 1)) * a.k.sn : 0) + 8 * g) * 4;
        f32x4 x[KS][2];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int i = 0; i < 2; ++i) x[ks][i] = there ? *reinterpret_cast<const f32x4 *>(kp + 64 * ks + 16 * i) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          bf16x8 kf[3];
          split8_cut(x[ks][0], x[ks][1], kf);
          sc = mfma_split<3>(qf[ks], kf, sc);
        }
      } else {
        const int ksn = (int)a.k.sn * 2;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int id = i ? id1 : id0, at = slot0 + 16 * i, rows = id < 0 ? 0 : min(held - at, 16);
          request_rows<D, 16, 1>(rows_rsrc<D>(kbase + (max(id, 0) * a.k.sb + (int64_t)(at & (p.page - 1)) * a.k.sn) * 2, rows, ksn), ksn, mine + i * T::bytes(16), 0, lane);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc = mfma32(qf[ks][0], T::rows_at(rows0, 0, ks), sc);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // (the next slots may be asked for)
      }
      sum = slot0 + 32 <= first_sees ? sum_rows<true>(sc, shift, see, slot, a.scale_log2e, g) : sum_rows<false>(sc, shift, see, slot, a.scale_log2e, g);
      if ((r < 16 ? id0 : id1) < 0) sum = 0.f;
    }
    sum = xhalf_sum(sum);
    if (g == 0 && slot < capacity) add_weight(a, (int64_t)bh * capacity + slot, sum);
  }
}

// Rows are asked for two steps of 32 ahead.  Where the slots make few workgroups the rows are cut into parts, whose sums a second kernel adds up (1536 rows over 512 slots: 11 us for 43 uncut).
template <int D, bool F32>
static constexpr int tile_weight_bytes() { return 2 * (F32 ? 3 : 1) * Tile<D>::bytes(32); }
template <int D, bool F32>
__device__ __forceinline__ void weights_of_tiles(const WeightArgs &a, unsigned block, char *lds_, float (&shift)[2][32], int (&see)[2][32]) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, NS = F32 ? 3 : 1, ESZ = F32 ? 4 : 2, STAGE = T::bytes(32), PER = 32 * T::PIECES / 256;
  char *const lds[2] = {lds_, lds_ + NS * STAGE};
  const Paged &p = a.p;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int row_part = block % a.row_parts, item = block / a.row_parts;
  const int bh = item / a.parts, b = bh / p.Hkv, hk = bh % p.Hkv, first = (item % a.parts) * 128, slot0 = first + 32 * w, slot = slot0 + r, capacity = p.capacity();
  const NewRows n(p, b);
  const int held = p.held(b), n_rows = n.n * p.G, before = held - n.all;      // before: slots ahead of the first new token's
  if (a.few && n_rows <= 32) return;
  const int id = slot < held ? p.page_of(b, slot) : -1;
  LongSum total;
  // steps of rows that see the workgroup's first slot, this part's
  const int steps = (n_rows + 31) / 32, step0 = first >= held ? steps : p.causal ? max(first - before, 0) * p.G / 32 : 0, count = max(steps - step0, 0);
  int R0 = 32 * (step0 + count * row_part / a.row_parts);
  const int R_end = 32 * (step0 + count * (row_part + 1) / a.row_parts);
  if (R0 < R_end) {
    struct Ahead {
      Row8 x[PER];
      float shift;
      int see;
    };
    auto request = [&](Ahead &y, int R) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int at = threadIdx.x + 256 * i, piece = at % T::PIECES;
        const WeightRow row(a, n, held, hk, R + at / T::PIECES);
        y.x[i] = load_row8<F32, true>(a.q.p, row.query, 8 * piece, 8 * piece + 4);
      }
      if (threadIdx.x < 32) {
        const WeightRow row(a, n, held, hk, R + r);
        y.shift = row.shift;
        y.see = row.see;
      }
    };
    auto deposit = [&](const Ahead &y, int stage) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int at = threadIdx.x + 256 * i, line = at / T::PIECES, piece = at % T::PIECES;
        char *to = lds[stage] + line * T::PITCH + ((piece ^ T::swz(line)) << 4);
        if constexpr (F32) {
          bf16x8 z[3];
          split8_cut(y.x[i].a, y.x[i].b, z);
#pragma unroll
          for (int s = 0; s < 3; ++s) *reinterpret_cast<bf16x8 *>(to + s * STAGE) = z[s];
        } else {
          *reinterpret_cast<bf16x8 *>(to) = __builtin_convertvector(__builtin_shufflevector(y.x[i].a, y.x[i].b, 0, 1, 2, 3, 4, 5, 6, 7), bf16x8);
        }
      }
      if (threadIdx.x < 32) {
        shift[stage][r] = y.shift;
        see[stage][r] = y.see;
      }
    };
    Ahead even{}, odd{};        // rows of the steps with an even and an odd distance from the first
    request(even, R0);
    request(odd, min(R0 + 32, R_end - 32));
    const char *kp = a.k.p + (hk * a.k.sh + (id < 0 ? 0 : id * a.k.sb + (int64_t)(slot & (p.page - 1)) * a.k.sn) + 8 * g) * ESZ;
    bf16x8 kf[KS][NS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (F32) {
        f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
        if (id >= 0) {
          lo = *reinterpret_cast<const f32x4 *>(kp + 64 * ks);
          hi = *reinterpret_cast<const f32x4 *>(kp + 64 * ks + 16);
        }
        split8_cut(lo, hi, kf[ks]);
      } else {
        kf[ks][0] = bf16x8{};
        if (id >= 0) kf[ks][0] = *reinterpret_cast<const bf16x8 *>(kp + 32 * ks);
      }
    }
    deposit(even, 0);
    __syncthreads();
    auto step = [&](Ahead &now, const Ahead &next, int stage) {      // (now: has been deposited, takes the rows of two steps on)
      if (R0 + 64 < R_end) request(now, R0 + 64);
      const unsigned rows0 = T::rows_base(lds[stage], lane);
      f32x16 sc;
#pragma unroll
      for (int y = 0; y < 16; ++y) sc[y] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 qf[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) qf[s] = T::rows_at(rows0, 0, ks, s * STAGE);
        sc = mfma_split<NS>(qf, kf[ks], sc);
      }
      // (a row that sees all of the wave's slots: so do those behind it)
      const int first_sees = p.causal ? min(held, before + R0 / p.G + 1) : held;
      total.add(slot0 + 32 <= first_sees && R0 + 32 <= n_rows && !__any(shift[stage][r] == -INFINITY) ? sum_rows<true>(sc, shift[stage], see[stage], slot, a.scale_log2e, g)
                                                                                                  : sum_rows<false>(sc, shift[stage], see[stage], slot, a.scale_log2e, g));
      if (R0 + 32 < R_end) deposit(next, stage ^ 1);
      __syncthreads();
      R0 += 32;
    };
    while (true) {
      step(even, odd, 0);
      if (R0 >= R_end) break;
      step(odd, even, 1);
      if (R0 >= R_end) break;
    }
    if (id < 0) total = LongSum{};
  }
  const float sum = xhalf_sum(total.value());
  if (g == 0 && slot < capacity) {
    const int64_t at = (int64_t)bh * capacity + slot;
    if (a.row_parts > 1) a.sums[(int64_t)row_part * p.B * p.Hkv * capacity + at] = sum;
    else add_weight(a, at, sum);
  }
}
template <int D, bool F32>
__global__ __launch_bounds__(256) void paged_weights_few_kernel(WeightArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[few_weight_bytes<D, F32>()];
  __shared__ float shift[32];
  __shared__ int see[32];
  weights_of_few<D, F32>(a, blockIdx.x, lds, shift, see);
}
template <int D, bool F32>
__global__ __launch_bounds__(256, 2) void paged_weights_tile_kernel(WeightArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[tile_weight_bytes<D, F32>()];
  __shared__ float shift[2][32];
  __shared__ int see[2][32];
  weights_of_tiles<D, F32>(a, blockIdx.x, lds, shift, see);
}
// Chunks beside single tokens: both in one launch, the first `tile_blocks` workgroups for tiles (a prompt of 512 tokens beside 31 over 4096 slots, 32 heads on 8: 75 us for 102 in two).
template <int D, bool F32>
__global__ __launch_bounds__(256, 2) void paged_weights_both_kernel(WeightArgs a, unsigned tile_blocks) {
  constexpr int FEW = few_weight_bytes<D, F32>(), TILE = tile_weight_bytes<D, F32>();
  __shared__ __attribute__((aligned(1024))) char lds[FEW > TILE ? FEW : TILE];
  __shared__ float shift[2][32];
  __shared__ int see[2][32];
  if (blockIdx.x < tile_blocks) weights_of_tiles<D, F32>(a, blockIdx.x, lds, shift, see);
  else weights_of_few<D, F32>(a, blockIdx.x - tile_blocks, lds, shift[0], see[0]);
}
__global__ __launch_bounds__(256) void paged_weights_join_kernel(WeightArgs a) {
  const Paged &p = a.p;
  const int64_t capacity = p.capacity(), all = (int64_t)p.B * p.Hkv * capacity, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= all || (a.few && NewRows(p, (int)(at / capacity / p.Hkv)).n * p.G <= 32)) return;
  float sum = 0.f;
  for (int i = 0; i < a.row_parts; ++i) sum += a.sums[i * all + at];
  add_weight(a, at, sum);
}

struct WeightPlan {
  bool few, tile;
  int blocks, row_parts;      // of 128 slots, of the rows
  size_t total;
};
WeightPlan weight_plan(const ha_paged_problem &p) {
  WeightPlan f{};
  const int64_t slots = (int64_t)p.max_pages * p.page, groups = (int64_t)p.B * p.H_kv, rows = (int64_t)p.max_new * (p.H / p.H_kv);
  f.blocks = (int)((slots + 127) / 128);
  f.few = rows <= 32 || p.q_offset;
  f.tile = rows > 32;
  // Parts until there are two workgroups to a CU, each with four steps of 32 rows.
  f.row_parts = f.tile && slots > 0 ? (int)std::max<int64_t>(1, std::min<int64_t>(512 / (groups * f.blocks), (rows + 31) / 32 / 4)) : 1;
  if (f.row_parts > 1) f.total = round256((size_t)f.row_parts * groups * slots * 4);
  return f;
}

template <int D, bool F32>
hipError_t launch_weights(const WeightArgs &a, unsigned tile_blocks, unsigned few_blocks, hipStream_t st) {
  if (tile_blocks && few_blocks) paged_weights_both_kernel<D, F32><<<tile_blocks + few_blocks, 256, 0, st>>>(a, tile_blocks);
  else if (tile_blocks) paged_weights_tile_kernel<D, F32><<<tile_blocks, 256, 0, st>>>(a);
  else paged_weights_few_kernel<D, F32><<<few_blocks, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" size_t hybrid_attn_paged_weights_workspace_bytes(const ha_paged_problem *p) {
  if (check_paged(p) != HA_OK) return 0;
  return weight_plan(*p).total;
}

extern "C" ha_status hybrid_attn_paged_weights(const ha_paged_problem *p, const ha_view *q, const ha_view *k_pages, const float *lse, const float *weights, float *weights_out,
                                               void *workspace, size_t workspace_bytes, void *hip_stream) {
  ha_status st = check_paged(p);
  if (st != HA_OK) return st;
  WeightArgs a{};
  if ((st = check_packed(*p, q, p->H, false, a.q)) != HA_OK || (st = check_pool(*p, k_pages, false, a.k)) != HA_OK) return st;
  const int64_t slots = (int64_t)p->max_pages * p->page, groups = (int64_t)p->B * p->H_kv;
  const WeightPlan f = weight_plan(*p);
  if (groups * f.blocks > (1 << 23)) return HA_ERR_UNSUPPORTED;
  if ((p->T > 0 && !lse) || (slots > 0 && !weights_out)) return HA_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(weights) | reinterpret_cast<uintptr_t>(weights_out)) & 3u) return HA_ERR_ALIGN;
  if ((st = check_workspace(workspace, workspace_bytes, f.total)) != HA_OK) return st;
  if (slots == 0) return HA_OK;
  a.p = paged_of(*p);
  a.lse = lse;
  a.weights = weights;
  a.out = weights_out;
  a.scale_log2e = p->softmax_scale * kLog2e;
  a.inv_G = 1.f / (float)a.p.G;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool f32 = p->dtype == HA_F32;
  hipError_t e;
  a.parts = f.blocks;
  a.few = f.few;
  a.row_parts = f.row_parts;
  a.sums = static_cast<float *>(workspace);
  a.few_parts = (int)std::max<int64_t>(1, std::min<int64_t>(f.blocks, 2048 / groups));
  const unsigned tile_blocks = f.tile ? (unsigned)(groups * f.blocks * f.row_parts) : 0, few_blocks = f.few ? (unsigned)(groups * a.few_parts) : 0;
  if (p->d_head == 128) e = f32 ? launch_weights<128, true>(a, tile_blocks, few_blocks, stream) : launch_weights<128, false>(a, tile_blocks, few_blocks, stream);
  else e = f32 ? launch_weights<64, true>(a, tile_blocks, few_blocks, stream) : launch_weights<64, false>(a, tile_blocks, few_blocks, stream);
  if (e != hipSuccess) return device_error(e);
  if (f.row_parts > 1) {
    paged_weights_join_kernel<<<(unsigned)((groups * slots + 255) / 256), 256, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
  }
  return HA_OK;
}
