// Block-sparse attention, gfx950: the gradients.
//
//   P = exp(scale S - lse),  dP = dO V^T,  dS = P (dP - delta) scale,  delta_i = dO_i . O_i,
//   dQ = dS K,   dK = dS^T Q,   dV = P^T dO      (the last two summed over the query heads of a key head)
//
// Two passes, neither with an atomic, so that the sums have one order: dQ by tiles of queries along their lists, as the forward walks them, and dK, dV by
// key blocks along the tiles that chose them.  S and dP are formed in both (seven products for five; writing dQ's terms from the second pass
// instead would be fp32 atomics, or T x n_select partial tiles in memory).  The inverse lists are built on the way: tiles in rising order for every key
// block, by counting in chunks of tiles.  Popular blocks (a first block that every tile keeps) would leave one workgroup with thousands of
// tiles, so a list is cut into parts whose sums a last kernel joins in order.
#include <climits>

#include "ha_sparse.h"

#include <algorithm>

namespace ha {
namespace {

constexpr int kPart = 64;        // tiles of an inverse list that one workgroup takes, at most
constexpr int kChunk = 8;        // tiles counted together while the inverse lists are built (training at 480p 3.66 ms with 8 and 16, 3.69 with 4; 4096 causal tokens 180, 182 and 183 us)

struct GradArgs {
  Sparse s;
  View q, k, v, dout, dq, dk, dv;      // inputs bf16 (fp32 tensors: the first pieces; the next stand piece_* elements behind)
  int64_t piece_q, piece_k;
  const int32_t *blocks;
  float *stat;                         // [B H][T qb / 32][2][32]: -lse / scale (-infinity for rows that take no part), -delta
  int32_t *hist;                       // [B Hkv][n_chunks][Tk]
  int32_t *first, *item0, *slot0;      // [B Hkv][Tk + 1]: a block's first place in inv, its first item and its first slot
  int32_t *inv;                        // [B Hkv][T sel] tiles
  int2 *work;                          // items in the order of their launch: {block of all heads' blocks, part}
  int32_t *n_work;                     // how many
  float *part;                         // [B Hkv][max_slots][dk | dv][kb][D]
  int n_chunks, max_items, max_slots, part_tiles;
  float scale, scale_log2e;
  unsigned items, share;
};

// ---- row statistics ----------------------------------------------------------------------------------------------------
// Bound by memory: 41 us for out and its gradient at 12 heads of 32760 x 128, 4.9 TB/s.
template <int D, bool F32>
__global__ __launch_bounds__(256) void sparse_delta_kernel(Sparse s, View out, View dout, const float *lse, float inv_scale, float *stat) {
  constexpr int TPR = D / 8, RPB = 256 / TPR;
  const int rows = s.T * s.qb;
  const int64_t at = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (at >= (int64_t)s.B * s.H * rows) return;
  const int bh = (int)(at / rows), n = (int)(at % rows), b = bh / s.H, h = bh % s.H, c = 8 * (threadIdx.x % TPR);
  float sum = 0.f;
  if (n < s.Nq) {
    const int64_t io = b * out.sb + h * out.sh + n * out.sn + c, id = b * dout.sb + h * dout.sh + n * dout.sn + c;
    if constexpr (F32) {
      const f32x4 *x = reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(out.p) + io), *y = reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(dout.p) + id);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += x[i][j] * y[i][j];
    } else {
      const bf16x8 x = *reinterpret_cast<const bf16x8 *>(out.p + io * 2), y = *reinterpret_cast<const bf16x8 *>(dout.p + id * 2);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += static_cast<float>(x[i]) * static_cast<float>(y[i]);
    }
  }
#pragma unroll
  for (int i = TPR / 2; i > 0; i >>= 1) sum += __shfl_xor(sum, i);
  if (c == 0) {
    const float l = n < s.Nq ? lse[(int64_t)bh * s.Nq + n] : -INFINITY;
    float *to = stat + (at >> 5) * 64 + (at & 31);
    to[0] = l == -INFINITY ? -INFINITY : -l * inv_scale;
    to[32] = l == -INFINITY ? 0.f : -sum;
  }
}

// ---- inverse lists -----------------------------------------------------------------------------------------------------
// Four small launches, 25 us of 3.6 ms at 480p (256 tiles of 64 entries, 512 blocks, 12 heads), 12 us for the smallest problems.  (Counted in memory instead of
// LDS, the first alone took 34.)
// hist[chunk][j]: how many times the chunk's tiles list block j.
constexpr int kCounted = 2048;   // blocks counted in LDS at a time
__global__ __launch_bounds__(256) void inverse_count_kernel(GradArgs a) {
  const Sparse &s = a.s;
  const int chunk = blockIdx.x, bh = blockIdx.y;
  int32_t *h = a.hist + ((int64_t)bh * a.n_chunks + chunk) * s.Tk;
  const int lo = chunk * kChunk * s.sel, hi = min((chunk + 1) * kChunk, s.T) * s.sel;
  const int32_t *list = a.blocks + (int64_t)bh * s.T * s.sel;
  __shared__ int n[kCounted];
  for (int j0 = 0; j0 < s.Tk; j0 += kCounted) {
    for (int j = threadIdx.x; j < kCounted; j += 256) n[j] = 0;
    __syncthreads();
    for (int i = lo + threadIdx.x; i < hi; i += 256) {
      const int j = list[i];
      if ((unsigned)j < (unsigned)s.Tk && (unsigned)(j - j0) < (unsigned)kCounted) atomicAdd(n + j - j0, 1);
    }
    __syncthreads();
    for (int j = threadIdx.x; j < min(kCounted, s.Tk - j0); j += 256) h[j0 + j] = n[j];
    __syncthreads();
  }
}

__device__ __forceinline__ int3 add3(int3 a, int3 b) { return int3{a.x + b.x, a.y + b.y, a.z + b.z}; }

// Per head: every block's first place, first item and first slot; hist becomes the chunk's first place within the block's list.
__global__ __launch_bounds__(1024) void inverse_scan_kernel(GradArgs a) {
  const Sparse &s = a.s;
  __shared__ int3 wave_sum[16];
  const int bh = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int32_t *h = a.hist + (int64_t)bh * a.n_chunks * s.Tk;
  int32_t *first = a.first + (int64_t)bh * (s.Tk + 1), *item0 = a.item0 + (int64_t)bh * (s.Tk + 1), *slot0 = a.slot0 + (int64_t)bh * (s.Tk + 1);
  int3 base = {0, 0, 0};
  for (int j0 = 0; j0 < s.Tk; j0 += 1024) {
    const int j = j0 + threadIdx.x;
    int n = 0;
    if (j < s.Tk)
      for (int c = 0; c < a.n_chunks; c += 8) {
        int x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c + i < a.n_chunks ? h[(int64_t)(c + i) * s.Tk + j] : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (c + i < a.n_chunks) h[(int64_t)(c + i) * s.Tk + j] = n;
          n += x[i];
        }
      }
    const int parts = j < s.Tk ? max(1, (n + a.part_tiles - 1) / a.part_tiles) : 0;
    const int3 mine = {n, parts, parts > 1 ? parts : 0};
    int3 sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int3 up = {__shfl_up(sum.x, d), __shfl_up(sum.y, d), __shfl_up(sum.z, d)};
      if (lane >= d) sum = add3(sum, up);
    }
    if (lane == 63) wave_sum[w] = sum;
    __syncthreads();
    int3 before = base, all = base;
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      if (u < w) before = add3(before, wave_sum[u]);
      all = add3(all, wave_sum[u]);
    }
    __syncthreads();
    const int3 at = {before.x + sum.x - mine.x, before.y + sum.y - mine.y, before.z + sum.z - mine.z};
    if (j < s.Tk) {
      first[j] = at.x;
      item0[j] = at.y;
      slot0[j] = at.z;
    }
    base = all;
  }
  if (threadIdx.x == 0) {
    first[s.Tk] = base.x;
    item0[s.Tk] = base.y;
    slot0[s.Tk] = base.z;
  }
}

// The order of the work: head by head, and in a head the parts with the most tiles first.  Workgroups that run at the same time then walk lists of one length
// over one head's tiles and stay side by side, which is what lets them share the tiles through the L2 of their XCD (a head's queries and gradients are
// several times its size).  Parts of one length stand in no particular order: it decides nothing but when they run.
__global__ __launch_bounds__(1024) void inverse_order_kernel(GradArgs a) {
  const Sparse &s = a.s;
  const int bh = blockIdx.x, heads = gridDim.x;
  __shared__ int before[16], bucket[kPart + 1];
  int n = 0;
  for (int i = threadIdx.x; i < bh; i += 1024) n += a.item0[(int64_t)i * (s.Tk + 1) + s.Tk];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) n += __shfl_down(n, d);
  if ((threadIdx.x & 63) == 0) before[threadIdx.x >> 6] = n;
  if (threadIdx.x <= kPart) bucket[threadIdx.x] = 0;
  __syncthreads();
  const int32_t *first = a.first + (int64_t)bh * (s.Tk + 1);
  for (int j = threadIdx.x; j < s.Tk; j += 1024) {
    const int len = first[j + 1] - first[j];
    if (len >= a.part_tiles) atomicAdd(&bucket[0], len / a.part_tiles);
    if (len % a.part_tiles || len == 0) atomicAdd(&bucket[a.part_tiles - len % a.part_tiles], 1);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int at = 0;
    for (int w = 0; w < 16; ++w) at += before[w];
    for (int i = 0; i <= a.part_tiles; ++i) {
      const int c = bucket[i];
      bucket[i] = at;
      at += c;
    }
    if (bh == heads - 1) *a.n_work = at;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < s.Tk; j += 1024) {
    const int len = first[j + 1] - first[j];
    const int full = len / a.part_tiles;
    if (full) {
      const int at = atomicAdd(&bucket[0], full);
      for (int i = 0; i < full; ++i) a.work[at + i] = int2{bh * s.Tk + j, i};
    }
    if (len % a.part_tiles || len == 0) a.work[atomicAdd(&bucket[a.part_tiles - len % a.part_tiles], 1)] = int2{bh * s.Tk + j, full};
  }
}

// The tiles of a chunk one after the other, so that every block's list rises; the entries of one tile side by side (one that stands twice takes two
// places of the same value).
__global__ __launch_bounds__(256) void inverse_fill_kernel(GradArgs a) {
  const Sparse &s = a.s;
  const int chunk = blockIdx.x, bh = blockIdx.y;
  int32_t *h = a.hist + ((int64_t)bh * a.n_chunks + chunk) * s.Tk;
  const int32_t *first = a.first + (int64_t)bh * (s.Tk + 1);
  int32_t *inv = a.inv + (int64_t)bh * s.T * s.sel;
  const int32_t *list = a.blocks + (int64_t)bh * s.T * s.sel;
  for (int t = chunk * kChunk; t < min((chunk + 1) * kChunk, s.T); ++t) {
    for (int i = threadIdx.x; i < s.sel; i += 256) {
      const int j = list[(int64_t)t * s.sel + i];
      if ((unsigned)j < (unsigned)s.Tk) inv[first[j] + atomicAdd(h + j, 1)] = t;
    }
    __syncthreads();                  // (every returned count has been used: the tile's are done)
  }
}

// ---- dQ --------------------------------------------------------------------------------------------------------------------
// The forward's walk with three products, S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T.  1.10 ms at 480p (1.1 PFLOP/s), matrix cores busy 63 % of the cycles.
// Tiles of 64 queries are two waves, which go 32 keys at a time where a CU has more than two of them: all gradients of 32 heads of 8192 tokens, 16 blocks of 64,
// 631 us for 657 with 64 keys at a time (d = 64: 332 for 343), of four heads 131 for 122 (90 for 87).
//
// dS is rounded to bf16 for the matrix cores, and delta stems from an output that was rounded, so a row's dS no longer add up to nothing, and what is left
// over goes with the mean key: to be seen where few keys share a row (of rounding apart, dQ is 0.18 % off at 1024 keys, 0.19 at 512, 0.25 at 64 and 0.3 at 16;
// rounding dQ itself adds 0.17 %).  Tiles of up to kFewKeys keys go along their list again and take sum(dS) P K away: 0.16 % off at all of these.  They also
// put delta right for dK.
constexpr int kFewKeys = 512;

template <int D, bool F32, int NW, int ROWS = Pieces<F32>::ROWS>
__global__ __launch_bounds__(64 * NW, F32 ? (NW == 2 && D == 64 ? 2 : 1) : NW == 4 || ROWS == 32 ? 2 : 1) void sparse_dq_kernel(GradArgs a) {
  typedef Tile<D> T;
  enum { ONLY, FIRST, SECOND };
  constexpr int KS = D / 16, RB = D / 32, NS = Pieces<F32>::N, STAGE = T::bytes(ROWS);
  constexpr int STAGES = F32 && NW == 2 ? 1 : 2;      // (two waves: one stage, and more workgroups to a CU)
  __shared__ __attribute__((aligned(1024))) char lds[STAGES * 2 * NS * STAGE];
  const unsigned item = xcd_item(blockIdx.x, a.share);
  if (item >= a.items) return;
  const Sparse &s = a.s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int t = item % s.T, bh = item / s.T, b = bh / s.H, h = bh % s.H, hk = h / s.G;
  const int held = s.held(b), start = s.start(b);
  const int q0 = t * s.qb + 32 * w, qi = q0 + r;
  const int limit = s.causal ? min(held, start + min((t + 1) * s.qb, s.Nq)) : held;
  const int wave_limit = s.causal ? min(held, start + q0 + 1) : held, row_limit = s.causal ? min(held, start + qi + 1) : held;
  const int32_t *list = a.blocks + ((int64_t)(b * s.Hkv + hk) * s.T + t) * s.sel;
  ListWalk<ROWS> walk(list, 0, s.sel, s, limit, lane);
  const char *kbase = a.k.p + (b * a.k.sb + hk * a.k.sh) * 2, *vbase = a.v.p + (b * a.v.sb + hk * a.v.sh) * 2;
  const int ksn = (int)a.k.sn * 2, vsn = (int)a.v.sn * 2;
  auto request = [&](int key, int stage) {
    char *to = lds + stage * (2 * NS * STAGE);
    const int rows = min(limit - key, ROWS);
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      request_rows<D, ROWS, NW>(rows_rsrc<D>(kbase + (key * a.k.sn + n * a.piece_k) * 2, rows, ksn), ksn, to + n * STAGE, w, lane);
      request_rows<D, ROWS, NW>(rows_rsrc<D>(vbase + (key * a.v.sn + n * a.piece_k) * 2, rows, vsn), vsn, to + (NS + n) * STAGE, w, lane);
    }
  };
  int key = walk.next();
  if (key >= 0) request(key, 0);
  bf16x8 qf[KS][NS], df[KS][NS];
  const int row = min(qi, s.Nq - 1);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      qf[ks][n] = *reinterpret_cast<const bf16x8 *>(a.q.p + (b * a.q.sb + h * a.q.sh + row * a.q.sn + n * a.piece_q + 16 * ks + 8 * g) * 2);
      df[ks][n] = *reinterpret_cast<const bf16x8 *>(a.dout.p + (b * a.dout.sb + h * a.dout.sh + row * a.dout.sn + n * a.piece_q + 16 * ks + 8 * g) * 2);
    }
  float *st = a.stat + ((int64_t)bh * s.T * s.qb + q0) * 2 + r;
  const float c = a.scale_log2e, minus_lse2 = st[0] * c, minus_delta = st[32];
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;
  const unsigned rows0 = T::rows_base(lds, lane), cols0 = T::cols_base(lds, lane);
  float total = 0.f, unrounded = 0.f;  // FIRST: of this lane's keys' dS, as the product takes them and before
  // One walk along the list: o += dS K, or (SECOND) o += (-total P) K.
  auto add = [&](auto pass) {
    constexpr int PASS = decltype(pass)::value;
    for (int stage = 0; key >= 0; stage ^= STAGES - 1) {
      const int next = walk.next();
      landed();
      if (STAGES == 2 && next >= 0) request(next, stage ^ 1);
      const unsigned rows = rows0 + stage * (2 * NS * STAGE), cols = cols0 + stage * (2 * NS * STAGE);
      const bool mask = key + ROWS > wave_limit;
#pragma unroll
      for (int i = 0; i < ROWS / 32; ++i) {
        f32x16 sc, dp;
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = dp[x] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          bf16x8 kf[NS], vf[NS];
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            kf[n] = T::rows_at(rows, 32 * i, ks, n * STAGE);
            if constexpr (PASS != SECOND) vf[n] = T::rows_at(rows, 32 * i, ks, (NS + n) * STAGE);
          }
          sc = mfma_split<NS>(kf, qf[ks], sc);
          if constexpr (PASS != SECOND) dp = mfma_split<NS>(vf, df[ks], dp);
        }
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = fast_exp2(__builtin_fmaf(sc[x], c, minus_lse2)) * (PASS == SECOND ? -total : dp[x] + minus_delta);
        if (mask) {
#pragma unroll
          for (int x = 0; x < 16; ++x) sc[x] = key + 32 * i + crow(x, g) < row_limit ? sc[x] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f32x8 ds;
#pragma unroll
          for (int x = 0; x < 8; ++x) ds[x] = sc[8 * u + x];
          bf16x8 db[NS];
          split8<NS>(ds, db);
          if constexpr (PASS == FIRST) {
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              total += static_cast<float>(db[0][x]);
              unrounded += ds[x];
            }
          }
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            bf16x8 kf[NS];
#pragma unroll
            for (int n = 0; n < NS; ++n) kf[n] = T::cols_at(cols, rb, 32 * i + 16 * u, n * STAGE);
            o[rb] = mfma_split<NS>(kf, db, o[rb]);
          }
        }
      }
      if (STAGES == 1) {
        __syncthreads();
        if (next >= 0) request(next, 0);
      }
      key = next;
    }
  };
  if constexpr (F32) {
    add(std::integral_constant<int, ONLY>());
  } else if (min(s.sel * s.kb, limit) <= kFewKeys) {
    add(std::integral_constant<int, FIRST>());
    total = xhalf_sum(total);
    st[32] = minus_delta - xhalf_sum(unrounded);      // for dK (both lanes of a row write the same)
    __syncthreads();
    walk = ListWalk<ROWS>(list, 0, s.sel, s, limit, lane);
    key = walk.next();
    if (key >= 0) request(key, 0);
    add(std::integral_constant<int, SECOND>());
  } else {
    add(std::integral_constant<int, ONLY>());
  }
  __syncthreads();
  constexpr int ESZ = F32 ? 4 : 2;
  store_rows<D, F32>(o, a.scale, lds + w * store_bytes<D, F32>(), a.dq.p + (b * a.dq.sb + h * a.dq.sh) * ESZ, a.dq.sn * ESZ, q0,
                         min((t + 1) * s.qb, s.Nq), lane);
}

// ---- dK, dV ----------------------------------------------------------------------------------------------------------------
// A workgroup takes 64 keys of a block and one part of its list, 32 queries ("a chunk") of one head at a time: S = Q K^T, dP = dO V^T, then
// dV^T += dO^T P and dK^T += Q^T dS with P and dS straight from the registers of the first two products.  Q and dO lie in LDS and are read both ways.

// The statistics of a chunk to LDS.
__device__ __forceinline__ void request_stat(const float *src, char *to, int lane) {
  const unsigned l = __builtin_amdgcn_readfirstlane(lds_offset(to));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(l), "v"(lane * 4), "s"(src) : "memory");
}

// Four waves: the halves of the keys by two chunks at a time.  Two workgroups to a CU, so that one's loads, waits and exponentials run under the other's
// products; that leaves 256 registers to a wave: 128 for dK and dV, 32 for S and dP, K and half of V; the other half of V lies in LDS.  S starts from
// -lse / scale and dP from -delta, so that exp2(c S) is P and P dP is dS; the d / 16 sums then round at the size of lse / scale, which puts a weight off by up to d / 16 lse 2^-24
// (1e-5 of it at lse = 20, where its rounding to bf16 is 4e-3).  1.65 ms at 480p for four products (1.0 PFLOP/s), matrix cores busy 56 %.  It is
// bound by how little of one workgroup's loads and vector work the other one covers, and by the L2 (items in another order miss it almost twice as often).
template <int D>
__global__ __launch_bounds__(256, 2) void sparse_dkv_kernel(GradArgs a) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, TILE = T::bytes(32), CHUNK = 2 * TILE + 256, VKEEP = KS / 2, VROW = 64 * (KS - VKEEP) * 16;
  __shared__ __attribute__((aligned(1024))) char lds[2 * 2 * CHUNK + 2 * VROW];      // [stage][chunk][q | dO | statistics], [half of the keys][ks][lane] of v
  const Sparse &s = a.s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5, kh = w & 1, cg = w >> 1;
  // (workgroups go to the eight XCDs in turn: the two halves of a block of 128 keys to one of them)
  const int subs = s.kb >> 6, within = blockIdx.x % (8 * subs), half = within >> 3, item = blockIdx.x / (8 * subs) * 8 + (within & 7);
  if (item >= *a.n_work) return;
  const int2 work = a.work[item];
  const int bh = work.x / s.Tk, j = work.x - bh * s.Tk, part = work.y, b = bh / s.Hkv, hk = bh % s.Hkv;
  const int64_t at_j = (int64_t)bh * (s.Tk + 1) + j;
  const int parts = a.item0[at_j + 1] - a.item0[at_j];
  const int held = s.held(b), start = s.start(b), Nq = s.Nq, qb = s.qb, G = s.G;
  const int key0 = j * s.kb + 64 * half, k0 = key0 + 32 * kh, ki = k0 + r;
  const int first = a.first[at_j] + part * a.part_tiles, n = key0 < held ? min(a.first[at_j + 1] - first, a.part_tiles) : 0;
  const int tile = lane < n ? a.inv[(int64_t)bh * s.T * s.sel + first + lane] : 0;      // (a part has at most 64 tiles)
  const int per_head = qb >> 5, steps = (n * G * per_head) >> 1;                         // (2 or 4 chunks of a head in a tile)
  const int qsn = (int)a.q.sn * 2, dsn = (int)a.dout.sn * 2;
  const int64_t qsh = a.q.sh * 2, dsh = a.dout.sh * 2, ssh = (int64_t)s.T * qb * 8;
  const char *qhead = a.q.p + (b * a.q.sb + hk * G * a.q.sh) * 2, *dhead = a.dout.p + (b * a.dout.sb + hk * G * a.dout.sh) * 2;
  const char *shead = reinterpret_cast<const char *>(a.stat) + ((int64_t)b * s.H + hk * G) * ssh;
  const int first_seen = s.causal ? key0 - start : INT_MIN;         // the first query that sees one of the keys
  int e = 0, hd = 0, sub = cg;                        // place in the list, head of the group, chunk of the tile: of the next request
  // Requests this wave's half of its next chunk and returns the chunk's first row, or -1: rows behind the last query, and (causal) chunks all of whose
  // rows stand before the keys, take no part.
  auto request = [&](int stage) {
    int row = __builtin_amdgcn_readlane(tile, e) * qb + 32 * sub;
    const int rows = min(Nq - row, 32);
    if (rows <= 0 || row + rows <= first_seen) {
      row = -1;
    } else {
      char *to = lds + (stage * 2 + cg) * CHUNK;
      request_rows<D, 32, 2>(rows_rsrc<D>(qhead + (int64_t)row * qsn, rows, qsn), qsn, to, kh, lane);
      request_rows<D, 32, 2>(rows_rsrc<D>(dhead + (int64_t)row * dsn, rows, dsn), dsn, to + TILE, kh, lane);
      if (kh == 0) request_stat(reinterpret_cast<const float *>(shead + (int64_t)row * 8), to + 2 * TILE, lane);
    }
    sub += 2;
    if (sub >= per_head) {
      sub = cg;
      ++hd;
      qhead += qsh;
      dhead += dsh;
      shead += ssh;
      if (hd == G) {
        hd = 0;
        ++e;
        qhead -= G * qsh;
        dhead -= G * dsh;
        shead -= G * ssh;
      }
    }
    return row;
  };
  bf16x8 *vrest = reinterpret_cast<bf16x8 *>(lds + 2 * 2 * CHUNK) + kh * (VROW / 16) + lane;
  bf16x8 kf[KS], vf[VKEEP];
  int row = -1;
  if (steps > 0) {
    row = request(0);
    const char *kp = a.k.p + (b * a.k.sb + hk * a.k.sh + min(ki, s.Nk - 1) * a.k.sn + 8 * g) * 2, *vp = a.v.p + (b * a.v.sb + hk * a.v.sh + min(ki, s.Nk - 1) * a.v.sn + 8 * g) * 2;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[ks] = *reinterpret_cast<const bf16x8 *>(kp + 32 * ks);
      const bf16x8 x = *reinterpret_cast<const bf16x8 *>(vp + 32 * ks);
      if (ks < VKEEP) vf[ks] = x;
      else if (cg == 0) vrest[(ks - VKEEP) * 64] = x;
    }
  }
  const float c = a.scale_log2e;
  f32x16 dk[RB], dv[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) dk[rb][x] = dv[rb][x] = 0.f;
  const unsigned rows0 = T::rows_base(lds + cg * CHUNK, lane), cols0 = T::cols_base(lds + cg * CHUNK, lane);

  for (int step = 0, stage = 0; step < steps; ++step, stage ^= 1) {
    landed();
    const int cur = row;
    if (step + 1 < steps) row = request(stage ^ 1);
    if (cur < 0) continue;
    const unsigned rows = rows0 + stage * (2 * CHUNK), cols = cols0 + stage * (2 * CHUNK);
    const float *stat = reinterpret_cast<const float *>(lds + (stage * 2 + cg) * CHUNK + 2 * TILE) + 4 * g;
    f32x16 sc, dp;
#pragma unroll
    for (int x4 = 0; x4 < 4; ++x4) {
      const f32x4 l4 = *reinterpret_cast<const f32x4 *>(stat + 8 * x4), d4 = *reinterpret_cast<const f32x4 *>(stat + 32 + 8 * x4);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        sc[4 * x4 + x] = l4[x];
        dp[4 * x4 + x] = d4[x];
      }
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sc = mfma32(T::rows_at(rows, 0, ks), kf[ks], sc);
      dp = mfma32(T::rows_at(rows, 0, ks, TILE), ks < VKEEP ? vf[ks < VKEEP ? ks : 0] : vrest[(ks - VKEEP) * 64], dp);
    }
    if (k0 + 32 > held || cur < first_seen + 32 * kh + 31) {
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        // (rows behind the last query see what it sees)
        const bool seen = ki < held && ki - key0 + first_seen <= min(cur + crow(x, g), Nq - 1);
        sc[x] = seen ? sc[x] : -INFINITY;
        dp[x] = seen ? dp[x] : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x8 p8, d8;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        p8[x] = fast_exp2(sc[8 * u + x] * c);
        d8[x] = p8[x] * dp[8 * u + x];
      }
      const bf16x8 pb = __builtin_convertvector(p8, bf16x8), db = __builtin_convertvector(d8, bf16x8);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        dv[rb] = mfma32(T::cols_at(cols, rb, 16 * u, TILE), pb, dv[rb]);
        dk[rb] = mfma32(T::cols_at(cols, rb, 16 * u), db, dk[rb]);
      }
    }
  }
  // the other chunk's sums to the first's, as register images [dk | dv][lane] of each wave
  f32x4 *image = reinterpret_cast<f32x4 *>(lds);
  constexpr int IMAGE = 2 * RB * 4 * 64;
  __syncthreads();
  if (cg == 1) {
    f32x4 *to = image + kh * IMAGE + lane;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        to[(rb * 4 + x4) * 64] = f32x4{dk[rb][4 * x4], dk[rb][4 * x4 + 1], dk[rb][4 * x4 + 2], dk[rb][4 * x4 + 3]};
        to[((RB + rb) * 4 + x4) * 64] = f32x4{dv[rb][4 * x4], dv[rb][4 * x4 + 1], dv[rb][4 * x4 + 2], dv[rb][4 * x4 + 3]};
      }
  }
  __syncthreads();
  if (cg == 1) return;
  {
    const f32x4 *of = image + kh * IMAGE + lane;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        const f32x4 k4 = of[(rb * 4 + x4) * 64], v4 = of[((RB + rb) * 4 + x4) * 64];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          dk[rb][4 * x4 + x] += k4[x];
          dv[rb][4 * x4 + x] += v4[x];
        }
      }
  }
  if (parts > 1) {
    float *to = a.part + (((int64_t)bh * a.max_slots + a.slot0[at_j] + part) * 2 * s.kb + 64 * half + 32 * kh + r) * D;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        *reinterpret_cast<f32x4 *>(to + 32 * rb + 8 * x4 + 4 * g) = f32x4{dk[rb][4 * x4], dk[rb][4 * x4 + 1], dk[rb][4 * x4 + 2], dk[rb][4 * x4 + 3]};
        *reinterpret_cast<f32x4 *>(to + s.kb * D + 32 * rb + 8 * x4 + 4 * g) = f32x4{dv[rb][4 * x4], dv[rb][4 * x4 + 1], dv[rb][4 * x4 + 2], dv[rb][4 * x4 + 3]};
      }
    return;
  }
  static_assert(2 * IMAGE * 16 <= 2 * 2 * CHUNK + 2 * VROW && store_bytes<D, false>() <= IMAGE * 16, "images, and the stores in a wave's own");
  char *stage = lds + kh * (IMAGE * 16);
  store_rows<D, false>(dk, a.scale, stage, a.dk.p + (b * a.dk.sb + hk * a.dk.sh) * 2, a.dk.sn * 2, k0, s.Nk, lane);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  store_rows<D, false>(dv, 1.f, stage, a.dv.p + (b * a.dv.sb + hk * a.dv.sh) * 2, a.dv.sn * 2, k0, s.Nk, lane);
}

// fp32 tensors: the keys' and values' pieces in registers, 32 keys to a wave, and every wave reads all queries.  All gradients of 32 heads of 8192 tokens
// (d = 128, tiles of 128 x 16 blocks of 64) take 3.5 ms, 97 TFLOP/s, 0.6 PFLOP/s of the matrix cores: the pieces fill the registers of one wave to a SIMD.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 1) void sparse_dkv_f32_kernel(GradArgs a) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, NS = Pieces<true>::N, ROWS = Pieces<true>::ROWS, STAGE = T::bytes(ROWS), STAT = 2 * 32 * 4;
  constexpr int STAGES = NW == 2 ? 1 : 2;             // (as for dQ)
  __shared__ __attribute__((aligned(1024))) char lds[STAGES * (2 * NS * STAGE + STAT)];      // [stage][q | dO][pieces][ROWS], lse2 | delta
  const Sparse &s = a.s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  if ((int)blockIdx.x >= *a.n_work) return;
  const int2 work = a.work[blockIdx.x];
  const int bh = work.x / s.Tk, j = work.x - bh * s.Tk, part = work.y, b = bh / s.Hkv, hk = bh % s.Hkv;
  const int64_t at_j = (int64_t)bh * (s.Tk + 1) + j;
  const int parts = a.item0[at_j + 1] - a.item0[at_j], first = a.first[at_j], last = a.first[at_j + 1];
  const int32_t *list = a.inv + (int64_t)bh * s.T * s.sel;
  const int held = s.held(b), start = s.start(b);
  const int key0 = j * s.kb, k0 = key0 + 32 * w, ki = k0 + r;
  // steps: (place in the list, head of the group, ROWS queries of the tile)
  const int subs = s.qb / ROWS;
  int at = first + part * a.part_tiles, end = min(at + a.part_tiles, last), head = 0, sub = 0;
  if (key0 >= held) at = end;
  struct Step { int h, row; };        // row < 0: none left
  auto next_step = [&]() {
    while (at < end) {
      const Step st = {hk * s.G + head, __builtin_amdgcn_readfirstlane(list[at]) * s.qb + ROWS * sub};
      if (++sub == subs) {
        sub = 0;
        if (++head == s.G) {
          head = 0;
          ++at;
        }
      }
      // rows behind the last query, and (causal) all of whose rows stand before the block, take no part
      if (st.row < s.Nq && !(s.causal && start + min(st.row + ROWS - 1, s.Nq - 1) < key0)) return st;
    }
    return Step{0, -1};
  };
  const int qsn = (int)a.q.sn * 2, dsn = (int)a.dout.sn * 2;
  auto request = [&](const Step &st, int stage) {
    char *to = lds + stage * (2 * NS * STAGE + STAT);
    const int rows = min(s.Nq - st.row, ROWS);
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      request_rows<D, ROWS, NW>(rows_rsrc<D>(a.q.p + (b * a.q.sb + st.h * a.q.sh + st.row * a.q.sn + n * a.piece_q) * 2, rows, qsn), qsn, to + n * STAGE, w, lane);
      request_rows<D, ROWS, NW>(rows_rsrc<D>(a.dout.p + (b * a.dout.sb + st.h * a.dout.sh + st.row * a.dout.sn + n * a.piece_q) * 2, rows, dsn), dsn,
                              to + (NS + n) * STAGE, w, lane);
    }
    if (w == 0) request_stat(a.stat + ((int64_t)(b * s.H + st.h) * s.T * s.qb + st.row) * 2, to + 2 * NS * STAGE, lane);
  };
  Step cur = next_step();
  if (cur.row >= 0) request(cur, 0);

  bf16x8 kf[KS][NS], vf[KS][NS];
  const int krow = min(ki, s.Nk - 1);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      kf[ks][n] = *reinterpret_cast<const bf16x8 *>(a.k.p + (b * a.k.sb + hk * a.k.sh + krow * a.k.sn + n * a.piece_k + 16 * ks + 8 * g) * 2);
      vf[ks][n] = *reinterpret_cast<const bf16x8 *>(a.v.p + (b * a.v.sb + hk * a.v.sh + krow * a.v.sn + n * a.piece_k + 16 * ks + 8 * g) * 2);
    }
  const float c = a.scale_log2e;
  f32x16 dk[RB], dv[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) dk[rb][x] = dv[rb][x] = 0.f;

  const unsigned rows0 = T::rows_base(lds, lane), cols0 = T::cols_base(lds, lane);
  for (int stage = 0; cur.row >= 0; stage ^= STAGES - 1) {
    const Step next = next_step();
    landed();
    if (STAGES == 2 && next.row >= 0) request(next, stage ^ 1);
    const char *tq = lds + stage * (2 * NS * STAGE + STAT);
    const unsigned rows = rows0 + stage * (2 * NS * STAGE + STAT), cols = cols0 + stage * (2 * NS * STAGE + STAT);
    const float *stat = reinterpret_cast<const float *>(tq + 2 * NS * STAGE);
    const bool mask = k0 + 32 > held || (s.causal && start + cur.row < k0 + 31);
#pragma unroll
    for (int i = 0; i < ROWS / 32; ++i) {
      f32x16 sc, dp;
#pragma unroll
      for (int x = 0; x < 16; ++x) sc[x] = dp[x] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 qf[NS], df[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          qf[n] = T::rows_at(rows, 32 * i, ks, n * STAGE);
          df[n] = T::rows_at(rows, 32 * i, ks, (NS + n) * STAGE);
        }
        sc = mfma_split<NS>(qf, kf[ks], sc);
        dp = mfma_split<NS>(df, vf[ks], dp);
      }
      // (the statistics come last: a sum that starts from -lse / scale rounds at its size, and P is 1.4e-6 off)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        const f32x4 l4 = *reinterpret_cast<const f32x4 *>(stat + 8 * x4 + 4 * g), d4 = *reinterpret_cast<const f32x4 *>(stat + 32 + 8 * x4 + 4 * g);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float p = fast_exp2(__builtin_fmaf(sc[4 * x4 + x], c, l4[x] * c));
          sc[4 * x4 + x] = p;
          dp[4 * x4 + x] = p * (dp[4 * x4 + x] + d4[x]);
        }
      }
      if (mask) {
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const bool seen = ki < held && (!s.causal || ki <= start + min(cur.row + 32 * i + crow(x, g), s.Nq - 1));    // (rows behind the last query see what it sees)
          sc[x] = seen ? sc[x] : 0.f;
          dp[x] = seen ? dp[x] : 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x8 p8, d8;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          p8[x] = sc[8 * u + x];
          d8[x] = dp[8 * u + x];
        }
        bf16x8 pb[NS], db[NS];
        split8<NS>(p8, pb);
        split8<NS>(d8, db);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          bf16x8 qf[NS], df[NS];
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            df[n] = T::cols_at(cols, rb, 32 * i + 16 * u, (NS + n) * STAGE);
            qf[n] = T::cols_at(cols, rb, 32 * i + 16 * u, n * STAGE);
          }
          // (a sum of six products rounds at its own size, not at that of the sum over thousands of queries)
          dv[rb] += mfma_split<NS>(df, pb, f32x16{});
          dk[rb] += mfma_split<NS>(qf, db, f32x16{});
        }
      }
    }
    if (STAGES == 1) {
      __syncthreads();
      if (next.row >= 0) request(next, 0);
    }
    cur = next;
  }
  if (parts > 1) {
    float *to = a.part + (((int64_t)bh * a.max_slots + a.slot0[at_j] + part) * 2 * s.kb + 32 * w + r) * D;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        *reinterpret_cast<f32x4 *>(to + 32 * rb + 8 * x4 + 4 * g) = f32x4{dk[rb][4 * x4], dk[rb][4 * x4 + 1], dk[rb][4 * x4 + 2], dk[rb][4 * x4 + 3]};
        *reinterpret_cast<f32x4 *>(to + s.kb * D + 32 * rb + 8 * x4 + 4 * g) = f32x4{dv[rb][4 * x4], dv[rb][4 * x4 + 1], dv[rb][4 * x4 + 2], dv[rb][4 * x4 + 3]};
      }
    return;
  }
  __syncthreads();
  constexpr int ESZ = 4;
  char *stage = lds + w * store_bytes<D, true>();
  store_rows<D, true>(dk, a.scale, stage, a.dk.p + (b * a.dk.sb + hk * a.dk.sh) * ESZ, a.dk.sn * ESZ, k0, s.Nk, lane);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  store_rows<D, true>(dv, 1.f, stage, a.dv.p + (b * a.dv.sb + hk * a.dv.sh) * ESZ, a.dv.sn * ESZ, k0, s.Nk, lane);
}

// Joins the parts of the blocks that have several: D / 4 threads to a row of dk or dv, a workgroup to 256 / (D / 4) of a block's rows.
// Bound by memory, 36 us at 480p.
template <int D, bool F32>
__global__ __launch_bounds__(256) void sparse_dkv_join_kernel(GradArgs a) {
  constexpr int TPR = D / 4, RPB = 256 / TPR;
  const Sparse &s = a.s;
  const int row = blockIdx.y * RPB + threadIdx.x / TPR, at = blockIdx.x;
  const int j = at % s.Tk, bh = at / s.Tk, b = bh / s.Hkv, hk = bh % s.Hkv;
  const int64_t at_j = (int64_t)bh * (s.Tk + 1) + j;
  const int parts = a.item0[at_j + 1] - a.item0[at_j];
  if (parts <= 1) return;
  const int c = 4 * (threadIdx.x % TPR);
  const float *from = a.part + (((int64_t)bh * a.max_slots + a.slot0[at_j]) * 2 * s.kb + row) * D + c;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = 0; i < parts; ++i) sum += *reinterpret_cast<const f32x4 *>(from + (int64_t)i * 2 * s.kb * D);
  const bool is_v = row >= s.kb;
  const int n = j * s.kb + (is_v ? row - s.kb : row);
  if (n >= s.Nk) return;
  const View &to = is_v ? a.dv : a.dk;
  if (!is_v) sum *= a.scale;
  const int64_t i = b * to.sb + hk * to.sh + n * to.sn + c;
  if constexpr (F32) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(to.p) + i) = sum;
  else *reinterpret_cast<bf16x4 *>(reinterpret_cast<__bf16 *>(to.p) + i) = __builtin_convertvector(sum, bf16x4);
}

struct GradPlanS {
  int n_chunks, max_items, max_slots, part_tiles;
  size_t off_q, off_k, off_v, off_do, off_stat, off_hist, off_first, off_item0, off_slot0, off_inv, off_work, off_n_work, off_part, total;
};

GradPlanS plan_grad(const ha_sparse_problem &p, const Sparse &s) {
  GradPlanS f{};
  const int64_t entries = (int64_t)s.T * s.sel;
  f.n_chunks = (s.T + kChunk - 1) / kChunk;
  // Parts of 64 tiles, shorter ones where the lists of all heads would not fill the chip twice, but at least some queries to a part, whose sums pass through
  // memory: 512 in bf16, 256 in fp32, where a query takes four times as long.  Passes (forward and gradients) with at least 8 tiles / 256 / 512 / 1024 queries
  // to a part, us: [2, 12 : 4, 1819] bf16 138 / 102 / 102 / 106, [1, 16 : 2, 411] 141 / 84 / 83 / 90, [2, 3 : 1, 3724] causal 126 / 142 / 129 / 123;
  // [2, 2 : 1, 4810] fp32 261 / 138 / 156 / 198, [2, 6 : 3, 305] 210 / 147 / 189 / 209.
  const int64_t rows = (int64_t)s.G * s.qb, fill = (int64_t)s.B * s.Hkv * entries / 512;
  int64_t part = std::max<int64_t>({fill, (p.dtype == HA_F32 ? 256 : 512) / rows, 1});
  // fp32: a sum over R queries in 16s is 2.4e-8 sqrt(R / 32) off by its roundings; parts of up to 8192 queries hold that under 4e-7
  if (p.dtype == HA_F32) part = std::min<int64_t>(part, std::max<int64_t>(8192 / rows, 1));
  f.part_tiles = (int)std::min<int64_t>(part, kPart);
  // ceil(n_j / part) parts of block j: over all blocks at most entries / part + Tk; those of blocks with several, of which there are
  // fewer than entries / part, at most 2 entries / part
  f.max_items = (int)(entries / f.part_tiles) + s.Tk;
  f.max_slots = (int)(2 * (entries / f.part_tiles));
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round256(bytes);
    return here;
  };
  const size_t nq = (size_t)s.B * s.H * s.Nq * p.d_head, nk = (size_t)s.B * s.Hkv * s.Nk * p.d_head, hk = (size_t)s.B * s.Hkv;
  if (p.dtype == HA_F32) {
    f.off_q = take(6 * nq);
    f.off_k = take(6 * nk);
    f.off_v = take(6 * nk);
    f.off_do = take(6 * nq);
  }
  f.off_stat = take((size_t)s.B * s.H * s.T * s.qb * 8);
  f.off_hist = take(hk * f.n_chunks * s.Tk * 4);
  f.off_first = take(hk * (s.Tk + 1) * 4);
  f.off_item0 = take(hk * (s.Tk + 1) * 4);
  f.off_slot0 = take(hk * (s.Tk + 1) * 4);
  f.off_inv = take(hk * entries * 4);
  f.off_work = take(hk * f.max_items * 8);
  f.off_n_work = take(4);
  f.off_part = take(hk * f.max_slots * 2 * s.kb * p.d_head * 4);
  f.total = at;
  if ((int64_t)hk * f.max_items > (1 << 22)) f.total = 0;      // (twice 256 threads to an item: more than a launch takes)
  return f;
}

template <int D, bool F32>
hipError_t launch_grad(const ha_sparse_problem &p, GradArgs &a, hipStream_t st) {
  const Sparse &s = a.s;
  hipError_t e;
  if (s.Nq > 0) {
    a.items = (unsigned)((int64_t)s.B * s.H * s.T);
    a.share = xcd_share(a.items);
    if (s.qb == 128) sparse_dq_kernel<D, F32, 4><<<8 * a.share, 256, 0, st>>>(a);
    else if (F32 || a.items <= 512) sparse_dq_kernel<D, F32, 2><<<8 * a.share, 128, 0, st>>>(a);
    else sparse_dq_kernel<D, F32, 2, 32><<<8 * a.share, 128, 0, st>>>(a);      // half the LDS, more workgroups to a CU
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (s.Nk > 0) {
    const unsigned items = (unsigned)((int64_t)s.B * s.Hkv * a.max_items);
    if constexpr (!F32) sparse_dkv_kernel<D><<<(items + 7) / 8 * 8 * (s.kb >> 6), 256, 0, st>>>(a);
    else if (s.kb == 128) sparse_dkv_f32_kernel<D, 4><<<items, 256, 0, st>>>(a);
    else sparse_dkv_f32_kernel<D, 2><<<items, 128, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.max_slots > 0) {
      sparse_dkv_join_kernel<D, F32><<<dim3((unsigned)((int64_t)s.B * s.Hkv * s.Tk), 2 * s.kb / (1024 / D)), 256, 0, st>>>(a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" size_t hybrid_attn_sparse_grad_workspace_bytes(const ha_sparse_problem *p) {
  if (check_sparse(p) != HA_OK) return 0;
  return plan_grad(*p, sparse_of(*p)).total;
}

extern "C" ha_status hybrid_attn_sparse_grad(const ha_sparse_problem *p, const ha_view *q, const ha_view *k, const ha_view *v, const int32_t *blocks,
                                             const ha_view *out, const float *lse, const ha_view *grad_out, const ha_view *grad_q, const ha_view *grad_k,
                                             const ha_view *grad_v, void *workspace, size_t workspace_bytes, void *hip_stream) {
  ha_status st = check_sparse(p);
  if (st != HA_OK) return st;
  GradArgs a{};
  View o;
  if ((st = check_view(*p, q, p->H, p->N_q, p->q_block, false, a.q)) != HA_OK || (st = check_view(*p, k, p->H_kv, p->N_k, p->k_block, false, a.k)) != HA_OK ||
      (st = check_view(*p, v, p->H_kv, p->N_k, p->k_block, false, a.v)) != HA_OK || (st = check_view(*p, out, p->H, p->N_q, p->q_block, false, o)) != HA_OK ||
      (st = check_view(*p, grad_out, p->H, p->N_q, p->q_block, false, a.dout)) != HA_OK ||
      (st = check_view(*p, grad_q, p->H, p->N_q, p->q_block, true, a.dq)) != HA_OK ||
      (st = check_view(*p, grad_k, p->H_kv, p->N_k, p->k_block, true, a.dk)) != HA_OK ||
      (st = check_view(*p, grad_v, p->H_kv, p->N_k, p->k_block, true, a.dv)) != HA_OK)
    return st;
  if (p->N_q > 0 && (!blocks || !lse)) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(blocks) & 3u || reinterpret_cast<uintptr_t>(lse) & 3u) return HA_ERR_ALIGN;
  const Sparse s = a.s = sparse_of(*p);
  const GradPlanS f = plan_grad(*p, s);
  if (f.total == 0) return HA_ERR_UNSUPPORTED;      // (any plan that is not refused has some bytes, without queries or keys too)
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < f.total) return HA_ERR_WORKSPACE;
  if (p->N_q == 0 && p->N_k == 0) return HA_OK;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(workspace);
  const int d = p->d_head;
  const bool f32 = p->dtype == HA_F32;
  float *stat = reinterpret_cast<float *>(ws + f.off_stat);
  hipError_t e;
  if (s.Nq > 0) {
    const int rpb = 256 / (d / 8);
    const unsigned n = (unsigned)(((int64_t)s.B * s.H * s.T * s.qb + rpb - 1) / rpb);
    if (d == 128) { if (f32) sparse_delta_kernel<128, true><<<n, 256, 0, stream>>>(s, o, a.dout, lse, 1.f / p->softmax_scale, stat); else sparse_delta_kernel<128, false><<<n, 256, 0, stream>>>(s, o, a.dout, lse, 1.f / p->softmax_scale, stat); }
    else { if (f32) sparse_delta_kernel<64, true><<<n, 256, 0, stream>>>(s, o, a.dout, lse, 1.f / p->softmax_scale, stat); else sparse_delta_kernel<64, false><<<n, 256, 0, stream>>>(s, o, a.dout, lse, 1.f / p->softmax_scale, stat); }
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
  }
  if (f32) {
    const SplitJob jobs[4] = {{a.q, reinterpret_cast<__bf16 *>(ws + f.off_q), s.H, s.Nq}, {a.k, reinterpret_cast<__bf16 *>(ws + f.off_k), s.Hkv, s.Nk},
                              {a.v, reinterpret_cast<__bf16 *>(ws + f.off_v), s.Hkv, s.Nk}, {a.dout, reinterpret_cast<__bf16 *>(ws + f.off_do), s.H, s.Nq}};
    if ((e = launch_split(s, d, jobs, 4, stream)) != hipSuccess) return device_error(e);
    a.q = split_view(jobs[0], d);
    a.k = split_view(jobs[1], d);
    a.v = split_view(jobs[2], d);
    a.dout = split_view(jobs[3], d);
    a.piece_q = (int64_t)s.B * s.H * s.Nq * d;
    a.piece_k = (int64_t)s.B * s.Hkv * s.Nk * d;
  }
  a.blocks = blocks;
  a.stat = stat;
  a.hist = reinterpret_cast<int32_t *>(ws + f.off_hist);
  a.first = reinterpret_cast<int32_t *>(ws + f.off_first);
  a.item0 = reinterpret_cast<int32_t *>(ws + f.off_item0);
  a.slot0 = reinterpret_cast<int32_t *>(ws + f.off_slot0);
  a.inv = reinterpret_cast<int32_t *>(ws + f.off_inv);
  a.work = reinterpret_cast<int2 *>(ws + f.off_work);
  a.n_work = reinterpret_cast<int32_t *>(ws + f.off_n_work);
  a.part = reinterpret_cast<float *>(ws + f.off_part);
  a.n_chunks = f.n_chunks;
  a.max_items = f.max_items;
  a.max_slots = f.max_slots;
  a.part_tiles = f.part_tiles;
  a.scale = p->softmax_scale;
  a.scale_log2e = p->softmax_scale * kLog2e;
  if (s.Nk > 0) {
    const unsigned heads = (unsigned)s.B * s.Hkv;
    if (f.n_chunks > 0) {
      inverse_count_kernel<<<dim3(f.n_chunks, heads), 256, 0, stream>>>(a);
      if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
    }
    inverse_scan_kernel<<<heads, 1024, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
    inverse_order_kernel<<<heads, 1024, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
    if (f.n_chunks > 0) {
      inverse_fill_kernel<<<dim3(f.n_chunks, heads), 256, 0, stream>>>(a);
      if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
    }
  }
  if (d == 128) e = f32 ? launch_grad<128, true>(*p, a, stream) : launch_grad<128, false>(*p, a, stream);
  else e = f32 ? launch_grad<64, true>(*p, a, stream) : launch_grad<64, false>(*p, a, stream);
  return e == hipSuccess ? HA_OK : device_error(e);
}
