// Block-sparse attention, gfx950: the gradients.
//
//   P = exp(scale S - lse),  dP = dO V^T,  dS = P (dP - delta) scale,  delta_i = dO_i . O_i,
//   dQ = dS K,   dK = dS^T Q,   dV = P^T dO      (the last two summed over the query heads of a key head)
//
// Two passes, neither with an atomic, so that the sums have one order: dQ by tiles of queries along their lists, as the forward walks them, and dK, dV by
// key blocks along the tiles that chose them.  S and dP are formed in both (seven products for five; writing dQ's terms from the second pass
// instead would be fp32 atomics, or T x n_select partial tiles in memory).  The inverse lists are built on the way: tiles in rising order for every key
// block, by counting in chunks of tiles.  Popular blocks (a first block that every tile keeps) would leave one workgroup with thousands of
// tiles, so a list is cut into parts of kPart tiles whose sums a last kernel joins in order.
#include "ha_sparse.h"

namespace ha {
namespace {

constexpr int kPart = 64;        // tiles of an inverse list that one workgroup takes
constexpr int kChunk = 16;       // tiles counted together while the inverse lists are built

struct GradArgs {
  Sparse s;
  View q, k, v, dout, dq, dk, dv;      // inputs bf16 (fp32 tensors: the first pieces; the next stand piece_* elements behind)
  int64_t piece_q, piece_k;
  const int32_t *blocks;
  const float *lse2, *delta;           // [B H][T qb]: lse log2 e (+infinity for rows that take no part), delta
  int32_t *hist;                       // [B Hkv][n_chunks][Tk]
  int32_t *first, *item0, *slot0;      // [B Hkv][Tk + 1]: a block's first place in inv, its first item and its first slot
  int32_t *inv;                        // [B Hkv][T sel] tiles
  int32_t *item_block;                 // [B Hkv][max_items] block of an item, -1 behind the last
  float *part;                         // [B Hkv][max_slots][dk | dv][kb][D]
  int n_chunks, max_items, max_slots;
  float scale, scale_log2e;
  unsigned items, share;
};

// ---- row statistics ----------------------------------------------------------------------------------------------------
template <int D, bool F32>
__global__ __launch_bounds__(256) void sparse_delta_kernel(Sparse s, View out, View dout, const float *lse, float *lse2, float *delta) {
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
    lse2[at] = l == -INFINITY ? INFINITY : l * kLog2e;
    delta[at] = l == -INFINITY ? 0.f : sum;
  }
}

// ---- inverse lists -----------------------------------------------------------------------------------------------------
// hist[chunk][j]: how many times the chunk's tiles list block j.
__global__ __launch_bounds__(256) void inverse_count_kernel(GradArgs a) {
  const Sparse &s = a.s;
  const int chunk = blockIdx.x, bh = blockIdx.y;
  int32_t *h = a.hist + ((int64_t)bh * a.n_chunks + chunk) * s.Tk;
  for (int j = threadIdx.x; j < s.Tk; j += 256) h[j] = 0;
  __threadfence();
  __syncthreads();
  const int lo = chunk * kChunk * s.sel, hi = min((chunk + 1) * kChunk, s.T) * s.sel;
  const int32_t *list = a.blocks + (int64_t)bh * s.T * s.sel;
  for (int i = lo + threadIdx.x; i < hi; i += 256) {
    const int j = list[i];
    if ((unsigned)j < (unsigned)s.Tk) atomicAdd(h + j, 1);
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
  int32_t *item_block = a.item_block + (int64_t)bh * a.max_items;
  int3 base = {0, 0, 0};
  for (int j0 = 0; j0 < s.Tk; j0 += 1024) {
    const int j = j0 + threadIdx.x;
    int n = 0;
    if (j < s.Tk)
      for (int c = 0; c < a.n_chunks; ++c) {
        const int x = h[(int64_t)c * s.Tk + j];
        h[(int64_t)c * s.Tk + j] = n;
        n += x;
      }
    const int parts = j < s.Tk ? max(1, (n + kPart - 1) / kPart) : 0;
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
      for (int i = 0; i < parts; ++i) item_block[at.y + i] = j;
    }
    base = all;
  }
  if (threadIdx.x == 0) {
    first[s.Tk] = base.x;
    item0[s.Tk] = base.y;
    slot0[s.Tk] = base.z;
  }
  for (int i = base.y + threadIdx.x; i < a.max_items; i += 1024) item_block[i] = -1;
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
template <int D, bool F32, int NW>
__global__ __launch_bounds__(64 * NW, !F32 && NW == 4 ? 2 : 1) void sparse_dq_kernel(GradArgs a) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, NS = Pieces<F32>::N, ROWS = Pieces<F32>::ROWS, STAGE = T::bytes(ROWS);
  __shared__ __attribute__((aligned(1024))) char lds[2 * 2 * NS * STAGE];
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
  const int64_t st = (int64_t)bh * s.T * s.qb + qi;
  const float lse2 = a.lse2[st], delta = a.delta[st], c = a.scale_log2e;
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;
  for (int stage = 0; key >= 0; stage ^= 1) {
    const int next = walk.next();
    landed();
    if (next >= 0) request(next, stage ^ 1);
    const char *tk = lds + stage * (2 * NS * STAGE), *tv = tk + NS * STAGE;
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
          kf[n] = T::rows(tk + n * STAGE, 32 * i, ks, lane);
          vf[n] = T::rows(tv + n * STAGE, 32 * i, ks, lane);
        }
        sc = mfma_split<NS>(kf, qf[ks], sc);
        dp = mfma_split<NS>(vf, df[ks], dp);
      }
#pragma unroll
      for (int x = 0; x < 16; ++x) sc[x] = fast_exp2(__builtin_fmaf(sc[x], c, -lse2)) * (dp[x] - delta);
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
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          bf16x8 kf[NS];
#pragma unroll
          for (int n = 0; n < NS; ++n) kf[n] = T::cols(tk + n * STAGE, rb, 32 * i + 16 * u, lane);
          o[rb] = mfma_split<NS>(kf, db, o[rb]);
        }
      }
    }
    key = next;
  }
  __syncthreads();
  constexpr int ESZ = F32 ? 4 : 2;
  store_rows<D, F32>(o, a.scale, lds + w * store_bytes<D, F32>(), a.dq.p + (b * a.dq.sb + h * a.dq.sh) * ESZ, a.dq.sn * ESZ, q0,
                         min((t + 1) * s.qb, s.Nq), lane);
}

// ---- dK, dV ----------------------------------------------------------------------------------------------------------------
// A workgroup takes one part of one key block's list: 32 keys to a wave, whose K and V stay in registers; 64 queries at a time lie in LDS, Q and dO,
// read as rows for S = Q K^T and dP = dO V^T and as columns for dK^T += Q^T dS and dV^T += dO^T P.
template <int D, bool F32, int NW>
__global__ __launch_bounds__(64 * NW, 1) void sparse_dkv_kernel(GradArgs a) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, NS = Pieces<F32>::N, ROWS = Pieces<F32>::ROWS, STAGE = T::bytes(ROWS), STAT = 2 * 64 * 4;
  __shared__ __attribute__((aligned(1024))) char lds[2 * (2 * NS * STAGE + STAT)];      // [2 stages][q | dO][pieces][ROWS], lse2 | delta
  const unsigned item = xcd_item(blockIdx.x, a.share);
  if (item >= a.items) return;
  const Sparse &s = a.s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int bh = item / a.max_items, it = item % a.max_items, b = bh / s.Hkv, hk = bh % s.Hkv;
  const int j = __builtin_amdgcn_readfirstlane(a.item_block[(int64_t)bh * a.max_items + it]);
  if (j < 0) return;
  const int part = it - a.item0[(int64_t)bh * (s.Tk + 1) + j], parts = a.item0[(int64_t)bh * (s.Tk + 1) + j + 1] - a.item0[(int64_t)bh * (s.Tk + 1) + j];
  const int first = a.first[(int64_t)bh * (s.Tk + 1) + j], last = a.first[(int64_t)bh * (s.Tk + 1) + j + 1];
  const int32_t *list = a.inv + (int64_t)bh * s.T * s.sel;
  const int held = s.held(b), start = s.start(b);
  const int key0 = j * s.kb, k0 = key0 + 32 * w, ki = k0 + r;
  // steps: (place in the list, head of the group, ROWS queries of the tile)
  const int subs = s.qb / ROWS;
  int at = first + part * kPart, end = min(at + kPart, last), head = 0, sub = 0;
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
    if (w < 2) {
      const float *src = (w == 0 ? a.lse2 : a.delta) + (int64_t)(b * s.H + st.h) * s.T * s.qb + st.row;
      const unsigned l = __builtin_amdgcn_readfirstlane(lds_offset(to + 2 * NS * STAGE) + w * 256);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(l), "v"(lane * 4), "s"(src) : "memory");
    }
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

  for (int stage = 0; cur.row >= 0; stage ^= 1) {
    const Step next = next_step();
    landed();
    if (next.row >= 0) request(next, stage ^ 1);
    const char *tq = lds + stage * (2 * NS * STAGE + STAT), *td = tq + NS * STAGE;
    const float *lse2 = reinterpret_cast<const float *>(tq + 2 * NS * STAGE), *delta = lse2 + 64;
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
          qf[n] = T::rows(tq + n * STAGE, 32 * i, ks, lane);
          df[n] = T::rows(td + n * STAGE, 32 * i, ks, lane);
        }
        sc = mfma_split<NS>(qf, kf[ks], sc);
        dp = mfma_split<NS>(df, vf[ks], dp);
      }
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        const f32x4 l4 = *reinterpret_cast<const f32x4 *>(lse2 + 32 * i + 8 * x4 + 4 * g), d4 = *reinterpret_cast<const f32x4 *>(delta + 32 * i + 8 * x4 + 4 * g);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          sc[4 * x4 + x] = fast_exp2(__builtin_fmaf(sc[4 * x4 + x], c, -l4[x]));
          dp[4 * x4 + x] = sc[4 * x4 + x] * (dp[4 * x4 + x] - d4[x]);
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
            df[n] = T::cols(td + n * STAGE, rb, 32 * i + 16 * u, lane);
            qf[n] = T::cols(tq + n * STAGE, rb, 32 * i + 16 * u, lane);
          }
          dv[rb] = mfma_split<NS>(df, pb, dv[rb]);
          dk[rb] = mfma_split<NS>(qf, db, dk[rb]);
        }
      }
    }
    cur = next;
  }
  if (parts > 1) {
    float *to = a.part + (((int64_t)bh * a.max_slots + a.slot0[(int64_t)bh * (s.Tk + 1) + j] + part) * 2 * s.kb + 32 * w + r) * D;
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
  constexpr int ESZ = F32 ? 4 : 2;
  char *stage = lds + w * store_bytes<D, F32>();
  store_rows<D, F32>(dk, a.scale, stage, a.dk.p + (b * a.dk.sb + hk * a.dk.sh) * ESZ, a.dk.sn * ESZ, k0, s.Nk, lane);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  store_rows<D, F32>(dv, 1.f, stage, a.dv.p + (b * a.dv.sb + hk * a.dv.sh) * ESZ, a.dv.sn * ESZ, k0, s.Nk, lane);
}

// Joins the parts of the blocks that have several: D / 4 threads to a row of dk or dv.
template <int D, bool F32>
__global__ __launch_bounds__(256) void sparse_dkv_join_kernel(GradArgs a) {
  constexpr int TPR = D / 4;
  const Sparse &s = a.s;
  const int j = blockIdx.x % s.Tk, bh = blockIdx.x / s.Tk, b = bh / s.Hkv, hk = bh % s.Hkv;
  const int64_t at = (int64_t)bh * (s.Tk + 1) + j;
  const int parts = a.item0[at + 1] - a.item0[at];
  if (parts <= 1) return;
  const float *from = a.part + ((int64_t)bh * a.max_slots + a.slot0[at]) * 2 * s.kb * D;
  const int c = 4 * (threadIdx.x % TPR);
  for (int row = threadIdx.x / TPR; row < 2 * s.kb; row += 256 / TPR) {
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < parts; ++i) sum += *reinterpret_cast<const f32x4 *>(from + ((int64_t)i * 2 * s.kb + row) * D + c);
    const bool is_v = row >= s.kb;
    const int n = j * s.kb + (is_v ? row - s.kb : row);
    if (n >= s.Nk) continue;
    const View &to = is_v ? a.dv : a.dk;
    if (!is_v) sum *= a.scale;
    const int64_t i = b * to.sb + hk * to.sh + n * to.sn + c;
    if constexpr (F32) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(to.p) + i) = sum;
    else *reinterpret_cast<bf16x4 *>(reinterpret_cast<__bf16 *>(to.p) + i) = __builtin_convertvector(sum, bf16x4);
  }
}

struct GradPlanS {
  int n_chunks, max_items, max_slots;
  size_t off_q, off_k, off_v, off_do, off_lse2, off_delta, off_hist, off_first, off_item0, off_slot0, off_inv, off_item, off_part, total;
};

GradPlanS plan_grad(const ha_sparse_problem &p, const Sparse &s) {
  GradPlanS f{};
  const int64_t entries = (int64_t)s.T * s.sel;
  f.n_chunks = (s.T + kChunk - 1) / kChunk;
  // ceil(n_j / kPart) parts of block j: over all blocks at most entries / kPart + Tk; those of blocks with several, of which there are
  // fewer than entries / kPart, at most 2 entries / kPart
  f.max_items = (int)(entries / kPart) + s.Tk;
  f.max_slots = (int)(2 * (entries / kPart));
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
  f.off_lse2 = take((size_t)s.B * s.H * s.T * s.qb * 4);
  f.off_delta = take((size_t)s.B * s.H * s.T * s.qb * 4);
  f.off_hist = take(hk * f.n_chunks * s.Tk * 4);
  f.off_first = take(hk * (s.Tk + 1) * 4);
  f.off_item0 = take(hk * (s.Tk + 1) * 4);
  f.off_slot0 = take(hk * (s.Tk + 1) * 4);
  f.off_inv = take(hk * entries * 4);
  f.off_item = take(hk * f.max_items * 4);
  f.off_part = take(hk * f.max_slots * 2 * s.kb * p.d_head * 4);
  f.total = at;
  if ((int64_t)hk * f.max_items > (1 << 30)) f.total = 0;      // (more workgroups than a launch is given)
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
    else sparse_dq_kernel<D, F32, 2><<<8 * a.share, 128, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (s.Nk > 0) {
    a.items = (unsigned)((int64_t)s.B * s.Hkv * a.max_items);
    a.share = xcd_share(a.items);
    if (s.kb == 128) sparse_dkv_kernel<D, F32, 4><<<8 * a.share, 256, 0, st>>>(a);
    else sparse_dkv_kernel<D, F32, 2><<<8 * a.share, 128, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.max_slots > 0) {
      sparse_dkv_join_kernel<D, F32><<<(unsigned)((int64_t)s.B * s.Hkv * s.Tk), 256, 0, st>>>(a);
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
  if (p->N_q > 0 && f.total == 0) return HA_ERR_UNSUPPORTED;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < f.total) return HA_ERR_WORKSPACE;
  if (p->N_q == 0 && p->N_k == 0) return HA_OK;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(workspace);
  const int d = p->d_head;
  const bool f32 = p->dtype == HA_F32;
  float *lse2 = reinterpret_cast<float *>(ws + f.off_lse2), *delta = reinterpret_cast<float *>(ws + f.off_delta);
  hipError_t e;
  if (s.Nq > 0) {
    const int rpb = 256 / (d / 8);
    const unsigned n = (unsigned)(((int64_t)s.B * s.H * s.T * s.qb + rpb - 1) / rpb);
    if (d == 128) { if (f32) sparse_delta_kernel<128, true><<<n, 256, 0, stream>>>(s, o, a.dout, lse, lse2, delta); else sparse_delta_kernel<128, false><<<n, 256, 0, stream>>>(s, o, a.dout, lse, lse2, delta); }
    else { if (f32) sparse_delta_kernel<64, true><<<n, 256, 0, stream>>>(s, o, a.dout, lse, lse2, delta); else sparse_delta_kernel<64, false><<<n, 256, 0, stream>>>(s, o, a.dout, lse, lse2, delta); }
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
  a.lse2 = lse2;
  a.delta = delta;
  a.hist = reinterpret_cast<int32_t *>(ws + f.off_hist);
  a.first = reinterpret_cast<int32_t *>(ws + f.off_first);
  a.item0 = reinterpret_cast<int32_t *>(ws + f.off_item0);
  a.slot0 = reinterpret_cast<int32_t *>(ws + f.off_slot0);
  a.inv = reinterpret_cast<int32_t *>(ws + f.off_inv);
  a.item_block = reinterpret_cast<int32_t *>(ws + f.off_item);
  a.part = reinterpret_cast<float *>(ws + f.off_part);
  a.n_chunks = f.n_chunks;
  a.max_items = f.max_items;
  a.max_slots = f.max_slots;
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
    if (f.n_chunks > 0) {
      inverse_fill_kernel<<<dim3(f.n_chunks, heads), 256, 0, stream>>>(a);
      if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
    }
  }
  if (d == 128) e = f32 ? launch_grad<128, true>(*p, a, stream) : launch_grad<128, false>(*p, a, stream);
  else e = f32 ? launch_grad<64, true>(*p, a, stream) : launch_grad<64, false>(*p, a, stream);
  return e == hipSuccess ? HA_OK : device_error(e);
}
