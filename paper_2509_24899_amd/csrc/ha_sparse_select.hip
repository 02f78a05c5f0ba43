// Block-sparse attention, gfx950: checks of its arguments, block means of the keys, and the choice of key blocks for every tile of queries.
//
//   mean_j = sum of the keys of block j / their number        score_tj = (sum of the queries of tile t over its heads) . mean_j
//
// Everything that decides is formed in double (in fp32 about one list in ten thousand changed with the order of summation).  The sums of 64 or 128 bf16 values
// are exact there, sums of fp32 values are not, and a score is a sum of d products rounded in double: scores that are closer than some 1e-15 of their terms
// may stand in either order, and rank by index only where the doubles are equal.  A list is the same bit for bit for one problem; the two ways of forming the
// scores (few_tiles) sum in different orders, so that such near ties may fall otherwise where the number of tiles is another.  The sums over q and k are bound by
// memory (12 heads of 32760 x 128 bf16, 100 MB: 20 us for keys and 20 for queries, 5 TB/s); the scores of 128 queries against a block of 64 keys take one
// product of d values.
#include <climits>
#include <cmath>

#include "ha_sparse.h"

namespace ha {

ha_status check_sparse(const ha_sparse_problem *p) {
  if (!p) return HA_ERR_NULL;
  if (p->B <= 0 || p->H <= 0 || p->H_kv <= 0 || p->N_q < 0 || p->N_k < 0 || p->d_head <= 0) return HA_ERR_SHAPE;
  if (p->H % p->H_kv || p->n_select < 1 || p->keep_first < 0 || p->near_tokens < -1) return HA_ERR_SHAPE;
  if (p->causal != 0 && p->causal != 1) return HA_ERR_SHAPE;
  if (!(p->softmax_scale >= 1e-30f && p->softmax_scale <= 1e30f)) return HA_ERR_SHAPE;      // (its reciprocal, and logits times it, are finite)
  if (p->dtype != HA_BF16 && p->dtype != HA_F32) return HA_ERR_UNSUPPORTED;
  if (p->d_head != 64 && p->d_head != 128) return HA_ERR_UNSUPPORTED;
  if ((p->q_block != 64 && p->q_block != 128) || (p->k_block != 64 && p->k_block != 128)) return HA_ERR_UNSUPPORTED;
  if ((int64_t)p->B * p->H > 65535 || p->N_q > (1 << 24) || p->N_k > (1 << 29) || p->n_select > (1 << 20) || p->near_tokens > (1 << 29)) return HA_ERR_UNSUPPORTED;
  const int64_t T = (p->N_q + p->q_block - 1) / p->q_block, Tk = (p->N_k + p->k_block - 1) / p->k_block, B = p->B;
  // (a launch takes 2^32 - 1 threads, 256 to a tile, a key block or 16 rows, and an index into one head's lists 31 bits)
  if (B * p->H * T > (1 << 20) || B * p->H_kv * Tk > (1 << 23) || T * p->n_select > (1 << 30)) return HA_ERR_UNSUPPORTED;
  if (reinterpret_cast<uintptr_t>(p->q_start) & 3u || reinterpret_cast<uintptr_t>(p->key_len) & 3u) return HA_ERR_ALIGN;
  return HA_OK;
}

ha_status check_view(const ha_sparse_problem &p, const ha_view *v, int heads, int n, int block, bool written, View &out) {
  if (!v) return HA_ERR_NULL;
  out = View{static_cast<char *>(v->data), v->stride_b, v->stride_h, v->stride_n};
  if (n == 0) return HA_OK;
  if (!v->data) return HA_ERR_NULL;
  const int esz = p.dtype == HA_BF16 ? 2 : 4, per16 = 16 / esz;
  if (n == 1) out.sn = p.d_head;
  if (heads == 1) out.sh = n * out.sn;
  if (p.B == 1) out.sb = heads * out.sh;
  if (out.sn < p.d_head || out.sh < 0 || out.sb < 0) return HA_ERR_SHAPE;
  if (written && (out.sh < p.d_head || out.sb < p.d_head)) return HA_ERR_SHAPE;
  if (out.sn > ((int64_t)1 << 31) / esz / (block + 1) || out.sh > (int64_t)1 << 44 || out.sb > (int64_t)1 << 44) return HA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(v->data) & 15u || out.sn % per16 || out.sh % per16 || out.sb % per16) return HA_ERR_ALIGN;
  return HA_OK;
}

Sparse sparse_of(const ha_sparse_problem &p) {
  return Sparse{p.B, p.H, p.H_kv, p.H / p.H_kv, p.N_q, p.N_k, (p.N_q + p.q_block - 1) / p.q_block, (p.N_k + p.k_block - 1) / p.k_block,
                p.q_block, p.k_block, p.n_select, p.causal, p.q_start, p.key_len};
}

namespace {

// ---- sums over rows ----------------------------------------------------------------------------------------------------
// Sum of rows [0, n) of up to 128 of one head, as 256 threads: D / 8 threads to a row, each eight columns.  acc is added to.
template <int D, bool F32>
__device__ __forceinline__ void add_rows(const char *base, int64_t stride, int n, double (&acc)[8]) {
  constexpr int TPR = D / 8, RPP = 256 / TPR;
  const int c = threadIdx.x % TPR, r0 = threadIdx.x / TPR;
#pragma unroll 4
  for (int r = r0; r < n; r += RPP) {
    if constexpr (F32) {
      const f32x4 *p = reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(base) + (int64_t)r * stride + 8 * c);
      const f32x4 x = p[0], y = p[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[i] += (double)x[i];
        acc[4 + i] += (double)y[i];
      }
    } else {
      const bf16x8 x = *reinterpret_cast<const bf16x8 *>(reinterpret_cast<const __bf16 *>(base) + (int64_t)r * stride + 8 * c);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += (double)static_cast<float>(x[i]);
    }
  }
}
// Joins the partial sums of the workgroup's row groups; thread t < D returns column t.
template <int D>
__device__ __forceinline__ double join_rows(const double (&acc)[8], double *lds) {
  constexpr int TPR = D / 8, RPP = 256 / TPR;
#pragma unroll
  for (int i = 0; i < 8; ++i) lds[(threadIdx.x / TPR) * (D + 1) + 8 * (threadIdx.x % TPR) + i] = acc[i];
  __syncthreads();
  double s = 0.;
  if (threadIdx.x < D)
    for (int r = 0; r < RPP; ++r) s += lds[r * (D + 1) + threadIdx.x];
  return s;
}

template <int D, bool F32>
__global__ __launch_bounds__(256) void key_means_kernel(Sparse s, View k, int only_last, int n_j, float *means) {
  __shared__ double lds[(256 / (D / 8)) * (D + 1)];
  const int bh = blockIdx.x / n_j, b = bh / s.Hkv, h = bh % s.Hkv, held = s.held(b);
  int j = blockIdx.x % n_j;
  if (only_last > 0) {
    j += (held + s.kb - 1) / s.kb - n_j;
    if (j < 0) return;
  }
  const int n = min(held - j * s.kb, s.kb);
  double acc[8] = {0., 0., 0., 0., 0., 0., 0., 0.};
  constexpr int ESZ = F32 ? 4 : 2;
  if (n > 0) add_rows<D, F32>(k.p + (b * k.sb + h * k.sh + (int64_t)j * s.kb * k.sn) * ESZ, k.sn, n, acc);
  const double sum = join_rows<D>(acc, lds);
  if (threadIdx.x < D) means[((int64_t)bh * s.Tk + j) * D + threadIdx.x] = (float)(n > 0 ? sum / n : 0.);
}

// Sum of a tile's queries over the heads that share the choice: double [B * Hkv * T][D].
template <int D, bool F32>
__global__ __launch_bounds__(256) void query_sums_kernel(Sparse s, View q, double *sums) {
  __shared__ double lds[(256 / (D / 8)) * (D + 1)];
  const int row = blockIdx.x, t = row % s.T, bh = row / s.T, b = bh / s.Hkv, h = bh % s.Hkv;
  const int n = min(s.Nq - t * s.qb, s.qb);
  double acc[8] = {0., 0., 0., 0., 0., 0., 0., 0.};
  constexpr int ESZ = F32 ? 4 : 2;
  for (int i = 0; i < s.G; ++i) add_rows<D, F32>(q.p + (b * q.sb + (int64_t)(h * s.G + i) * q.sh + (int64_t)t * s.qb * q.sn) * ESZ, q.sn, n, acc);
  const double sum = join_rows<D>(acc, lds);
  if (threadIdx.x < D) sums[(int64_t)row * D + threadIdx.x] = sum;
}

// Order of doubles as that of unsigned integers (NaN above all); 0 is kept for blocks that may not be chosen.
__device__ __forceinline__ uint64_t ordered(double x) {
  if (x != x) return ~(uint64_t)0 - 1;
  const uint64_t u = __double_as_longlong(x + 0.);     // (-0 as 0)
  return (u >> 63) ? ~u : u | ((uint64_t)1 << 63);
}

struct ScoreArgs {
  Sparse s;
  View q;
  double *sums;
  const float *means;
  uint64_t *keys;
  int32_t *blocks;
  int keep_first, near_tokens;
};
// Key of block j for tile t: its score's order, all ones where the block is always kept, 0 where it may not be chosen.
__device__ __forceinline__ uint64_t rank_key(const ScoreArgs &a, int held, int start, int t, int j, double score) {
  const Sparse &s = a.s;
  const int lo_key = j * s.kb, hi_key = lo_key + s.kb - 1, lo = start + t * s.qb, hi = start + min((t + 1) * s.qb, s.Nq) - 1;
  uint64_t key = ordered(score);
  if (j < a.keep_first || (a.near_tokens >= 0 && hi_key >= lo - a.near_tokens && lo_key <= hi + (s.causal ? 0 : a.near_tokens))) key = ~(uint64_t)0;
  if (lo_key >= held || (s.causal && lo_key > hi)) key = 0;
  return key;
}

// Scores of kTiles tiles against 16 blocks by one wave on the fp64 matrix cores: lane l holds the sums of tile l % 16 (rows) and the mean of block l % 16
// (columns) at columns 16 i + 4 (l / 16) + u of every 16, the contraction's k of product (i, u); register v of the result is tile 4 v + l / 16,
// block l % 16.  (As vector products the sums came from LDS for every block, and that bound it: 22 us for 15 at 256 tiles by 512 blocks of 12 heads.)
constexpr int kTiles = 16;
constexpr int kFusedBlocks = 1024;     // keys of kTiles tiles that fit LDS
constexpr int kRowBlocks = 256;        // keys of a tile that one wave holds in four registers: one launch (4 x 256: 7.4 us for 11.5 in two, 256 x 256: 8.1 for 17.9)
typedef double f64x4 __attribute__((ext_vector_type(4)));
template <int D>
__device__ __forceinline__ void load_sums(const ScoreArgs &a, int bh, int t0, int lane, f64x4 (&q)[D / 16]) {
  const int t = min(t0 + (lane & 15), a.s.T - 1);
  const f64x4 *p = reinterpret_cast<const f64x4 *>(a.sums + ((int64_t)bh * a.s.T + t) * D) + (lane >> 4);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) q[i] = p[4 * i];
}
template <int D>
__device__ __forceinline__ void load_means(const ScoreArgs &a, int bh, int j0, int lane, f32x4 (&m)[D / 16]) {
  const f32x4 *p = reinterpret_cast<const f32x4 *>(a.means + ((int64_t)bh * a.s.Tk + min(j0 + (lane & 15), a.s.Tk - 1)) * D) + (lane >> 4);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) m[i] = p[4 * i];
}
template <int D>
__device__ __forceinline__ f64x4 scores_of_blocks(const f32x4 (&m)[D / 16], const f64x4 (&q)[D / 16]) {
  f64x4 c[2] = {{0., 0., 0., 0.}, {0., 0., 0., 0.}};
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int u = 0; u < 4; ++u) c[u & 1] = __builtin_amdgcn_mfma_f64_16x16x4f64(q[i][u], (double)m[i][u], c[u & 1], 0, 0, 0);
  return c[0] + c[1];
}
// Every wave of WAVES its groups of 16 blocks of [lo, hi); done(j0, scores).
template <int D, int WAVES, typename Done>
__device__ __forceinline__ void score_range(const ScoreArgs &a, int bh, int lo, int hi, int w, int lane, const f64x4 (&q)[D / 16], Done done) {
  for (int j0 = lo + 16 * w; j0 < hi; j0 += 16 * WAVES) {
    f32x4 m[D / 16];
    load_means<D>(a, bh, j0, lane, m);
    done(j0, scores_of_blocks<D>(m, q));
  }
}

// Very many blocks: the keys go through memory, [rows][Tk].
template <int D>
__global__ __launch_bounds__(512) void scores_kernel(ScoreArgs a) {
  const Sparse &s = a.s;
  const int bh = blockIdx.z, b = bh / s.Hkv, t0 = blockIdx.x * kTiles, lane = threadIdx.x & 63, held = s.held(b), start = s.start(b);
  f64x4 q[D / 16];
  load_sums<D>(a, bh, t0, lane, q);
  score_range<D, 8>(a, bh, blockIdx.y * 1024, min(s.Tk, (int)(blockIdx.y + 1) * 1024), threadIdx.x >> 6, lane, q, [&](int j0, f64x4 score) {
    const int j = j0 + (lane & 15);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int t = t0 + 4 * v + (lane >> 4);
      if (t < s.T && j < s.Tk) a.keys[((int64_t)bh * s.T + t) * s.Tk + j] = rank_key(a, held, start, t, j, score[v]);
    }
  });
}

// ---- the choice ------------------------------------------------------------------------------------------------------
// A list is the blocks whose keys reach a threshold: the largest that at least n_select keys reach is found bit by bit from the top (the search ends as
// soon as exactly n_select do), then the blocks are written in rising order.  If more reach it, it is the n_select-th largest key itself, and of
// the blocks whose keys equal it the first are taken.
// One wave, with the keys of blocks l, l + 64, .. in lane l.  The upper halves of the keys decide almost always; the lower ones are looked at where they do not.
template <int V>
__device__ __forceinline__ void choose_wave(const uint64_t *keys, int sel, int32_t *out, int lane) {
  uint32_t hi[V], lo[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint64_t k = keys[64 * i + lane];
    hi[i] = (uint32_t)(k >> 32);
    lo[i] = (uint32_t)k;
  }
  auto reach = [&](uint32_t y) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) c += __popcll(__ballot(hi[i] >= y));
    return c;
  };
  uint32_t x = 1, y = 0;                // the threshold's halves (a key that may be chosen has an upper half of 1 or more)
  int n = reach(1);                     // keys that reach it
  if (n > sel) {
    // Every lane's largest key reaches the smallest of these, so that at least 64 keys do: the threshold lies between it and the largest key of all, and what
    // the two have in common (sign and most of the exponent, as a rule) need not be searched.
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) most = max(most, hi[i]);
    uint32_t least = sel <= 64 ? most : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      most = max(most, (uint32_t)__shfl_xor(most, d));
      least = min(least, (uint32_t)__shfl_xor(least, d));
    }
    most = __builtin_amdgcn_readfirstlane(most);
    least = __builtin_amdgcn_readfirstlane(least);
    const int bits = most == least ? 0 : 32 - __builtin_clz(most ^ least);
    x = bits == 32 ? 0 : most >> bits << bits;
    n = INT_MAX;
    for (int bit = bits - 1; bit >= 0 && n != sel; --bit) {
      const int c = reach(x | 1u << bit);
      if (c >= sel) {
        x |= 1u << bit;
        n = c;
      }
    }
    if (n == INT_MAX) n = reach(x);
    if (n > sel) {
      const int above = x == ~0u ? 0 : reach(x + 1);
      for (int bit = 31; bit >= 0 && n != sel; --bit) {
        int c = above;
#pragma unroll
        for (int i = 0; i < V; ++i) c += __popcll(__ballot(hi[i] == x && lo[i] >= (y | 1u << bit)));
        if (c >= sel) {
          y |= 1u << bit;
          n = c;
        }
      }
    }
  }
  // more than sel reach it: it is the sel-th largest key itself, and of the blocks whose keys equal it the first are taken
  const bool ties = n > sel;
  const uint64_t cut = (uint64_t)x << 32 | y;
  int equal_left = 0, at = 0;
  if (ties) {
    equal_left = sel;
#pragma unroll
    for (int i = 0; i < V; ++i) equal_left -= __popcll(__ballot(((uint64_t)hi[i] << 32 | lo[i]) > cut));
  }
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint64_t k = (uint64_t)hi[i] << 32 | lo[i];
    const bool eq = ties && k == cut, over = ties ? k > cut : k >= cut;
    const uint64_t m_eq = __ballot(eq), m_over = __ballot(over);
    const int eq_before = __popcll(m_eq & below), place = at + __popcll(m_over & below) + min(eq_before, equal_left);
    if (over || (eq && eq_before < equal_left)) out[place] = i * 64 + lane;
    const int taken = min((int)__popcll(m_eq), equal_left);
    at += __popcll(m_over) + taken;
    equal_left -= taken;
  }
  for (int i = at + lane; i < sel; i += 64) out[i] = -1;
}

// Many tiles: a workgroup scores kTiles of them against all blocks (at most 64 V), then every wave makes one tile's choice.  26 us at 256 tiles x 512 blocks
// of 12 heads (480p), 15 of them the scores: 192 workgroups, one to a CU, each a chain of loads, products, barrier and search, matrix cores busy 28 % of the cycles.
// Sixteen waves take all registers of a CU, so that no second workgroup runs beside one: 591 tiles x 591 blocks of 24 heads (720p with guidance), 888 workgroups,
// are four rounds of such chains, 111 us, matrix cores busy 31 %.
template <int D, int V>
__global__ __launch_bounds__(1024) void score_and_choose_kernel(ScoreArgs a) {
  const Sparse &s = a.s;
  __shared__ uint64_t keys[kTiles][64 * V];
  const int bh = blockIdx.y, b = bh / s.Hkv, t0 = blockIdx.x * kTiles, lane = threadIdx.x & 63, w = threadIdx.x >> 6, held = s.held(b), start = s.start(b);
  {
    f64x4 q[D / 16];
    load_sums<D>(a, bh, t0, lane, q);
    const int last = (s.Tk + 15) & ~15;
    score_range<D, 16>(a, bh, 0, last, w, lane, q, [&](int j0, f64x4 score) {
      const int j = j0 + (lane & 15);
#pragma unroll
      for (int v = 0; v < 4; ++v) keys[4 * v + (lane >> 4)][j] = j < s.Tk ? rank_key(a, held, start, t0 + 4 * v + (lane >> 4), j, score[v]) : 0;
    });
    for (int i = threadIdx.x; i < kTiles * (64 * V - last); i += 1024) keys[i % kTiles][last + i / kTiles] = 0;
  }
  __syncthreads();
  if (t0 + w < s.T) choose_wave<V>(keys[w], s.sel, a.blocks + ((int64_t)bh * s.T + t0 + w) * s.sel, lane);
}

// Few tiles.  A workgroup of WAVES waves forms the keys of one tile for blocks [lo, hi) from its queries on: their sum, then the scores, a block's mean to
// eight lanes.  `part` is WAVES rows of D doubles.
template <int D, bool F32, int WAVES>
__device__ __forceinline__ void keys_of_tile(const ScoreArgs &a, int row, int lo, int hi, double (*part)[D], uint64_t *keys) {
  const Sparse &s = a.s;
  constexpr int TPR = D / 8, LPM = 8, PER = D / 32, ESZ = F32 ? 4 : 2, AT_ONCE = WAVES * 64 / LPM;
  const int t = row % s.T, bh = row / s.T, b = bh / s.Hkv, h = bh % s.Hkv, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int held = s.held(b), start = s.start(b), n_rows = min(s.Nq - t * s.qb, s.qb);
  double acc[8] = {0., 0., 0., 0., 0., 0., 0., 0.};
  {
    const int c = threadIdx.x % TPR, total = s.G * n_rows;
    for (int i = threadIdx.x / TPR; i < total; i += WAVES * 64 / TPR) {
      const int hd = i / n_rows;
      const char *p = a.q.p + (b * a.q.sb + (int64_t)(h * s.G + hd) * a.q.sh + (int64_t)(t * s.qb + i - hd * n_rows) * a.q.sn + 8 * c) * ESZ;
      if constexpr (F32) {
        const f32x4 x = reinterpret_cast<const f32x4 *>(p)[0], y = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          acc[u] += (double)x[u];
          acc[4 + u] += (double)y[u];
        }
      } else {
        const bf16x8 x = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[u] += (double)static_cast<float>(x[u]);
      }
    }
#pragma unroll
    for (int d = TPR; d < 64; d <<= 1)
#pragma unroll
      for (int u = 0; u < 8; ++u) acc[u] += __shfl_xor(acc[u], d);
    if (lane < TPR)
#pragma unroll
      for (int u = 0; u < 8; ++u) part[w][8 * c + u] = acc[u];
    __syncthreads();
    if (threadIdx.x < D) {
      double sum = part[0][threadIdx.x];
#pragma unroll
      for (int i = 1; i < WAVES; ++i) sum += part[i][threadIdx.x];
      part[0][threadIdx.x] = sum;       // (its own column: nobody else reads it before the barrier)
    }
    __syncthreads();
  }
  const int c = lane % LPM;
  double q[PER][4];
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int u = 0; u < 4; ++u) q[i][u] = part[0][32 * i + 4 * c + u];
  for (int j0 = lo; j0 < hi; j0 += AT_ONCE) {
    const int j = j0 + (int)threadIdx.x / LPM;
    const float *mean = a.means + ((int64_t)bh * s.Tk + min(j, s.Tk - 1)) * D + 4 * c;
    f32x4 x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = *reinterpret_cast<const f32x4 *>(mean + 32 * i);
    double score = 0.;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) score = __builtin_fma((double)x[i][u], q[i][u], score);
#pragma unroll
    for (int d = 1; d < LPM; d <<= 1) score += __shfl_xor(score, d);
    if (c == 0 && j < hi) keys[j] = rank_key(a, held, start, t, j, score);
  }
}

// Up to 256 blocks: the whole choice of a tile in one launch.
template <int D, bool F32>
__global__ __launch_bounds__(512) void choose_row_kernel(ScoreArgs a) {
  __shared__ double part[8][D];
  __shared__ uint64_t keys[kRowBlocks];
  if (threadIdx.x < kRowBlocks && (int)threadIdx.x >= a.s.Tk) keys[threadIdx.x] = 0;
  keys_of_tile<D, F32, 8>(a, blockIdx.x, 0, a.s.Tk, part, keys);
  __syncthreads();
  if (threadIdx.x < 64) choose_wave<kRowBlocks / 64>(keys, a.s.sel, a.blocks + (int64_t)blockIdx.x * a.s.sel, threadIdx.x);
}

// More: the means are many, so that a workgroup takes 128 of them, and a second launch makes the choice.
template <int D, bool F32>
__global__ __launch_bounds__(1024) void keys_kernel(ScoreArgs a) {
  __shared__ double part[16][D];
  keys_of_tile<D, F32, 16>(a, blockIdx.y, blockIdx.x * 128, min(a.s.Tk, (int)(blockIdx.x + 1) * 128), part, a.keys + (int64_t)blockIdx.y * a.s.Tk);
}
template <int V>
__global__ __launch_bounds__(64) void choose_list_kernel(const uint64_t *keys, int Tk, int sel, int32_t *blocks) {
  __shared__ uint64_t k[64 * V];
  const int64_t row = blockIdx.x;
#pragma unroll
  for (int i = 0; i < V; ++i) k[64 * i + threadIdx.x] = 64 * i + (int)threadIdx.x < Tk ? keys[row * Tk + 64 * i + threadIdx.x] : 0;
  choose_wave<V>(k, sel, blocks + row * sel, threadIdx.x);       // (every lane reads what it wrote)
}

// Very many blocks: 256 threads to a list, keys read from memory for every bit.
__global__ __launch_bounds__(256) void choose_kernel(const uint64_t *all_keys, int Tk, int sel, int32_t *blocks) {
  __shared__ int count[2][4], chosen[2][2][4];
  const int64_t row = blockIdx.x;
  const uint64_t *keys = all_keys + row * Tk;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, rounds = (Tk + 255) / 256;
  auto key = [&](int i) { return i * 256 + (int)threadIdx.x < Tk ? keys[i * 256 + threadIdx.x] : 0; };
  int turn = 0;
  auto reach = [&](uint64_t x) {
    int c = 0;
    for (int i = 0; i < rounds; ++i) c += __popcll(__ballot(key(i) >= x));
    if (lane == 0) count[turn][w] = c;
    __syncthreads();
    c = count[turn][0] + count[turn][1] + count[turn][2] + count[turn][3];
    turn ^= 1;
    return c;
  };
  uint64_t x = 1;
  int n = reach(1);
  if (n > sel) {
    x = 0;
    for (int bit = 63; bit >= 0 && n != sel; --bit) {
      const uint64_t y = x | (uint64_t)1 << bit;
      const int c = reach(y);
      if (c >= sel) {
        x = y;
        n = c;
      }
    }
  }
  const bool ties = n > sel;
  int equal_left = ties ? sel - (x == ~(uint64_t)0 ? 0 : reach(x + 1)) : 0, at = 0;
  int32_t *out = blocks + row * sel;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int i = 0; i < rounds; ++i) {
    const uint64_t k = key(i);
    const bool eq = ties && k == x, over = ties ? k > x : k >= x;
    const uint64_t m_eq = __ballot(eq), m_over = __ballot(over);
    if (lane == 0) {
      chosen[i & 1][0][w] = __popcll(m_eq);
      chosen[i & 1][1][w] = __popcll(m_over);
    }
    __syncthreads();
    int eq_before = 0, over_before = 0, eq_all = 0, over_all = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = chosen[i & 1][0][u], o = chosen[i & 1][1][u];
      if (u < w) {
        eq_before += e;
        over_before += o;
      }
      eq_all += e;
      over_all += o;
    }
    eq_before += __popcll(m_eq & below);
    over_before += __popcll(m_over & below);
    if (over || (eq && eq_before < equal_left)) out[at + over_before + min(eq_before, equal_left)] = i * 256 + threadIdx.x;
    const int taken = min(eq_all, equal_left);
    at += over_all + taken;
    equal_left -= taken;
  }
  for (int i = at + threadIdx.x; i < sel; i += 256) out[i] = -1;
}

// ---- fp32 tensors as three bf16 images -----------------------------------------------------------------------------------
// One pass at the rate of memory: 4 bytes of a value read, 6 written (30 M values 49 us, 6.3 TB/s).
struct SplitJobs {
  SplitJob job[4];
  unsigned end[4];                      // how many groups of rows up to this job's
};
template <int D>
__global__ __launch_bounds__(256) void split_kernel(Sparse s, SplitJobs jobs) {
  constexpr int TPR = D / 8, RPB = 256 / TPR;
  int at = 0;
  for (unsigned i = blockIdx.x; i < jobs.end[3]; i += gridDim.x) {
    while (i >= jobs.end[at]) ++at;
    const SplitJob &j = jobs.job[at];
    const int64_t row = (int64_t)(i - (at ? jobs.end[at - 1] : 0)) * RPB + threadIdx.x / TPR, rows = (int64_t)s.B * j.heads * j.n;
    if (row >= rows) continue;
    const int c = 8 * (threadIdx.x % TPR), n = (int)(row % j.n), h = (int)(row / j.n % j.heads), b = (int)(row / j.n / j.heads);
    const f32x4 *p = reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(j.in.p) + b * j.in.sb + h * j.in.sh + n * j.in.sn + c);
    bf16x8 out[3];
    split8_any(p[0], p[1], out);
#pragma unroll
    for (int p3 = 0; p3 < 3; ++p3) *reinterpret_cast<bf16x8 *>(j.out + (p3 * rows + row) * D + c) = out[p3];
  }
}

size_t sums_bytes(const Sparse &s, int d) { return round256((size_t)s.B * s.Hkv * s.T * d * 8); }

// Few tiles make their choice from the queries on, a workgroup or several each; many share passes over the means.  Us at d = 128, sixteen of the blocks:
//   tiles x blocks      4 x 16  512 x 16  256 x 256  1024 x 256  4096 x 240  |  4 x 500  128 x 500  256 x 500  512 x 500  256 x 940
//   on their own           4.5       6.1        8.1        17.6        55.3  |     11.0       17.2       26.5       43.1       42.0
//   sums and scores        7.2       9.0       21.4        25.2        38.9  |     19.1       27.8       27.6       28.1       38.8
bool few_tiles(const Sparse &s) { return (int64_t)s.B * s.Hkv * s.T <= (s.Tk <= kRowBlocks ? 1024 : 128); }

// The choice from keys in memory: a wave that holds them where they are up to 2048.
void launch_choose(const Sparse &s, const uint64_t *keys, int32_t *blocks, hipStream_t st) {
  const unsigned rows = (unsigned)s.B * s.Hkv * s.T;
  if (s.Tk <= 1024) choose_list_kernel<16><<<rows, 64, 0, st>>>(keys, s.Tk, s.sel, blocks);
  else if (s.Tk <= 2048) choose_list_kernel<32><<<rows, 64, 0, st>>>(keys, s.Tk, s.sel, blocks);
  else choose_kernel<<<rows, 256, 0, st>>>(keys, s.Tk, s.sel, blocks);
}

// Whether a list holds the blocks that are always kept.  A count that no place of the tiles exceeds decides first; where it does not fit and the places are
// known (q_start lies on the device), the blocks of every tile are counted.
bool holds_kept_blocks(const ha_sparse_problem &p) {
  const int64_t kb = p.k_block, Tk = (p.N_k + kb - 1) / kb, before = p.near_tokens, behind = p.causal ? 0 : p.near_tokens;
  if (p.n_select >= Tk) return true;
  int64_t most = p.keep_first;
  if (p.near_tokens >= 0) most += ((p.N_q < p.q_block ? p.N_q : p.q_block) + before + behind - 1 + kb - 1) / kb + 1;
  if (most <= p.n_select) return true;
  if (p.q_start) return false;
  auto block = [&](int64_t key) { return key >= 0 ? key / kb : -((-key + kb - 1) / kb); };
  for (int64_t i = 0; i < p.N_q; i += p.q_block) {
    const int64_t lo = (int64_t)p.N_k - p.N_q + i, hi = lo + (p.N_q - i < p.q_block ? p.N_q - i : p.q_block) - 1;      // the tile's positions
    const int64_t last = p.causal && block(hi) < Tk - 1 ? block(hi) : Tk - 1;                                      // the last block that it may see
    const int64_t first_kept = p.keep_first < last + 1 ? p.keep_first : last + 1;
    int64_t n = first_kept > 0 ? first_kept : 0;
    if (p.near_tokens >= 0) {
      const int64_t from = block(lo - before) > n ? block(lo - before) : n, to = block(hi + behind) < last ? block(hi + behind) : last;
      if (to >= from) n += to - from + 1;
    }
    if (n > p.n_select) return false;
  }
  return true;
}

}  // namespace

hipError_t launch_split(const Sparse &s, int d, const SplitJob *jobs, int n_jobs, hipStream_t st) {
  SplitJobs all{};
  unsigned blocks = 0;
  const int rpb = 256 / (d / 8);
  for (int i = 0; i < 4; ++i) {
    if (i < n_jobs) {
      all.job[i] = jobs[i];
      blocks += (unsigned)(((int64_t)s.B * jobs[i].heads * jobs[i].n + rpb - 1) / rpb);
    }
    all.end[i] = blocks;
  }
  if (blocks == 0) return hipSuccess;
  if (blocks > 1 << 23) blocks = 1 << 23;
  if (d == 128) split_kernel<128><<<blocks, 256, 0, st>>>(s, all);
  else split_kernel<64><<<blocks, 256, 0, st>>>(s, all);
  return hipGetLastError();
}

}  // namespace ha

using namespace ha;

extern "C" ha_status hybrid_attn_sparse_validate(const ha_sparse_problem *p) { return check_sparse(p); }

extern "C" ha_status hybrid_attn_key_means(const ha_sparse_problem *p, const ha_view *k, int32_t only_last, float *means, void *hip_stream) {
  ha_status st = check_sparse(p);
  if (st != HA_OK) return st;
  View kv;
  if ((st = check_view(*p, k, p->H_kv, p->N_k, p->k_block, false, kv)) != HA_OK) return st;
  if (only_last < 0) return HA_ERR_SHAPE;
  if (p->N_k == 0) return HA_OK;
  if (!means) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(means) & 15u) return HA_ERR_ALIGN;
  const Sparse s = sparse_of(*p);
  const int n_j = only_last > 0 && only_last < s.Tk ? only_last : s.Tk;
  const unsigned blocks = (unsigned)s.B * s.Hkv * n_j;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
#define HA_MEANS(D, F) key_means_kernel<D, F><<<blocks, 256, 0, stream>>>(s, kv, only_last, n_j, means)
  if (p->d_head == 128) { if (p->dtype == HA_F32) HA_MEANS(128, true); else HA_MEANS(128, false); }
  else { if (p->dtype == HA_F32) HA_MEANS(64, true); else HA_MEANS(64, false); }
#undef HA_MEANS
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? HA_OK : device_error(e);
}

extern "C" size_t hybrid_attn_select_workspace_bytes(const ha_sparse_problem *p) {
  if (check_sparse(p) != HA_OK) return 0;
  const Sparse s = sparse_of(*p);
  if (few_tiles(s) && s.Tk <= kRowBlocks) return 0;
  return sums_bytes(s, p->d_head) + (!few_tiles(s) && s.Tk <= kFusedBlocks ? 0 : round256((size_t)s.B * s.Hkv * s.T * s.Tk * 8));
}

extern "C" ha_status hybrid_attn_select_blocks(const ha_sparse_problem *p, const ha_view *q, const float *means, int32_t *blocks, void *workspace,
                                               size_t workspace_bytes, void *hip_stream) {
  ha_status st = check_sparse(p);
  if (st != HA_OK) return st;
  View qv;
  if ((st = check_view(*p, q, p->H, p->N_q, p->q_block, false, qv)) != HA_OK) return st;
  const Sparse s = sparse_of(*p);
  if (p->causal && p->near_tokens < 0) return HA_ERR_SHAPE;
  if (!holds_kept_blocks(*p)) return HA_ERR_SHAPE;
  if (p->N_q == 0) return HA_OK;
  if (!blocks || (p->N_k > 0 && !means)) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(means) & 15u || reinterpret_cast<uintptr_t>(blocks) & 3u) return HA_ERR_ALIGN;
  const size_t need = hybrid_attn_select_workspace_bytes(p);
  if (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < need)) return HA_ERR_WORKSPACE;
  double *sums = static_cast<double *>(workspace);
  uint64_t *keys = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + sums_bytes(s, p->d_head));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const unsigned rows = (unsigned)s.B * s.Hkv * s.T;
  const ScoreArgs a{s, qv, sums, means, keys, blocks, p->keep_first, p->near_tokens};
  hipError_t e;
  if (few_tiles(s)) {
#define HA_ROW(K, ...) do { \
    if (p->d_head == 128) { if (p->dtype == HA_F32) K<128, true>__VA_ARGS__(a); else K<128, false>__VA_ARGS__(a); } \
    else { if (p->dtype == HA_F32) K<64, true>__VA_ARGS__(a); else K<64, false>__VA_ARGS__(a); } } while (0)
    if (s.Tk <= kRowBlocks) {
      HA_ROW(choose_row_kernel, <<<rows, 512, 0, stream>>>);
    } else {
      HA_ROW(keys_kernel, <<<dim3((s.Tk + 127) / 128, rows), 1024, 0, stream>>>);
      if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
      launch_choose(s, keys, blocks, stream);
    }
#undef HA_ROW
    e = hipGetLastError();
    return e == hipSuccess ? HA_OK : device_error(e);
  }
#define HA_SUMS(D, F) query_sums_kernel<D, F><<<rows, 256, 0, stream>>>(s, qv, sums)
  if (p->d_head == 128) { if (p->dtype == HA_F32) HA_SUMS(128, true); else HA_SUMS(128, false); }
  else { if (p->dtype == HA_F32) HA_SUMS(64, true); else HA_SUMS(64, false); }
#undef HA_SUMS
  if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
  const unsigned groups = (s.T + kTiles - 1) / kTiles, heads = (unsigned)s.B * s.Hkv;
  if (s.Tk <= kFusedBlocks) {
#define HA_FUSED(V) (p->d_head == 128 ? score_and_choose_kernel<128, V><<<dim3(groups, heads), 1024, 0, stream>>>(a) \
                                      : score_and_choose_kernel<64, V><<<dim3(groups, heads), 1024, 0, stream>>>(a))
    // A list's keys in four registers, eight, twelve or sixteen: every one that holds nothing costs its part of the search, and its LDS.  Us with as many as hold
    // the blocks / with 16, d = 128: 4096 tiles 240 blocks 38.9 / 47.7, 500 47.1 / 52.7, 513 49.9 / 52.5, 768 53.0 / 55.2; 768 tiles 513 blocks 34.5 / 37.0, 768 37.0 / 38.9;
    // 14 thousand tiles 513 blocks 185 / 195, 768 198 / 206.  (Ten are 2 - 4 % sooner than twelve where they hold them.)
    if (s.Tk <= 256) HA_FUSED(4);
    else if (s.Tk <= 512) HA_FUSED(8);
    else if (s.Tk <= 768) HA_FUSED(12);
    else HA_FUSED(16);
#undef HA_FUSED
  } else {
    const dim3 grid(groups, (s.Tk + 1023) / 1024, heads);
    if (p->d_head == 128) scores_kernel<128><<<grid, 512, 0, stream>>>(a);
    else scores_kernel<64><<<grid, 512, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
    launch_choose(s, keys, blocks, stream);
  }
  e = hipGetLastError();
  return e == hipSuccess ? HA_OK : device_error(e);
}
