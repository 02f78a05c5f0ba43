// Block-sparse attention, gfx950: the forward.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - m_i),   j over the keys of the blocks in the tile's list
//
// in one pass over the list: m_i follows the largest logit seen, and what has been summed is rescaled when it has moved far.  A workgroup takes
// one tile of queries of one head, 32 queries to a wave, and walks the list 32 keys at a time; keys and values lie in LDS (how many steps of them, and how far ahead
// they are asked for, stands at each kernel) and every wave reads all of them.  Per wave and 32 keys: S^T = K Q^T on the matrix cores, exponentials,
// O^T += V^T P^T with P straight from the registers that hold S.  Few tiles: the list is cut into ranges, a workgroup each, whose sums a second kernel joins.
//
// The logits, the weights' sums and O are fp32.  Of bf16 tensors the weights are rounded to bf16 for the second product, since a matrix instruction takes both
// its operands in one type and V is bf16; the sum that divides is that of the unrounded ones.  A weight is off by half a step at most, 2^-8, and the output by 0.23 %
// on the average where its own rounding alone makes 0.17; the weights in two pieces would be half as many products again of the second kind, a quarter of all.
// Of fp32 tensors all operands are three bf16 pieces, six products each.
#include <cmath>
#include <type_traits>

#include "ha_sparse.h"

#include <algorithm>

namespace ha {
namespace {

struct FwdArgs {
  Sparse s;
  View q, k, v, out;          // as they are (fp32 tensors: k and v are the first bf16 pieces, the next stand piece_k elements behind)
  int64_t piece_k;
  const int32_t *blocks;
  float *lse;
  int n_split;                // ranges of the list
  float *po, *pm, *pl;        // n_split > 1: [n_split][B H N_q][D], [n_split][B H N_q]
  float scale, scale_log2e;
  unsigned items, share;
};

// bf16 tensors: 32 keys to a step, four steps' keys and values in LDS, asked for three steps ahead.  A step forms the logits of the next keys under the
// exponentials of its own, then O^T += V^T P^T over the maxima of the next ones, so that the matrix cores and the vector units of a SIMD have work
// of one wave at the same time, and of two with two workgroups to a CU.  12 heads of 32760 tokens, 64 blocks of 64: 0.81 ms, 1.0 PFLOP/s, matrix cores busy
// 54 % of the cycles at 1.73 GHz; what bounds it is power and, behind that, the L2 (lists that all name the same blocks take 0.77 ms).
//
// Tiles of 64 queries are two waves, and four steps in LDS would leave a CU with four of them at d = 128.  So they hold two steps' keys and three steps' values,
// asked for two steps ahead: 32 heads of 8192 tokens, 16 blocks of 64, 183 us for 231 (d = 64: 101 for 116); with a workgroup or two to a CU there is nothing to
// win at d = 128, and four steps it is (DEEP; four heads: 30 us for 35, at d = 64 28 for 27).
template <int D, int NW, bool DEEP>
__global__ __launch_bounds__(64 * NW, !DEEP && D == 64 ? 3 : DEEP && NW == 2 ? 1 : 2) void sparse_fwd_kernel(FwdArgs a) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, TILE = T::bytes(32);
  constexpr int AHEAD = DEEP ? 3 : 2, KSLOTS = DEEP ? 4 : 2, VSLOTS = DEEP ? 4 : 3;      // (a step's keys go ahead of its values)
  // a step's place
  constexpr auto k_at = [](int step) { return DEEP ? step % KSLOTS * 2 * TILE : step % KSLOTS * TILE; };
  constexpr auto v_at = [](int step) { return DEEP ? step % VSLOTS * 2 * TILE + TILE : (KSLOTS + step % VSLOTS) * TILE; };
  __shared__ __attribute__((aligned(1024))) char lds[(KSLOTS + VSLOTS) * TILE];      // keys of KSLOTS steps, values of VSLOTS
  const unsigned item = xcd_item(blockIdx.x, a.share);
  if (item >= a.items) return;
  const Sparse &s = a.s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int range = item % a.n_split, t = item / a.n_split % s.T, bh = item / a.n_split / s.T, b = bh / s.H, h = bh % s.H, hk = h / s.G;
  const int held = s.held(b), start = s.start(b);
  const int q0 = t * s.qb + 32 * w, qi = q0 + r;      // this wave's first query, this lane's
  const int tile_last = min((t + 1) * s.qb, s.Nq) - 1;
  // keys that the tile, this wave's first query and this lane's query see
  const int limit = s.causal ? min(held, start + tile_last + 1) : held;
  const int wave_limit = s.causal ? min(held, start + q0 + 1) : held, row_limit = s.causal ? min(held, start + qi + 1) : held;
  const int32_t *list = a.blocks + ((int64_t)(b * s.Hkv + hk) * s.T + t) * s.sel;
  ListWalk<32> walk(list, (int)((int64_t)range * s.sel / a.n_split), (int)((int64_t)(range + 1) * s.sel / a.n_split), s, limit, lane);

  const char *kbase = a.k.p + (b * a.k.sb + hk * a.k.sh) * 2, *vbase = a.v.p + (b * a.v.sb + hk * a.v.sh) * 2;
  const int ksn = (int)a.k.sn * 2, vsn = (int)a.v.sn * 2;
  constexpr int REQUESTS = 2 * T::chunks(32) / NW;
  // (behind the list's last key zeros are requested: every step has as many requests, which is what the waits count)
  auto request = [&](int key, int step) {
    char *to = lds + k_at(step);
    const int rows = key < 0 ? 0 : min(limit - key, 32), at = max(key, 0);
    request_rows<D, 32, NW>(rows_rsrc<D>(kbase + (int64_t)at * ksn, rows, ksn), ksn, to, w, lane);
    request_rows<D, 32, NW>(rows_rsrc<D>(vbase + (int64_t)at * vsn, rows, vsn), vsn, to + (v_at(step) - k_at(step)), w, lane);
  };
  int key0 = walk.next(), key1 = walk.next(), key2 = DEEP ? walk.next() : -1;
  const float c = a.scale_log2e;
  float m = -INFINITY, top = -INFINITY, l = 0.f;      // what the sums are expressed against, the largest logit and the sum of weights (this lane's keys)
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;
  if (key0 >= 0) {
    request(key0, 0);
    request(key1, 1);
    if constexpr (DEEP) request(key2, 2);
    bf16x8 qf[KS];
    const char *qp = a.q.p + (b * a.q.sb + h * a.q.sh + (int64_t)min(qi, s.Nq - 1) * a.q.sn + 8 * g) * 2;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(qp + 32 * ks);
    // addresses of all operands of a step; the slot goes into the instruction
    unsigned rows[KS], cols[RB][2];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) rows[ks] = T::rows_base(lds, lane) ^ (ks << 5);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int i = 0; i < 2; ++i) cols[rb][i] = T::cols_base(lds, lane) ^ (rb << 6) ^ (i << 5);
    auto read_k = [&](int step, int ks) { return T::row_piece(rows[ks] + k_at(step)); };
    auto read_v = [&](int step, int rb, int u) {
      const int at = v_at(step) + 16 * u * T::PITCH;
      return T::col_piece(cols[rb][0] + at, cols[rb][1] + at + 8 * T::PITCH);
    };
    const float gap = 8.f / c;
    float mc = 0.f;
    // logits of keys that this wave's queries do not all see (a key of -1: of none), then the running maximum.  What has been summed follows it when
    // some query's has moved by 8 in the exponent (weights stay below 2^8).
    auto mask = [&](f32x16 &sc, int key) {
      if (key < 0 || key + 32 > wave_limit) {
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = key >= 0 && key + crow(x, g) < row_limit ? sc[x] : -INFINITY;
      }
    };
    auto follow = [&](const f32x16 &sc) {
#pragma unroll
      for (int x = 0; x < 16; ++x) top = fmaxf(top, sc[x]);
      if (__any(top - m > gap)) {
        top = xhalf_max(top);
        const float f = top == m ? 1.f : fast_exp2((m - top) * c);      // (neither may have seen a key)
        l *= f;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int x = 0; x < 16; ++x) o[rb][x] *= f;
        m = top;
        mc = m == -INFINITY ? 0.f : m * c;
      }
    };
    const f32x16 none = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    f32x16 s_a, s_b;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 1) * REQUESTS) : "memory");
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s_a = mfma32(read_k(0, ks), qf[ks], ks == 0 ? none : s_a);
    mask(s_a, key0);
    follow(s_a);
    auto step = [&](f32x16 &sc, f32x16 &sn, auto now_c) {
      constexpr int now = decltype(now_c)::value, next = now + 1;
      // the next keys have landed, and no wave reads those of the step before any more
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 2) * REQUESTS) : "memory");
      __syncthreads();
      bf16x8 kf[KS], vf[2 * RB], pb[2];
      kf[0] = read_k(next, 0);
      kf[1] = read_k(next, 1);
      const int further = walk.next();
      request(further, now + AHEAD);
      constexpr int PER = 16 / KS;         // logits to a product: 2 at d = 128, 4 at d = 64
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + 2 < KS) kf[ks + 2] = read_k(next, ks + 2);
        else vf[ks + 2 - KS] = read_v(now, ks + 2 - KS, 0);
        HA_FENCE();
        sn = mfma32(kf[ks], qf[ks], ks == 0 ? none : sn);
#pragma unroll
        for (int y = 0; y < PER; ++y) {
          const int x = ks * PER + y;
          sc[x] = fast_exp2(__builtin_fmaf(sc[x], c, -mc));
          l += sc[x];
          if (x % 8 == 7) {
            f32x8 p;
#pragma unroll
            for (int z = 0; z < 8; ++z) p[z] = sc[x - 7 + z];
            pb[x / 8] = __builtin_convertvector(p, bf16x8);
          }
        }
        HA_FENCE();
      }
#pragma unroll
      for (int n = 0; n < 2 * RB; ++n) {   // n = RB u + rb
        if (n + 2 < 2 * RB) vf[n + 2] = read_v(now, (n + 2) % RB, (n + 2) / RB);
        HA_FENCE();
        o[n % RB] = mfma32(vf[n], pb[n / RB], o[n % RB]);
      }
      mask(sn, key1);
      follow(sn);
      key0 = key1;
      key1 = DEEP ? key2 : further;
      key2 = further;
    };
    while (true) {
      step(s_a, s_b, std::integral_constant<int, 0>{});
      if (key0 < 0) break;
      step(s_b, s_a, std::integral_constant<int, 1>{});
      if (key0 < 0) break;
      step(s_a, s_b, std::integral_constant<int, 2>{});
      if (key0 < 0) break;
      step(s_b, s_a, std::integral_constant<int, 3>{});
      if (key0 < 0) break;
      if constexpr (!DEEP) {
        step(s_a, s_b, std::integral_constant<int, 4>{});
        if (key0 < 0) break;
        step(s_b, s_a, std::integral_constant<int, 5>{});
        if (key0 < 0) break;
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  l = xhalf_sum(l);
  if (a.n_split > 1) {
    const int64_t row = ((int64_t)range * s.B * s.H + bh) * s.Nq + qi;
    if (qi < s.Nq) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int x4 = 0; x4 < 4; ++x4)
          *reinterpret_cast<f32x4 *>(a.po + row * D + 32 * rb + 8 * x4 + 4 * g) = f32x4{o[rb][4 * x4], o[rb][4 * x4 + 1], o[rb][4 * x4 + 2], o[rb][4 * x4 + 3]};
      if (g == 0) {
        a.pm[row] = m;
        a.pl[row] = l;
      }
    }
    return;
  }
  if (a.lse && g == 0 && qi < s.Nq) a.lse[(int64_t)bh * s.Nq + qi] = l > 0.f ? m * a.scale + logf(l) : l == 0.f ? -INFINITY : l;
  __syncthreads();                                    // the slots become the staging area of the stores
  store_rows<D, false>(o, l == 0.f ? 0.f : 1.f / l, lds + w * store_bytes<D, false>(), a.out.p + (b * a.out.sb + h * a.out.sh) * 2, a.out.sn * 2,
                       q0, min((t + 1) * s.qb, s.Nq), lane);
}

// fp32 tensors: 32 keys at a time in three pieces, six products for one.  One stage of LDS, so that other workgroups of the CU cover the loads: 32 heads of
// 8192 tokens (d = 128, tiles of 128 x 16 blocks of 64) take 675 us (204 TFLOP/s, 1.2 PFLOP/s of the matrix cores) and 807 with two stages and one
// workgroup to a CU; four heads, which leave a CU with one, 132 and 130.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void sparse_fwd_f32_kernel(FwdArgs a) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, NS = Pieces<true>::N, ROWS = Pieces<true>::ROWS, STAGE = T::bytes(ROWS);
  __shared__ __attribute__((aligned(1024))) char lds[2 * NS * STAGE];      // [k | v][pieces][ROWS]
  const unsigned item = xcd_item(blockIdx.x, a.share);
  if (item >= a.items) return;
  const Sparse &s = a.s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int range = item % a.n_split, t = item / a.n_split % s.T, bh = item / a.n_split / s.T, b = bh / s.H, h = bh % s.H, hk = h / s.G;
  const int held = s.held(b), start = s.start(b);
  const int q0 = t * s.qb + 32 * w, qi = q0 + r;      // this wave's first query, this lane's
  const int tile_last = min((t + 1) * s.qb, s.Nq) - 1;
  // keys that the tile, this wave's first query and this lane's query see
  const int limit = s.causal ? min(held, start + tile_last + 1) : held;
  const int wave_limit = s.causal ? min(held, start + q0 + 1) : held, row_limit = s.causal ? min(held, start + qi + 1) : held;
  const int32_t *list = a.blocks + ((int64_t)(b * s.Hkv + hk) * s.T + t) * s.sel;
  ListWalk<ROWS> walk(list, (int)((int64_t)range * s.sel / a.n_split), (int)((int64_t)(range + 1) * s.sel / a.n_split), s, limit, lane);

  const char *kbase = a.k.p + (b * a.k.sb + hk * a.k.sh) * 2, *vbase = a.v.p + (b * a.v.sb + hk * a.v.sh) * 2;
  const int ksn = (int)a.k.sn * 2, vsn = (int)a.v.sn * 2;
  auto request = [&](int key) {
    const int rows = min(limit - key, ROWS);
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      request_rows<D, ROWS, NW>(rows_rsrc<D>(kbase + (key * a.k.sn + n * a.piece_k) * 2, rows, ksn), ksn, lds + n * STAGE, w, lane);
      request_rows<D, ROWS, NW>(rows_rsrc<D>(vbase + (key * a.v.sn + n * a.piece_k) * 2, rows, vsn), vsn, lds + (NS + n) * STAGE, w, lane);
    }
  };
  int key = walk.next();
  if (key >= 0) request(key);

  bf16x8 qf[KS][NS];
  {
    const float *at = reinterpret_cast<const float *>(a.q.p) + b * a.q.sb + h * a.q.sh + (int64_t)min(qi, s.Nq - 1) * a.q.sn + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) split8_any(*reinterpret_cast<const f32x4 *>(at + 16 * ks), *reinterpret_cast<const f32x4 *>(at + 16 * ks + 4), qf[ks]);
  }
  const float c = a.scale_log2e;
  float m = -INFINITY, l = 0.f;                       // this query's largest logit (lagging, see below), its sum of weights (this lane's keys)
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;

  const unsigned rows = T::rows_base(lds, lane), cols = T::cols_base(lds, lane);
  while (key >= 0) {
    landed();
    f32x16 sc[ROWS / 32];
#pragma unroll
    for (int i = 0; i < ROWS / 32; ++i) {
#pragma unroll
      for (int x = 0; x < 16; ++x) sc[i][x] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) kf[n] = T::rows_at(rows, 32 * i, ks, n * STAGE);
        sc[i] = mfma_split<NS>(kf, qf[ks], sc[i]);
      }
    }
    if (key + ROWS > wave_limit) {
#pragma unroll
      for (int i = 0; i < ROWS / 32; ++i)
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[i][x] = key + 32 * i + crow(x, g) < row_limit ? sc[i][x] : -INFINITY;
    }
    float top = sc[0][0];
#pragma unroll
    for (int i = 0; i < ROWS / 32; ++i)
#pragma unroll
      for (int x = 0; x < 16; ++x) top = fmaxf(top, sc[i][x]);
    top = xhalf_max(top);
    // the accumulators follow the maximum when some query's has moved by 8 in the exponent (weights stay below 2^8)
    if (__any(top > m + 8.f / c)) {
      const float to = fmaxf(m, top), f = m == -INFINITY ? 0.f : fast_exp2((m - to) * c);
      l *= f;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[rb][x] *= f;
      m = to;
    }
    const float mc = m == -INFINITY ? 0.f : m * c;    // (nothing seen yet: every logit is -infinity, every weight 0)
#pragma unroll
    for (int i = 0; i < ROWS / 32; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x8 p;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          p[x] = fast_exp2(__builtin_fmaf(sc[i][8 * u + x], c, -mc));
          l += p[x];
        }
        bf16x8 pb[NS];
        split8<NS>(p, pb);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          bf16x8 vf[NS];
#pragma unroll
          for (int n = 0; n < NS; ++n) vf[n] = T::cols_at(cols, rb, 32 * i + 16 * u, (NS + n) * STAGE);
          o[rb] = mfma_split<NS>(vf, pb, o[rb]);
        }
      }
    __syncthreads();                                  // every wave is done with the stage
    key = walk.next();
    if (key >= 0) request(key);
  }
  l = xhalf_sum(l);
  if (a.n_split > 1) {
    const int64_t row = ((int64_t)range * s.B * s.H + bh) * s.Nq + qi;
    if (qi < s.Nq) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int x4 = 0; x4 < 4; ++x4)
          *reinterpret_cast<f32x4 *>(a.po + row * D + 32 * rb + 8 * x4 + 4 * g) = f32x4{o[rb][4 * x4], o[rb][4 * x4 + 1], o[rb][4 * x4 + 2], o[rb][4 * x4 + 3]};
      if (g == 0) {
        a.pm[row] = m;
        a.pl[row] = l;
      }
    }
    return;
  }
  if (a.lse && g == 0 && qi < s.Nq) a.lse[(int64_t)bh * s.Nq + qi] = l > 0.f ? m * a.scale + logf(l) : l == 0.f ? -INFINITY : l;
  __syncthreads();                                    // the stage becomes the staging area of the stores
  store_rows<D, true>(o, l == 0.f ? 0.f : 1.f / l, lds + w * store_bytes<D, true>(), a.out.p + (b * a.out.sb + h * a.out.sh) * 4, a.out.sn * 4,
                         q0, min((t + 1) * s.qb, s.Nq), lane);
}

// The sums of four waves that walked keys of one group's range: joined through LDS (`image`: 4 x 32 D values) and stored.
template <int D>
static constexpr int image_bytes() { return 4 * 32 * D * 4; }
template <int D, bool F32>
__device__ __forceinline__ void join_waves(const FwdArgs &a, const f32x16 (&o)[D / 32], float m, float l, char *lds, float (&stats)[2][4][32], int range, int b, int hk, int w, int lane) {
  constexpr int RB = D / 32, IMAGE = RB * 4 * 64;
  const Sparse &s = a.s;
  const int r = lane & 31, g = lane >> 5, rows = s.G * s.Nq;
  const float c = a.scale_log2e;
  l = xhalf_sum(l);
  __syncthreads();
  f32x4 *image = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x4 = 0; x4 < 4; ++x4)
      image[w * IMAGE + (rb * 4 + x4) * 64 + lane] = f32x4{o[rb][4 * x4], o[rb][4 * x4 + 1], o[rb][4 * x4 + 2], o[rb][4 * x4 + 3]};
  if (g == 0) {
    stats[0][w][r] = m;
    stats[1][w][r] = l;
  }
  __syncthreads();
  if (w >= RB || r >= rows) return;
  const int h = hk * s.G + r / s.Nq, n = r % s.Nq;
  // wave w: columns 32 w .. of the joined rows
  float top = stats[0][0][r], total = 0.f;
#pragma unroll
  for (int i = 1; i < 4; ++i) top = fmaxf(top, stats[0][i][r]);
  f32x4 y[4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float mi = stats[0][i][r], f = mi == top ? 1.f : fast_exp2((mi - top) * c);
    total += stats[1][i][r] * f;
#pragma unroll
    for (int x4 = 0; x4 < 4; ++x4) y[x4] += image[i * IMAGE + (w * 4 + x4) * 64 + lane] * f;
  }
  const int64_t row = ((int64_t)b * s.H + h) * s.Nq + n;
  if (a.n_split > 1) {
    const int64_t at = (int64_t)range * s.B * s.H * s.Nq + row;
#pragma unroll
    for (int x4 = 0; x4 < 4; ++x4) *reinterpret_cast<f32x4 *>(a.po + at * D + 32 * w + 8 * x4 + 4 * g) = y[x4];
    if (w == 0 && g == 0) {
      a.pm[at] = top;
      a.pl[at] = total;
    }
    return;
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int x4 = 0; x4 < 4; ++x4) {
    char *to = a.out.p + (b * a.out.sb + h * a.out.sh + n * a.out.sn + 32 * w + 8 * x4 + 4 * g) * (F32 ? 4 : 2);
    if constexpr (F32) *reinterpret_cast<f32x4 *>(to) = y[x4] * inv;
    else *reinterpret_cast<bf16x4 *>(to) = __builtin_convertvector(y[x4] * inv, bf16x4);
  }
  if (a.lse && w == 0 && g == 0) a.lse[row] = total > 0.f ? top * a.scale + logf(total) : total == 0.f ? -INFINITY : total;
}

// Few queries (a decoding step): all queries of all heads of a key head, 32 at most, are the columns of one product, so that keys and values are read once
// for the group.  What bounds it is memory, so every wave walks keys of its own, every fourth step of the range, with its own two stages in LDS and no
// barrier; the four waves' sums are joined behind the list.  Four sequences of 12 heads on 4 with 32 blocks of 64 of 60000 keys: 8 us (and 4.5 of joining) for
// 17 MB, which is the time of a few dependent loads, not of the bytes; 64 sequences 41 us, 6.5 TB/s.
template <int D>
__global__ __launch_bounds__(256) void sparse_few_kernel(FwdArgs a) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, TILE = T::bytes(32), SLOT = 2 * TILE, REQUESTS = 2 * T::chunks(32);
  __shared__ __attribute__((aligned(1024))) char lds[4 * 2 * SLOT];      // [wave][stage][k | v]; then [wave][register image]
  static_assert(image_bytes<D>() <= 4 * 2 * SLOT, "the images fit the stages");
  __shared__ float stats[2][4][32];
  const Sparse &s = a.s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int range = blockIdx.x % a.n_split, bh = blockIdx.x / a.n_split, b = bh / s.Hkv, hk = bh % s.Hkv;
  const int held = s.held(b), start = s.start(b), rows = s.G * s.Nq, col = min(r, rows - 1), h = hk * s.G + col / s.Nq, n = col % s.Nq;
  const int limit = s.causal ? min(held, start + s.Nq) : held, all_see = s.causal ? min(held, start + 1) : held, row_limit = s.causal ? min(held, start + n + 1) : held;
  ListWalk<32> walk(a.blocks + (int64_t)bh * s.sel, (int)((int64_t)range * s.sel / a.n_split), (int)((int64_t)(range + 1) * s.sel / a.n_split), s, limit, lane);
  const char *kbase = a.k.p + (b * a.k.sb + hk * a.k.sh) * 2, *vbase = a.v.p + (b * a.v.sb + hk * a.v.sh) * 2;
  const int ksn = (int)a.k.sn * 2, vsn = (int)a.v.sn * 2;
  char *mine = lds + w * (2 * SLOT);
  auto request = [&](int key, int stage) {
    const int n_keys = min(limit - key, 32);
    request_rows<D, 32, 1>(rows_rsrc<D>(kbase + (int64_t)key * ksn, n_keys, ksn), ksn, mine + stage * SLOT, 0, lane);
    request_rows<D, 32, 1>(rows_rsrc<D>(vbase + (int64_t)key * vsn, n_keys, vsn), vsn, mine + stage * SLOT + TILE, 0, lane);
  };
  int key = -1;
  for (int i = 0; i <= w; ++i) key = walk.next();
  if (key >= 0) request(key, 0);
  bf16x8 qf[KS];
  const char *qp = a.q.p + (b * a.q.sb + h * a.q.sh + n * a.q.sn + 8 * g) * 2;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(qp + 32 * ks);
  const unsigned rows0 = T::rows_base(mine, lane), cols0 = T::cols_base(mine, lane);
  const float c = a.scale_log2e;
  float m = -INFINITY, l = 0.f;
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;
  for (int stage = 0; key >= 0; stage ^= 1) {
    int next = -1;
    for (int i = 0; i < 4; ++i) next = walk.next();
    if (next >= 0) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (the last step's reads of that stage are done)
      request(next, stage ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(REQUESTS) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    const unsigned kt = rows0 + stage * SLOT, vt = cols0 + stage * SLOT;
    f32x16 sc;
#pragma unroll
    for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) sc = mfma32(T::rows_at(kt, 0, ks), qf[ks], sc);
    if (key + 32 > all_see) {
#pragma unroll
      for (int x = 0; x < 16; ++x) sc[x] = key + crow(x, g) < row_limit ? sc[x] : -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int x = 0; x < 16; ++x) top = fmaxf(top, sc[x]);
    top = xhalf_max(top);
    const float f = top == m ? 1.f : fast_exp2((m - top) * c), mc = top == -INFINITY ? 0.f : top * c;
    m = top;
    l *= f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[rb][x] *= f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x8 p;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        p[x] = fast_exp2(__builtin_fmaf(sc[8 * u + x], c, -mc));
        l += p[x];
      }
      const bf16x8 pb = __builtin_convertvector(p, bf16x8);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) o[rb] = mfma32(T::cols_at(vt, rb, 16 * u, TILE), pb, o[rb]);
    }
    key = next;
  }
  join_waves<D, false>(a, o, m, l, lds, stats, range, b, hk, w, lane);
}

// The same of fp32 tensors, whose chosen rows are split on the way: each wave takes them from memory to registers (a row of keys to a lane, eight rows of a
// column of the values), so that a step reads the chosen rows once and not the whole cache.  Keys are requested a step ahead.  Three sequences of 8 heads on 4,
// d = 64, 41 blocks of 128 of some ten thousand keys: 15 us; splitting the whole cache ahead 152 us and 51 behind it.
template <int D>
__global__ __launch_bounds__(256, 1) void sparse_few_f32_kernel(FwdArgs a) {
  constexpr int KS = D / 16, RB = D / 32;
  __shared__ __attribute__((aligned(1024))) char lds[image_bytes<D>()];
  __shared__ float stats[2][4][32];
  const Sparse &s = a.s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int range = blockIdx.x % a.n_split, bh = blockIdx.x / a.n_split, b = bh / s.Hkv, hk = bh % s.Hkv;
  const int held = s.held(b), start = s.start(b), rows = s.G * s.Nq, col = min(r, rows - 1), h = hk * s.G + col / s.Nq, n = col % s.Nq;
  const int limit = s.causal ? min(held, start + s.Nq) : held, all_see = s.causal ? min(held, start + 1) : held, row_limit = s.causal ? min(held, start + n + 1) : held;
  ListWalk<32> walk(a.blocks + (int64_t)bh * s.sel, (int)((int64_t)range * s.sel / a.n_split), (int)((int64_t)(range + 1) * s.sel / a.n_split), s, limit, lane);
  const float *kbase = reinterpret_cast<const float *>(a.k.p) + b * a.k.sb + hk * a.k.sh + 8 * g, *vbase = reinterpret_cast<const float *>(a.v.p) + b * a.v.sb + hk * a.v.sh + r;
  f32x4 kr[KS][2];
  // (rows behind the last visible key are that key's: their weights are zero)
  auto request = [&](int key) {
    const float *p = kbase + min(key + r, limit - 1) * a.k.sn;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i) kr[ks][i] = *reinterpret_cast<const f32x4 *>(p + 16 * ks + 4 * i);
  };
  int key = -1;
  for (int i = 0; i <= w; ++i) key = walk.next();
  if (key >= 0) request(key);
  bf16x8 qf[KS][3];
  const float *qp = reinterpret_cast<const float *>(a.q.p) + b * a.q.sb + h * a.q.sh + n * a.q.sn + 8 * g;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) split8_any(*reinterpret_cast<const f32x4 *>(qp + 16 * ks), *reinterpret_cast<const f32x4 *>(qp + 16 * ks + 4), qf[ks]);
  const float c = a.scale_log2e;
  float m = -INFINITY, l = 0.f;
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;
  while (key >= 0) {
    float vr[2][RB][8];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float *p = vbase + min(key + crow(8 * u + x, g), limit - 1) * a.v.sn;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) vr[u][rb][x] = p[32 * rb];
      }
    f32x16 sc;
#pragma unroll
    for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 kf[3];
      split8_any(kr[ks][0], kr[ks][1], kf);
      sc = mfma_split<3>(kf, qf[ks], sc);
    }
    const int at = key;
    for (int i = 0; i < 4; ++i) key = walk.next();
    if (key >= 0) request(key);
    if (at + 32 > all_see) {
#pragma unroll
      for (int x = 0; x < 16; ++x) sc[x] = at + crow(x, g) < row_limit ? sc[x] : -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int x = 0; x < 16; ++x) top = fmaxf(top, sc[x]);
    top = xhalf_max(top);
    const float f = top == m ? 1.f : fast_exp2((m - top) * c), mc = top == -INFINITY ? 0.f : top * c;
    m = top;
    l *= f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[rb][x] *= f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x8 p;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        p[x] = fast_exp2(__builtin_fmaf(sc[8 * u + x], c, -mc));
        l += p[x];
      }
      bf16x8 pb[3];
      split8<3>(p, pb);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float(&v)[8] = vr[u][rb];
        bf16x8 vf[3];
        split8_any(f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]}, vf);
        o[rb] = mfma_split<3>(vf, pb, o[rb]);
      }
    }
  }
  join_waves<D, true>(a, o, m, l, lds, stats, range, b, hk, w, lane);
}

// Joins the ranges of a row, at most 64: a wave to a row.  Lane i has range i's maximum and sum; D / 4 lanes take four columns each, ranges in turn.
// (4.5 us for 48 rows of 16 ranges: a launch and two loads one behind the other.)
template <int D, bool F32>
__global__ __launch_bounds__(256) void sparse_join_kernel(FwdArgs a) {
  constexpr int LPR = D / 4, AT_ONCE = 64 / LPR;
  const Sparse &s = a.s;
  const int64_t rows = (int64_t)s.B * s.H * s.Nq, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int lane = threadIdx.x & 63, c4 = 4 * (lane % LPR);
  const bool has = lane < a.n_split;
  const float mi = has ? a.pm[lane * rows + row] : -INFINITY;
  float m = mi;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  const float f = mi == m ? 1.f : fast_exp2((mi - m) * a.scale_log2e);
  float l = has ? a.pl[lane * rows + row] * f : 0.f;          // (a range that saw nothing has 0, or the NaN that has to show)
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < a.n_split; i0 += 4 * AT_ONCE) {
    f32x4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = min(i0 + u * AT_ONCE + lane / LPR, a.n_split - 1);
      x[u] = *reinterpret_cast<const f32x4 *>(a.po + (i * rows + row) * D + c4);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * AT_ONCE + lane / LPR;
      const float fi = __shfl(f, min(i, 63));
      if (i < a.n_split) o += x[u] * fi;
    }
  }
#pragma unroll
  for (int d = LPR; d < 64; d <<= 1)
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] += __shfl_xor(o[u], d);
  if (lane >= LPR) return;
  const int b = (int)(row / s.Nq / s.H), h = (int)(row / s.Nq % s.H), n = (int)(row % s.Nq);
  if (a.lse && lane == 0) a.lse[row] = l > 0.f ? m * a.scale + logf(l) : l == 0.f ? -INFINITY : l;
  o *= l == 0.f ? 0.f : 1.f / l;
  const int64_t at = b * a.out.sb + h * a.out.sh + n * a.out.sn + c4;
  if constexpr (F32) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out.p) + at) = o;
  else *reinterpret_cast<bf16x4 *>(reinterpret_cast<__bf16 *>(a.out.p) + at) = __builtin_convertvector(o, bf16x4);
}

struct FwdPlan {
  bool few;
  int n_split;
  size_t off_k, off_v, off_po, off_pm, off_pl, total;
};

FwdPlan plan_forward(const ha_sparse_problem &p, const Sparse &s) {
  FwdPlan f{};
  // Workgroups: a tile of a head each, or all queries of a key head's group where they are 32 at most.  Us with that / with tiles: 12 query heads on 4 key
  // heads, 32 blocks of 64, one query 9.7 / 17.2, in batches of 16 18.6 / 45.3, of 64 41 / 111; lists of 4 blocks for 64 x 12 heads that share no keys 27.4 / 23.4.
  f.few = s.T == 1 && s.G * (int64_t)s.Nq <= 32;
  // The list is cut until every CU has a workgroup, but a wave keeps a step of 32 keys, a workgroup of tiles eight.  Us so / uncut: that one query 9.7 / 28.1;
  // twelve heads of 128 queries, 16 blocks 15.8 / 24.6, of 256 and 32 20.6 / 44.0, of 1200 (120 tiles) 40 / 46.  With at
  // least 16 steps the first two of these take 20.0 and 22.3; with two workgroups to a CU the batch of 16 above takes 22.6.
  const int64_t groups = (int64_t)s.B * (f.few ? s.Hkv : s.H * (int64_t)s.T), steps = (int64_t)s.sel * s.kb / 32;
  // Two workgroups to a CU where each keeps 64 steps: 156 tiles with lists of 256 steps 108 us for 161, of 64 46 for 46, of 16 33 for 16 (their join).
  const int64_t most = f.few ? (steps + 3) / 4 : (steps + 7) / 8;
  int64_t parts = 1;
  if (groups > 0) {
    parts = std::min(256 / groups, most);
    if (!f.few) parts = std::max(parts, std::min(512 / groups, steps / 64));
  }
  f.n_split = (int)std::max<int64_t>(parts, 1);
  if (f.n_split > s.sel) f.n_split = s.sel;
  if (f.n_split > 64) f.n_split = 64;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round256(bytes);
    return here;
  };
  if (p.dtype == HA_F32 && !f.few) {
    f.off_k = take((size_t)6 * s.B * s.Hkv * s.Nk * p.d_head);
    f.off_v = take((size_t)6 * s.B * s.Hkv * s.Nk * p.d_head);
  }
  if (f.n_split > 1) {
    const size_t rows = (size_t)f.n_split * s.B * s.H * s.Nq;
    f.off_po = take(rows * p.d_head * 4);
    f.off_pm = take(rows * 4);
    f.off_pl = take(rows * 4);
  }
  f.total = at;
  return f;
}

template <int D, bool F32, int NW>
hipError_t launch_fwd(const FwdArgs &a, hipStream_t st) {
  if constexpr (F32) sparse_fwd_f32_kernel<D, NW><<<8 * a.share, 64 * NW, 0, st>>>(a);
  else if (NW == 4 || (D == 128 && a.items <= 512)) sparse_fwd_kernel<D, NW, NW == 4 || D == 128><<<8 * a.share, 64 * NW, 0, st>>>(a);
  else sparse_fwd_kernel<D, NW, NW == 4><<<8 * a.share, 64 * NW, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" size_t hybrid_attn_sparse_workspace_bytes(const ha_sparse_problem *p) {
  if (check_sparse(p) != HA_OK) return 0;
  return plan_forward(*p, sparse_of(*p)).total;
}

extern "C" ha_status hybrid_attn_sparse_forward(const ha_sparse_problem *p, const ha_view *q, const ha_view *k, const ha_view *v, const int32_t *blocks,
                                                const ha_view *out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
  ha_status st = check_sparse(p);
  if (st != HA_OK) return st;
  FwdArgs a{};
  if ((st = check_view(*p, q, p->H, p->N_q, p->q_block, false, a.q)) != HA_OK || (st = check_view(*p, k, p->H_kv, p->N_k, p->k_block, false, a.k)) != HA_OK ||
      (st = check_view(*p, v, p->H_kv, p->N_k, p->k_block, false, a.v)) != HA_OK || (st = check_view(*p, out, p->H, p->N_q, p->q_block, true, a.out)) != HA_OK)
    return st;
  if (p->N_q == 0) return HA_OK;
  if (!blocks) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(blocks) & 3u || reinterpret_cast<uintptr_t>(lse) & 3u) return HA_ERR_ALIGN;
  const Sparse s = a.s = sparse_of(*p);
  const FwdPlan f = plan_forward(*p, s);
  if (f.total > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < f.total)) return HA_ERR_WORKSPACE;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(workspace);
  hipError_t e;
  const int d = p->d_head;
  const bool f32 = p->dtype == HA_F32;
  if (f32 && !f.few) {
    const SplitJob jobs[2] = {{a.k, reinterpret_cast<__bf16 *>(ws + f.off_k), s.Hkv, s.Nk}, {a.v, reinterpret_cast<__bf16 *>(ws + f.off_v), s.Hkv, s.Nk}};
    if ((e = launch_split(s, d, jobs, 2, stream)) != hipSuccess) return device_error(e);
    a.k = split_view(jobs[0], d);
    a.v = split_view(jobs[1], d);
    a.piece_k = (int64_t)s.B * s.Hkv * s.Nk * d;
  }
  a.blocks = blocks;
  a.lse = lse;
  a.n_split = f.n_split;
  a.po = reinterpret_cast<float *>(ws + f.off_po);
  a.pm = reinterpret_cast<float *>(ws + f.off_pm);
  a.pl = reinterpret_cast<float *>(ws + f.off_pl);
  a.scale = p->softmax_scale;
  a.scale_log2e = p->softmax_scale * kLog2e;
  a.items = (unsigned)((int64_t)s.B * s.H * s.T * f.n_split);
  a.share = xcd_share(a.items);
  if (f.few) {
    const unsigned n = (unsigned)s.B * s.Hkv * f.n_split;
    if (f32) {
      if (d == 128) sparse_few_f32_kernel<128><<<n, 256, 0, stream>>>(a);
      else sparse_few_f32_kernel<64><<<n, 256, 0, stream>>>(a);
    } else if (d == 128) {
      sparse_few_kernel<128><<<n, 256, 0, stream>>>(a);
    } else {
      sparse_few_kernel<64><<<n, 256, 0, stream>>>(a);
    }
    e = hipGetLastError();
  } else if (d == 128) {
    if (f32) e = s.qb == 128 ? launch_fwd<128, true, 4>(a, stream) : launch_fwd<128, true, 2>(a, stream);
    else e = s.qb == 128 ? launch_fwd<128, false, 4>(a, stream) : launch_fwd<128, false, 2>(a, stream);
  } else {
    if (f32) e = s.qb == 128 ? launch_fwd<64, true, 4>(a, stream) : launch_fwd<64, true, 2>(a, stream);
    else e = s.qb == 128 ? launch_fwd<64, false, 4>(a, stream) : launch_fwd<64, false, 2>(a, stream);
  }
  if (e != hipSuccess) return device_error(e);
  if (f.n_split > 1) {
    const unsigned blocks_j = (unsigned)(((int64_t)s.B * s.H * s.Nq + 3) / 4);
    if (d == 128) { if (f32) sparse_join_kernel<128, true><<<blocks_j, 256, 0, stream>>>(a); else sparse_join_kernel<128, false><<<blocks_j, 256, 0, stream>>>(a); }
    else { if (f32) sparse_join_kernel<64, true><<<blocks_j, 256, 0, stream>>>(a); else sparse_join_kernel<64, false><<<blocks_j, 256, 0, stream>>>(a); }
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
  }
  return HA_OK;
}
