// Block-sparse attention, gfx950: checks of its arguments, block means of the keys, and the choice of key blocks for every tile of queries.
//
//   mean_j = sum of the keys of block j / their number        score_tj = (sum of the queries of tile t over its heads) . mean_j
//
// Everything that decides is formed in double: the sums of 64 or 128 bf16 values are exact there, and two scores that differ at all are in the
// right order, whatever the order of summation (in fp32 about one list in ten thousand changed with it).  The sums over q and k are bound by
// memory; the scores of 128 queries against a block of 64 keys take one product of d values.
#include <cmath>
#include <limits>

#include "ha_sparse.h"

namespace ha {

ha_status check_sparse(const ha_sparse_problem *p) {
  if (!p) return HA_ERR_NULL;
  if (p->B <= 0 || p->H <= 0 || p->H_kv <= 0 || p->N_q < 0 || p->N_k < 0 || p->d_head <= 0) return HA_ERR_SHAPE;
  if (p->H % p->H_kv || p->n_select < 1 || p->keep_first < 0 || p->near_tokens < -1) return HA_ERR_SHAPE;
  if (p->causal != 0 && p->causal != 1) return HA_ERR_SHAPE;
  if (!(p->softmax_scale > 0.f) || !std::isfinite(p->softmax_scale)) return HA_ERR_SHAPE;
  if (p->dtype != HA_BF16 && p->dtype != HA_F32) return HA_ERR_UNSUPPORTED;
  if (p->d_head != 64 && p->d_head != 128) return HA_ERR_UNSUPPORTED;
  if ((p->q_block != 64 && p->q_block != 128) || (p->k_block != 64 && p->k_block != 128)) return HA_ERR_UNSUPPORTED;
  if ((int64_t)p->B * p->H > 65535 || p->N_q > (1 << 24) || p->N_k > (1 << 29) || p->n_select > (1 << 20) || p->near_tokens > (1 << 29)) return HA_ERR_UNSUPPORTED;
  const int64_t T = (p->N_q + p->q_block - 1) / p->q_block, Tk = (p->N_k + p->k_block - 1) / p->k_block, BH = (int64_t)p->B * p->H;
  // (a launch takes 2^31 - 1 workgroups, and an index into one head's lists 31 bits)
  if (BH * T > (1 << 24) || BH * Tk > (1 << 25) || T * p->n_select > (1 << 30)) return HA_ERR_UNSUPPORTED;
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

// Scores of TILES tiles against 256 blocks, a block a thread, as ordered integers [rows][Tk].
struct ScoreArgs {
  Sparse s;
  const double *sums;
  const float *means;
  uint64_t *keys;
  int keep_first, near_tokens;
};
template <int D, int TILES>
__global__ __launch_bounds__(256) void scores_kernel(ScoreArgs a) {
  const Sparse &s = a.s;
  __shared__ double q[TILES][D];
  const int bh = blockIdx.z, b = bh / s.Hkv, t0 = blockIdx.y * TILES, j = blockIdx.x * 256 + threadIdx.x;
  for (int i = threadIdx.x; i < TILES * D; i += 256) q[i / D][i % D] = t0 + i / D < s.T ? a.sums[((int64_t)bh * s.T + t0) * D + i] : 0.;
  __syncthreads();
  if (j >= s.Tk) return;
  const f32x4 *m = reinterpret_cast<const f32x4 *>(a.means + ((int64_t)bh * s.Tk + j) * D);
  double acc[TILES];
#pragma unroll
  for (int i = 0; i < TILES; ++i) acc[i] = 0.;
#pragma unroll 2
  for (int c = 0; c < D / 4; ++c) {
    const f32x4 x = m[c];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < TILES; ++i) acc[i] = __builtin_fma((double)x[u], q[i][4 * c + u], acc[i]);
  }
  const int held = s.held(b), lo_key = j * s.kb, hi_key = lo_key + s.kb - 1, start = s.start(b);
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    const int t = t0 + i;
    if (t >= s.T) break;
    const int lo = start + t * s.qb, hi = start + min((t + 1) * s.qb, s.Nq) - 1;
    uint64_t key = ordered(acc[i]);
    if (j < a.keep_first || (a.near_tokens >= 0 && hi_key >= lo - a.near_tokens && lo_key <= hi + (s.causal ? 0 : a.near_tokens))) key = ~(uint64_t)0;
    if (lo_key >= held || (s.causal && lo_key > hi)) key = 0;
    a.keys[((int64_t)bh * s.T + t) * s.Tk + j] = key;
  }
}

// ---- the choice ------------------------------------------------------------------------------------------------------
// One workgroup to a list: the largest threshold that at least n_select keys reach is found bit by bit, then the blocks are written in rising order.
// V > 0: thread t holds blocks t, t + 256, ..; V = 0: any number, read again for every bit.
template <int V>
struct Keys {
  uint64_t k[V];
  int n;
  __device__ __forceinline__ Keys(const uint64_t *keys, int n_) : n(n_) {
#pragma unroll
    for (int i = 0; i < V; ++i) k[i] = i * 256 + (int)threadIdx.x < n ? keys[i * 256 + threadIdx.x] : 0;
  }
  __device__ __forceinline__ int rounds() const { return V; }
  __device__ __forceinline__ uint64_t at(int i) const { return k[i]; }
};
template <>
struct Keys<0> {
  const uint64_t *p;
  int n;
  __device__ __forceinline__ Keys(const uint64_t *keys, int n_) : p(keys), n(n_) {}
  __device__ __forceinline__ int rounds() const { return (n + 255) / 256; }
  __device__ __forceinline__ uint64_t at(int i) const { return i * 256 + (int)threadIdx.x < n ? p[i * 256 + threadIdx.x] : 0; }
};

template <int V>
__global__ __launch_bounds__(256) void choose_kernel(const uint64_t *keys, int Tk, int sel, int32_t *blocks) {
  __shared__ int count[2][4];
  const int64_t row = blockIdx.x;
  const Keys<V> k(keys + row * Tk, Tk);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int turn = 0;
  // keys that are >= x, of the whole workgroup
  auto reach = [&](uint64_t x) {
    int c = 0;
    if constexpr (V > 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) c += __popcll(__ballot(k.at(i) >= x));
    } else {
      for (int i = 0; i < k.rounds(); ++i) c += __popcll(__ballot(k.at(i) >= x));
    }
    if (lane == 0) count[turn][w] = c;
    __syncthreads();
    c = count[turn][0] + count[turn][1] + count[turn][2] + count[turn][3];
    turn ^= 1;
    return c;
  };
  // x: reached by at least sel keys (or 1: by all that may be chosen), with as many bits decided as it takes
  uint64_t x = 0;
  int n = reach(1);
  if (n <= sel) {
    x = 1;
  } else {
    for (int bit = 63; bit >= 0 && n != sel; --bit) {
      const uint64_t y = x | (uint64_t)1 << bit;
      const int c = reach(y);
      if (c >= sel) {
        x = y;
        n = c;
      }
    }
  }
  // n keys reach x.  If they are more than sel, x is the sel-th largest key itself: of those equal to it the first are taken
  int equal_left = sel;
  if (n > sel) equal_left = sel - (x == ~(uint64_t)0 ? 0 : reach(x + 1));
  else equal_left = n;
  const bool ties = n > sel;
  int32_t *out = blocks + row * sel;
  int at = 0;
  __shared__ int chosen[2][2][4];
  for (int i = 0; i < k.rounds(); ++i) {
    const uint64_t v = k.at(i);
    const bool eq = ties && v == x, over = ties ? v > x : v >= x;
    const uint64_t m_eq = __ballot(eq), m_over = __ballot(over), below = ((uint64_t)1 << lane) - 1;
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
    const int taken_before = over_before + (ties ? min(eq_before, equal_left) : 0);
    if (over || (eq && eq_before < equal_left)) out[at + taken_before] = i * 256 + threadIdx.x;
    at += over_all + (ties ? min(eq_all, equal_left) : 0);
    equal_left -= ties ? min(eq_all, equal_left) : 0;
  }
  for (int i = at + threadIdx.x; i < sel; i += 256) out[i] = -1;
}

// ---- fp32 tensors as three bf16 images -----------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void split_kernel(Sparse s, SplitJob j) {
  constexpr int TPR = D / 8, RPB = 256 / TPR;
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR, rows = (int64_t)s.B * j.heads * j.n;
  if (row >= rows) return;
  const int c = 8 * (threadIdx.x % TPR), n = (int)(row % j.n), h = (int)(row / j.n % j.heads), b = (int)(row / j.n / j.heads);
  const f32x4 *p = reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(j.in.p) + b * j.in.sb + h * j.in.sh + n * j.in.sn + c);
  const f32x4 a = p[0], d = p[1];
  const f32x8 x = {a.x, a.y, a.z, a.w, d.x, d.y, d.z, d.w};
  bf16x8 out[3];
  split8<3>(x, out);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (!__builtin_isfinite(x[i])) out[1][i] = out[2][i] = static_cast<__bf16>(0.f);      // (inf - inf)
#pragma unroll
  for (int p3 = 0; p3 < 3; ++p3) *reinterpret_cast<bf16x8 *>(j.out + (p3 * rows + row) * D + c) = out[p3];
}

size_t sums_bytes(const Sparse &s, int d) { return round256((size_t)s.B * s.Hkv * s.T * d * 8); }

// Blocks that are always kept, at most.
int64_t forced_blocks(const ha_sparse_problem &p) {
  int64_t n = p.keep_first;
  if (p.near_tokens >= 0) {
    const int64_t span = (p.N_q < p.q_block ? p.N_q : p.q_block) + (int64_t)p.near_tokens * (p.causal ? 1 : 2);
    n += (span - 1 + p.k_block - 1) / p.k_block + 1;
  }
  return n;
}

}  // namespace

hipError_t launch_split(const Sparse &s, int d, const SplitJob *jobs, int n_jobs, hipStream_t st) {
  for (int i = 0; i < n_jobs; ++i) {
    const int64_t rows = (int64_t)s.B * jobs[i].heads * jobs[i].n;
    if (rows == 0) continue;
    const int rpb = 256 / (d / 8);
    const unsigned blocks = (unsigned)((rows + rpb - 1) / rpb);
    if (d == 128) split_kernel<128><<<blocks, 256, 0, st>>>(s, jobs[i]);
    else split_kernel<64><<<blocks, 256, 0, st>>>(s, jobs[i]);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
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
  return sums_bytes(s, p->d_head) + round256((size_t)s.B * s.Hkv * s.T * s.Tk * 8);
}

extern "C" ha_status hybrid_attn_select_blocks(const ha_sparse_problem *p, const ha_view *q, const float *means, int32_t *blocks, void *workspace,
                                               size_t workspace_bytes, void *hip_stream) {
  ha_status st = check_sparse(p);
  if (st != HA_OK) return st;
  View qv;
  if ((st = check_view(*p, q, p->H, p->N_q, p->q_block, false, qv)) != HA_OK) return st;
  const Sparse s = sparse_of(*p);
  if (p->causal && p->near_tokens < 0) return HA_ERR_SHAPE;
  if (p->n_select < s.Tk && forced_blocks(*p) > p->n_select) return HA_ERR_SHAPE;
  if (p->N_q == 0) return HA_OK;
  if (!blocks || (p->N_k > 0 && !means)) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(means) & 15u || reinterpret_cast<uintptr_t>(blocks) & 3u) return HA_ERR_ALIGN;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < hybrid_attn_select_workspace_bytes(p)) return HA_ERR_WORKSPACE;
  double *sums = static_cast<double *>(workspace);
  uint64_t *keys = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + sums_bytes(s, p->d_head));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const unsigned rows = (unsigned)s.B * s.Hkv * s.T;
  hipError_t e;
  if (s.Tk > 0) {
#define HA_SUMS(D, F) query_sums_kernel<D, F><<<rows, 256, 0, stream>>>(s, qv, sums)
    if (p->d_head == 128) { if (p->dtype == HA_F32) HA_SUMS(128, true); else HA_SUMS(128, false); }
    else { if (p->dtype == HA_F32) HA_SUMS(64, true); else HA_SUMS(64, false); }
#undef HA_SUMS
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
    constexpr int TILES = 8;
    const ScoreArgs a{s, sums, means, keys, p->keep_first, p->near_tokens};
    const dim3 grid((s.Tk + 255) / 256, (s.T + TILES - 1) / TILES, s.B * s.Hkv);
    if (p->d_head == 128) scores_kernel<128, TILES><<<grid, 256, 0, stream>>>(a);
    else scores_kernel<64, TILES><<<grid, 256, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
  }
#define HA_CHOOSE(V) choose_kernel<V><<<rows, 256, 0, stream>>>(keys, s.Tk, s.sel, blocks)
  if (s.Tk <= 256) HA_CHOOSE(1);
  else if (s.Tk <= 512) HA_CHOOSE(2);
  else if (s.Tk <= 1024) HA_CHOOSE(4);
  else if (s.Tk <= 2048) HA_CHOOSE(8);
  else HA_CHOOSE(0);
#undef HA_CHOOSE
  e = hipGetLastError();
  return e == hipSuccess ? HA_OK : device_error(e);
}
