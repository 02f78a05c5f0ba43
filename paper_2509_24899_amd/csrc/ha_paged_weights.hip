// The weight that every slot of a paged cache gets from new tokens, gfx950.
//
//   w_j += sum over rows R that see slot j of exp(scale q_R . k_j - lse_R)
//
// A wave owns 32 slots, whose keys stay in its registers, and walks the rows 32 at a time: S = Q K^T with the slot as the lane's column, so that a slot's sum is a
// lane's own.  Single tokens: bound by reading the keys.  Chunks: an exponential for every row and slot next to 2 d operations of the matrix cores, which
// take about as long.
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
  int blocks;                 // of 128 slots, in a sequence
};

template <int D, bool F32>
__global__ __launch_bounds__(256) void paged_weights_kernel(WeightArgs a) {
  constexpr int KS = D / 16, NS = F32 ? 3 : 1, ESZ = F32 ? 4 : 2;
  __shared__ float shift[4][32];      // [wave][row]: - lse log2 e
  __shared__ int sees[4][32];         // slots that the row sees
  const Paged &p = a.p;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int bh = blockIdx.x / a.blocks, b = bh / p.Hkv, hk = bh % p.Hkv, slot0 = (blockIdx.x % a.blocks) * 128 + 32 * w, slot = slot0 + r;
  const NewRows n(p, b);
  const int held = p.held(b), n_rows = n.n * p.G, before = held - n.all;      // before: slots ahead of the first new token's
  if (slot0 >= p.capacity()) return;
  float sum = 0.f;
  if (slot0 < held && n_rows > 0) {
    const int R_first = p.causal ? max(slot0 - before, 0) * p.G / 32 * 32 : 0;      // (of the 32 rows with the first that sees the wave's first slot)
    const int id = slot < held ? p.page_of(b, slot) : -1;
    const char *kp = a.k.p + (hk * a.k.sh + (id < 0 ? 0 : (int64_t)id * a.k.sb + (int64_t)(slot & (p.page - 1)) * a.k.sn) + 8 * g) * ESZ;
    bf16x8 kf[KS][NS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (F32) {
        f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
        if (id >= 0) {
          lo = *reinterpret_cast<const f32x4 *>(kp + 64 * ks);
          hi = *reinterpret_cast<const f32x4 *>(kp + 64 * ks + 16);
        }
        split8_any(lo, hi, kf[ks]);
      } else {
        bf16x8 x = {};
        if (id >= 0) x = *reinterpret_cast<const bf16x8 *>(kp + 32 * ks);
        kf[ks][0] = x;
      }
    }
    for (int R0 = R_first; R0 < n_rows; R0 += 32) {
      const int R = R0 + r, Rc = min(R, n_rows - 1), i = Rc / p.G, h = hk * p.G + Rc - i * p.G;
      const int64_t token = n.first + i;
      const char *qp = a.q.p + (h * a.q.sh + token * a.q.sn + 8 * g) * ESZ;
      const float x = a.lse[token * p.H + h];
      const int see = p.causal ? min(held, before + i + 1) : held;
      if (g == 0) {
        shift[w][r] = R < n_rows && x != -INFINITY ? -x * kLog2e : -INFINITY;
        sees[w][r] = see;
      }
      f32x16 sc;
#pragma unroll
      for (int y = 0; y < 16; ++y) sc[y] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 qf[NS];
        if constexpr (F32) split8_any(*reinterpret_cast<const f32x4 *>(qp + 64 * ks), *reinterpret_cast<const f32x4 *>(qp + 64 * ks + 16), qf);
        else qf[0] = *reinterpret_cast<const bf16x8 *>(qp + 32 * ks);
        sc = mfma_split<NS>(qf, kf[ks], sc);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // (a wave's LDS instructions execute in order)
#pragma unroll
      for (int y4 = 0; y4 < 4; ++y4) {
        const f32x4 t = *reinterpret_cast<const f32x4 *>(&shift[w][8 * y4 + 4 * g]);
        const int *s = &sees[w][8 * y4 + 4 * g];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const float e = fast_exp2(__builtin_fmaf(sc[4 * y4 + y], a.scale_log2e, t[y]));
          sum += slot < s[y] && t[y] != -INFINITY ? e : 0.f;
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    if (id < 0) sum = 0.f;
  }
  sum = xhalf_sum(sum);
  if (g == 0 && slot < p.capacity()) {
    const int64_t at = (int64_t)bh * p.capacity() + slot;
    a.out[at] = (a.weights ? a.weights[at] : 0.f) + sum;
  }
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" size_t hybrid_attn_paged_weights_workspace_bytes(const ha_paged_problem *p) {
  (void)p;
  return 0;
}

extern "C" ha_status hybrid_attn_paged_weights(const ha_paged_problem *p, const ha_view *q, const ha_view *k_pages, const float *lse, const float *weights, float *weights_out,
                                               void *workspace, size_t workspace_bytes, void *hip_stream) {
  ha_status st = check_paged(p);
  if (st != HA_OK) return st;
  WeightArgs a{};
  if ((st = check_packed(*p, q, p->H, false, a.q)) != HA_OK || (st = check_pool(*p, k_pages, false, a.k)) != HA_OK) return st;
  const int64_t slots = (int64_t)p->max_pages * p->page, blocks = (slots + 127) / 128;
  if ((int64_t)p->B * p->H_kv * blocks > (1 << 23)) return HA_ERR_UNSUPPORTED;
  if ((p->T > 0 && !lse) || (slots > 0 && !weights_out)) return HA_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(weights) | reinterpret_cast<uintptr_t>(weights_out)) & 3u) return HA_ERR_ALIGN;
  if ((st = check_workspace(workspace, workspace_bytes, hybrid_attn_paged_weights_workspace_bytes(p))) != HA_OK) return st;
  if (slots == 0) return HA_OK;
  a.p = paged_of(*p);
  a.lse = lse;
  a.weights = weights;
  a.out = weights_out;
  a.scale_log2e = p->softmax_scale * kLog2e;
  a.blocks = (int)blocks;
  const unsigned grid = (unsigned)(p->B * p->H_kv * blocks);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool f32 = p->dtype == HA_F32;
  if (p->d_head == 128) { if (f32) paged_weights_kernel<128, true><<<grid, 256, 0, stream>>>(a); else paged_weights_kernel<128, false><<<grid, 256, 0, stream>>>(a); }
  else { if (f32) paged_weights_kernel<64, true><<<grid, 256, 0, stream>>>(a); else paged_weights_kernel<64, false><<<grid, 256, 0, stream>>>(a); }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? HA_OK : device_error(e);
}
