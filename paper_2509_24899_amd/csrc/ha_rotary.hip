// Rotary positions, alone and behind the norm of every head's row, gfx950: forward and gradients.
//
//   out = R (w n),  n = x r,  r = (mean x^2 + eps)^-1/2            g = R^T dout,  h = w g,  dx = r (h - n mean(h n)),  dw = sum over rows of g n
//
// Memory is what bounds these: a row is read once (the gradient: two rows) and written once.  D / 8 threads hold a row, a workgroup 16 or 32 tokens of all
// heads: the angles of a token, which take some 200 instructions a thread, are formed once and serve every head.
#include <cmath>

#include "ha_rows.h"

#include <algorithm>

namespace ha {

ha_status check_rotary(const ha_rotary *r, int d_head, int64_t tokens, bool one_list, Rotary &out) {
  if (!r) return HA_ERR_NULL;
  out = Rotary{r->freq, r->axis, r->positions, r->positions_stride_b, r->rot_dim, r->n_axes, r->magnitude};
  if (r->rot_dim < 0 || r->rot_dim > d_head || r->rot_dim % 2) return HA_ERR_SHAPE;
  if (r->interleaved != 0 && r->interleaved != 1) return HA_ERR_SHAPE;
  if (!r->interleaved && r->rot_dim % 8) return HA_ERR_UNSUPPORTED;
  if (r->rot_dim == 0) {
    out.axis = nullptr;
    return HA_OK;
  }
  if (r->n_axes < 1 || r->n_axes > 4 || !std::isfinite(r->magnitude)) return HA_ERR_SHAPE;
  if (r->positions_stride_b != 0 && (one_list || r->positions_stride_b < tokens * r->n_axes || r->positions_stride_b > (int64_t)1 << 44)) return HA_ERR_SHAPE;
  if (!r->freq || (!r->positions && tokens > 0)) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(r->freq) & 7u || reinterpret_cast<uintptr_t>(r->axis) & 3u || reinterpret_cast<uintptr_t>(r->positions) & 3u) return HA_ERR_ALIGN;
  return HA_OK;
}

ha_status check_rows(int B, int heads, int64_t n, int d, int dtype, const ha_view *v, bool written, View &out) {
  if (!v) return HA_ERR_NULL;
  out = View{static_cast<char *>(v->data), v->stride_b, v->stride_h, v->stride_n};
  if (n == 0 || heads == 0) return HA_OK;
  if (!v->data) return HA_ERR_NULL;
  const int64_t per16 = dtype == HA_BF16 ? 8 : 4, most = (int64_t)1 << 44;
  if (n == 1) out.sn = d;
  if (heads == 1) out.sh = n * out.sn;
  if (B == 1) out.sb = heads * out.sh;
  if (out.sn < 0 || out.sh < 0 || out.sb < 0 || (written && (out.sn < d || out.sh < d || out.sb < d))) return HA_ERR_SHAPE;
  if (out.sn > most || out.sh > most || out.sb > most) return HA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(v->data) & 15u || out.sn % per16 || out.sh % per16 || out.sb % per16) return HA_ERR_ALIGN;
  return HA_OK;
}

namespace {

struct RowsArgs {
  int N, H, heads;            // heads: H of the queries, then those of the keys
  unsigned groups;            // of tokens, in a batch entry
  View x[2], g[2], y[2];      // queries and keys: inputs, gradients of the outputs, what is written
  const float *w[2];
  Rotary rot;
  float eps, sign;            // sign of the sine: -1 transposes
  float *partial;             // gradient: [workgroup][2][D]
};

template <int D>
struct Group {
  static constexpr int TPR = D / 8, ROWS = 256 / TPR;      // threads to a row, tokens to a workgroup
};

// U: heads whose rows are asked for at once.  Four where there are many tokens (12 + 12 heads of 2 x 75600 tokens: forward 341 us with four, 346 with one, gradients 506 and 502), one
// where the launch is short and what counts is the code that has to be fetched (two heads of 1024 tokens: 3.5 us with one, 3.8 with four).
template <int D, bool F32, bool NEXT, bool NORM, int U, bool ONCE>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a) {
  typedef Group<D> G;
  const int t = threadIdx.x % G::TPR;
  const int64_t b = blockIdx.x / a.groups;
  const int n_ = (blockIdx.x % a.groups) * G::ROWS + threadIdx.x / G::TPR;
  const bool there = n_ < a.N;
  const int n = there ? n_ : a.N - 1;
  int ca, cb;
  own_channels<NEXT>(t, a.rot.rot, ca, cb);
  f32x4 c, s;
  pair_angles(a.rot, a.rot.positions + b * a.rot.positions_sb + (int64_t)n * a.rot.n_axes, t, c, s);
  s *= a.sign;
  const int pairs = a.rot.rot / 2 - 4 * t;
  Row8 w[2];
  if constexpr (NORM) {
    w[0] = weight8(a.w[0], ca, cb);
    w[1] = weight8(a.w[1], ca, cb);
  }
  for (int h0 = blockIdx.y * U; h0 < a.heads; h0 += gridDim.y * U) {
    Row8 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int hh = min(h0 + u, a.heads - 1), k = hh >= a.H;
      const View &v = a.x[k];
      x[u] = load_row8<F32, NEXT, ONCE>(v.p, b * v.sb + (hh - (k ? a.H : 0)) * v.sh + n * v.sn, ca, cb);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int hh = h0 + u, k = hh >= a.H;
      if (hh >= a.heads) break;
      if constexpr (NORM) x[u] = times(times(x[u], inverse_rms<D>(x[u], a.eps)), k ? w[1] : w[0]);
      const Row8 y = turn<NEXT>(x[u], c, s, pairs);
      const View &v = a.y[k];
      if (there) store_row8<F32, NEXT, ONCE>(v.p, b * v.sb + (hh - (k ? a.H : 0)) * v.sh + n * v.sn, ca, cb, y);
    }
  }
}

// The gradient.  A workgroup walks groups of tokens and leaves its sums over rows of the weights' gradients, which a second kernel adds up.  (12 + 12 heads of 2 x 75600 tokens: 506 us
// for three streams, 5.5 TB/s; the forward 341 us for two, 5.4.  Sums by atomics would be in another order every time.)
template <int D, bool F32, bool NEXT, bool SUMS, int U, bool ONCE>
__global__ __launch_bounds__(256) void rows_grad_kernel(RowsArgs a, unsigned all_groups) {
  typedef Group<D> G;
  __shared__ float lds[SUMS ? G::ROWS * D : 1];
  const int t = threadIdx.x % G::TPR, row = threadIdx.x / G::TPR;
  int ca, cb;
  own_channels<NEXT>(t, a.rot.rot, ca, cb);
  const Row8 w[2] = {weight8(a.w[0], ca, cb), weight8(a.w[1], ca, cb)};
  const int pairs = a.rot.rot / 2 - 4 * t;
  const f32x4 none = {0.f, 0.f, 0.f, 0.f};
  Row8 sum[2] = {{none, none}, {none, none}};
  for (unsigned group = blockIdx.x; group < all_groups; group += gridDim.x) {
    const int64_t b = group / a.groups;
    const int n_ = (group % a.groups) * G::ROWS + row;
    const bool there = n_ < a.N;
    const int n = there ? n_ : a.N - 1;
    f32x4 c, s;
    pair_angles(a.rot, a.rot.positions + b * a.rot.positions_sb + (int64_t)n * a.rot.n_axes, t, c, s);
    for (int h0 = blockIdx.y * U; h0 < a.heads; h0 += gridDim.y * U) {
      Row8 x[U], g[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int hh = min(h0 + u, a.heads - 1), k = hh >= a.H;
        const int64_t h = hh - (k ? a.H : 0);
        x[u] = load_row8<F32, NEXT, ONCE>(a.x[k].p, b * a.x[k].sb + h * a.x[k].sh + n * a.x[k].sn, ca, cb);
        g[u] = load_row8<F32, NEXT, ONCE>(a.g[k].p, b * a.g[k].sb + h * a.g[k].sh + n * a.g[k].sn, ca, cb);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int hh = h0 + u, k = hh >= a.H;
        if (hh >= a.heads) break;
        const int64_t h = hh - (k ? a.H : 0);
        const Row8 gt = turn<NEXT>(g[u], c, -s, pairs), gw = times(gt, k ? w[1] : w[0]);
        const float r = inverse_rms<D>(x[u], a.eps);
        const Row8 nx = times(x[u], r);
        const float mean = row_sum<D>(dot4(gw.a, nx.a) + dot4(gw.b, nx.b)) * (1.f / D);
        const Row8 y = Row8{(gw.a - nx.a * mean) * r, (gw.b - nx.b * mean) * r};
        if (there) {
          store_row8<F32, NEXT, ONCE>(a.y[k].p, b * a.y[k].sb + h * a.y[k].sh + n * a.y[k].sn, ca, cb, y);
          if constexpr (SUMS) {
            if (k) {
              sum[1].a += gt.a * nx.a;
              sum[1].b += gt.b * nx.b;
            } else {
              sum[0].a += gt.a * nx.a;
              sum[0].b += gt.b * nx.b;
            }
          }
        }
      }
    }
  }
  if constexpr (SUMS) {
    float *out = a.partial + (int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * 2 * D;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      __syncthreads();
      *reinterpret_cast<f32x4 *>(lds + row * D + ca) = sum[k].a;
      *reinterpret_cast<f32x4 *>(lds + row * D + cb) = sum[k].b;
      __syncthreads();
      if (threadIdx.x < D) {
        float total = 0.f;
        for (int i = 0; i < G::ROWS; ++i) total += lds[i * D + threadIdx.x];
        out[k * D + threadIdx.x] = total;
      }
    }
  }
}

// Sum of the workgroups' sums, 16 columns to a workgroup, in double (1024 of them: 6.7 us).
__global__ __launch_bounds__(1024) void weight_sums_kernel(const float *partial, int n, int width, int D, float *dw_q, float *dw_k) {
  constexpr int U = 8;        // loads in flight
  __shared__ double lds[64][17];
  const int c = threadIdx.x % 16, r = threadIdx.x / 16, col = blockIdx.x * 16 + c;
  double sum = 0.;
  for (int i = r; i < n; i += 64 * U) {
    float x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = i + 64 * u < n ? partial[(int64_t)(i + 64 * u) * width + col] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) sum += (double)x[u];
  }
  lds[r][c] = sum;
  __syncthreads();
  for (int half = 32; half > 0; half /= 2) {
    if (r < half) lds[r][c] += lds[r + half][c];
    __syncthreads();
  }
  float *out = col < D ? dw_q : dw_k;
  if (r == 0 && out) out[col % D] = (float)lds[0][c];
}

ha_status check_problem(const ha_rows_problem *p) {
  if (!p) return HA_ERR_NULL;
  if (p->B <= 0 || p->H <= 0 || p->H_kv < 0 || p->N < 0 || p->d_head <= 0) return HA_ERR_SHAPE;
  if (!(p->eps >= 0.f) || !std::isfinite(p->eps)) return HA_ERR_SHAPE;
  if (p->dtype != HA_BF16 && p->dtype != HA_F32) return HA_ERR_UNSUPPORTED;
  if (p->d_head != 64 && p->d_head != 128) return HA_ERR_UNSUPPORTED;
  if ((int64_t)p->B * p->H > 65535 || (int64_t)p->B * p->H_kv > 65535 || (int64_t)p->B * p->N > (1 << 27)) return HA_ERR_UNSUPPORTED;
  return HA_OK;
}
ha_status check_both(const ha_rows_problem *p, const ha_rotary *r, RowsArgs &a) {
  ha_status st = check_problem(p);
  if (st != HA_OK || (st = check_rotary(r, p->d_head, p->N, false, a.rot)) != HA_OK) return st;
  a.N = p->N;
  a.H = p->H;
  a.heads = p->H + p->H_kv;
  a.eps = p->eps;
  a.sign = 1.f;
  const int rows = 256 / (p->d_head / 8);
  a.groups = (p->N + rows - 1) / rows;
  return HA_OK;
}
ha_status check_weight(const float *w) { return reinterpret_cast<uintptr_t>(w) & 15u ? HA_ERR_ALIGN : HA_OK; }

// Workgroups: a group of tokens each, of all heads; where those are few, the heads are dealt to several and taken one at a time.
bool is_short(int64_t groups) { return groups < 512; }
dim3 grid_of(int64_t groups, int heads) { return dim3((unsigned)groups, is_short(groups) ? (unsigned)std::min<int64_t>(heads, (512 + groups - 1) / groups) : 1); }
int64_t groups_of(const ha_rows_problem &p) {
  const int rows = 256 / (p.d_head / 8);
  return (int64_t)p.B * ((p.N + rows - 1) / rows);
}
dim3 grad_grid(const ha_rows_problem &p) { return grid_of(std::min<int64_t>(std::max<int64_t>(groups_of(p), 1), 1024), p.H + p.H_kv); }

enum Form { kShort, kMany, kOnce };
Form form_of(const ha_rows_problem &p, int streams) {
  if (is_short(groups_of(p))) return kShort;
  return stream_once((int64_t)streams * p.B * (p.H + p.H_kv) * p.N * p.d_head * (p.dtype == HA_F32 ? 4 : 2)) ? kOnce : kMany;
}
template <int D, bool F32, bool NEXT, bool NORM>
hipError_t launch_rows(const RowsArgs &a, dim3 grid, Form form, hipStream_t st) {
  if (form == kShort) rows_kernel<D, F32, NEXT, NORM, 1, false><<<grid, 256, 0, st>>>(a);
  else if (form == kMany) rows_kernel<D, F32, NEXT, NORM, 4, false><<<grid, 256, 0, st>>>(a);
  else rows_kernel<D, F32, NEXT, NORM, 4, true><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}
template <int D, bool F32>
hipError_t launch_rows(const RowsArgs &a, dim3 grid, Form form, bool next, bool norm, hipStream_t st) {
  if (next) return norm ? launch_rows<D, F32, true, true>(a, grid, form, st) : launch_rows<D, F32, true, false>(a, grid, form, st);
  return norm ? launch_rows<D, F32, false, true>(a, grid, form, st) : launch_rows<D, F32, false, false>(a, grid, form, st);
}
hipError_t launch_rows(const ha_rows_problem &p, const RowsArgs &a, bool next, bool norm, hipStream_t st) {
  const dim3 grid = grid_of(groups_of(p), a.heads);
  const Form form = form_of(p, 2);
  if (p.d_head == 128) return p.dtype == HA_F32 ? launch_rows<128, true>(a, grid, form, next, norm, st) : launch_rows<128, false>(a, grid, form, next, norm, st);
  return p.dtype == HA_F32 ? launch_rows<64, true>(a, grid, form, next, norm, st) : launch_rows<64, false>(a, grid, form, next, norm, st);
}
template <int D, bool F32, bool NEXT, bool SUMS>
hipError_t launch_grad(const RowsArgs &a, dim3 grid, unsigned groups, Form form, hipStream_t st) {
  if (form == kShort) rows_grad_kernel<D, F32, NEXT, SUMS, 1, false><<<grid, 256, 0, st>>>(a, groups);
  else if (form == kMany) rows_grad_kernel<D, F32, NEXT, SUMS, 4, false><<<grid, 256, 0, st>>>(a, groups);
  else rows_grad_kernel<D, F32, NEXT, SUMS, 4, true><<<grid, 256, 0, st>>>(a, groups);
  return hipGetLastError();
}
template <int D, bool F32>
hipError_t launch_grad(const RowsArgs &a, dim3 grid, unsigned groups, Form form, bool next, hipStream_t st) {
  if (a.partial) return next ? launch_grad<D, F32, true, true>(a, grid, groups, form, st) : launch_grad<D, F32, false, true>(a, grid, groups, form, st);
  return next ? launch_grad<D, F32, true, false>(a, grid, groups, form, st) : launch_grad<D, F32, false, false>(a, grid, groups, form, st);
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" ha_status hybrid_attn_rotary_validate(const ha_rows_problem *p, const ha_rotary *r) {
  RowsArgs a{};
  return check_both(p, r, a);
}

extern "C" ha_status hybrid_attn_rotate(const ha_rows_problem *p, const ha_rotary *r, const ha_view *x, const ha_view *out, int32_t transposed, void *hip_stream) {
  RowsArgs a{};
  ha_status st = check_both(p, r, a);
  if (st != HA_OK) return st;
  if (p->H_kv != 0 || (transposed != 0 && transposed != 1)) return HA_ERR_SHAPE;
  if ((st = check_rows(p->B, p->H, p->N, p->d_head, p->dtype, x, false, a.x[0])) != HA_OK ||
      (st = check_rows(p->B, p->H, p->N, p->d_head, p->dtype, out, true, a.y[0])) != HA_OK)
    return st;
  if (p->N == 0) return HA_OK;
  a.sign = transposed ? -1.f : 1.f;
  const hipError_t e = launch_rows(*p, a, r->interleaved, false, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? HA_OK : device_error(e);
}

extern "C" ha_status hybrid_attn_norm_rotate(const ha_rows_problem *p, const ha_rotary *r, const ha_view *q, const ha_view *k, const float *w_q, const float *w_k,
                                             const ha_view *q_out, const ha_view *k_out, void *hip_stream) {
  RowsArgs a{};
  ha_status st = check_both(p, r, a);
  if (st != HA_OK) return st;
  if ((st = check_rows(p->B, p->H, p->N, p->d_head, p->dtype, q, false, a.x[0])) != HA_OK ||
      (st = check_rows(p->B, p->H, p->N, p->d_head, p->dtype, q_out, true, a.y[0])) != HA_OK || (st = check_weight(w_q)) != HA_OK)
    return st;
  a.w[0] = w_q;
  if (p->H_kv > 0) {
    if ((st = check_rows(p->B, p->H_kv, p->N, p->d_head, p->dtype, k, false, a.x[1])) != HA_OK ||
        (st = check_rows(p->B, p->H_kv, p->N, p->d_head, p->dtype, k_out, true, a.y[1])) != HA_OK || (st = check_weight(w_k)) != HA_OK)
      return st;
    a.w[1] = w_k;
  }
  if (p->N == 0) return HA_OK;
  const hipError_t e = launch_rows(*p, a, r->interleaved, true, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? HA_OK : device_error(e);
}

extern "C" size_t hybrid_attn_norm_rotate_grad_workspace_bytes(const ha_rows_problem *p) {
  if (check_problem(p) != HA_OK) return 0;
  const dim3 g = grad_grid(*p);
  return (size_t)g.x * g.y * 2 * p->d_head * 4;
}

extern "C" ha_status hybrid_attn_norm_rotate_grad(const ha_rows_problem *p, const ha_rotary *r, const ha_view *grad_q, const ha_view *grad_k, const ha_view *q, const ha_view *k,
                                                  const float *w_q, const float *w_k, const ha_view *grad_in_q, const ha_view *grad_in_k, float *grad_w_q, float *grad_w_k,
                                                  void *workspace, size_t workspace_bytes, void *hip_stream) {
  RowsArgs a{};
  ha_status st = check_both(p, r, a);
  if (st != HA_OK) return st;
  const bool keys = p->H_kv > 0;
  for (int i = 0; i < (keys ? 2 : 1); ++i) {
    const int heads = i ? p->H_kv : p->H;
    if ((st = check_rows(p->B, heads, p->N, p->d_head, p->dtype, i ? grad_k : grad_q, false, a.g[i])) != HA_OK ||
        (st = check_rows(p->B, heads, p->N, p->d_head, p->dtype, i ? k : q, false, a.x[i])) != HA_OK ||
        (st = check_rows(p->B, heads, p->N, p->d_head, p->dtype, i ? grad_in_k : grad_in_q, true, a.y[i])) != HA_OK || (st = check_weight(i ? w_k : w_q)) != HA_OK)
      return st;
    a.w[i] = i ? w_k : w_q;
  }
  if (reinterpret_cast<uintptr_t>(grad_w_q) & 3u || (keys && reinterpret_cast<uintptr_t>(grad_w_k) & 3u)) return HA_ERR_ALIGN;
  if (!keys) grad_w_k = nullptr;
  const dim3 grid = grad_grid(*p);
  const int d = p->d_head;
  if (grad_w_q || grad_w_k) {
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) & 255u || workspace_bytes < (size_t)grid.x * grid.y * 2 * d * 4) return HA_ERR_WORKSPACE;
    a.partial = static_cast<float *>(workspace);
  }
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  const unsigned groups = (unsigned)p->B * a.groups;      // (without tokens the sums are those of no rows)
  if (p->N == 0 && !a.partial) return HA_OK;
  const Form form = form_of(*p, 3);
  const bool next = r->interleaved;
  if (d == 128) e = p->dtype == HA_F32 ? launch_grad<128, true>(a, grid, groups, form, next, stream) : launch_grad<128, false>(a, grid, groups, form, next, stream);
  else e = p->dtype == HA_F32 ? launch_grad<64, true>(a, grid, groups, form, next, stream) : launch_grad<64, false>(a, grid, groups, form, next, stream);
  if (e != hipSuccess) return device_error(e);
  if (a.partial) {
    weight_sums_kernel<<<2 * d / 16, 1024, 0, stream>>>(a.partial, (int)(grid.x * grid.y), 2 * d, d, grad_w_q, grad_w_k);
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
  }
  return HA_OK;
}
