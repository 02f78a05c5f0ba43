// Global gradient norm, clipping and the update of many parameters, gfx950.
//
//   norm = sqrt(sum g^2) over all tensors, factor = min(1, max_norm / norm), clipped g = factor g, update with factor g.
//
// All of it is bound by memory: the norm reads every gradient once, the clip reads and writes them once more, AdamW moves 28 bytes a value
// (30 with a bf16 copy).  So tensors are cut into pieces of one size, a workgroup each, whatever tensor they belong to: many small tensors
// cost what one large tensor costs, and a launch takes as many tensors as its arguments hold.  The sum of squares is kept in double (a square of
// an fp32 value cannot overflow there, and 2^30 terms lose nothing that fp32 would show) and joined in the order of the pieces.
//
// 71 M values in 240 tensors (fp32 gradients, AdamW, bf16 copies of the weights): norm 82 us in two launches (3.5 TB/s) and 5 us of joining, update 370 us in
// five (5.8 TB/s); of 2.4 M values in eight the launches are what it takes (norm 7.3 us, clip 4.5).
#include "ha_plan.h"
#include "ha_update.h"

#include "../../include/hybrid_attn_optim.h"

namespace ha {
namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));    // (16-byte accesses need no more than the element's alignment)
typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr uint64_t kPiece = 8192;        // elements of a workgroup's piece, a multiple of 4 * 256 (norm and update of 71 M values: 520 us, 520 with 4096, 555 with 16384)
constexpr uint64_t kMaxPieces = 16384;   // beyond, pieces grow: the joining workgroup reads them all
constexpr uint64_t kFewPieces = 1024;   // fewer than these, and pieces are smaller (piece_size)
constexpr int kThreads = 256;

template <bool F32>
__device__ __forceinline__ f32x4 load4(const void *p, uint64_t i) {
  if constexpr (F32) return *reinterpret_cast<const f32x4u *>(static_cast<const float *>(p) + i);
  else return __builtin_convertvector(static_cast<bf16x4>(*reinterpret_cast<const bf16x4u *>(static_cast<const __bf16 *>(p) + i)), f32x4);
}
template <bool F32>
__device__ __forceinline__ float load1(const void *p, uint64_t i) {
  if constexpr (F32) return static_cast<const float *>(p)[i];
  else return static_cast<float>(static_cast<const __bf16 *>(p)[i]);
}
__device__ __forceinline__ void store4(void *p, uint64_t i, f32x4 x, bool f32) {
  if (f32) *reinterpret_cast<f32x4u *>(static_cast<float *>(p) + i) = x;
  else *reinterpret_cast<bf16x4u *>(static_cast<__bf16 *>(p) + i) = __builtin_convertvector(x, bf16x4);
}
__device__ __forceinline__ void store1(void *p, uint64_t i, float x, bool f32) {
  if (f32) static_cast<float *>(p)[i] = x;
  else static_cast<__bf16 *>(p)[i] = static_cast<__bf16>(x);
}

// Tensors of one launch: first[t] is the number of pieces ahead of tensor t within it.
template <int MAX>
struct Pieces {
  uint64_t piece;             // elements of a piece
  uint32_t first[MAX + 1];
  int n;
  // tensor of piece b
  __device__ __forceinline__ int tensor(uint32_t b) const {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= b) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  }
};

constexpr int kNormTensors = 128;
struct NormArgs {
  const void *data[kNormTensors];
  uint64_t n[kNormTensors];
  uint8_t f32[kNormTensors];
  Pieces<kNormTensors> at;
  double *partial;            // of the launch's first piece
};

template <bool F32, int THREADS>
__device__ __forceinline__ double sum_squares(const void *p, uint64_t lo, uint64_t hi) {
  const unsigned thread = threadIdx.x % THREADS;
  double s[4] = {0., 0., 0., 0.};
  const uint64_t full = lo + ((hi - lo) & ~(uint64_t)3);
#pragma unroll 4
  for (uint64_t i = lo + 4 * thread; i < full; i += 4 * THREADS) {
    const f32x4 x = load4<F32>(p, i);
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = __builtin_fma((double)x[j], (double)x[j], s[j]);
  }
  if (full + thread < hi) {
    const double x = (double)load1<F32>(p, full + thread);
    s[0] = __builtin_fma(x, x, s[0]);
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Sum over the workgroup in a fixed order; thread 0 has it.
template <int THREADS>
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[THREADS / 64];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_down(x, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = part[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) s += part[w];
  return s;
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(NormArgs a) {
  const uint32_t b = blockIdx.x;
  const int t = a.at.tensor(b);
  const uint64_t lo = (uint64_t)(b - a.at.first[t]) * a.at.piece, hi = lo + a.at.piece < a.n[t] ? lo + a.at.piece : a.n[t];
  const double s = block_sum<kThreads>(a.f32[t] ? sum_squares<true, kThreads>(a.data[t], lo, hi) : sum_squares<false, kThreads>(a.data[t], lo, hi));
  if (threadIdx.x == 0) a.partial[b] = s;
}

__device__ __forceinline__ void store_result(double sum, float max_norm, float *result) {
  const double norm = sqrt(sum);
  result[0] = (float)norm;
  result[1] = !(norm < (double)INFINITY) ? NAN : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}

__global__ __launch_bounds__(1024) void grad_norm_join_kernel(const double *partial, uint32_t n, float max_norm, float *result) {
  double s = 0.;
  for (uint32_t i = threadIdx.x; i < n; i += 1024) s += partial[i];
  s = block_sum<1024>(s);
  if (threadIdx.x == 0) store_result(s, max_norm, result);
}

// All of it in one launch where the gradients are few: the waves of one workgroup take pieces in turn, three each at most.  Us with this kernel / the two
// above: 8192 values 4.9 / 7.3, 33 thousand in eight tensors (40 pieces) 4.9 / 7.3, 64 pieces 5.8 / 7.2 and 7.6 / 7.4 (in 4 and 64 tensors), 130 thousand 13.0 / 7.2.
constexpr uint64_t kSmallPiece = 1024, kSmallPieces = 48;
__global__ __launch_bounds__(1024) void grad_norm_small_kernel(NormArgs a, float max_norm, float *result) {
  double s = 0.;
  for (uint32_t b = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); b < a.at.first[a.at.n]; b += 16) {
    const int t = a.at.tensor(b);
    const uint64_t lo = (uint64_t)(b - a.at.first[t]) * kSmallPiece, hi = lo + kSmallPiece < a.n[t] ? lo + kSmallPiece : a.n[t];
    s += a.f32[t] ? sum_squares<true, 64>(a.data[t], lo, hi) : sum_squares<false, 64>(a.data[t], lo, hi);
  }
  s = block_sum<1024>(s);
  if (threadIdx.x == 0) store_result(s, max_norm, result);
}

constexpr int kClipTensors = 96;
struct ClipArgs {
  const void *in[kClipTensors];
  void *out[kClipTensors];
  uint64_t n[kClipTensors];
  uint8_t kind[kClipTensors];   // bit 0: in is fp32, bit 1: out is
  Pieces<kClipTensors> at;
  const float *result;
};

template <bool F32>
__device__ __forceinline__ void clip_piece(const void *in, void *out, uint64_t lo, uint64_t hi, float f, bool out_f32) {
  const uint64_t full = lo + ((hi - lo) & ~(uint64_t)3);
#pragma unroll 4
  for (uint64_t i = lo + 4 * threadIdx.x; i < full; i += 4 * kThreads) store4(out, i, load4<F32>(in, i) * f, out_f32);
  if (full + threadIdx.x < hi) store1(out, full + threadIdx.x, load1<F32>(in, full + threadIdx.x) * f, out_f32);
}

__global__ __launch_bounds__(kThreads) void grad_clip_kernel(ClipArgs a) {
  const float f = a.result[1];
  if (!__builtin_isfinite(f)) return;
  const uint32_t b = blockIdx.x;
  const int t = a.at.tensor(b);
  if (f == 1.f && a.in[t] == a.out[t]) return;
  const uint64_t lo = (uint64_t)(b - a.at.first[t]) * a.at.piece, hi = lo + a.at.piece < a.n[t] ? lo + a.at.piece : a.n[t];
  if (a.kind[t] & 1) clip_piece<true>(a.in[t], a.out[t], lo, hi, f, a.kind[t] & 2);
  else clip_piece<false>(a.in[t], a.out[t], lo, hi, f, a.kind[t] & 2);
}

constexpr int kUpdateTensors = 56;
struct ManyArgs {
  float *master[kUpdateTensors];
  const void *grad[kUpdateTensors];
  float *m[kUpdateTensors], *v[kUpdateTensors];
  void *io[kUpdateTensors];
  uint64_t n[kUpdateTensors];
  uint8_t kind[kUpdateTensors];   // bit 0: the gradient is fp32, bit 1: the copy is
  Pieces<kUpdateTensors> at;
  UpdateRates r;
  const float *result;
};

template <bool ADAMW, bool F32>
__device__ __forceinline__ void update_piece(const ManyArgs &a, int t, uint64_t lo, uint64_t hi, float scale) {
  float *master = a.master[t], *mm = a.m[t], *vv = a.v[t];
  const void *grad = a.grad[t];
  void *io = a.io[t];
  const bool io_f32 = a.kind[t] & 2;
  const uint64_t full = lo + ((hi - lo) & ~(uint64_t)3);
#pragma unroll 2
  for (uint64_t i = lo + 4 * threadIdx.x; i < full; i += 4 * kThreads) {
    const f32x4 g = load4<F32>(grad, i);
    f32x4 p = load4<true>(master, i), m = {0.f, 0.f, 0.f, 0.f}, v = m;
    if constexpr (ADAMW) {
      m = load4<true>(mm, i);
      v = load4<true>(vv, i);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float pj = p[j], mj = m[j], vj = v[j];
      update_element<ADAMW>(a.r, scale * g[j], pj, mj, vj);
      p[j] = pj;
      m[j] = mj;
      v[j] = vj;
    }
    if constexpr (ADAMW) {
      store4(mm, i, m, true);
      store4(vv, i, v, true);
    }
    store4(master, i, p, true);
    if (io) store4(io, i, p, io_f32);
  }
  if (const uint64_t i = full + threadIdx.x; i < hi) {
    float p = master[i], m = 0.f, v = 0.f;
    if constexpr (ADAMW) {
      m = mm[i];
      v = vv[i];
    }
    update_element<ADAMW>(a.r, scale * load1<F32>(grad, i), p, m, v);
    if constexpr (ADAMW) {
      mm[i] = m;
      vv[i] = v;
    }
    master[i] = p;
    if (io) store1(io, i, p, io_f32);
  }
}

template <bool ADAMW>
__global__ __launch_bounds__(kThreads) void param_update_many_kernel(ManyArgs a) {
  float scale = a.r.grad_scale;
  if (a.result) {
    const float f = a.result[1];
    if (!__builtin_isfinite(f)) return;
    scale *= f;
  }
  const uint32_t b = blockIdx.x;
  const int t = a.at.tensor(b);
  const uint64_t lo = (uint64_t)(b - a.at.first[t]) * a.at.piece, hi = lo + a.at.piece < a.n[t] ? lo + a.at.piece : a.n[t];
  if (a.kind[t] & 1) update_piece<ADAMW, true>(a, t, lo, hi, scale);
  else update_piece<ADAMW, false>(a, t, lo, hi, scale);
}

// Smaller where that would leave workgroups few and each with rounds of loads to wait for, down to one load of each tensor a thread.
// Us of norm / clip / AdamW so and with pieces of 8192: 33 thousand values 5.9 / 3.7 / 4.2 and 5.9 / 4.0 / 5.4, 200 thousand 7.9 / 4.7 / 4.1 and 7.7 / 5.0 / 7.3,
// 2.4 million 7.6 / 5.2 / 11.9 and 7.9 / 6.1 / 13.3; from 10 million on they are the same.
uint64_t piece_size(uint64_t total) {
  if (const uint64_t most = (total + kMaxPieces - 1) / kMaxPieces; most > kPiece) return (most + kPiece - 1) / kPiece * kPiece;
  uint64_t piece = kPiece;
  while (piece > 4 * kThreads && piece * kFewPieces > total) piece /= 2;
  return piece;
}
uint64_t pieces_of(uint64_t n, uint64_t piece) { return (n + piece - 1) / piece; }

constexpr uint64_t kMaxElements = (uint64_t)1 << 40;

// Sizes, types and alignment of a list of tensors; the sum of the sizes.
ha_status check_tensors(int32_t count, const ha_tensor *t, uint64_t &total) {
  total = 0;
  if (count < 0 || count > (1 << 24)) return HA_ERR_SHAPE;
  if (count > 0 && !t) return HA_ERR_NULL;
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].dtype != HA_BF16 && t[i].dtype != HA_F32) return HA_ERR_UNSUPPORTED;
    if (t[i].reserved != 0 || t[i].n > kMaxElements) return HA_ERR_SHAPE;
    if (t[i].n > 0 && !t[i].data) return HA_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(t[i].data) & (t[i].dtype == HA_F32 ? 3u : 1u)) return HA_ERR_ALIGN;
    total += t[i].n;
    if (total > kMaxElements) return HA_ERR_SHAPE;
  }
  return HA_OK;
}

uint64_t total_pieces(int32_t count, const ha_tensor *t, uint64_t piece) {
  uint64_t s = 0;
  for (int32_t i = 0; i < count; ++i) s += pieces_of(t[i].n, piece);
  return s;
}

// Takes tensors from i on; the first that is left.
int32_t fill_norm(NormArgs &a, const ha_tensor *grads, int32_t i, int32_t n_tensors, uint64_t piece) {
  a.at.piece = piece;
  a.at.n = 0;
  a.at.first[0] = 0;
  for (; i < n_tensors && a.at.n < kNormTensors; ++i) {
    if (grads[i].n == 0) continue;
    const int t = a.at.n++;
    a.data[t] = grads[i].data;
    a.n[t] = grads[i].n;
    a.f32[t] = grads[i].dtype == HA_F32;
    a.at.first[t + 1] = a.at.first[t] + (uint32_t)pieces_of(grads[i].n, piece);
  }
  return i;
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" size_t hybrid_attn_grad_norm_workspace_bytes(int32_t n_tensors, const ha_tensor *grads) {
  uint64_t total;
  if (check_tensors(n_tensors, grads, total) != HA_OK) return 0;
  const uint64_t n = total_pieces(n_tensors, grads, piece_size(total));
  return (n > 0 ? n : 1) * sizeof(double);
}

extern "C" ha_status hybrid_attn_grad_norm(int32_t n_tensors, const ha_tensor *grads, float max_norm, float *result, void *workspace,
                                           size_t workspace_bytes, void *hip_stream) {
  uint64_t total;
  if (const ha_status s = check_tensors(n_tensors, grads, total); s != HA_OK) return s;
  if (!result) return HA_ERR_NULL;
  if (!(max_norm > 0.f)) return HA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(result) & 3u || reinterpret_cast<uintptr_t>(workspace) & 7u) return HA_ERR_ALIGN;
  const uint64_t piece = piece_size(total), need = total_pieces(n_tensors, grads, piece) * sizeof(double);
  if (!workspace || workspace_bytes < need) return HA_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  uint32_t done = 0;
  NormArgs a;
  if (n_tensors <= kNormTensors && total_pieces(n_tensors, grads, kSmallPiece) <= kSmallPieces) {
    fill_norm(a, grads, 0, n_tensors, kSmallPiece);
    grad_norm_small_kernel<<<1, 1024, 0, st>>>(a, max_norm, result);
    return (e = hipGetLastError()) == hipSuccess ? HA_OK : device_error(e);
  }
  for (int32_t i = 0; i < n_tensors;) {
    i = fill_norm(a, grads, i, n_tensors, piece);
    a.partial = static_cast<double *>(workspace) + done;
    if (a.at.n == 0) break;
    const uint32_t blocks = a.at.first[a.at.n];
    grad_norm_kernel<<<blocks, kThreads, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return device_error(e);
    done += blocks;
  }
  grad_norm_join_kernel<<<1, 1024, 0, st>>>(static_cast<const double *>(workspace), done, max_norm, result);
  return (e = hipGetLastError()) == hipSuccess ? HA_OK : device_error(e);
}

extern "C" ha_status hybrid_attn_grad_clip(int32_t n_tensors, const ha_tensor *grads, const ha_tensor *out, const float *result, void *hip_stream) {
  uint64_t total, total_out;
  if (const ha_status s = check_tensors(n_tensors, grads, total); s != HA_OK) return s;
  if (const ha_status s = check_tensors(n_tensors, out, total_out); s != HA_OK) return s;
  if (!result) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(result) & 3u) return HA_ERR_ALIGN;
  for (int32_t i = 0; i < n_tensors; ++i)
    if (grads[i].n != out[i].n || (grads[i].n > 0 && grads[i].data == out[i].data && grads[i].dtype != out[i].dtype)) return HA_ERR_SHAPE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  ClipArgs a;
  a.at.piece = piece_size(total);
  a.result = result;
  for (int32_t i = 0; i < n_tensors;) {
    a.at.n = 0;
    a.at.first[0] = 0;
    for (; i < n_tensors && a.at.n < kClipTensors; ++i) {
      if (grads[i].n == 0) continue;
      const int t = a.at.n++;
      a.in[t] = grads[i].data;
      a.out[t] = out[i].data;
      a.n[t] = grads[i].n;
      a.kind[t] = (grads[i].dtype == HA_F32) | (out[i].dtype == HA_F32) << 1;
      a.at.first[t + 1] = a.at.first[t] + (uint32_t)pieces_of(grads[i].n, a.at.piece);
    }
    if (a.at.n == 0) break;
    grad_clip_kernel<<<a.at.first[a.at.n], kThreads, 0, st>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return device_error(e);
  }
  return HA_OK;
}

extern "C" ha_status hybrid_attn_param_update_many(const ha_optimizer *opt, int32_t n_params, const ha_param *params, const float *result,
                                                   void *hip_stream) {
  if (!opt) return HA_ERR_NULL;
  if (const ha_status s = check_optimizer(opt); s != HA_OK) return s;
  if (n_params < 0 || n_params > (1 << 24)) return HA_ERR_SHAPE;
  if (n_params > 0 && !params) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(result) & 3u) return HA_ERR_ALIGN;
  const bool adamw = opt->kind == HA_OPT_ADAMW;
  uint64_t total = 0;
  for (int32_t i = 0; i < n_params; ++i) {
    const ha_param &p = params[i];
    if (p.n > kMaxElements || (total += p.n) > kMaxElements) return HA_ERR_SHAPE;
    if ((p.grad_dtype != HA_BF16 && p.grad_dtype != HA_F32) || (p.param_io && p.io_dtype != HA_BF16 && p.io_dtype != HA_F32)) return HA_ERR_UNSUPPORTED;
    if (p.n > 0 && (!p.master || !p.grad || (adamw && (!p.m || !p.v)))) return HA_ERR_NULL;
    for (const void *t : {static_cast<const void *>(p.master), static_cast<const void *>(p.m), static_cast<const void *>(p.v)})
      if (reinterpret_cast<uintptr_t>(t) & 3u) return HA_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(p.grad) & (p.grad_dtype == HA_F32 ? 3u : 1u)) return HA_ERR_ALIGN;
    if (p.param_io && (reinterpret_cast<uintptr_t>(p.param_io) & (p.io_dtype == HA_BF16 ? 1u : 3u))) return HA_ERR_ALIGN;
    if (p.n > 0 && p.param_io == p.master) return HA_ERR_SHAPE;
  }
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  ManyArgs a;
  a.at.piece = piece_size(total);
  a.r = update_rates(*opt);
  a.result = result;
  for (int32_t i = 0; i < n_params;) {
    a.at.n = 0;
    a.at.first[0] = 0;
    for (; i < n_params && a.at.n < kUpdateTensors; ++i) {
      const ha_param &p = params[i];
      if (p.n == 0) continue;
      const int t = a.at.n++;
      a.master[t] = p.master;
      a.grad[t] = p.grad;
      a.m[t] = p.m;
      a.v[t] = p.v;
      a.io[t] = p.param_io;
      a.n[t] = p.n;
      a.kind[t] = (p.grad_dtype == HA_F32) | (p.param_io && p.io_dtype == HA_F32) << 1;
      a.at.first[t + 1] = a.at.first[t] + (uint32_t)pieces_of(p.n, a.at.piece);
    }
    if (a.at.n == 0) break;
    if (adamw) param_update_many_kernel<true><<<a.at.first[a.at.n], kThreads, 0, st>>>(a);
    else param_update_many_kernel<false><<<a.at.first[a.at.n], kThreads, 0, st>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return device_error(e);
  }
  return HA_OK;
}
