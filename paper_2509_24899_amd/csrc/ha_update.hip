// Parameter update of the attention-distillation loop (Attention Surgery, Sec. 3.3, Alg. "distil": the line
// phi <- phi - eta grad_phi L; the training details name AdamW with learning rate 1e-3 for this stage), gfx950.
// Elementwise and HBM-bound: one pass over the fp32 master copy, the gradient and (AdamW) the two moments, which also
// writes the parameter in the dtype the forward reads.  fp32 arithmetic; the bias corrections of AdamW are formed on
// the host in double precision.
#include "ha_update.h"

namespace {

struct UpdateArgs {
  float *master;
  const float *grad;
  float *m, *v;
  void *param_io;
  int64_t n;
  ha::UpdateRates r;
};

template <bool ADAMW, int IO>   // IO 0: no copy, 1: bf16, 2: fp32
__global__ __launch_bounds__(256) void param_update_kernel(UpdateArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.n) return;
  const float g = a.r.grad_scale * a.grad[i];
  float p = a.master[i], m = 0.f, v = 0.f;
  if constexpr (ADAMW) {
    m = a.m[i];
    v = a.v[i];
  }
  ha::update_element<ADAMW>(a.r, g, p, m, v);
  if constexpr (ADAMW) {
    a.m[i] = m;
    a.v[i] = v;
  }
  a.master[i] = p;
  if constexpr (IO == 1) static_cast<__bf16 *>(a.param_io)[i] = static_cast<__bf16>(p);
  if constexpr (IO == 2) static_cast<float *>(a.param_io)[i] = p;
}

}  // namespace

extern "C" ha_status hybrid_attn_param_update(const ha_optimizer *opt, size_t n, float *master, const float *grad, float *m,
                                              float *v, void *param_io, int32_t io_dtype, void *hip_stream) {
  if (!opt || !master || !grad) return HA_ERR_NULL;
  if (opt->kind != HA_OPT_SGD && opt->kind != HA_OPT_ADAMW) return HA_ERR_UNSUPPORTED;
  const bool adamw = opt->kind == HA_OPT_ADAMW;
  if (adamw && (!m || !v)) return HA_ERR_NULL;
  if (param_io && io_dtype != HA_BF16 && io_dtype != HA_F32) return HA_ERR_UNSUPPORTED;
  if (const ha_status s = ha::check_optimizer(opt); s != HA_OK) return s;
  for (const void *t : {static_cast<const void *>(master), static_cast<const void *>(grad), static_cast<const void *>(m),
                        static_cast<const void *>(v)})
    if (reinterpret_cast<uintptr_t>(t) & 3u) return HA_ERR_ALIGN;
  if (param_io && (reinterpret_cast<uintptr_t>(param_io) & (io_dtype == HA_BF16 ? 1u : 3u))) return HA_ERR_ALIGN;
  if (param_io == master) return HA_ERR_SHAPE;
  if (n == 0) return HA_OK;
  if (n > ((size_t)1 << 40)) return HA_ERR_SHAPE;
  UpdateArgs a;
  a.master = master; a.grad = grad; a.m = m; a.v = v; a.param_io = param_io; a.n = (int64_t)n;
  a.r = ha::update_rates(*opt);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const unsigned blocks = (unsigned)((n + 255) / 256);
  const int io = !param_io ? 0 : (io_dtype == HA_BF16 ? 1 : 2);
#define HA_UPD(A, IO) param_update_kernel<A, IO><<<blocks, 256, 0, st>>>(a)
  if (adamw) { if (io == 0) HA_UPD(true, 0); else if (io == 1) HA_UPD(true, 1); else HA_UPD(true, 2); }
  else { if (io == 0) HA_UPD(false, 0); else if (io == 1) HA_UPD(false, 1); else HA_UPD(false, 2); }
#undef HA_UPD
  return hipGetLastError() == hipSuccess ? HA_OK : HA_ERR_DEVICE;
}
