// The parameter update's arithmetic and its host checks, shared by the call of one tensor (ha_update.hip) and the call of many (ha_optim.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/hybrid_attn.h"

namespace ha {

struct UpdateRates {
  float lr, grad_scale, beta1, beta2, eps, decay_factor, step_size, inv_sqrt_bc2;
};

// One element: parameter p and moments m, v (AdamW) by the scaled gradient g.  The roundings are spelled out, so that both calls give the same bits.
template <bool ADAMW>
static __device__ __forceinline__ void update_element(const UpdateRates &a, float g, float &p, float &m, float &v) {
  if constexpr (ADAMW) {
    m = __builtin_fmaf(1.0f - a.beta1, g, a.beta1 * m);
    v = __builtin_fmaf(g, (1.0f - a.beta2) * g, a.beta2 * v);
    p = __builtin_fmaf(a.decay_factor, p, -(a.step_size * m / __builtin_fmaf(sqrtf(v), a.inv_sqrt_bc2, a.eps)));
  } else {
    p = __builtin_fmaf(-a.lr, g, p);
  }
}

static inline ha_status check_optimizer(const ha_optimizer *opt) {
  if (opt->kind != HA_OPT_SGD && opt->kind != HA_OPT_ADAMW) return HA_ERR_UNSUPPORTED;
  auto finite = [](float x) { return std::isfinite(x); };
  if (!finite(opt->lr) || !finite(opt->grad_scale) || opt->lr < 0.f) return HA_ERR_SHAPE;
  if (opt->kind == HA_OPT_ADAMW) {
    if (opt->step < 1) return HA_ERR_SHAPE;
    if (!(opt->beta1 >= 0.f && opt->beta1 < 1.f) || !(opt->beta2 >= 0.f && opt->beta2 < 1.f)) return HA_ERR_SHAPE;
    if (!finite(opt->eps) || opt->eps < 0.f || !finite(opt->weight_decay) || opt->weight_decay < 0.f) return HA_ERR_SHAPE;
  }
  return HA_OK;
}

// (the bias corrections of AdamW in double precision, of the betas that ha_optimizer holds: floats, as 1 - beta is in update_element)
static inline UpdateRates update_rates(const ha_optimizer &opt) {
  UpdateRates a{opt.lr, opt.grad_scale, opt.beta1, opt.beta2, opt.eps, 1.f, 0.f, 1.f};
  if (opt.kind == HA_OPT_ADAMW) {
    const double bc1 = 1.0 - std::pow((double)opt.beta1, (double)opt.step);
    const double bc2 = 1.0 - std::pow((double)opt.beta2, (double)opt.step);
    a.decay_factor = (float)(1.0 - (double)opt.lr * (double)opt.weight_decay);
    a.step_size = (float)((double)opt.lr / bc1);
    a.inv_sqrt_bc2 = (float)(1.0 / std::sqrt(bc2));
  }
  return a;
}

}  // namespace ha
