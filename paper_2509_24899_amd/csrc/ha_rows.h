// Building blocks of kernels that work on rows of heads (gfx950): a row's channels in the threads that own them, the rotation of pairs by positions, the norm.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hybrid_attn_rotary.h"
#include "ha_sparse.h"

namespace ha {

struct Rotary {
  const double *freq;
  const int32_t *axis, *positions;
  int64_t positions_sb;
  int rot, n_axes;
  float magnitude;
};

// D / 8 threads own a row, thread t two pieces of four channels that hold both halves of its pairs 4 t .. 4 t + 3: NEXT, channels 8 t .. 8 t + 7; otherwise
// 4 t .. and rot / 2 + 4 t .. while those are rotated, and 8 t .. of what is not.  So a row is read once, with no exchange between threads, and can be written in place.
template <bool NEXT>
static __device__ __forceinline__ void own_channels(int t, int rot, int &ca, int &cb) {
  const bool half = !NEXT && 8 * t < rot;
  ca = half ? 4 * t : 8 * t;
  cb = half ? 4 * t + rot / 2 : 8 * t + 4;
}

struct Row8 {
  f32x4 a, b;
};
static __device__ __forceinline__ Row8 times(const Row8 &x, float f) { return Row8{x.a * f, x.b * f}; }
static __device__ __forceinline__ Row8 times(const Row8 &x, const Row8 &w) { return Row8{x.a * w.a, x.b * w.b}; }
static __device__ __forceinline__ Row8 weight8(const float *w, int ca, int cb) {
  if (!w) return Row8{f32x4{1.f, 1.f, 1.f, 1.f}, f32x4{1.f, 1.f, 1.f, 1.f}};
  return Row8{*reinterpret_cast<const f32x4 *>(w + ca), *reinterpret_cast<const f32x4 *>(w + cb)};
}
// Streams that are read or written once and that the memory-side cache cannot hold go past it (ONCE).  Loads only where one instruction takes whole lines: 12 + 12 heads of
// 2 x 75600 bf16 tokens, forward and gradients 861 us for 911, of which the stores make 18; fp32 gradients of 5003 tokens 32 us with such loads and 25 without.
template <bool ONCE, typename T>
static __device__ __forceinline__ T load_as(const void *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(static_cast<const T *>(p));
  else return *static_cast<const T *>(p);
}
template <bool ONCE, typename T>
static __device__ __forceinline__ void store_as(void *p, T x) {
  if constexpr (ONCE) __builtin_nontemporal_store(x, static_cast<T *>(p));
  else *static_cast<T *>(p) = x;
}
static inline bool stream_once(int64_t bytes) { return bytes > (int64_t)128 << 20; }      // (read and written)

template <bool F32, bool NEXT, bool ONCE = false>
static __device__ __forceinline__ Row8 load_row8(const char *p, int64_t row, int ca, int cb) {
  if constexpr (F32) {
    const float *x = reinterpret_cast<const float *>(p) + row;
    return Row8{*reinterpret_cast<const f32x4 *>(x + ca), *reinterpret_cast<const f32x4 *>(x + cb)};
  } else if constexpr (NEXT) {
    const f32x8 f = __builtin_convertvector(load_as<ONCE, bf16x8>(reinterpret_cast<const __bf16 *>(p) + row + ca), f32x8);
    return Row8{__builtin_shufflevector(f, f, 0, 1, 2, 3), __builtin_shufflevector(f, f, 4, 5, 6, 7)};
  } else {
    const __bf16 *x = reinterpret_cast<const __bf16 *>(p) + row;
    return Row8{__builtin_convertvector(*reinterpret_cast<const bf16x4 *>(x + ca), f32x4), __builtin_convertvector(*reinterpret_cast<const bf16x4 *>(x + cb), f32x4)};
  }
}
template <bool F32, bool NEXT, bool ONCE = false>
static __device__ __forceinline__ void store_row8(char *p, int64_t row, int ca, int cb, const Row8 &y) {
  if constexpr (F32) {
    float *x = reinterpret_cast<float *>(p) + row;
    store_as<ONCE>(x + ca, y.a);
    store_as<ONCE>(x + cb, y.b);
  } else if constexpr (NEXT) {
    store_as<ONCE>(reinterpret_cast<__bf16 *>(p) + row + ca, __builtin_convertvector(__builtin_shufflevector(y.a, y.b, 0, 1, 2, 3, 4, 5, 6, 7), bf16x8));
  } else {
    __bf16 *x = reinterpret_cast<__bf16 *>(p) + row;
    store_as<ONCE>(x + ca, __builtin_convertvector(y.a, bf16x4));
    store_as<ONCE>(x + cb, __builtin_convertvector(y.b, bf16x4));
  }
}

// cos and sin of a thread's four pairs at the position `at` (n_axes numbers).  The angle in turns is formed in double and reduced there; what is left, half a
// turn at most, goes to the library's fp32 sine and cosine of multiples of pi.
static __device__ __forceinline__ void pair_angles(const Rotary &r, const int32_t *at, int t, f32x4 &c, f32x4 &s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pair = 4 * t + i;
    c[i] = 1.f;
    s[i] = 0.f;
    if (2 * pair < r.rot) {
      const int axis = r.axis ? min(max(r.axis[pair], 0), r.n_axes - 1) : 0;
      double turns = at[axis] * (r.freq[pair] * 0.15915494309189533577);
      turns -= rint(turns);
      float sn, cs;
      sincospif(2.f * (float)turns, &sn, &cs);
      c[i] = cs * r.magnitude;
      s[i] = sn * r.magnitude;
    }
  }
}
// The first `pairs` of a thread's four are rotated (an infinity in a channel that is not must not reach its neighbour).
template <bool NEXT>
static __device__ __forceinline__ Row8 turn(const Row8 &x, f32x4 c, f32x4 s, int pairs) {
  Row8 y = x;
  if constexpr (NEXT) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (i < pairs) {
        y.a[2 * i] = x.a[2 * i] * c[i] - x.a[2 * i + 1] * s[i];
        y.a[2 * i + 1] = x.a[2 * i] * s[i] + x.a[2 * i + 1] * c[i];
      }
      if (2 + i < pairs) {
        y.b[2 * i] = x.b[2 * i] * c[2 + i] - x.b[2 * i + 1] * s[2 + i];
        y.b[2 * i + 1] = x.b[2 * i] * s[2 + i] + x.b[2 * i + 1] * c[2 + i];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < pairs) {
        y.a[i] = x.a[i] * c[i] - x.b[i] * s[i];
        y.b[i] = x.a[i] * s[i] + x.b[i] * c[i];
      }
    }
  }
  return y;
}

// Sum over the D / 8 threads of a row, in all of them: 8 or 16 neighbouring lanes, which DPP moves reach.
template <int CTRL>
static __device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int D>
static __device__ __forceinline__ float row_sum(float x) {
  x = dpp_add<0xB1>(x);       // lane ^ 1
  x = dpp_add<0x4E>(x);       // lane ^ 2
  x = dpp_add<0x141>(x);      // 7 - lane, of every eight: the other four
  if constexpr (D == 128) x = dpp_add<0x140>(x);      // 15 - lane
  return x;
}
static __device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return (a[0] * b[0] + a[1] * b[1]) + (a[2] * b[2] + a[3] * b[3]); }
template <int D>
static __device__ __forceinline__ float inverse_rms(const Row8 &x, float eps) {
  return rsqrtf(row_sum<D>(dot4(x.a, x.a) + dot4(x.b, x.b)) * (1.f / D) + eps);
}

// ---- host ----------------------------------------------------------------------------------------------------------
ha_status check_rotary(const ha_rotary *r, int d_head, int64_t tokens, bool one_list, Rotary &out);
// data, strides and alignment of a [B, heads, n, d] view; the strides of dimensions of one entry are set to those of a contiguous tensor in `out`.
ha_status check_rows(int B, int heads, int64_t n, int d, int dtype, const ha_view *v, bool written, View &out);

}  // namespace ha
