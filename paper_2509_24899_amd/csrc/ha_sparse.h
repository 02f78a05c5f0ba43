// Building blocks of block-sparse attention (gfx950): the problem as the kernels see it, and tiles of rows in LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hybrid_attn_sparse.h"
#include "ha_mlp128.h"
#include "ha_plan.h"

namespace ha {

// A [B, heads, N, d] tensor of bf16 or fp32, strides in elements.
struct View {
  char *p;
  int64_t sb, sh, sn;
};

struct Sparse {
  int B, H, Hkv, G, Nq, Nk, T, Tk, qb, kb, sel, causal;
  const int32_t *q_start, *key_len;
  __device__ __forceinline__ int held(int b) const { return key_len ? min(max(key_len[b], 0), Nk) : Nk; }
  __device__ __forceinline__ int start(int b) const { return q_start ? q_start[b] : Nk - Nq; }
};

// Consecutive workgroups go to the eight XCDs in turn; work item of workgroup `id` such that every XCD walks one contiguous
// range of items (neighbouring tiles of one head, which read much the same keys, share its L2).  The grid is 8 xcd_share(n) workgroups, those
// whose item is n or more have none.  (Forward at 480p 820 us for 825 with items in the order of workgroups; training with 4096 causal tokens 180 us for 187.)
static __host__ __device__ inline unsigned xcd_share(unsigned n) { return (n + 7) / 8; }
static __device__ __forceinline__ unsigned xcd_item(unsigned id, unsigned share) { return (id & 7) * share + (id >> 3); }

// ---- tiles of rows in LDS ------------------------------------------------------------------------------------------
// R rows of D bf16 lie in LDS as they lie in memory, 2 D bytes each, but the 16-byte pieces of row r stand at piece ^ swz(r).  With that,
// both ways of reading a tile spread over all banks: 16 consecutive rows of one piece (the operand whose rows are the tile's) fall into 16
// different pieces of 256 bytes, and so do four consecutive rows of four neighbouring pieces (the transposed operand).  The tile is filled
// with direct-to-LDS loads, where a lane's place in LDS is fixed, so the permutation is in the addresses the lanes read.
static __device__ __forceinline__ unsigned lds_offset(const void *p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }
template <int D>
struct Tile {
  static constexpr int PIECES = D / 8, PITCH = 2 * D, ROWS_PER_CHUNK = 64 / PIECES;
  static constexpr int bytes(int rows) { return rows * PITCH; }
  static constexpr int chunks(int rows) { return rows / ROWS_PER_CHUNK; }
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    else return ((row << 1) & 4) | ((row >> 2) & 3);
  }
  // Operand with the tile's rows as its rows: rows row0 + r, contraction slots (g, t) = columns 16 ks + 8 g + t ("natural").
  // Operand with the tile's columns 32 cb .. as its rows and its rows row0 .. row0 + 15 as the contraction, "chained" order.
  // Both from a lane's address that is formed once for a tile (whose place in LDS is a multiple of PITCH): the piece is the low bits of the address, so
  // that one exclusive or gives any other; row0 is a multiple of 16 and, like a distance between tiles (`further`), goes into the instruction.
  static __device__ __forceinline__ unsigned rows_base(const char *tile, int lane) {
    const int row = lane & 31;
    return lds_offset(tile) + row * PITCH + (((lane >> 5) ^ swz(row)) << 4);
  }
  static __device__ __forceinline__ bf16x8 row_piece(unsigned at) { return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8 *>(static_cast<uintptr_t>(at)); }
  static __device__ __forceinline__ bf16x8 rows_at(unsigned base, int row0, int ks, int further = 0) { return row_piece((base ^ (ks << 5)) + row0 * PITCH + further); }
  static __device__ __forceinline__ unsigned cols_base(const char *tile, int lane) {
    const int row = 4 * (lane >> 5) + ((lane & 15) >> 2), piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    return lds_offset(tile) + row * PITCH + ((piece ^ swz(row)) << 4) + (lane & 1) * 8;
  }
  static __device__ __forceinline__ bf16x8 col_piece(unsigned at0, unsigned at8) {
    return join(__builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4_ptr>(static_cast<uintptr_t>(at0))),
                __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4_ptr>(static_cast<uintptr_t>(at8))));
  }
  static __device__ __forceinline__ bf16x8 cols_at(unsigned base, int cb, int row0, int further = 0) {
    // (eight rows further down the permutation differs in piece bit 1)
    const unsigned at = base ^ (cb << 6);
    return col_piece(at + row0 * PITCH + further, (at ^ 32) + (row0 + 8) * PITCH + further);
  }
};

typedef int i32x4 __attribute__((ext_vector_type(4)));
// Descriptor of `rows` rows of D bf16 at base (wave-uniform); rows behind them read as zero.
template <int D>
static __device__ __forceinline__ i32x4 rows_rsrc(const char *base, int rows, int64_t stride_bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const int n = rows > 0 ? (int)((rows - 1) * stride_bytes) + 2 * D : 0;
  return i32x4{(int)__builtin_amdgcn_readfirstlane((int)(uint32_t)p), (int)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32) & 0xffff),
               (int)__builtin_amdgcn_readfirstlane(n), 0x00020000};
}

// Requests the tile of ROWS rows described by `rsrc` into `lds`: one instruction moves 64 lanes x 16 bytes, the chunks are dealt round-robin
// to the NW waves.  Completion is awaited by the caller (vmcnt), which then synchronises the workgroup.
template <int D, int ROWS, int NW>
static __device__ __forceinline__ void request_rows(const i32x4 &rsrc, int stride_bytes, char *lds, int w, int lane) {
  typedef Tile<D> T;
  static_assert(T::chunks(ROWS) % NW == 0, "chunks are dealt evenly");
#pragma unroll
  for (int i = 0; i < T::chunks(ROWS) / NW; ++i) {
    const int c = i * NW + w, row = c * T::ROWS_PER_CHUNK + lane / T::PIECES;
    const int off = row * stride_bytes + (((lane % T::PIECES) ^ T::swz(row)) << 4);
    const unsigned l = __builtin_amdgcn_readfirstlane(lds_offset(lds) + c * 1024);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(l), "v"(off), "s"(rsrc) : "memory");
  }
}
static __device__ __forceinline__ void landed() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// bf16 pieces of eight fp32 values: each the rounding of what the ones before it leave.  Three hold all 24 bits.
template <int NS>
static __device__ __forceinline__ void split8(f32x8 x, bf16x8 (&out)[NS]) {
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    out[n] = __builtin_convertvector(x, bf16x8);
    if (n + 1 < NS)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] -= static_cast<float>(out[n][i]);
  }
}
// Any values: infinities and NaN have one piece (infinity less infinity is none), and the first piece of a finite value above bf16's largest, which would
// round to infinity, is cut off instead of rounded.
static __device__ __forceinline__ void split8_any(f32x4 lo, f32x4 hi, bf16x8 (&out)[3]) {
  const f32x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  split8<3>(x, out);
  bool any = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) any |= !__builtin_isfinite(static_cast<float>(out[0][i]));
  if (!any) return;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (!__builtin_isfinite(static_cast<float>(out[0][i]))) {
      const float first = __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u), rest = __builtin_isfinite(x[i]) ? x[i] - first : 0.f;
      if (__builtin_isfinite(x[i])) out[0][i] = static_cast<__bf16>(first);
      out[1][i] = static_cast<__bf16>(rest);
      out[2][i] = static_cast<__bf16>(rest - static_cast<float>(out[1][i]));
    }
}
// a b with both in pieces, small terms first; of three pieces the products that stay below the last bit are left out (six of nine are formed).
template <int NS>
static __device__ __forceinline__ f32x16 mfma_split(const bf16x8 (&a)[NS], const bf16x8 (&b)[NS], f32x16 c) {
#pragma unroll
  for (int order = NS - 1; order >= 0; --order)
#pragma unroll
    for (int n = 0; n <= order; ++n) c = mfma32(a[order - n], b[n], c);
  return c;
}
// Pieces of a tensor, and rows of a step of the kernels that take both types (fp32 forward, dQ, fp32 dK and dV): one or two steps' keys and values, or queries and
// gradients, in all their pieces lie in LDS.
template <bool F32>
struct Pieces {
  static constexpr int N = F32 ? 3 : 1, ROWS = F32 ? 32 : 64;
};

// Writes a 32-row tile held as C^T (NB blocks of 32 columns; the row is the lane's) times `f` through `stage` (this wave's own LDS, 32 rows
// of D values and 16 bytes) to rows first .. of `out`, those below `limit`.
template <int D, bool F32>
static __device__ __forceinline__ void store_rows(const f32x16 (&o)[D / 32], float f, char *stage, char *out, int64_t stride_bytes, int first,
                                                  int limit, int lane) {
  constexpr int PASSES = F32 ? 2 : 1, DP = D / PASSES, ESZ = F32 ? 4 : 2, PITCH = DP * ESZ + 16, CPR = DP * ESZ / 16;
  const int r = lane & 31, g = lane >> 5;
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
#pragma unroll
    for (int b = 0; b < D / 32 / PASSES; ++b)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        const int col = 32 * b + 8 * x4 + 4 * g;
        const f32x16 &t = o[pass * (D / 32 / PASSES) + b];
        const f32x4 y = {t[4 * x4] * f, t[4 * x4 + 1] * f, t[4 * x4 + 2] * f, t[4 * x4 + 3] * f};
        if constexpr (F32) *reinterpret_cast<f32x4 *>(stage + r * PITCH + col * 4) = y;
        else *reinterpret_cast<bf16x4 *>(stage + r * PITCH + col * 2) = __builtin_convertvector(y, bf16x4);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // (a wave's LDS instructions execute in order)
#pragma unroll
    for (int i = lane; i < 32 * CPR; i += 64) {
      const int row = i / CPR, ch = i % CPR;
      if (first + row < limit)
        *reinterpret_cast<f32x4 *>(out + (int64_t)(first + row) * stride_bytes + pass * DP * ESZ + ch * 16) = *reinterpret_cast<const f32x4 *>(stage + row * PITCH + ch * 16);
    }
    if (PASSES > 1) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}
template <int D, bool F32>
static constexpr int store_bytes() { return 32 * ((F32 ? D / 2 * 4 : D * 2) + 16); }

// Walks a list STEP keys at a time: the steps whose keys someone in the tile may see.
template <int STEP>
struct ListWalk {
  const int32_t *list;
  int at, end, sub, subs, Tk, kb, limit, lane, held_from;
  int entry;                  // lane l: list[held_from + l]
  __device__ __forceinline__ ListWalk(const int32_t *l, int lo, int hi, const Sparse &s, int lim, int lane_)
      : list(l), at(lo), end(hi), sub(0), subs(s.kb / STEP), Tk(s.Tk), kb(s.kb), limit(lim), lane(lane_), held_from(lo) { fetch(); }
  __device__ __forceinline__ void fetch() { entry = held_from + lane < end ? list[held_from + lane] : -1; }
  // first key of the next step, or -1
  __device__ __forceinline__ int next() {
    while (at < end) {
      if (at - held_from == 64) {
        held_from = at;
        fetch();
      }
      const int j = __builtin_amdgcn_readlane(entry, at - held_from), key = j * kb + STEP * sub;
      if (++sub == subs) {
        sub = 0;
        ++at;
      }
      if ((unsigned)j < (unsigned)Tk && key < limit) return key;
      if ((unsigned)j >= (unsigned)Tk && sub) {
        sub = 0;
        ++at;
      }
    }
    return -1;
  }
};

// ---- host ----------------------------------------------------------------------------------------------------------
ha_status check_sparse(const ha_sparse_problem *p);
// data, strides and alignment of a view of `heads` heads of n rows in blocks of `block`; the strides of dimensions of one entry are set to
// those of a contiguous tensor in `out`.
ha_status check_view(const ha_sparse_problem &p, const ha_view *v, int heads, int n, int block, bool written, View &out);
Sparse sparse_of(const ha_sparse_problem &p);
static inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
// The three bf16 images of an fp32 view, contiguous [3][B, heads, N, d]; split_view is that of the first.
struct SplitJob {
  View in;
  __bf16 *out;
  int heads, n;
};
static inline View split_view(const SplitJob &j, int d) {
  const int64_t n = j.n * (int64_t)d;
  return View{reinterpret_cast<char *>(j.out), j.heads * n, n, d};
}
hipError_t launch_split(const Sparse &s, int d, const SplitJob *jobs, int n_jobs, hipStream_t st);

}  // namespace ha
