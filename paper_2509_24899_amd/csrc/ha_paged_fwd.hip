// Attention of new tokens over a paged cache, gfx950.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - m_i),   j over the slots that new token i sees
//
// All query heads of a key head are rows of one product (row R of a sequence is token R / G, head R % G of the group), so that keys and values are read once for a
// group.  Logits, sums and the output's sums are fp32; of bf16 tensors the weights of tiles are rounded to bf16 for the second product (half a step, 2^-8 of each, the sum
// that divides is that of the unrounded ones), of fp32 tensors every operand is three bf16 pieces, six products each.
//   few   32 rows at most (single tokens): bound by memory, which leaves time for weights in two pieces (a result is off by 0.17 % on the average, the rounding of the
//         output alone, where weights in one piece make it 0.22).  A workgroup takes a range of a sequence's slots for a key head, every wave slots of its own.
//   tile  128 rows, 32 to a wave: bound by the matrix cores.  All waves read the same slots out of LDS.
// Where either leaves compute units idle the slots are cut into ranges, whose sums a second kernel joins.
#include <cmath>

#include "ha_paged.h"

#include <algorithm>
#include <type_traits>

namespace ha {

ha_status check_paged(const ha_paged_problem *p) {
  if (!p) return HA_ERR_NULL;
  if (p->B <= 0 || p->H <= 0 || p->H_kv <= 0 || p->H % p->H_kv || p->T < 0 || p->d_head <= 0) return HA_ERR_SHAPE;
  if (p->n_pages < 0 || p->max_pages < 0 || p->max_new < 0 || p->max_new > p->T) return HA_ERR_SHAPE;
  if (p->causal != 0 && p->causal != 1) return HA_ERR_SHAPE;
  if (!(p->softmax_scale >= 1e-30f && p->softmax_scale <= 1e30f)) return HA_ERR_SHAPE;
  if (!p->q_offset && (int64_t)p->B * p->max_new != p->T) return HA_ERR_SHAPE;
  if (p->dtype != HA_BF16 && p->dtype != HA_F32) return HA_ERR_UNSUPPORTED;
  if (p->d_head != 64 && p->d_head != 128) return HA_ERR_UNSUPPORTED;
  if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128 && p->page != 256) return HA_ERR_UNSUPPORTED;
  if ((int64_t)p->max_pages * p->page > (1 << 30) || (int64_t)p->n_pages * p->page > ((int64_t)1 << 40)) return HA_ERR_UNSUPPORTED;
  if (p->B > 65535 || p->H > 65535 || (int64_t)p->B * p->H_kv > 65535 || (int64_t)p->T * (p->H / p->H_kv) > (1 << 20) || (int64_t)p->T * p->H > (1 << 24)) return HA_ERR_UNSUPPORTED;
  if (!p->key_len || (!p->page_table && p->max_pages > 0)) return HA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(p->page_table) & 3u || reinterpret_cast<uintptr_t>(p->key_len) & 3u || reinterpret_cast<uintptr_t>(p->q_offset) & 3u) return HA_ERR_ALIGN;
  return HA_OK;
}

Paged paged_of(const ha_paged_problem &p) {
  return Paged{p.B, p.H, p.H_kv, p.H / p.H_kv, p.T, p.n_pages, p.page, __builtin_ctz(p.page), p.max_pages, p.max_new, p.causal, p.page_table, p.key_len, p.q_offset};
}

ha_status check_pool(const ha_paged_problem &p, const ha_view *v, bool written, View &out) {
  const ha_status st = check_rows(p.n_pages, p.H_kv, p.n_pages ? p.page : 0, p.d_head, p.dtype, v, written, out);
  if (st != HA_OK) return st;
  if (p.n_pages && out.sn > ((int64_t)1 << 31) / (p.dtype == HA_BF16 ? 2 : 4) / (p.page + 1)) return HA_ERR_SHAPE;
  return HA_OK;
}

namespace {

// The first step of range i of n, n <= 64 (of 2^25 steps at most: the product fits 32 bits).
static __device__ __forceinline__ int part_of(int i, int steps, int n) { return (int)((unsigned)i * (unsigned)steps / (unsigned)n); }

struct FwdArgs {
  Paged p;
  View q, k, v, out;
  float *lse;
  int n_split, tiles;         // tile: ranges of the slots, tiles of a key head
  int each;                   // tile: tiles of every sequence, or 0: as the offsets place them
  int leave_few;              // tile: sequences of 32 rows or fewer are another launch's
  int wanted, line_blocks;    // few: ranges that a key head's sequences are to be cut into, together; fours of rows that a sequence may have
  int split_from;             // few: steps of a sequence that is cut
  int32_t *map;               // few, more than 64 sequences: [2][B + 1] ranges and places of the sequences ahead of each
  int32_t *heads;             // few: [place] sequence and ranges where it is a sequence's first place, otherwise -1
  float *po, *pm, *pl;        // sums of ranges: [place][rows][D], [place][rows]
  float scale, scale_log2e;
  unsigned items, share;
};

// What 32 rows of a wave are: row R of a sequence.
struct RowsOf {
  int h, token, see, n_rows;  // this lane's query head, row of T, slots that it sees
  __device__ __forceinline__ RowsOf(const Paged &p, const NewRows &n, int held, int hk, int R) {
    n_rows = n.n * p.G;
    R = min(R, n_rows - 1);
    const int i = R / p.G;
    h = hk * p.G + R - i * p.G;
    token = n.first + i;
    see = p.causal ? min(held, held - n.all + i + 1) : held;
  }
};

// 32 slots from `key` on (-1: none) and the pages that hold the first and the last sixteen of them (-1: it is not there).
struct Step {
  int key, id0, id1;
};
// Walks the slots of a sequence for one key head, 32 at a time, steps at .. end - 1, and describes the rows of keys and values that have to be read for each.
// SMALL: pages of 16 slots, two to a step (k0, v0 and k1, v1), whose addresses are formed for 64 pages at once, one in each lane; otherwise a step lies in one page, and the next
// one of that page is 32 rows further.  There is one scalar unit for all waves of a CU, so that what a step does here is kept short.
template <int ESZ, int D, bool SMALL>
struct Cursor {
  const Paged &p;
  PageWalk walk;
  const View &kv, &vv;
  const uint64_t k_base, v_base;      // of the head
  int at, end, limit, left;
  i32x4 k0, v0, k1, v1;       // descriptors of rows
  int id;
  uint64_t ka, va;
  int from;
  unsigned klo, khi, vlo, vhi;        // SMALL: this lane's page's (khi = ~0: it is not there)
  __device__ __forceinline__ Cursor(const FwdArgs &a, int b, int hk, int at_, int end_, int limit_, int lane)
      : p(a.p), walk(a.p, b, lane), kv(a.k), vv(a.v), k_base(reinterpret_cast<uint64_t>(a.k.p + hk * a.k.sh * ESZ)), v_base(reinterpret_cast<uint64_t>(a.v.p + hk * a.v.sh * ESZ)),
        at(at_), end(end_), limit(limit_), left(0), id(-1), ka(0), va(0), from(-64), klo(0), khi(0), vlo(0), vhi(0) {
    k0 = v0 = k1 = v1 = i32x4{0, 0, 0, 0x00020000};
  }
  // Bytes from the first of `rows` rows of stride `sn` elements to the end of the last.
  static __device__ __forceinline__ int span(int rows, int64_t sn) { return rows > 0 ? ((rows - 1) * (int)sn + D) * ESZ : 0; }
  __device__ __forceinline__ Step next() {
    Step s{-1, -1, -1};
    if (at >= end) {
      k0[2] = v0[2] = k1[2] = v1[2] = 0;
      return s;
    }
    const int key = 32 * at, seen = limit - key;
    s.key = key;
    ++at;
    if constexpr (SMALL) {
      const int index = key >> 4;
      if (index - from > 62) {
        from = index;
        const int page = index + walk.lane, number = page < p.max_pages ? walk.list[page] : -1;
        const bool there = (unsigned)number < (unsigned)p.n_pages;
        const uint64_t k = k_base + (uint64_t)(there ? number : 0) * kv.sb * ESZ, v = v_base + (uint64_t)(there ? number : 0) * vv.sb * ESZ;
        klo = (unsigned)k;
        khi = there ? (unsigned)(k >> 32) & 0xffff : ~0u;
        vlo = (unsigned)v;
        vhi = (unsigned)(v >> 32) & 0xffff;
      }
      const int i = index - from;
      k0[0] = __builtin_amdgcn_readlane(klo, i);
      k0[1] = __builtin_amdgcn_readlane(khi, i);
      v0[0] = __builtin_amdgcn_readlane(vlo, i);
      v0[1] = __builtin_amdgcn_readlane(vhi, i);
      k1[0] = __builtin_amdgcn_readlane(klo, i + 1);
      k1[1] = __builtin_amdgcn_readlane(khi, i + 1);
      v1[0] = __builtin_amdgcn_readlane(vlo, i + 1);
      v1[1] = __builtin_amdgcn_readlane(vhi, i + 1);
      s.id0 = k0[1] < 0 ? -1 : 0;
      s.id1 = k1[1] < 0 ? -1 : 0;
      k0[2] = k1[2] = span(16, kv.sn);
      v0[2] = v1[2] = span(16, vv.sn);
      if (seen < 32) {
        k0[2] = span(min(seen, 16), kv.sn);
        v0[2] = span(min(seen, 16), vv.sn);
        k1[2] = span(min(seen - 16, 16), kv.sn);
        v1[2] = span(min(seen - 16, 16), vv.sn);
      }
      if (s.id0 < 0) k0[1] = k0[2] = v0[2] = 0;
      if (s.id1 < 0) k1[1] = k1[2] = v1[2] = 0;
    } else {
      if (left == 0) {
        id = walk.at(key >> p.page_log2);
        left = (p.page - (key & (p.page - 1))) >> 5;
        const int64_t page = max(id, 0), row = key & (p.page - 1);
        ka = k_base + (page * kv.sb + row * kv.sn) * ESZ;
        va = v_base + (page * vv.sb + row * vv.sn) * ESZ;
      } else {
        ka += 32 * ESZ * kv.sn;
        va += 32 * ESZ * vv.sn;
      }
      --left;
      s.id0 = s.id1 = id;
      k0[0] = (int)(unsigned)ka;
      k0[1] = (int)(unsigned)(ka >> 32) & 0xffff;
      v0[0] = (int)(unsigned)va;
      v0[1] = (int)(unsigned)(va >> 32) & 0xffff;
      k0[2] = span(32, kv.sn);
      v0[2] = span(32, vv.sn);
      if (seen < 32 || id < 0) {
        k0[2] = span(id < 0 ? 0 : seen, kv.sn);
        v0[2] = span(id < 0 ? 0 : seen, vv.sn);
      }
    }
    return s;
  }
};
// A wave's requests of rows of a step (2 W bytes each): chunk i of its CHUNKS (every NW-th of the tile's) into `to`, from the half or the step that it lies in.
template <int W, bool SMALL, int NW>
struct Requests {
  typedef Tile<W> T;
  static constexpr int CHUNKS = T::chunks(32) / NW;
  int off[CHUNKS];
  unsigned to[CHUNKS];
  bool second[CHUNKS];
  __device__ __forceinline__ Requests(const char *lds, int stride_bytes, int w, int lane) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int chunk = i * NW + w, first = chunk * T::ROWS_PER_CHUNK, row = first + lane / T::PIECES;
      second[i] = first >= 16;
      off[i] = (SMALL ? row % 16 : row) * stride_bytes + (((lane % T::PIECES) ^ T::swz(row)) << 4);
      to[i] = __builtin_amdgcn_readfirstlane(lds_offset(lds) + chunk * 1024);
    }
  }
  __device__ __forceinline__ void operator()(const i32x4 &r0, const i32x4 &r1, int further) const {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      i32x4 r = r0;
      if (SMALL && second[i]) r = r1;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to[i] + further), "v"(off[i]), "s"(r) : "memory");
    }
  }
  // The same of rows that nothing else will read.
  __device__ __forceinline__ void once(const i32x4 &r0, const i32x4 &r1) const {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      i32x4 r = r0;
      if (SMALL && second[i]) r = r1;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(to[i]), "v"(off[i]), "s"(r) : "memory");
    }
  }
};

// Bytes of a slot's row from the pool's first (the head's part is in `base`).
static __device__ __forceinline__ int64_t slot_offset(const Paged &p, const View &v, int id, int slot, int esz) {
  return ((int64_t)id * v.sb + (int64_t)(slot & (p.page - 1)) * v.sn) * esz;
}
static __device__ __forceinline__ Step step_at(const Paged &p, PageWalk &walk, int key) {
  const int index = key >> p.page_log2;
  Step s{key, walk.at(index), -1};
  s.id1 = p.page > 16 ? s.id0 : index + 1 < p.max_pages ? walk.at(index + 1) : -1;
  return s;
}
// Logits of slots that this lane's row does not see.
static __device__ __forceinline__ void mask_step(f32x16 &sc, const Step &s, int see, int all_see, int g) {
  if (s.key + 32 > all_see || s.id0 < 0 || s.id1 < 0) {
    const int see0 = s.id0 < 0 ? 0 : see, see1 = s.id1 < 0 ? 0 : see;
#pragma unroll
    for (int x = 0; x < 16; ++x) sc[x] = s.key + crow(x, g) < (x < 8 ? see0 : see1) ? sc[x] : -INFINITY;
  }
}

static __device__ __forceinline__ float log_sum(float m, float l, float scale) { return l > 0.f ? m * scale + logf(l) : l == 0.f ? -INFINITY : l; }

// ---- few rows --------------------------------------------------------------------------------------------------------
// Steps of 32 slots that the rows of sequence b see, -1 where it has no rows or more than 32 of them.
static __device__ __forceinline__ int few_steps(const Paged &p, int b) {
  const NewRows n(p, b);
  if (n.n <= 0 || n.n * p.G > 32) return -1;
  const int held = p.held(b);
  return ((p.causal ? max(min(held, held - n.all + n.n), 0) : held) + 31) / 32;
}
// One token of 12 heads, d = 128, uncut and cut: 512 slots 9.1 and 9.7 us, 640 10.1 and 9.7, 768 11.1 and 9.8, 1000 13.3 and 9.8 (d = 64: 640 8.0 and 8.6, 768 8.8 and 8.5); fp32: 192 slots 13.7
// and 15.5, 256 13.9 and 13.4 (d = 64: 256 8.6 and 10, 384 10.8 and 10.2).
static inline int split_from(bool f32, int D) { return !f32 ? 24 : D == 128 ? 9 : 12; }
// Every sequence of as many steps is cut into as many ranges as is its share of `wanted`, rounded down, with four steps each and 64 ranges at most, and one at least: long ones among short
// ones do not take longer.  Those with several have a place for each range's sums, `wanted` at most.
static __device__ __forceinline__ int ranges_of(int steps, double all, int wanted, int from) {
  if (steps < from) return steps < 0 ? 0 : 1;
  // (the quotient of whole numbers below 2^42 is not rounded up to the next one)
  return max(1, min(min(64, steps / 4), (int)((double)wanted * steps / all)));
}
struct Share {
  int b, n, range, place;     // sequence (-1: none), its ranges, this one, the place of its first range's sums
  int places;                 // of all sequences
};
// Range x of all.  Where no sequence is cut, sequence x; otherwise up to 64 sequences are a lane each; of more a kernel has written the sums.
static __device__ __forceinline__ Share share_of(const FwdArgs &a, int x, int lane) {
  const Paged &p = a.p;
  Share s{-1, 0, 0, 0, 0};
  if (a.wanted == 1) {
    if (x < p.B && few_steps(p, x) >= 0) {
      s.b = x;
      s.n = 1;
    }
    return s;
  }
  if (a.map) {
    const int32_t *ranges = a.map, *places = a.map + p.B + 1;
    s.places = places[p.B];
    if (x >= ranges[p.B]) return s;
    s.b = last_not_above(p.B, x, lane, [&](int b) { return ranges[b]; });
    s.n = ranges[s.b + 1] - ranges[s.b];
    s.place = places[s.b];
    s.range = x - ranges[s.b];
    return s;
  }
  const int steps = lane < p.B ? few_steps(p, lane) : -1;
  const unsigned all = (unsigned)__builtin_amdgcn_readlane(sum_upto(max(steps, 0)), 63);      // (64 sequences of 2^25 steps at most)
  const int n = ranges_of(steps, all, a.wanted, a.split_from), places = n > 1 ? n : 0, upto_places = sum_upto(places), upto = sum_upto(n);
  s.places = __builtin_amdgcn_readlane(upto_places, 63);
  const uint64_t found = __ballot(upto > x);
  if (!found) return s;
  s.b = __ffsll((long long)found) - 1;
  s.n = __builtin_amdgcn_readlane(n, s.b);
  s.place = __builtin_amdgcn_readlane(upto_places - places, s.b);
  s.range = x - __builtin_amdgcn_readlane(upto - n, s.b);
  return s;
}
// The share of a workgroup of the kernels of few rows.  It says what the places are for: the first of a sequence's, or (the x-th range's workgroup, of place x) that there is none.
static __device__ __forceinline__ Share my_share(const FwdArgs &a, unsigned block, int lane) {
  const int x = block / a.p.Hkv, hk = block % a.p.Hkv;
  const Share s = share_of(a, x, lane);
  if (threadIdx.x == 0 && a.wanted > 1) {
    int32_t *heads = a.heads + (int64_t)hk * a.wanted * 2;
    if (x < a.wanted && x >= s.places) heads[2 * x] = -1;
    if (s.b >= 0 && s.n > 1) {
      heads[2 * (s.place + s.range)] = s.range ? -1 : s.b;
      heads[2 * (s.place + s.range) + 1] = s.n;
    }
  }
  return s;
}
__global__ __launch_bounds__(1024) void paged_map_kernel(FwdArgs a) {
  __shared__ double part[16];
  __shared__ int sums[2][16];
  const Paged &p = a.p;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  double all = 0.;
  for (int b = threadIdx.x; b < p.B; b += 1024) all += max(few_steps(p, b), 0);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) all += __shfl_xor(all, d);
  if (lane == 0) part[w] = all;
  __syncthreads();
  all = 0.;
  for (int i = 0; i < 16; ++i) all += part[i];
  int before[2] = {0, 0};
  for (int b0 = 0; b0 < p.B; b0 += 1024) {
    const int b = b0 + threadIdx.x, n = b < p.B ? ranges_of(few_steps(p, b), all, a.wanted, a.split_from) : 0, upto[2] = {sum_upto(n), sum_upto(n > 1 ? n : 0)};
    __syncthreads();
    if (lane == 63) {
      sums[0][w] = upto[0];
      sums[1][w] = upto[1];
    }
    __syncthreads();
    for (int k = 0; k < 2; ++k) {
      int ahead = before[k];
      for (int i = 0; i < 16; ++i) {
        ahead += i < w ? sums[k][i] : 0;
        before[k] += sums[k][i];
      }
      if (b < p.B) a.map[k * (p.B + 1) + b + 1] = ahead + upto[k];
    }
  }
  if (threadIdx.x < 2) a.map[threadIdx.x * (p.B + 1)] = 0;
}

template <int D>
static constexpr int image_bytes() { return 4 * 32 * D * 4; }
// The sums of four waves that walked slots of one range: joined through LDS (`image`: 4 x 32 D values) and stored.
template <int D, bool F32>
__device__ __forceinline__ void join_waves(const FwdArgs &a, const f32x16 (&o)[D / 32], float m, float l, char *lds, float (&stats)[2][4][32], int place, const RowsOf &row, int w, int lane) {
  constexpr int RB = D / 32, IMAGE = RB * 4 * 64;
  const int r = lane & 31, g = lane >> 5;
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
  if (w >= RB || r >= row.n_rows) return;
  float top = stats[0][0][r], total = 0.f;      // wave w: columns 32 w .. of the joined rows
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
  if (place >= 0) {
    const int64_t at = (int64_t)place * 32 + r;
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
    char *to = a.out.p + (row.h * a.out.sh + row.token * a.out.sn + 32 * w + 8 * x4 + 4 * g) * (F32 ? 4 : 2);
    if constexpr (F32) *reinterpret_cast<f32x4 *>(to) = y[x4] * inv;
    else *reinterpret_cast<bf16x4 *>(to) = __builtin_convertvector(y[x4] * inv, bf16x4);
  }
  if (a.lse && w == 0 && g == 0) a.lse[(int64_t)row.token * a.p.H + row.h] = log_sum(top, total, a.scale);
}

// Sums of one step: logits sc of 32 slots and the running maximum, sum and output.
template <int RB>
static __device__ __forceinline__ void follow(const f32x16 &sc, float c, float &m, float &mc, LongSum &l, f32x16 (&o)[RB]) {
  float top = m;
#pragma unroll
  for (int x = 0; x < 16; ++x) top = fmaxf(top, sc[x]);
  top = xhalf_max(top);
  const float f = top == m ? 1.f : fast_exp2((m - top) * c);      // (neither may have seen a slot)
  mc = top == -INFINITY ? 0.f : top * c;
  m = top;
  l.scale(f);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] *= f;
}

// A wave has 32 slots' keys and values in LDS, and asks for the next keys when it has read these, and for the next values likewise, so that one or the other is
// always on its way; two workgroups to a CU (fp32, 128 wide, whose rows are split into pieces behind LDS: one).  Values are asked for past the caches, which leaves those to the keys, that
// the slots' weights are formed from next: 394 MB of both 66 us for 77, up to 260 MB the same to within 1.5 us.  (Four tokens of 12 heads on 4 over up to 60000 128-wide slots: 61 us,
// 6.0 TB/s.)
template <int D, bool F32>
static constexpr int few_bytes() { return 4 * 2 * Tile<D * (F32 ? 4 : 2) / 2>::bytes(32); }      // [wave][k | v]; then [wave][register image]
template <int D, bool F32, bool SMALL>
__device__ __forceinline__ void few_rows(const FwdArgs &a, unsigned block, char *lds, float (&stats)[2][4][32]) {
  constexpr int ESZ = F32 ? 4 : 2, W = D * ESZ / 2, KS = D / 16, RB = D / 32, NS = F32 ? 3 : 1, PS = F32 ? 3 : 2;      // W: a row in twos of bytes; pieces of a value, of a weight
  typedef Tile<W> T;
  constexpr int TILE = T::bytes(32), REQUESTS = T::chunks(32);
  static_assert(image_bytes<D>() <= few_bytes<D, F32>(), "the images fit the stages");
  const Paged &p = a.p;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const int hk = block % p.Hkv;
  const Share share = my_share(a, block, lane);
  const int b = __builtin_amdgcn_readfirstlane(share.b), n_split = __builtin_amdgcn_readfirstlane(share.n), range = __builtin_amdgcn_readfirstlane(share.range);
  if (b < 0) return;
  const NewRows n(p, b);
  const int held = p.held(b);
  const RowsOf row(p, n, held, hk, r);
  const int limit = p.causal ? max(min(held, held - n.all + n.n), 0) : held, all_see = p.causal ? min(held, held - n.all + 1) : held;
  const int steps = (limit + 31) / 32;
  // (a wave has a quarter of the range, so that its steps follow one another)
  const int first = part_of(range, steps, n_split), count = part_of(range + 1, steps, n_split) - first;
  Cursor<ESZ, D, SMALL> cursor(a, b, hk, first + part_of(w, count, 4), first + part_of(w + 1, count, 4), limit, lane);
  const int ksn = (int)a.k.sn * ESZ, vsn = (int)a.v.sn * ESZ;
  char *mine = lds + w * (2 * TILE);
  const Requests<W, SMALL, 1> keys(mine, ksn, 0, lane), values(mine + TILE, vsn, 0, lane);
  Step now = cursor.next();
  if (now.key >= 0) {
    keys(cursor.k0, cursor.k1, 0);
    values.once(cursor.v0, cursor.v1);
  }
  bf16x8 qf[KS][NS];
  const char *qp = a.q.p + (row.h * a.q.sh + row.token * a.q.sn + 8 * g) * ESZ;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    if constexpr (F32) split8_cut(*reinterpret_cast<const f32x4 *>(qp + 64 * ks), *reinterpret_cast<const f32x4 *>(qp + 64 * ks + 16), qf[ks]);
    else qf[ks][0] = *reinterpret_cast<const bf16x8 *>(qp + 32 * ks);
  }
  const unsigned rows0 = T::rows_base(mine, lane), cols0 = T::cols_base(mine + TILE, lane);
  auto key_piece = [&](int ks, bf16x8 (&kf)[NS]) {
    if constexpr (F32) {      // eight columns of the lane's row: two pieces of 16 bytes
      const char *line = mine + r * T::PITCH;
      split8_cut(*reinterpret_cast<const f32x4 *>(line + (((4 * ks + 2 * g) ^ T::swz(r)) << 4)), *reinterpret_cast<const f32x4 *>(line + (((4 * ks + 2 * g + 1) ^ T::swz(r)) << 4)), kf);
    } else {
      kf[0] = T::rows_at(rows0, 0, ks);
    }
  };
  auto value_piece = [&](int rb, int u, bf16x8 (&vf)[NS]) {
    if constexpr (F32) {      // eight rows of the lane's column
      f32x8 x;
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int line = crow(8 * u + y, g);
        x[y] = *reinterpret_cast<const float *>(mine + TILE + line * T::PITCH + (((8 * rb + (r >> 2)) ^ T::swz(line)) << 4) + (r & 3) * 4);
      }
      split8_cut(__builtin_shufflevector(x, x, 0, 1, 2, 3), __builtin_shufflevector(x, x, 4, 5, 6, 7), vf);
    } else {
      vf[0] = T::cols_at(cols0, rb, 16 * u);
    }
  };
  const float c = a.scale_log2e;
  float m = -INFINITY, mc = 0.f;
  LongSum l;
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;
  while (now.key >= 0) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(REQUESTS) : "memory");
    f32x16 sc;
#pragma unroll
    for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 kf[NS];
      key_piece(ks, kf);
      sc = mfma_split<NS>(kf, qf[ks], sc);
    }
    const Step next = cursor.next();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // (the keys have been read)
    // (behind the last step nothing is read, but as many requests are made: the waits count them)
    keys(cursor.k0, cursor.k1, 0);
    mask_step(sc, now, row.see, all_see, g);
    follow(sc, c, m, mc, l, o);
    bf16x8 pb[2][PS];
    float step_sum = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x8 pr;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        pr[x] = fast_exp2(__builtin_fmaf(sc[8 * u + x], c, -mc));
        step_sum += pr[x];
      }
      if constexpr (F32) {
        split8<PS>(pr, pb[u]);
      } else {              // cut off, and what that leaves, which is never 0 of a weight that is not: an infinite value's product with it would be NaN
        f32x8 cut;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          cut[x] = __uint_as_float(__float_as_uint(pr[x]) & 0xffff0000u);
          pr[x] = fmaxf(pr[x] - cut[x], pr[x] * 0x1p-20f);
        }
        pb[u][0] = __builtin_convertvector(cut, bf16x8);
        pb[u][1] = __builtin_convertvector(pr, bf16x8);
      }
    }
    l.add(step_sum);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(REQUESTS) : "memory");
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        bf16x8 vf[NS];
        value_piece(rb, u, vf);
        if constexpr (F32) {
          o[rb] = mfma_split<NS>(vf, pb[u], o[rb]);
        } else {
          o[rb] = mfma32(vf[0], pb[u][1], o[rb]);
          o[rb] = mfma32(vf[0], pb[u][0], o[rb]);
        }
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    values.once(cursor.v0, cursor.v1);
    now = next;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // (the stages become the images)
  join_waves<D, F32>(a, o, m, l.value(), lds, stats, n_split > 1 ? hk * a.wanted + share.place + range : -1, row, w, lane);
}
template <int D, bool F32, bool SMALL>
__global__ __launch_bounds__(256, F32 && D == 128 ? 1 : 2) void paged_few_kernel(FwdArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[few_bytes<D, F32>()];
  __shared__ float stats[2][4][32];
  few_rows<D, F32, SMALL>(a, blockIdx.x, lds, stats);
}

// ---- tiles of rows ---------------------------------------------------------------------------------------------------
// The tiles of 128 rows of sequence b are those from here on, as many as it needs.  There are two ways to count them, of which the host takes the one of fewer tiles: as many for every
// sequence as the longest may need, or by the offsets, T G / 128 + B of them; some hold nothing.
static __device__ __forceinline__ int first_tile(const FwdArgs &a, int b) { return a.each ? b * a.each : a.p.offset(b) * a.p.G / 128 + b; }

// Writes a 32-row tile held as C^T (the row is the lane's) times `f` through `stage` (this wave's own LDS) to the rows at to(r), those below `rows`.
template <int D, bool F32, typename To>
static __device__ __forceinline__ void store_tile(const f32x16 (&o)[D / 32], float f, char *stage, int rows, int lane, To to) {
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
      if (row < rows) *reinterpret_cast<f32x4 *>(to(row) + pass * DP * ESZ + ch * 16) = *reinterpret_cast<const f32x4 *>(stage + row * PITCH + ch * 16);
    }
    if (PASSES > 1) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// What a workgroup of tiles works on; n_rows = 0: nothing.
struct TileOf {
  int hk, range, b, row0, n_rows;      // row0: the tile's first row of the sequence
  __device__ __forceinline__ TileOf(const Paged &p, const FwdArgs &a, unsigned item, int lane) {
    range = item % a.n_split;
    const int tile = item / a.n_split % a.tiles;
    hk = item / a.n_split / a.tiles;
    b = last_not_above(p.B, tile, lane, [&](int s) { return first_tile(a, s); });
    const NewRows n(p, b);
    row0 = (tile - first_tile(a, b)) * 128;
    n_rows = n.n * p.G;
    if (row0 < 0 || row0 >= n_rows || (a.leave_few && n_rows <= 32)) row0 = n_rows = 0;      // (a row of such a tile is never below n_rows; ahead of the first sequence row0 was negative)
  }
};

template <int D>
__device__ __forceinline__ void store_partial(const FwdArgs &a, const f32x16 (&o)[D / 32], float m, float l, unsigned item, int w, int lane) {
  const int r = lane & 31, g = lane >> 5;
  const int64_t row = (int64_t)item * 128 + 32 * w + r;
#pragma unroll
  for (int rb = 0; rb < D / 32; ++rb)
#pragma unroll
    for (int x4 = 0; x4 < 4; ++x4)
      *reinterpret_cast<f32x4 *>(a.po + row * D + 32 * rb + 8 * x4 + 4 * g) = f32x4{o[rb][4 * x4], o[rb][4 * x4 + 1], o[rb][4 * x4 + 2], o[rb][4 * x4 + 3]};
  if (g == 0) {
    a.pm[row] = m;
    a.pl[row] = l;
  }
}

// bf16: 32 slots to a step, four steps' keys and values in LDS, asked for three steps ahead.  A step forms the logits of the next slots under the exponentials of its own,
// then O^T += V^T P^T over the maxima of the next ones, so that the matrix cores and the vector units of a SIMD have work of one wave at the same time, and of two
// with two workgroups to a CU.  (1560 tokens of 12 128-wide heads over 34320 slots, 329 GFLOP: 808 thousand cycles, 368 us in a run of calls and up to 420 in short profiled ones, by the clock: the matrix cores are busy 39 % of them, a wave
// issues 45 % of its time.)
constexpr int kTileSlots = 4;
template <int D>
static constexpr int tile_bytes() { return kTileSlots * 2 * Tile<D>::bytes(32); }
template <int D, bool SMALL>
__device__ __forceinline__ void tile_rows(const FwdArgs &a, unsigned block, char *lds) {
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, TILE = T::bytes(32), SLOTS = kTileSlots, AHEAD = 3, REQUESTS = 2 * T::chunks(32) / 4;
  constexpr auto k_at = [](int step) { return step % SLOTS * 2 * TILE; };
  constexpr auto v_at = [](int step) { return step % SLOTS * 2 * TILE + TILE; };
  static_assert(4 * store_bytes<D, false>() <= tile_bytes<D>(), "the stores' staging areas fit");
  const unsigned item = xcd_item(block, a.share);
  if (item >= a.items) return;
  const Paged &p = a.p;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const TileOf tile(p, a, item, lane);
  if (tile.n_rows <= 0) return;
  const int b = tile.b, hk = tile.hk;
  const NewRows n(p, b);
  const int held = p.held(b), R0 = tile.row0 + 32 * w;
  const RowsOf row(p, n, held, hk, R0 + r);
  const int last = min(tile.row0 + 127, tile.n_rows - 1) / p.G;      // the tile's last token
  const int limit = p.causal ? max(min(held, held - n.all + last + 1), 0) : held;
  const int all_see = p.causal ? min(held, held - n.all + min(R0, tile.n_rows - 1) / p.G + 1) : held;
  const int steps = (limit + 31) / 32, end = part_of(tile.range + 1, steps, a.n_split);
  Cursor<2, D, SMALL> cursor(a, b, hk, part_of(tile.range, steps, a.n_split), end, limit, lane);
  const int ksn = (int)a.k.sn * 2, vsn = (int)a.v.sn * 2;
  const Requests<D, SMALL, 4> keys(lds, ksn, w, lane), values(lds + TILE, vsn, w, lane);
  // (behind the last step nothing is read, but as many requests are made: the waits count them)
  auto request = [&](int step) {
    const Step s = cursor.next();
    keys(cursor.k0, cursor.k1, k_at(step));
    values(cursor.v0, cursor.v1, k_at(step));
    return s;
  };
  const float c = a.scale_log2e;
  float m = -INFINITY, top = -INFINITY;               // what the sums are expressed against, the largest logit and the sum of weights (this lane's slots)
  LongSum weights;
  float some = 0.f;           // of the last one to four steps, which are added together (12 64-wide heads of 1560 tokens over 34320 slots: 251 us, each for itself 253, one sum 248)
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;
  Step s0 = request(0), s1 = request(1), s2 = request(2);
  if (s0.key >= 0 && R0 >= tile.n_rows) {             // a wave without rows has its part of the loads and barriers only
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 1) * REQUESTS) : "memory");
    __syncthreads();
    for (int now = 0; s0.key >= 0; ++now) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 2) * REQUESTS) : "memory");
      __syncthreads();
      const Step further = request(now + AHEAD);
      s0 = s1;
      s1 = s2;
      s2 = further;
    }
  } else if (s0.key >= 0) {
    bf16x8 qf[KS];
    const char *qp = a.q.p + (row.h * a.q.sh + row.token * a.q.sn + 8 * g) * 2;
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
      const int at_ = v_at(step) + 16 * u * T::PITCH;
      return T::col_piece(cols[rb][0] + at_, cols[rb][1] + at_ + 8 * T::PITCH);
    };
    const float gap = 8.f / c;
    float mc = 0.f;
    // What has been summed follows the maximum when some row's has moved by 8 in the exponent (weights stay below 2^8).
    auto mask = [&](f32x16 &sc, const Step &s) {
      if (s.key < 0) {
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = -INFINITY;
      } else {
        mask_step(sc, s, row.see, all_see, g);
      }
    };
    auto follow_far = [&](const f32x16 &sc) {
#pragma unroll
      for (int x = 0; x < 16; ++x) top = fmaxf(top, sc[x]);
      if (__any(top - m > gap)) {
        top = xhalf_max(top);
        const float f = top == m ? 1.f : fast_exp2((m - top) * c);      // (neither may have seen a slot)
        weights.scale(f);
        some *= f;
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
    mask(s_a, s0);
    follow_far(s_a);
    auto step = [&](f32x16 &sc, f32x16 &sn, auto now_c) {
      constexpr int now = decltype(now_c)::value, next = now + 1;
      // the next slots have landed, and no wave reads those of the step before any more
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 2) * REQUESTS) : "memory");
      __syncthreads();
      bf16x8 kf[KS], vf[2 * RB], pb[2];
      kf[0] = read_k(next, 0);
      kf[1] = read_k(next, 1);
      const Step further = request(now + AHEAD);
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
          some += sc[x];
          if (x % 8 == 7) {
            f32x8 pr;
#pragma unroll
            for (int z = 0; z < 8; ++z) pr[z] = sc[x - 7 + z];
            pb[x / 8] = __builtin_convertvector(pr, bf16x8);
          }
        }
        HA_FENCE();
      }
      if constexpr (now == SLOTS - 1) {
        weights.add(some);
        some = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 2 * RB; ++i) {   // i = RB u + rb
        if (i + 2 < 2 * RB) vf[i + 2] = read_v(now, (i + 2) % RB, (i + 2) / RB);
        HA_FENCE();
        o[i % RB] = mfma32(vf[i], pb[i / RB], o[i % RB]);
      }
      mask(sn, s1);
      follow_far(sn);
      s0 = s1;
      s1 = s2;
      s2 = further;
    };
    while (true) {
      step(s_a, s_b, std::integral_constant<int, 0>{});
      if (s0.key < 0) break;
      step(s_b, s_a, std::integral_constant<int, 1>{});
      if (s0.key < 0) break;
      step(s_a, s_b, std::integral_constant<int, 2>{});
      if (s0.key < 0) break;
      step(s_b, s_a, std::integral_constant<int, 3>{});
      if (s0.key < 0) break;
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  weights.add(some);
  const float l = xhalf_sum(weights.value());
  if (a.n_split > 1) {
    store_partial<D>(a, o, m, l, item, w, lane);
    return;
  }
  if (a.lse && g == 0 && R0 + r < tile.n_rows) a.lse[(int64_t)row.token * p.H + row.h] = log_sum(m, l, a.scale);
  __syncthreads();                                    // the slots become the staging area of the stores
  store_tile<D, false>(o, l == 0.f ? 0.f : 1.f / l, lds + w * store_bytes<D, false>(), tile.n_rows - R0, lane, [&](int line_) {
    const int R = R0 + line_, i = R / p.G;
    return a.out.p + ((hk * p.G + R - i * p.G) * a.out.sh + (int64_t)(n.first + i) * a.out.sn) * 2;
  });
}

template <int D, bool SMALL>
__global__ __launch_bounds__(256, 2) void paged_tile_kernel(FwdArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[tile_bytes<D>()];
  tile_rows<D, SMALL>(a, blockIdx.x, lds);
}
// Chunks beside single tokens: both in one launch, the few rows in the places that tiles leave, and behind them (64-wide, 12 heads on 4, over 8192 slots: a batch of four prompts and
// four tokens 57.6 us, with the few rows first 63.5, in launches of their own 68; one prompt of 512 beside 31 tokens over 4096, 128-wide, 32 on 8: 102, 140 and 150).
template <int D, bool SMALL>
__global__ __launch_bounds__(256, 2) void paged_both_kernel(FwdArgs few, FwdArgs tile) {
  constexpr int FEW = few_bytes<D, false>(), TILE = tile_bytes<D>();
  __shared__ __attribute__((aligned(1024))) char lds[FEW > TILE ? FEW : TILE];
  __shared__ float stats[2][4][32];
  if (blockIdx.x < 8 * tile.share) tile_rows<D, SMALL>(tile, blockIdx.x, lds);
  else few_rows<D, false, SMALL>(few, blockIdx.x - 8 * tile.share, lds, stats);
}

// fp32: 32 slots to a step, in registers a step ahead and in one stage of LDS in three pieces.  (A step of one workgroup takes 4.4 us, of two 6.9, 3.2 of them products: 24 heads on 8 of 2 x 512
// 128-wide tokens over 4096 slots 294 us, joins 19.)
template <int D>
__global__ __launch_bounds__(256, 2) void paged_tile_f32_kernel(FwdArgs a) {
  constexpr bool F32 = true;
  typedef Tile<D> T;
  constexpr int KS = D / 16, RB = D / 32, NS = 3, STAGE = T::bytes(32), ESZ = 4, PER = 32 * T::PIECES / 256;
  constexpr int LDS = 2 * NS * STAGE > 4 * store_bytes<D, F32>() ? 2 * NS * STAGE : 4 * store_bytes<D, F32>();
  __shared__ __attribute__((aligned(1024))) char lds[LDS];      // [k | v][piece][32 rows]
  const unsigned item = xcd_item(blockIdx.x, a.share);
  if (item >= a.items) return;
  const Paged &p = a.p;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
  const TileOf tile(p, a, item, lane);
  if (tile.n_rows <= 0) return;
  const int b = tile.b, hk = tile.hk;
  const NewRows n(p, b);
  const int held = p.held(b), R0 = tile.row0 + 32 * w;
  const RowsOf row(p, n, held, hk, R0 + r);
  const int last = min(tile.row0 + 127, tile.n_rows - 1) / p.G;      // the tile's last token, this wave's first
  const int limit = p.causal ? max(min(held, held - n.all + last + 1), 0) : held;
  const int all_see = p.causal ? min(held, held - n.all + min(R0, tile.n_rows - 1) / p.G + 1) : held;
  const int steps = (limit + 31) / 32;
  int at = part_of(tile.range, steps, a.n_split);
  const int end = part_of(tile.range + 1, steps, a.n_split);
  PageWalk walk(p, b, lane);
  const char *kbase = a.k.p + hk * a.k.sh * ESZ, *vbase = a.v.p + hk * a.v.sh * ESZ;
  Row8 kr[PER], vr[PER];
  const f32x4 none = {0.f, 0.f, 0.f, 0.f};
  auto request = [&](const Step &s) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at_ = threadIdx.x + 256 * i, line = at_ / T::PIECES, piece = at_ % T::PIECES, id = line < 16 ? s.id0 : s.id1, slot = s.key + line;
      kr[i] = vr[i] = Row8{none, none};
      if (id >= 0 && slot < limit) {
        kr[i] = load_row8<F32, true>(kbase + slot_offset(p, a.k, id, slot, ESZ), 0, 8 * piece, 8 * piece + 4);
        vr[i] = load_row8<F32, true>(vbase + slot_offset(p, a.v, id, slot, ESZ), 0, 8 * piece, 8 * piece + 4);
      }
    }
  };
  auto deposit = [&]() {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at_ = threadIdx.x + 256 * i, line = at_ / T::PIECES, piece = at_ % T::PIECES;
      char *to = lds + line * T::PITCH + ((piece ^ T::swz(line)) << 4);
      bf16x8 x[3];
      split8_cut(kr[i].a, kr[i].b, x);
#pragma unroll
      for (int s = 0; s < 3; ++s) *reinterpret_cast<bf16x8 *>(to + s * STAGE) = x[s];
      split8_cut(vr[i].a, vr[i].b, x);
#pragma unroll
      for (int s = 0; s < 3; ++s) *reinterpret_cast<bf16x8 *>(to + (3 + s) * STAGE) = x[s];
    }
  };
  Step now{};
  if (at < end) {
    now = step_at(p, walk, 32 * at);
    request(now);
  }
  bf16x8 qf[KS][NS];
  const char *qp = a.q.p + (row.h * a.q.sh + row.token * a.q.sn + 8 * g) * ESZ;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) split8_cut(*reinterpret_cast<const f32x4 *>(qp + 64 * ks), *reinterpret_cast<const f32x4 *>(qp + 64 * ks + 16), qf[ks]);
  const unsigned rows0 = T::rows_base(lds, lane), cols0 = T::cols_base(lds, lane);
  const float c = a.scale_log2e;
  float m = -INFINITY, mc = 0.f;
  LongSum weights;
  f32x16 o[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[rb][x] = 0.f;
  while (at < end) {
    deposit();
    __syncthreads();
    Step next{};
    ++at;
    if (at < end) {
      next = step_at(p, walk, 32 * at);
      request(next);
    }
    f32x16 sc;
#pragma unroll
    for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 kf[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) kf[s] = T::rows_at(rows0, 0, ks, s * STAGE);
      sc = mfma_split<NS>(kf, qf[ks], sc);
    }
    mask_step(sc, now, row.see, all_see, g);
    follow(sc, c, m, mc, weights, o);
    float step_sum = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x8 pr;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        pr[x] = fast_exp2(__builtin_fmaf(sc[8 * u + x], c, -mc));
        step_sum += pr[x];
      }
      bf16x8 pb[NS];
      split8<NS>(pr, pb);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        bf16x8 vf[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) vf[s] = T::cols_at(cols0, rb, 16 * u, (NS + s) * STAGE);
        o[rb] = mfma_split<NS>(vf, pb, o[rb]);
      }
    }
    weights.add(step_sum);
    __syncthreads();                                  // every wave is done with the stage
    now = next;
  }
  const float l = xhalf_sum(weights.value());
  if (a.n_split > 1) {
    store_partial<D>(a, o, m, l, item, w, lane);
    return;
  }
  if (a.lse && g == 0 && R0 + r < tile.n_rows) a.lse[(int64_t)row.token * p.H + row.h] = log_sum(m, l, a.scale);
  store_tile<D, F32>(o, l == 0.f ? 0.f : 1.f / l, lds + w * store_bytes<D, F32>(), tile.n_rows - R0, lane, [&](int line) {
    const int R = R0 + line, i = R / p.G;
    return a.out.p + ((hk * p.G + R - i * p.G) * a.out.sh + (int64_t)(n.first + i) * a.out.sn) * ESZ;
  });
}

// Largest number and sum over a wave, in all lanes, as sum_upto goes.
template <int CTRL, int ROWS>
static __device__ __forceinline__ float dpp_rows(float none, float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
template <typename Join>
static __device__ __forceinline__ float wave_join(float x, float none, Join join) {
  x = join(x, dpp_rows<0x111, 0xf>(none, x));
  x = join(x, dpp_rows<0x112, 0xf>(none, x));
  x = join(x, dpp_rows<0x114, 0xf>(none, x));
  x = join(x, dpp_rows<0x118, 0xf>(none, x));
  x = join(x, dpp_rows<0x142, 0xa>(none, x));
  x = join(x, dpp_rows<0x143, 0xc>(none, x));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
static __device__ __forceinline__ float wave_max(float x) { return wave_join(x, -INFINITY, [](float a, float b) { return fmaxf(a, b); }); }
static __device__ __forceinline__ float wave_sum(float x) { return wave_join(x, 0.f, [](float a, float b) { return a + b; }); }

// Joins the ranges of a row, at most 64: a wave to a row (6.1 us for single tokens, 10.7 for a frame's 31 MB: loads that wait for each other; four rows to a wave were no faster).  Lane i has range i's maximum and sum; D / 4 lanes take four columns each, ranges in turn.
template <int D, bool F32, int ROWS>
__device__ __forceinline__ void join_ranges(const FwdArgs &a, unsigned block) {
  constexpr int LPR = D / 4, AT_ONCE = 64 / LPR;
  const Paged &p = a.p;
  const int lane = threadIdx.x & 63, c4 = 4 * (lane % LPR);
  const int blocks = ROWS == 32 ? a.line_blocks : ROWS / 4, line = __builtin_amdgcn_readfirstlane(block % blocks * 4 + (threadIdx.x >> 6)), group = block / blocks;
  int b, hk, R, n_rows, n_split;
  int64_t at0;                // place of the row in the first range's sums; range i's: at0 + i ROWS
  if constexpr (ROWS == 32) {
    hk = group / a.wanted;
    b = a.heads[2 * group];
    n_split = a.heads[2 * group + 1];
    if (b < 0) return;
    R = line;
    n_rows = NewRows(p, b).n * p.G;
    at0 = (int64_t)group * ROWS + line;
  } else {
    const TileOf tile(p, a, (unsigned)group * a.n_split, lane);
    b = tile.b;
    hk = tile.hk;
    R = tile.row0 + line;
    n_rows = tile.n_rows;
    if (R >= n_rows) return;
    n_split = a.n_split;
    at0 = (int64_t)group * n_split * ROWS + line;
  }
  const bool has = lane < n_split;
  const float mi = has ? a.pm[at0 + (int64_t)lane * ROWS] : -INFINITY, li = has ? a.pl[at0 + (int64_t)lane * ROWS] : 0.f;
  f32x4 x[4];
  auto request = [&](int i0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = min(i0 + u * AT_ONCE + lane / LPR, n_split - 1);
      x[u] = *reinterpret_cast<const f32x4 *>(a.po + (at0 + (int64_t)i * ROWS) * D + c4);
    }
  };
  request(0);
  if (ROWS == 32 && R >= n_rows) return;        // (what has been asked for is nobody's, but there)
  const float m = wave_max(mi), f = mi == m ? 1.f : fast_exp2((mi - m) * a.scale_log2e);
  const float l = wave_sum(has ? li * f : 0.f);                // (a range that saw nothing has 0, or the NaN that has to show)
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < n_split; i0 += 4 * AT_ONCE) {
    if (i0 > 0) request(i0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * AT_ONCE + lane / LPR;
      const float fi = __shfl(f, min(i, 63));
      if (i < n_split) o += x[u] * fi;
    }
  }
#pragma unroll
  for (int d = LPR; d < 64; d <<= 1)
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] += __shfl_xor(o[u], d);
  if (lane >= LPR) return;
  const int i = R / p.G, h = hk * p.G + R - i * p.G;
  const int64_t token = p.offset(b) + i;
  if (a.lse && lane == 0) a.lse[token * p.H + h] = log_sum(m, l, a.scale);
  o *= l == 0.f ? 0.f : 1.f / l;
  const int64_t to = h * a.out.sh + token * a.out.sn + c4;
  if constexpr (F32) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out.p) + to) = o;
  else *reinterpret_cast<bf16x4 *>(reinterpret_cast<__bf16 *>(a.out.p) + to) = __builtin_convertvector(o, bf16x4);
}

// tile_blocks workgroups join those of tiles, the others those of few rows.
template <int D, bool F32>
__global__ __launch_bounds__(256) void paged_join_kernel(FwdArgs few, FwdArgs tile, unsigned tile_blocks) {
  if (blockIdx.x < tile_blocks) join_ranges<D, F32, 128>(tile, blockIdx.x);
  else join_ranges<D, F32, 32>(few, blockIdx.x - tile_blocks);
}

struct Sums {
  size_t po, pm, pl, heads;   // offsets
};
struct FwdPlan {
  bool few, tile;             // which launches there are
  int wanted, n_split, groups, each;      // few: see FwdArgs; tile: ranges, tiles of all key heads, of a sequence (see FwdArgs)
  Sums few_sums, tile_sums;
  bool map;                   // few: more than 64 sequences
  size_t off_map, total;
};

// Ranges of the slots of `tiles` tiles: as many as take the least time by this reckoning, whose unit is a step of all the workgroups that a CU holds.  With fewer of them a CU takes
// `alone` of it at least; a workgroup starts in `start`; joining takes `join` and `join_each` for every workgroup.  Fitted to times of 1 to 64 ranges of 99 batches (1 to
// 384 tiles of 4 to 1876 steps): what this chooses takes 0.3 to 1.4 % longer than the best of them on the average of a type and width, and 15 % at most.  300 tiles of 512 steps,
// 128-wide: 358 us in five ranges, 476 in one; 256 of 1073: 606 in two, 988 in one; six fp32 ones of 12: 17 in 12, 52 in one.
int ranges_of_tiles(const ha_paged_problem &p, int64_t tiles, int64_t steps) {
  const bool f32 = p.dtype == HA_F32, wide = p.d_head == 128;
  const int resident = wide ? 2 : 3;
  const double alone = wide ? (f32 ? 0.9 : 0.85) : f32 ? 0.5 : 0.45, start = f32 || !wide ? 1. : 2., join = f32 ? 1.5 : wide ? 7. : 5.5, join_each = f32 ? (wide ? 0.005 : 0.008) : wide ? 0.04 : 0.02;
  int best = 1;
  double least = 0.;
  for (int n = 1; n <= 64 && n <= steps && (n == 1 || tiles * n <= 2048); ++n) {
    const int64_t most = (tiles * n + 255) / 256, left = most % resident;      // workgroups of the CU that has the most
    const double time = (most / resident + (left ? alone + (1. - alone) * left / resident : 0.)) * ((steps + n - 1) / n + start) + (n > 1 ? join + join_each * (tiles * n) : 0.);
    if (n == 1 || time < least) {
      best = n;
      least = time;
    }
  }
  return best;
}

FwdPlan plan_forward(const ha_paged_problem &p) {
  FwdPlan f{};
  const int64_t G = p.H / p.H_kv, steps = ((int64_t)p.max_pages * p.page + 31) / 32;
  f.few = p.T > 0 && p.max_new > 0 && (p.max_new * G <= 32 || p.q_offset);
  f.tile = p.max_new * G > 32;
  size_t at = 0;
  auto take = [&](size_t places, int rows) {
    Sums s;
    s.po = at;
    at += round256(places * rows * p.d_head * 4);
    s.pm = at;
    at += round256(places * rows * 4);
    s.pl = at;
    at += round256(places * rows * 4);
    s.heads = at;
    if (rows == 32) at += round256(places * 8);
    return s;
  };
  // (ranges of all sequences and key heads: two workgroups to a CU, of 128-wide fp32 heads one: 16 sequences of 4000 slots, 4 key heads, 54 us for 63 with two)
  const int resident_few = p.dtype == HA_F32 && p.d_head == 128 ? 256 : 512;
  f.wanted = steps >= split_from(p.dtype == HA_F32, p.d_head) ? std::max(1, resident_few / p.H_kv) : 1;
  if (f.few && f.wanted > 1) f.few_sums = take((size_t)f.wanted * p.H_kv, 32);
  if ((f.map = f.few && p.B > 64 && f.wanted > 1)) {
    f.off_map = at;
    at += round256((size_t)(p.B + 1) * 8);
  }
  // (rows of no sequence have no tiles: one chunk of 64 tokens in 8192 rows, 32 heads on 8: 43 MB of workspace for 4.4 GB with tiles for all rows)
  const int64_t each = (p.max_new * G + 127) / 128, full = p.B * each * p.H_kv, placed = (p.T * G / 128 + p.B) * p.H_kv, groups = p.q_offset ? std::min(placed, full) : full;
  f.each = groups == full ? (int)each : 0;
  f.groups = (int)groups;
  f.n_split = f.tile ? ranges_of_tiles(p, groups, steps) : 1;
  if (f.tile && f.n_split > 1) f.tile_sums = take((size_t)groups * f.n_split, 128);
  f.total = at;
  return f;
}

template <int D, bool F32>
hipError_t launch_forward(const FwdArgs &all, const FwdPlan &f, char *ws, hipStream_t st) {
  hipError_t e = hipSuccess;
  FwdArgs few = all, tile = all;
  auto sums = [&](FwdArgs &a, const Sums &x) {
    a.po = reinterpret_cast<float *>(ws + x.po);
    a.pm = reinterpret_cast<float *>(ws + x.pm);
    a.pl = reinterpret_cast<float *>(ws + x.pl);
    a.heads = reinterpret_cast<int32_t *>(ws + x.heads);
  };
  const Paged &p = all.p;
  unsigned few_blocks = 0, few_joins = 0, tile_joins = 0;
  if (f.few) {
    sums(few, f.few_sums);
    few.wanted = f.wanted;
    few.split_from = split_from(F32, D);
    few.line_blocks = (std::min(32, p.max_new * p.G) + 3) / 4;
    few.map = f.map ? reinterpret_cast<int32_t *>(ws + f.off_map) : nullptr;
    few_blocks = (unsigned)(f.wanted + p.B) * p.Hkv;      // (ranges of all sequences: their shares rounded down, or one)
    if (f.wanted > 1) few_joins = (unsigned)f.wanted * p.Hkv * few.line_blocks;
    if (f.map) {
      paged_map_kernel<<<1, 1024, 0, st>>>(few);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (f.tile) {
    sums(tile, f.tile_sums);
    tile.n_split = f.n_split;
    tile.each = f.each;
    tile.tiles = f.groups / p.Hkv;
    tile.leave_few = f.few;
    tile.items = (unsigned)f.groups * f.n_split;
    tile.share = xcd_share(tile.items);
    if (f.n_split > 1) tile_joins = (unsigned)f.groups * 32;
  }
  if (!F32 && f.few && f.tile) {
    if (p.page == 16) paged_both_kernel<D, true><<<8 * tile.share + few_blocks, 256, 0, st>>>(few, tile);
    else paged_both_kernel<D, false><<<8 * tile.share + few_blocks, 256, 0, st>>>(few, tile);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    if (f.tile) {
      if constexpr (F32) paged_tile_f32_kernel<D><<<8 * tile.share, 256, 0, st>>>(tile);
      else if (p.page == 16) paged_tile_kernel<D, true><<<8 * tile.share, 256, 0, st>>>(tile);
      else paged_tile_kernel<D, false><<<8 * tile.share, 256, 0, st>>>(tile);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (f.few) {
      if (p.page == 16) paged_few_kernel<D, F32, true><<<few_blocks, 256, 0, st>>>(few);
      else paged_few_kernel<D, F32, false><<<few_blocks, 256, 0, st>>>(few);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (tile_joins + few_joins > 0) {
    paged_join_kernel<D, F32><<<tile_joins + few_joins, 256, 0, st>>>(few, tile, tile_joins);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" ha_status hybrid_attn_paged_validate(const ha_paged_problem *p) { return check_paged(p); }

extern "C" size_t hybrid_attn_paged_workspace_bytes(const ha_paged_problem *p) {
  if (check_paged(p) != HA_OK) return 0;
  return plan_forward(*p).total;
}

extern "C" ha_status hybrid_attn_paged_forward(const ha_paged_problem *p, const ha_view *q, const ha_view *k_pages, const ha_view *v_pages, const ha_view *out, float *lse,
                                               void *workspace, size_t workspace_bytes, void *hip_stream) {
  ha_status st = check_paged(p);
  if (st != HA_OK) return st;
  FwdArgs a{};
  if ((st = check_packed(*p, q, p->H, false, a.q)) != HA_OK || (st = check_pool(*p, k_pages, false, a.k)) != HA_OK || (st = check_pool(*p, v_pages, false, a.v)) != HA_OK ||
      (st = check_packed(*p, out, p->H, true, a.out)) != HA_OK)
    return st;
  if (reinterpret_cast<uintptr_t>(lse) & 3u) return HA_ERR_ALIGN;
  if (p->T == 0) return HA_OK;
  const FwdPlan f = plan_forward(*p);
  if ((st = check_workspace(workspace, workspace_bytes, f.total)) != HA_OK) return st;
  a.p = paged_of(*p);
  a.lse = lse;
  a.scale = p->softmax_scale;
  a.scale_log2e = p->softmax_scale * kLog2e;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(workspace);
  const bool f32 = p->dtype == HA_F32;
  const hipError_t e = p->d_head == 128 ? (f32 ? launch_forward<128, true>(a, f, ws, stream) : launch_forward<128, false>(a, f, ws, stream))
                                        : (f32 ? launch_forward<64, true>(a, f, ws, stream) : launch_forward<64, false>(a, f, ws, stream));
  return e == hipSuccess ? HA_OK : device_error(e);
}
