// What the attention kernels share: the segment table and how its work is dealt out, staged tiles
// and their products, the number of splits.  (wm_attend.hip: attention to a program's keys;
// wm_prefix.hip: to a program's keys and the sequence's own.)
//
// All products are computed transposed, S^T = K . Q^T, so that a row is a
// lane's column of the accumulators: its softmax statistics are per-lane values
// completed across the lane pair (L, L ^ 32), and the probabilities are the
// operand of the next product where they are (its contraction runs over the
// accumulators' own row order).  The other operand of that product is the
// staged tile read by columns: LDS reads that transpose (bf16), single words
// (float32).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "wm_device.h"
#include "wm_internal.h"

namespace wm {
namespace attend {

constexpr int MAX_SEGS = 128;               // segments per launch (the table is a kernel argument)
constexpr int XCDS = 8;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// Weights against a maximum that is out of date are fine until a row's sum over one
// step passes this: the accumulators are seldom rescaled, and the maximum is seldom
// looked for (half an instruction per score, and a branch).
constexpr float SUM_LIMIT = 1024.0f;

// Segments of a launch, those with the longest loops first.  A segment's (key head,
// tile) pairs are dealt out evenly over the XCDs (workgroups go to them in turn), in
// runs that share a head's keys in an XCD's L2: dealing whole segments to XCDs
// left some with twice the work of others where key counts differ.
struct Table {
  int32_t n;
  struct {
    int32_t q0, lq, k0, lk;
  } seg[MAX_SEGS];
  int32_t off[MAX_SEGS + 1];                // pairs per XCD, summed
};

template <class T>
constexpr bool IS_BF = std::is_same<T, __bf16>::value;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// v of the lane pair (L, L ^ 32) combined
__device__ __forceinline__ float pair_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ float pair_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  return __uint_as_float(a) + __uint_as_float(b);
}

// Scores leave the products in units of log2 in float32 (an operand is scaled when it is
// loaded, and a score that is the maximum in use weighs exactly 1), unscaled in bf16 (a
// scaled operand would be rounded once more).
template <class T>
__device__ __forceinline__ float log2_units(float s, float c2) { return IS_BF<T> ? s * c2 : s; }
template <class T>
__device__ __forceinline__ float weight(float s, float c2, float at) { return exp2_of(IS_BF<T> ? fmaf(s, c2, -at) : s - at); }

// --------------------------------------------------------------------------
// A staged tile: rows of DH elements in 16-byte units; unit u of row r lies at
// u ^ swz(r).  The LDS serves 16 lanes of a 16-byte read together (256 bytes):
// 16 neighbouring rows, one unit, have to fall on different bank groups.  The column
// reads take 4 neighbouring rows x 4 units (bf16) or a row and the fourth
// after it x 8 units (float32) together.
template <class T, int DH>
struct Tile {
  static constexpr int E = IS_BF<T> ? 8 : 4;            // elements per unit
  static constexpr int UPR = DH / E;                    // units per row
  static constexpr int DB = DH / 32;                    // 32-column blocks
  static constexpr int NR = IS_BF<T> ? DH / 16 : DH / 8;   // 16-byte registers of one row operand
  using Op = u32x4[NR];

  static __device__ __forceinline__ int swz(int r) {
    if constexpr (IS_BF<T>) {
      if constexpr (DH == 32) return (r >> 2) & 3;
      else if constexpr (DH == 64) return ((r << 1) & 4) | ((r >> 1) & 2) | ((r >> 3) & 1);
      else return ((r & 3) << 2) | ((r >> 2) & 3);
    } else {
      if constexpr (DH == 32) return (r >> 1) & 7;
      else return ((r & 4) << 1) | ((r & 8) >> 1) | (r & 3);
    }
  }
  // Row operand: 32 columns (one per lane of a half) from rows of global memory.
  // bf16: register kk holds features 16 kk + 8 h ..; float32: register i features h DH/2 + 4 i ..
  static __device__ __forceinline__ void load_op(Op& op, const T* row, int h) {
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int f = IS_BF<T> ? 16 * i + 8 * h : h * (DH / 2) + 4 * i;
      op[i] = *reinterpret_cast<const u32x4*>(row + f);
    }
  }
  // float32: the operand times f, so that scores come out in units of log2
  static __device__ __forceinline__ void scale_op(Op& op, float f) {
    if constexpr (!IS_BF<T>) {
#pragma unroll
      for (int i = 0; i < NR; ++i) op[i] = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, op[i]) * f);
    }
  }
  // do_c . o_c of a lane's column c, by the products that form do . v (the same sums bit
  // for bit where o is a v: a row with one key has dS = 0)
  static __device__ __forceinline__ float dot_cols(const Op& x, const Op& y, int lane) {
    f32x16 acc = {};
#pragma unroll
    for (int i = 0; i < NR; ++i) acc = mm_one(x[i], y[i], acc);
    float d = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) d = acc_row(lane >> 5, r) == (lane & 31) ? acc[r] : d;
    return pair_sum(d);                         // the other half of the pair has 0
  }
  // one 16-byte register of both operands
  static __device__ __forceinline__ f32x16 mm_one(u32x4 x, u32x4 y, f32x16 acc) {
    if constexpr (IS_BF<T>) {
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
    } else {
      const f32x4 a = __builtin_bit_cast(f32x4, x), b = __builtin_bit_cast(f32x4, y);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], acc, 0, 0, 0);
    }
    return acc;
  }
  // sum over features of tile rows base .. base + 31 (accumulator rows) and the operand's columns
  static __device__ __forceinline__ f32x16 mm_row(const T* tile, int base, const Op& op, int lane) {
    const int h = lane >> 5, row = base + (lane & 31);
    f32x16 acc = {};
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int unit = IS_BF<T> ? 2 * i + h : h * (DH / 8) + i;
      const u32x4 u = *reinterpret_cast<const u32x4*>(tile + row * DH + (unit ^ swz(row)) * E);
      acc = mm_one(u, op[i], acc);
    }
    return acc;
  }
  // acc[b] += sum over tile rows base + acc_row(h, r) of column 32 b + c of the tile and p[r].
  // bf16: p (probabilities, score gradients) is rounded to bf16 to be a matrix operand; float32
  // products run at a seventh of the rate.  It costs the second of two roundings: results are
  // 1.9e-3 to 2.4e-3 off (2-norm), where the rounding of the result alone gives 1.7e-3.
  static __device__ __forceinline__ void mm_col(const T* tile, int base, const f32x16& p, f32x16 (&acc)[DB], int lane) {
    const int h = lane >> 5;
    if constexpr (IS_BF<T>) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        bf16x8 pf;
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[j] = (__bf16)p[8 * f + j];
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          s16x4 half[2];
#pragma unroll
          for (int jj = 0; jj < 2; ++jj) {
            const int row = base + 16 * f + 8 * jj + 4 * h + ((lane >> 2) & 3);
            const int unit = 4 * b + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
            const T* at = tile + row * DH + (unit ^ swz(row)) * 8 + 4 * (lane & 1);
            half[jj] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at));
          }
          typedef short s16x8 __attribute__((ext_vector_type(8)));
          const s16x8 a = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), pf, acc[b], 0, 0, 0);
        }
      }
    } else {
      const int c = lane & 31;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = base + acc_row(h, r);
        const float pr = p[r];
#pragma unroll
        for (int b = 0; b < DB; ++b)
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[row * DH + ((8 * b + (c >> 2)) ^ swz(row)) * 4 + (c & 3)], pr, acc[b], 0, 0, 0);
      }
    }
  }
};

// Rows per staged tile: two tiles of two matrices stay within 64 KiB (bf16) so
// that two workgroups share a compute unit, and within 128 KiB in every case.
template <class T, int DH>
constexpr int TILE_ROWS = (!IS_BF<T> && DH == 128) ? 32 : 64;

// Copy of `rows` <= ROWS rows into a tile; offset(row) gives a row's byte offset from the
// buffer's base, BAD for a row that is to read as zero.
constexpr uint32_t BAD = 0x80000000u;       // past every buffer's end: such lanes read zero
template <class T, int DH, int ROWS, int NT, class Off>
__device__ __forceinline__ void copy_tile(u32x4 buf, T* tile, int tid, Off offset) {
  using TL = Tile<T, DH>;
  constexpr int N = ROWS * TL::UPR / NT;
  static_assert(ROWS * TL::UPR % NT == 0, "whole units per thread");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int u = i * NT + tid, row = u / TL::UPR, unit = (u % TL::UPR) ^ TL::swz(row);
    const uint32_t o = offset(row);
    copy16(buf, tile + (size_t)(i * NT + (tid & ~63)) * TL::E, o == BAD ? BAD : o + unit * 16);
  }
}

// The problem of a workgroup: segment, key head, tile, split of its loop.
struct Prob {
  int q0, R, k0, Lk, hk, tile, split;
};
// false: none (a segment's pairs need not divide by the XCDs).  rows_per_tile: of the tiled axis (R, or Lk
// for keys).
template <bool KEYS, class Args>
__device__ __forceinline__ bool problem(const Table& t, const Args& a, int rows_per_tile, Prob& p, int block = blockIdx.x) {
  const int x = block % XCDS, i = block / XCDS;
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.off[mid] <= i) lo = mid; else hi = mid - 1;
  }
  p.q0 = t.seg[lo].q0;
  p.R = t.seg[lo].lq * a.G;
  p.k0 = t.seg[lo].k0;
  p.Lk = t.seg[lo].lk;
  const int tiles = ((KEYS ? p.Lk : p.R) + rows_per_tile - 1) / rows_per_tile;
  // XCD x's share, another first XCD for every segment so that the shares' remainders spread
  const int n = tiles * a.kv_heads * a.splits, y = (x + 3 * lo) % XCDS, at = (int)((int64_t)n * y / XCDS) + i - t.off[lo];
  const int pair = at / a.splits;
  p.split = at - pair * a.splits;
  p.hk = pair / tiles;
  p.tile = pair - p.hk * tiles;
  return at < (int)((int64_t)n * (y + 1) / XCDS);
}

// Which of the `n` keys from `key` on are seen, one bit each (64 at most).
__device__ __forceinline__ uint64_t in_range(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }

// Accumulators of a lane's column: rows (features) 32 b + acc_row(h, r), four neighbours at a time.
template <class T, int DB>
__device__ __forceinline__ void store_cols(T* row, const f32x16 (&acc)[DB], float f, int h) {
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      typedef T t4 __attribute__((ext_vector_type(4)));
      t4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (T)(acc[b][4 * q + i] * f);
      *reinterpret_cast<t4*>(row + 32 * b + acc_row(h, 4 * q)) = x;
    }
}

// --------------------------------------------------------------------------
// Host side.

inline size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Into how many splits the loops of `blocks` workgroups, `units` steps of unit_us each on
// average (`longest` at most), are cut: the number of rounds that 256 x per_cu
// places take times a split's length, plus what the partial sums cost (part_us a
// split; a launch that joins them).  A split of the longest loop keeps at least
// `least` steps; all loops are cut alike, so that splits of short ones may be empty,
// and a long loop among many short ones gets the splits of the average.
// One split of 520 workgroups on 512 places took 400 us (a second round of eight), four
// 310 and 21 for the sums.
inline int splits_for(int64_t blocks, double units, int64_t longest, int64_t least, int per_cu, double unit_us, double part_us) {
  int best = 1;
  double cost = 1e30;
  for (int s = 1; s <= 64 && (s == 1 || s <= longest / least); ++s) {
    const double c = (double)cdiv(blocks * s, 256 * per_cu) * std::ceil(units / s) * unit_us + (s > 1 ? s * part_us + 4.0 : 0.0);
    if (c < 0.98 * cost) {
      cost = c;
      best = s;
    }
  }
  return best;
}

// whether a matrix of n rows [heads][head_dim] has rows that the kernels can take
inline bool rows_ok(const wm_attention* a, const void* p, int64_t ld, int64_t n, int heads) {
  const int64_t e = a->dtype == WM_BF16 ? 2 : 4;
  return n == 0 || (p && (uintptr_t)p % 16 == 0 && ld >= (int64_t)heads * a->head_dim && ld * e % 16 == 0 && ld <= (1 << 22));
}

// Calls go(table, workgroups) for runs of at most MAX_SEGS segments, sorted by the length of their
// workgroups' loops; tiles(lq, lk) is a segment's number of tiles.
template <class Tiles, class Go>
hipError_t each_run(const wm_attention* a, bool keys, int splits, Tiles tiles, Go go) {
  for (int s0 = 0; s0 < a->S; s0 += MAX_SEGS) {
    Table t = {};
    for (int i = s0; i < std::min(a->S, s0 + MAX_SEGS); ++i)
      t.seg[t.n++] = {a->q_off[i], a->q_off[i + 1] - a->q_off[i], a->k_off[i], a->k_off[i + 1] - a->k_off[i]};
    std::stable_sort(t.seg, t.seg + t.n, [&](const auto& x, const auto& y) { return keys ? x.lq > y.lq : x.lk > y.lk; });
    for (int i = 0; i < t.n; ++i) t.off[i + 1] = t.off[i] + (int32_t)cdiv(tiles(t.seg[i].lq, t.seg[i].lk) * a->kv_heads * splits, XCDS);
    if (t.off[t.n] == 0) continue;
    go(t, t.off[t.n] * XCDS);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// f(T{}, integral_constant<DH>)
template <class F>
auto typed(const wm_attention* a, F f) {
  auto width = [&](auto t) {
    using T = decltype(t);
    if (a->head_dim == 32) return f(t, std::integral_constant<int, 32>{});
    if (a->head_dim == 64) return f(T{}, std::integral_constant<int, 64>{});
    return f(T{}, std::integral_constant<int, 128>{});
  };
  return a->dtype == WM_BF16 ? width(__bf16{}) : width(float{});
}

// wm_attention's checks, and what a call that does more needs of its plan.
struct Shared {
  int64_t nq, nk, max_lk, max_r;
};
wm_status check_shared(const wm_attention* w, Shared* sh);

}  // namespace attend
}  // namespace wm
