// Cross attention to encoded states of another length: forward and gradients.
//
// Segment s (a program) has query rows [q_off[s], q_off[s+1]) and key rows
// [k_off[s], k_off[s+1]); the G = heads / kv_heads query heads that share a
// key head are stacked, so (segment, key head) is one problem of R = Lq G rows
// (row r: query r / G, head hk G + r % G) against Lk keys, and the keys'
// gradients sum a group's heads by themselves.
#include <string>

#include "wm_attend.h"

using namespace wm;

namespace wm {
namespace attend {

struct Args {
  const void *q, *k, *v, *o, *d_o;
  int64_t ld_q, ld_k, ld_v, ld_o, ld_do;
  const uint8_t* mask;
  float c2, scale;                          // scale log2(e), scale
  int heads, kv_heads, G, splits;
  void *out, *out2;                         // o; dq; dk and dv
  int64_t ld_out, ld_out2;
  float* lse;                               // forward: out (may be null); gradient: in
  float* stat;                              // gradient: [Nq heads][2] (lse log2 e, delta)
  float* part;                              // partial sums [splits][rows][DH] (dkv: [splits][2][rows][DH])
  float* part_ml;                           // forward: [splits][rows][2] maximum (log2 units), sum
  int64_t part_rows;
};

// --------------------------------------------------------------------------
// Forward.  A workgroup of 4 wavefronts takes 128 / WK rows (32 per wavefront);
// WK wavefronts share rows and take every WK-th block of 32 keys (the form for at
// most 32 rows per key head, where a wavefront of its own per 32 rows would leave three idle:
// 16 streams of one query over 10k keys, 645 MB, 158 us, 4.1 TB/s, what a
// large read reaches here).  Tiles of K and V are staged two deep by copies straight
// to LDS; softmax online.  Long forms are bound by the vector unit: an exponential (as
// long as two instructions) and six instructions per score keep it busy 69% of the
// time, the matrix cores 33%, at 2.6 wavefronts per SIMD: 32k rows on 256 to 2048
// keys, 12 heads of 64 in bf16, 100 GFLOP, 141 us (711 TFLOP/s).
template <class T, int DH, int WK>
constexpr int FWD_PER_CU = 4 * (WK > 1 ? 32 * WK : TILE_ROWS<T, DH>) * DH * (int)sizeof(T) <= 80 * 1024 ? 2 : 1;
template <class T, int DH, int WK>
__global__ __launch_bounds__(256, (FWD_PER_CU<T, DH, WK>)) void forward_kernel(const Table t, const Args a) {
  using TL = Tile<T, DH>;
  constexpr int WR = 4 / WK, DB = TL::DB;
  constexpr int KB = WK > 1 ? 32 * WK : TILE_ROWS<T, DH>;     // keys per tile
  constexpr int NV = (KB + 63) / 64;                          // visibility words per tile
  __shared__ __attribute__((aligned(16))) T lds[4 * KB * DH];
  T* const ks = lds;                                          // [2][KB][DH]
  T* const vs = lds + 2 * KB * DH;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, wr = wave % WR, wk = wave / WR;
  Prob p;
  if (!problem<false>(t, a, 32 * WR, p)) return;
  const int row = p.tile * (32 * WR) + wr * 32 + (lane & 31);       // may pass R: computed, not stored
  const int rr = min(row, p.R - 1), head = p.hk * a.G + rr % a.G;
  const int64_t qrow = (int64_t)p.q0 + rr / a.G;
  typename TL::Op qf;
  TL::load_op(qf, static_cast<const T*>(a.q) + qrow * a.ld_q + head * DH, h);
  TL::scale_op(qf, a.c2);

  const int tiles = (p.Lk + KB - 1) / KB, split = p.split;
  const int t0 = (int)((int64_t)tiles * split / a.splits), t1 = (int)((int64_t)tiles * (split + 1) / a.splits);
  const uint8_t* mask = a.mask ? a.mask + p.k0 : nullptr;
  auto mask_byte = [&](int tile, int w) -> int {
    const int key = tile * KB + 64 * w + lane;
    return (KB >= 64 || lane < KB) && key < p.Lk ? mask[key] : 0;
  };
  auto copy = [&](int tile, const uint64_t (&vis)[NV]) {
    const int64_t first = (int64_t)p.k0 + (int64_t)tile * KB;
    const u32x4 kb = buffer_of(static_cast<const T*>(a.k) + first * a.ld_k + p.hk * DH, BAD - 1);
    const u32x4 vb = buffer_of(static_cast<const T*>(a.v) + first * a.ld_v + p.hk * DH, BAD - 1);
    auto seen = [&](int r) { return (vis[NV > 1 ? r >> 6 : 0] >> (r & 63)) & 1; };
    copy_tile<T, DH, KB, 256>(kb, ks + (tile & 1) * KB * DH, tid,
                              [&](int r) { return seen(r) ? (uint32_t)(r * a.ld_k * sizeof(T)) : BAD; });
    copy_tile<T, DH, KB, 256>(vb, vs + (tile & 1) * KB * DH, tid,
                              [&](int r) { return seen(r) ? (uint32_t)(r * a.ld_v * sizeof(T)) : BAD; });
  };
  uint64_t vis[NV], next[NV];
  int mb[NV];
  auto look = [&](int tile, uint64_t (&v)[NV], bool load) {   // visibility of a tile (mask bytes loaded before)
#pragma unroll
    for (int w = 0; w < NV; ++w) {
      if (load && mask) mb[w] = mask_byte(tile, w);
      v[w] = mask ? __ballot(mb[w] != 0) : in_range(min(p.Lk - tile * KB - 64 * w, KB));
    }
  };

  f32x16 acc[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b] = f32x16{};
  float mx = -INFINITY, sum = 0.0f;
  bool started = false;                       // every row has a maximum
  if (t0 < t1) {
    look(t0, vis, true);
    copy(t0, vis);
    if (mask && t0 + 1 < t1)
#pragma unroll
      for (int w = 0; w < NV; ++w) mb[w] = mask_byte(t0 + 1, w);
  }
  for (int ti = t0; ti < t1; ++ti) {
    wait_counts<0, true>();
    raw_barrier();
    if (ti + 1 < t1) {
      look(ti + 1, next, false);
      copy(ti + 1, next);
      if (mask && ti + 2 < t1)
#pragma unroll
        for (int w = 0; w < NV; ++w) mb[w] = mask_byte(ti + 2, w);
    }
    const T* kt = ks + (ti & 1) * KB * DH;
    const T* vt = vs + (ti & 1) * KB * DH;
    // The keys of this wavefront in the tile, 32 at a time; weights are formed
    // against the maximum in use, and only where their sum grows past 2^10 (or a
    // key is hidden, or there is no maximum yet) the maximum is looked for.
    constexpr int NB = KB / 32 / WK;
    f32x16 s[NB];
    uint32_t seen[NB];
    bool all = true;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      const int base = 32 * (kb * WK + wk);
      seen[kb] = (uint32_t)(vis[NV > 1 ? base >> 6 : 0] >> (base & 63));
      all = all && seen[kb] == ~0u;
    }
    float bs;
    bool look_for_max = !started || !all;
    // a second time, scores and all, with the maximum that the first lacked
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) s[kb] = TL::mm_row(kt, 32 * (kb * WK + wk), qf, lane);
      if (!all) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
          uint32_t m = seen[kb] >> (4 * h);
          asm volatile("" : "+v"(m));               // keeps this a branch: seldom taken, 48 instructions
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = (m >> acc_row(0, r)) & 1 ? s[kb][r] : -INFINITY;
        }
      }
      if (look_for_max) {
        float bm = s[0][0];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) bm = fmaxf(bm, s[kb][r]);
        bm = pair_max(bm);
        const float f = bm > mx ? exp2_of(log2_units<T>(mx - bm, a.c2)) : 1.0f;
        sum *= f;
#pragma unroll
        for (int b = 0; b < DB; ++b) acc[b] *= f;
        mx = bm > mx ? bm : mx;
        started = !__any(mx == -INFINITY);
      }
      const float mc = mx == -INFINITY ? 0.0f : log2_units<T>(mx, a.c2);      // only keys of weight 0 so far
      bs = 0.0f;
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {             // weights in the scores' place
          s[kb][r] = weight<T>(s[kb][r], a.c2, mc);
          bs += s[kb][r];
        }
      if (!__any(bs > SUM_LIMIT)) break;           // infinite or NaN scores stay what they are
      look_for_max = true;
    }
    sum += bs;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) TL::mm_col(vt, 32 * (kb * WK + wk), s[kb], acc, lane);
#pragma unroll
    for (int w = 0; w < NV; ++w) vis[w] = next[w];
  }
  sum = pair_sum(sum);
  float m2 = mx == -INFINITY ? -INFINITY : log2_units<T>(mx, a.c2);
  if constexpr (WK > 1) {       // join the wavefronts that share rows
    __syncthreads();
    constexpr int LW = DH + 4;
    float* x = reinterpret_cast<float*>(lds);                 // [4][32][LW]
    float* ml = x + 4 * 32 * LW;                              // [4][32][2]
    static_assert((4 * 32 * LW + 256) * 4 <= sizeof(lds), "the exchange takes the tiles' place");
    if (wk > 0) {
      store_cols<float, DB>(x + (wave * 32 + (lane & 31)) * LW, acc, 1.0f, h);
      if (h == 0) {
        ml[(wave * 32 + lane) * 2] = m2;
        ml[(wave * 32 + lane) * 2 + 1] = sum;
      }
    }
    __syncthreads();
    if (wk > 0) return;
    float top = m2;
#pragma unroll
    for (int k = 1; k < WK; ++k) top = fmaxf(top, ml[((wr + WR * k) * 32 + (lane & 31)) * 2]);
    const float at = top == -INFINITY ? 0.0f : top;
    float f = exp2_of(m2 - at);
    sum *= f;
#pragma unroll
    for (int b = 0; b < DB; ++b) acc[b] *= f;
#pragma unroll
    for (int k = 1; k < WK; ++k) {
      const int w = (wr + WR * k) * 32 + (lane & 31);
      f = exp2_of(ml[2 * w] - at);
      sum = fmaf(ml[2 * w + 1], f, sum);
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const f32x16 y = load_acc(x + w * LW + 32 * b, h);
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[b][r] = fmaf(y[r], f, acc[b][r]);
      }
    }
    m2 = top;
  }
  if (row >= p.R) return;
  const int64_t orow = qrow * a.heads + head;
  if (a.splits > 1) {
    const int64_t prow = split * a.part_rows + orow;
    store_cols<float, DB>(a.part + prow * DH, acc, 1.0f, h);
    if (h == 0) {
      a.part_ml[2 * prow] = m2;
      a.part_ml[2 * prow + 1] = sum;
    }
    return;
  }
  store_cols<T, DB>(static_cast<T*>(a.out) + qrow * a.ld_out + head * DH, acc, sum == 0.0f ? 0.0f : 1.0f / sum, h);
  if (a.lse && h == 0) a.lse[orow] = sum == 0.0f ? -INFINITY : (m2 + __builtin_amdgcn_logf(sum)) * LN2;
}

// Joins the key splits of every row: 16-byte quads of a row's features, one per thread.
template <class T, int DH>
__global__ __launch_bounds__(256) void join_kernel(const Args a, int64_t rows) {
  constexpr int Q = DH / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * Q) return;
  const int64_t r = i / Q;
  const int d = (int)(i % Q) * 4;
  float top = -INFINITY;
  for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.part_ml[2 * (s * a.part_rows + r)]);
  const float at = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < a.splits; ++s) {
    const int64_t p = s * a.part_rows + r;
    const float f = exp2_of(a.part_ml[2 * p] - at);
    sum = fmaf(a.part_ml[2 * p + 1], f, sum);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part + p * DH + d);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = fmaf(x[j], f, acc[j]);
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 y;
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = (T)(acc[j] * inv);
  *reinterpret_cast<t4*>(static_cast<T*>(a.out) + (r / a.heads) * a.ld_out + (r % a.heads) * DH + d) = y;
  if (a.lse && d == 0) a.lse[r] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
}

// --------------------------------------------------------------------------
// Gradients.  P = exp(S - lse) is formed again; delta = do . o; dS = P (do . v - delta).
// Sums are in a fixed order, without atomics: one kernel owns rows (dq), one
// owns keys (dk, dv).

// dq, and every row's (lse log2 e, delta) for the other kernel.  As the forward
// kernel with 128 rows per workgroup: three products of which two are formed again,
// against one that would have to pass dS through memory.  Vector unit busy 57% of the time, matrix
// cores 42%: 28k rows on 1024 to 2048 keys, 12 heads of 64 in bf16, 161 GFLOP, 190 us.
template <class T, int DH>
__global__ __launch_bounds__(256, (IS_BF<T> && DH <= 64) ? 2 : 1) void dq_kernel(const Table t, const Args a) {
  using TL = Tile<T, DH>;
  constexpr int DB = TL::DB, KB = TILE_ROWS<T, DH>;
  __shared__ __attribute__((aligned(16))) T lds[4 * KB * DH];
  T* const ks = lds;
  T* const vs = lds + 2 * KB * DH;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5;
  Prob p;
  if (!problem<false>(t, a, 128, p)) return;
  const int row = p.tile * 128 + wave * 32 + (lane & 31);
  const int rr = min(row, p.R - 1), head = p.hk * a.G + rr % a.G;
  const int64_t qrow = (int64_t)p.q0 + rr / a.G, orow = qrow * a.heads + head;
  typename TL::Op qf, gf;
  TL::load_op(qf, static_cast<const T*>(a.q) + qrow * a.ld_q + head * DH, h);
  TL::scale_op(qf, a.c2);
  TL::load_op(gf, static_cast<const T*>(a.d_o) + qrow * a.ld_do + head * DH, h);
  float delta;
  {
    typename TL::Op of;
    TL::load_op(of, static_cast<const T*>(a.o) + qrow * a.ld_o + head * DH, h);
    delta = TL::dot_cols(of, gf, lane);
  }
  const float lse = a.lse[orow];
  // a row without a visible key has lse = -inf: its P is 0
  const float l2 = lse == -INFINITY ? INFINITY : lse * LOG2E;
  const int split = p.split;
  if (split == 0 && h == 0 && row < p.R) {
    a.stat[2 * orow] = l2;
    a.stat[2 * orow + 1] = delta;
  }
  const int tiles = (p.Lk + KB - 1) / KB;
  const int t0 = (int)((int64_t)tiles * split / a.splits), t1 = (int)((int64_t)tiles * (split + 1) / a.splits);
  const uint8_t* mask = a.mask ? a.mask + p.k0 : nullptr;
  auto mask_byte = [&](int tile) -> int {
    const int key = tile * KB + lane;
    return (KB >= 64 || lane < KB) && key < p.Lk ? mask[key] : 0;
  };
  auto copy = [&](int tile, uint64_t vis) {
    const int64_t first = (int64_t)p.k0 + (int64_t)tile * KB;
    const u32x4 kb = buffer_of(static_cast<const T*>(a.k) + first * a.ld_k + p.hk * DH, BAD - 1);
    const u32x4 vb = buffer_of(static_cast<const T*>(a.v) + first * a.ld_v + p.hk * DH, BAD - 1);
    copy_tile<T, DH, KB, 256>(kb, ks + (tile & 1) * KB * DH, tid,
                              [&](int r) { return (vis >> r) & 1 ? (uint32_t)(r * a.ld_k * sizeof(T)) : BAD; });
    copy_tile<T, DH, KB, 256>(vb, vs + (tile & 1) * KB * DH, tid,
                              [&](int r) { return (vis >> r) & 1 ? (uint32_t)(r * a.ld_v * sizeof(T)) : BAD; });
  };
  auto look = [&](int tile, int mb) { return mask ? __ballot(mb != 0) : in_range(min(p.Lk - tile * KB, KB)); };
  f32x16 acc[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b] = f32x16{};
  uint64_t vis = 0, next = 0;
  int mb = 0;
  if (t0 < t1) {
    if (mask) mb = mask_byte(t0);
    vis = look(t0, mb);
    copy(t0, vis);
    if (mask && t0 + 1 < t1) mb = mask_byte(t0 + 1);
  }
  for (int ti = t0; ti < t1; ++ti) {
    wait_counts<0, true>();
    raw_barrier();
    if (ti + 1 < t1) {
      next = look(ti + 1, mb);
      copy(ti + 1, next);
      if (mask && ti + 2 < t1) mb = mask_byte(ti + 2);
    }
    const T* kt = ks + (ti & 1) * KB * DH;
    const T* vt = vs + (ti & 1) * KB * DH;
#pragma unroll
    for (int kb = 0; kb < KB / 32; ++kb) {
      const uint32_t seen = (uint32_t)(vis >> (32 * kb));
      if (seen == 0) continue;
      f32x16 s = TL::mm_row(kt, 32 * kb, qf, lane);
      const f32x16 dp = TL::mm_row(vt, 32 * kb, gf, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = weight<T>(s[r], a.c2, l2) * (dp[r] - delta);
      if (seen != ~0u) {
        uint32_t m = seen >> (4 * h);
        asm volatile("" : "+v"(m));             // keeps this a branch: seldom taken, 48 instructions
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = (m >> acc_row(0, r)) & 1 ? s[r] : 0.0f;
      }
      TL::mm_col(kt, 32 * kb, s, acc, lane);
    }
    vis = next;
  }
  if (row >= p.R) return;
  if (a.splits > 1) store_cols<float, DB>(a.part + (split * a.part_rows + orow) * DH, acc, a.scale, h);
  else store_cols<T, DB>(static_cast<T*>(a.out) + qrow * a.ld_out + head * DH, acc, a.scale, h);
}

// dk and dv of 128 keys (32 per wavefront, in registers as row operands); the
// rows' q and do pass through LDS.  Vector unit busy 49% of the time, matrix cores 33%, LDS
// 25%, which 1.6 wavefronts per SIMD overlap in part: the same rows and keys, 214 GFLOP,
// 311 us (688 TFLOP/s) and 21 to add four splits' sums.
template <class T, int DH>
__global__ __launch_bounds__(256, (IS_BF<T> && DH <= 64) ? 2 : 1) void dkv_kernel(const Table t, const Args a) {
  using TL = Tile<T, DH>;
  constexpr int DB = TL::DB, RB = TILE_ROWS<T, DH>;
  __shared__ __attribute__((aligned(16))) T lds[4 * RB * DH];
  __shared__ __attribute__((aligned(16))) float st[2][2][RB];      // [buffer][lse log2 e, delta][row]
  T* const qs = lds;
  T* const gs = lds + 2 * RB * DH;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5;
  Prob p;
  if (!problem<true>(t, a, 128, p)) return;
  const int key = p.tile * 128 + wave * 32 + (lane & 31), kc = min(key, p.Lk - 1);
  const int64_t krow = (int64_t)p.k0 + kc;
  const bool seen = !a.mask || a.mask[krow] != 0;
  typename TL::Op kf, vf;
  TL::load_op(kf, static_cast<const T*>(a.k) + krow * a.ld_k + p.hk * DH, h);
  TL::load_op(vf, static_cast<const T*>(a.v) + krow * a.ld_v + p.hk * DH, h);
  TL::scale_op(kf, a.c2);
  const int tiles = (p.R + RB - 1) / RB, split = p.split;
  const int t0 = (int)((int64_t)tiles * split / a.splits), t1 = (int)((int64_t)tiles * (split + 1) / a.splits);
  auto copy = [&](int tile) {
    const int r0 = tile * RB, first = r0 / a.G;            // the tile's first query
    const u32x4 qb = buffer_of(static_cast<const T*>(a.q) + ((int64_t)p.q0 + first) * a.ld_q + p.hk * a.G * DH, BAD - 1);
    const u32x4 gb = buffer_of(static_cast<const T*>(a.d_o) + ((int64_t)p.q0 + first) * a.ld_do + p.hk * a.G * DH, BAD - 1);
    auto off = [&](int r, int64_t ld) {
      const int x = r0 + r, qi = x / a.G;
      return x < p.R ? (uint32_t)(((qi - first) * ld + (x - qi * a.G) * DH) * sizeof(T)) : BAD;
    };
    copy_tile<T, DH, RB, 256>(qb, qs + (tile & 1) * RB * DH, tid, [&](int r) { return off(r, a.ld_q); });
    copy_tile<T, DH, RB, 256>(gb, gs + (tile & 1) * RB * DH, tid, [&](int r) { return off(r, a.ld_do); });
  };
  float2 sv = make_float2(INFINITY, 0.0f);
  auto load_stat = [&](int tile) {
    sv = make_float2(INFINITY, 0.0f);                      // rows past the end: P = 0
    const int x = tile * RB + tid;
    if (tid < RB && x < p.R) {
      const int qi = x / a.G;
      sv = *reinterpret_cast<const float2*>(a.stat + 2 * (((int64_t)p.q0 + qi) * a.heads + p.hk * a.G + x - qi * a.G));
    }
  };
  auto put_stat = [&](int tile) {
    if (tid < RB) {
      st[tile & 1][0][tid] = sv.x;
      st[tile & 1][1][tid] = sv.y;
    }
  };
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) dk[b] = dv[b] = f32x16{};
  if (t0 < t1) {
    copy(t0);
    load_stat(t0);
    put_stat(t0);
  }
  for (int ti = t0; ti < t1; ++ti) {
    wait_counts<0, true>();
    raw_barrier();
    if (ti + 1 < t1) {
      copy(ti + 1);
      load_stat(ti + 1);
    }
    const T* qt = qs + (ti & 1) * RB * DH;
    const T* gt = gs + (ti & 1) * RB * DH;
#pragma unroll
    for (int rb = 0; rb < RB / 32; ++rb) {               // rows past the end have P = 0
      // bf16: the branch keeps the blocks apart (without it the compiler holds both, in 244
      // registers instead of 210: a training step of 375 GFLOP 644 us, with it 631); float32
      // is faster without (275 and 265)
      if (IS_BF<T> && ti * RB + 32 * rb >= p.R) break;
      f32x16 s = TL::mm_row(qt, 32 * rb, kf, lane);
      const f32x16 dp = TL::mm_row(gt, 32 * rb, vf, lane);
      const f32x16 l2 = load_acc(&st[ti & 1][0][32 * rb], h), de = load_acc(&st[ti & 1][1][32 * rb], h);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = weight<T>(s[r], a.c2, l2[r]);
      TL::mm_col(gt, 32 * rb, s, dv, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= dp[r] - de[r];
      TL::mm_col(qt, 32 * rb, s, dk, lane);
    }
    if (ti + 1 < t1) put_stat(ti + 1);
  }
  if (key >= p.Lk) return;
  if (!seen) {                                             // also where such a key holds NaN
#pragma unroll
    for (int b = 0; b < DB; ++b) dk[b] = dv[b] = f32x16{};
  }
  if (a.splits > 1) {
    const int64_t prow = krow * a.kv_heads + p.hk;
    store_cols<float, DB>(a.part + ((2 * split) * a.part_rows + prow) * DH, dk, a.scale, h);
    store_cols<float, DB>(a.part + ((2 * split + 1) * a.part_rows + prow) * DH, dv, 1.0f, h);
  } else {
    store_cols<T, DB>(static_cast<T*>(a.out) + krow * a.ld_out + p.hk * DH, dk, a.scale, h);
    store_cols<T, DB>(static_cast<T*>(a.out2) + krow * a.ld_out2 + p.hk * DH, dv, 1.0f, h);
  }
}

// out[row] = sum of the splits' rows, in order; blockIdx.y picks dk or dv.
template <class T, int DH>
__global__ __launch_bounds__(256) void add_kernel(const float* part, int64_t rows, int splits, int sets, int heads,
                                                  void* out0, int64_t ld0, void* out1, int64_t ld1) {
  constexpr int Q = DH / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * Q) return;
  const int set = blockIdx.y;
  const int64_t r = i / Q, ld = set ? ld1 : ld0;
  const int d = (int)(i % Q) * 4;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < splits; ++s) acc += *reinterpret_cast<const f32x4*>(part + (((int64_t)s * sets + set) * rows + r) * DH + d);
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 y;
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = (T)acc[j];
  *reinterpret_cast<t4*>(static_cast<T*>(set ? out1 : out0) + (r / heads) * ld + (r % heads) * DH + d) = y;
}

// --------------------------------------------------------------------------
// Host side.

struct Plan {
  int64_t nq, nk;                 // rows
  int64_t max_lk, max_r;          // longest key run, most stacked rows of a segment
  bool few;                       // forward: rows of 32 per workgroup, its wavefronts sharing them
  int fwd_splits, dq_splits, dkv_splits;
  size_t o_part, o_ml, o_stat, bytes;
};

wm_status check(const wm_attention* a, Plan* p, bool grad) {
  auto bad = [](const char* m) { return set_error(WM_ERR_INVALID_ARGUMENT, m); };
  if (!a) return bad("attention arguments are NULL");
  if (a->dtype != WM_FP32 && a->dtype != WM_BF16) return bad("dtype must be WM_FP32 or WM_BF16");
  if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads) return bad("heads must be a positive multiple of kv_heads");
  if (a->heads > 1024) return set_error(WM_ERR_UNSUPPORTED, "more than 1024 heads");
  if (a->head_dim != 32 && a->head_dim != 64 && a->head_dim != 128)
    return set_error(WM_ERR_UNSUPPORTED, "head_dim must be 32, 64 or 128");
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale * LOG2E)) return bad("scale must be positive and below 2e38");
  if (a->S < 1 || a->S > WM_MAX_SEGMENTS) return bad("S must be in [1, WM_MAX_SEGMENTS]");
  if (!a->q_off || !a->k_off) return bad("q_off/k_off is NULL");
  if (a->q_off[0] != 0 || a->k_off[0] != 0) return bad("q_off and k_off must start at 0");
  p->max_lk = p->max_r = 0;
  const int G = a->heads / a->kv_heads;
  for (int s = 0; s < a->S; ++s) {
    const int64_t lq = (int64_t)a->q_off[s + 1] - a->q_off[s], lk = (int64_t)a->k_off[s + 1] - a->k_off[s];
    if (lq < 0 || lk < 0) return bad("q_off and k_off must not decrease");
    if (lq * G > INT32_MAX) return set_error(WM_ERR_UNSUPPORTED, "a segment has more than 2^31 rows of one key head");
    p->max_lk = std::max(p->max_lk, lk);
    p->max_r = std::max(p->max_r, lq * G);
  }
  p->nq = a->q_off[a->S];
  p->nk = a->k_off[a->S];
  const int64_t e = a->dtype == WM_BF16 ? 2 : 4;
  if (!rows_ok(a, a->q, a->ld_q, p->nq, a->heads) || !rows_ok(a, a->k, a->ld_k, p->nk, a->kv_heads) ||
      !rows_ok(a, a->v, a->ld_v, p->nk, a->kv_heads))
    return bad("q, k and v need 16-byte aligned rows: pointer, stride at least the row's width, at most 2^22 elements");
  // tiles of the kernels and steps of their loops, over all segments
  const bool bf = a->dtype == WM_BF16;
  const int dh = a->head_dim, wi = dh == 32 ? 0 : dh == 64 ? 1 : 2;
  const bool wide32 = !bf && dh == 128;
  const int few_rows = wide32 ? 64 : 32, few_keys = wide32 ? 64 : 128, tile = wide32 ? 32 : 64;
  int64_t row_tiles = 0, few_tiles = 0, key_tiles = 0;
  double row_steps = 0, few_steps = 0, key_steps = 0;
  for (int s = 0; s < a->S; ++s) {
    const int64_t r = ((int64_t)a->q_off[s + 1] - a->q_off[s]) * G, lk = (int64_t)a->k_off[s + 1] - a->k_off[s];
    row_tiles += cdiv(r, 128);
    few_tiles += cdiv(r, few_rows);
    key_tiles += cdiv(lk, 128);
    row_steps += (double)cdiv(r, 128) * cdiv(lk, tile);
    few_steps += (double)cdiv(r, few_rows) * cdiv(lk, few_keys);
    key_steps += (double)cdiv(lk, 128) * cdiv(r, tile);
  }
  const int64_t most = INT32_MAX / 64 / 8;               // 64: splits
  if (row_tiles * a->kv_heads > most || few_tiles * a->kv_heads > most || key_tiles * a->kv_heads > most)
    return set_error(WM_ERR_UNSUPPORTED, "too many row or key tiles");
  const int64_t rows_all = p->nq * a->heads, kv_all = p->nk * a->kv_heads;
  // workgroups that share a compute unit (registers, LDS), us of a step when they do (rates that the
  // kernels reach: 600 TFLOP/s in bf16, 90 in float32, a step of the few-row form its bytes at 4.5 TB/s; not
  // below 1 us), us to write and read a split's partial sums
  static const int fwd_cu[2][3] = {{3, 2, 2}, {4, 3, 2}}, few_cu[2][3] = {{2, 1, 1}, {4, 2, 1}};
  static const int dq_cu[2][3] = {{2, 2, 1}, {4, 3, 1}}, dkv_cu[2][3] = {{2, 1, 1}, {3, 2, 1}};
  auto step_us = [&](int products, int per_cu) {
    return std::max(1.0, products * 2.0 * 128 * tile * dh * 256 * per_cu / (bf ? 600e6 : 90e6));
  };
  auto part_us = [&](int64_t values) { return 2.0 * values * dh * 4 / 4.5e6; };
  auto avg = [](double steps, int64_t tiles) { return tiles ? steps / tiles : 0.0; };
  p->few = p->max_r <= few_rows;
  if (p->few) {
    const int cu = few_cu[bf][wi];
    p->fwd_splits = splits_for(few_tiles * a->kv_heads, avg(few_steps, few_tiles), cdiv(p->max_lk, few_keys), 2, cu,
                               std::max(1.0, 2.0 * few_keys * dh * e * 256 * cu / 4.5e6), part_us(rows_all));
  } else {
    const int cu = fwd_cu[bf][wi];
    p->fwd_splits = splits_for(row_tiles * a->kv_heads, avg(row_steps, row_tiles), cdiv(p->max_lk, tile), 2, cu, step_us(2, cu), part_us(rows_all));
  }
  p->dq_splits = splits_for(row_tiles * a->kv_heads, avg(row_steps, row_tiles), cdiv(p->max_lk, tile), 2, dq_cu[bf][wi],
                            step_us(3, dq_cu[bf][wi]), part_us(rows_all));
  p->dkv_splits = splits_for(key_tiles * a->kv_heads, avg(key_steps, key_tiles), cdiv(p->max_r, tile), 2, dkv_cu[bf][wi],
                             step_us(4, dkv_cu[bf][wi]), part_us(2 * kv_all));
  size_t at = 0;
  p->o_part = p->o_ml = p->o_stat = 0;
  auto take = [&](size_t n) { const size_t o = at; at = al256(at + n); return o; };
  if (!grad) {
    if (p->fwd_splits > 1) {
      p->o_part = take((size_t)p->fwd_splits * rows_all * a->head_dim * 4);
      p->o_ml = take((size_t)p->fwd_splits * rows_all * 8);
    }
  } else {
    p->o_stat = take((size_t)rows_all * 8);
    size_t part = 0;              // dq's and then dk's and dv's, one after the other on the stream
    if (p->dq_splits > 1) part = (size_t)p->dq_splits * rows_all * a->head_dim * 4;
    if (p->dkv_splits > 1) part = std::max(part, (size_t)p->dkv_splits * 2 * kv_all * a->head_dim * 4);
    if (part) p->o_part = take(part);
  }
  p->bytes = workspace_of(at);
  return WM_OK;
}

Args base_args(const wm_attention* w) {
  Args a = {};
  a.q = w->q; a.k = w->k; a.v = w->v;
  a.ld_q = w->ld_q; a.ld_k = w->ld_k; a.ld_v = w->ld_v;
  a.mask = w->kv_mask;
  a.scale = w->scale;
  a.c2 = w->scale * LOG2E;
  a.heads = w->heads; a.kv_heads = w->kv_heads; a.G = w->heads / w->kv_heads;
  return a;
}

hipError_t forward(const wm_attention* w, const Plan& p, const Args& a, hipStream_t st) {
  return typed(w, [&](auto tv, auto dh) {
    using T = decltype(tv);
    constexpr int DH = decltype(dh)::value;
    constexpr int WK = (!IS_BF<T> && DH == 128) ? 2 : 4;
    const int rows = p.few ? 128 / WK : 128;
    hipError_t e = each_run(w, false, a.splits, [&](int64_t lq, int64_t) { return cdiv(lq * a.G, rows); },
                            [&](const Table& t, int blocks) {
                              const dim3 grid(blocks);
                              if (p.few) hipLaunchKernelGGL((forward_kernel<T, DH, WK>), grid, dim3(256), 0, st, t, a);
                              else hipLaunchKernelGGL((forward_kernel<T, DH, 1>), grid, dim3(256), 0, st, t, a);
                            });
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t n = p.nq * a.heads;
    hipLaunchKernelGGL((join_kernel<T, DH>), dim3((unsigned)cdiv(n * (DH / 4), 256)), dim3(256), 0, st, a, n);
    return hipGetLastError();
  });
}

hipError_t grad_rows(const wm_attention* w, const Plan& p, const Args& a, hipStream_t st) {
  return typed(w, [&](auto tv, auto dh) {
    using T = decltype(tv);
    constexpr int DH = decltype(dh)::value;
    hipError_t e = each_run(w, false, a.splits, [&](int64_t lq, int64_t) { return cdiv(lq * a.G, 128); },
                            [&](const Table& t, int blocks) {
                              hipLaunchKernelGGL((dq_kernel<T, DH>), dim3(blocks), dim3(256), 0, st, t, a);
                            });
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t n = p.nq * a.heads;
    hipLaunchKernelGGL((add_kernel<T, DH>), dim3((unsigned)cdiv(n * (DH / 4), 256), 1), dim3(256), 0, st, a.part, n,
                       a.splits, 1, a.heads, a.out, a.ld_out, nullptr, (int64_t)0);
    return hipGetLastError();
  });
}

hipError_t grad_keys(const wm_attention* w, const Plan& p, const Args& a, hipStream_t st) {
  return typed(w, [&](auto tv, auto dh) {
    using T = decltype(tv);
    constexpr int DH = decltype(dh)::value;
    hipError_t e = each_run(w, true, a.splits, [&](int64_t, int64_t lk) { return cdiv(lk, 128); },
                            [&](const Table& t, int blocks) {
                              hipLaunchKernelGGL((dkv_kernel<T, DH>), dim3(blocks), dim3(256), 0, st, t, a);
                            });
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t n = p.nk * a.kv_heads;
    hipLaunchKernelGGL((add_kernel<T, DH>), dim3((unsigned)cdiv(n * (DH / 4), 256), 2), dim3(256), 0, st, a.part, n,
                       a.splits, 2, a.kv_heads, a.out, a.ld_out, a.out2, a.ld_out2);
    return hipGetLastError();
  });
}

wm_status check_shared(const wm_attention* w, Shared* sh) {
  Plan p;
  const wm_status s = check(w, &p, true);
  if (s != WM_OK) return s;
  sh->nq = p.nq;
  sh->nk = p.nk;
  sh->max_r = p.max_r;
  sh->max_lk = p.max_lk;
  return WM_OK;
}

}  // namespace attend
}  // namespace wm

using namespace wm::attend;

#define WM_AT(CALL)                                                                        \
  do {                                                                                     \
    timing_begin(TK_ATTEND, st);                                                           \
    hipError_t e_ = (CALL);                                                                \
    timing_end(TK_ATTEND, st);                                                             \
    if (e_ != hipSuccess) return set_error(WM_ERR_DEVICE, std::string("kernel launch: ") + hipGetErrorString(e_)); \
  } while (0)

extern "C" {

size_t wm_cross_attention_workspace_bytes(const wm_attention* a, int32_t grad) {
  Plan p;
  return check(a, &p, grad != 0) == WM_OK ? std::max(p.bytes, NO_WORKSPACE) : 0;
}

wm_status wm_cross_attention(const wm_attention* w, void* o, int64_t ld_o, float* lse, void* ws, size_t ws_bytes,
                             void* stream) {
  Plan p;
  const wm_status s = check(w, &p, false);
  if (s != WM_OK) return s;
  if (!rows_ok(w, o, ld_o, p.nq, w->heads)) return set_error(WM_ERR_INVALID_ARGUMENT, "o needs 16-byte aligned rows");
  if (p.bytes && (!ws || (uintptr_t)ws % 256 || ws_bytes < p.bytes))
    return set_error(WM_ERR_INVALID_ARGUMENT, "workspace is NULL, not 256-byte aligned or too small");
  if (p.nq == 0) return clear_error();
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  Args a = base_args(w);
  a.out = o;
  a.ld_out = ld_o;
  a.lse = lse;
  a.splits = p.fwd_splits;
  a.part = reinterpret_cast<float*>(w8 + p.o_part);
  a.part_ml = reinterpret_cast<float*>(w8 + p.o_ml);
  a.part_rows = p.nq * w->heads;
  WM_AT(forward(w, p, a, st));
  return clear_error();
}

wm_status wm_cross_attention_grad(const wm_attention* w, const void* o, int64_t ld_o, const float* lse, const void* d_o,
                                  int64_t ld_do, void* dq, int64_t ld_dq, void* dk, int64_t ld_dk, void* dv, int64_t ld_dv,
                                  void* ws, size_t ws_bytes, void* stream) {
  Plan p;
  const wm_status s = check(w, &p, true);
  if (s != WM_OK) return s;
  if (!rows_ok(w, o, ld_o, p.nq, w->heads) || !rows_ok(w, d_o, ld_do, p.nq, w->heads) ||
      !rows_ok(w, dq, ld_dq, p.nq, w->heads) || !rows_ok(w, dk, ld_dk, p.nk, w->kv_heads) ||
      !rows_ok(w, dv, ld_dv, p.nk, w->kv_heads))
    return set_error(WM_ERR_INVALID_ARGUMENT, "o, d_o, dq, dk and dv need 16-byte aligned rows");
  if (p.nq > 0 && !lse) return set_error(WM_ERR_INVALID_ARGUMENT, "lse is NULL");
  if (p.bytes && (!ws || (uintptr_t)ws % 256 || ws_bytes < p.bytes))
    return set_error(WM_ERR_INVALID_ARGUMENT, "workspace is NULL, not 256-byte aligned or too small");
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  Args a = base_args(w);
  a.o = o; a.ld_o = ld_o;
  a.d_o = d_o; a.ld_do = ld_do;
  a.lse = const_cast<float*>(lse);
  a.stat = reinterpret_cast<float*>(w8 + p.o_stat);
  a.part = reinterpret_cast<float*>(w8 + p.o_part);
  if (p.nq > 0) {
    a.out = dq; a.ld_out = ld_dq;
    a.splits = p.dq_splits;
    a.part_rows = p.nq * w->heads;
    WM_AT(grad_rows(w, p, a, st));
  }
  if (p.nk > 0) {
    a.out = dk; a.ld_out = ld_dk;
    a.out2 = dv; a.ld_out2 = ld_dv;
    a.splits = p.dkv_splits;
    a.part_rows = p.nk * w->kv_heads;
    WM_AT(grad_keys(w, p, a, st));
  }
  return clear_error();
}

}  // extern "C"
