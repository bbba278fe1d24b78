// Rotation of packed rows by position, and appending keys and values to a paged cache with the rotation
// applied on the way.  Both move every element once: what bounds them is memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "wm_device.h"
#include "wm_internal.h"

using namespace wm;

namespace wm {
namespace cache {

constexpr int MAX_DIM = 512;

struct Args {
  const int32_t *off, *first;
  const float* freq;
  int32_t* status;
  int64_t rows;
  int B, T_max;
  const void *q, *k, *v;                    // rotate: q alone
  int64_t ld_q, ld_k, ld_v, ld_out;
  void* out;                                // of q
  int heads, kv_heads, dim, rot, interleaved, inverse;
  // append
  void *k_cache, *v_cache;
  const int32_t *pages, *lens;
  int max_pages, n_pages, lps;
};

// How the pairs of a head lie in 16-byte units: HALVES: 8 (float32: 4) pairs are a unit of the first half and one
// of the second; NEIGHBOURS: within units; SINGLE: a rotation that does not divide into units, pair by pair.
enum Form { HALVES, NEIGHBOURS, SINGLE };

// sin and cos of position x freq.  In turns: freq / (2 pi) in two doubles (107 bits), its product with the position exact but for the
// lower one's, each part taken modulo 1, which is exact: for |freq| up to 2^32 at every position the turns are right to 2^-43.  (One
// product in 64 bits left an error of 2^-53 of the product, angles wrong by 4.9e-7 at 2^31 radians and by 0.2 at 2^51.)  Quarter turns
// leave an argument of at most pi / 4, where the Taylor sums of degree 11 and 12 are right to float32's rounding.
__device__ __forceinline__ float2 sincos_of(int64_t position, float freq) {
#pragma clang fp contract(off)              // p's rounding is the one that `rest` takes up
  constexpr double TURN = 0x1.45f306dc9c883p-3, TURN_REST = -0x1.6b01ec5417056p-57;        // 1 / (2 pi)
  const double at = (double)position, f = (double)freq;
  const double upper = f * TURN, lower = fma(f, TURN, -upper) + f * TURN_REST;
  const double p = at * upper, rest = fma(at, upper, -p);
  const double turns = (p - __builtin_rint(p)) + ((rest - __builtin_rint(rest)) + at * lower);
  const double quarters = turns * 4.0, n = __builtin_rint(quarters);
  const float x = (float)(quarters - n) * 1.57079632679489662f;
  const int q = (int)((long long)n & 3);
  const float x2 = x * x;
  float s = fmaf(-2.50521084e-8f, x2, 2.75573192e-6f);
  s = fmaf(s, x2, -1.98412698e-4f);
  s = fmaf(s, x2, 8.33333333e-3f);
  s = fmaf(s, x2, -1.66666667e-1f);
  s = fmaf(s * x2, x, x);
  float c = fmaf(2.08767570e-9f, x2, -2.75573192e-7f);
  c = fmaf(c, x2, 2.48015873e-5f);
  c = fmaf(c, x2, -1.38888889e-3f);
  c = fmaf(c, x2, 4.16666667e-2f);
  c = fmaf(c, x2, -0.5f);
  c = fmaf(c, x2, 1.0f);
  const float a = q & 1 ? c : s, b = q & 1 ? s : c;
  return make_float2(q & 2 ? -a : a, (q == 1 || q == 2) ? -b : b);
}

// What the row of a block needs: its sequence's slot and position.
struct Row {
  int64_t at;                               // element of key head 0 in the caches
  int write, real;                          // the slot exists; the row belongs to a sequence
};

// RB rows per workgroup: their sequences, slots and angles first (sin and cos of a row's pairs are formed
// once for all its heads), then all their units, one per thread at a time.  Memory bounds it: 45884 rows of 12 heads of 64, 16 bits,
// 27 us (5.1 TB/s), an append of 17892 rows of 48 heads of 128 88 us (5.0 TB/s).
template <class T, Form FORM, bool APPEND, int RB>
__global__ __launch_bounds__(256) void rotate_kernel(const Args a) {
  constexpr int V = 16 / (int)sizeof(T);
  using Unit = T __attribute__((ext_vector_type(V)));
  __shared__ Row info[RB];
  __shared__ int64_t position[RB];
  __shared__ float2 turn[RB][MAX_DIM / 2];          // (sin, cos)
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (a.status) {
    for (int64_t s = (int64_t)blockIdx.x * 256 + tid; s <= a.B; s += (int64_t)gridDim.x * 256) {
      const int64_t x = a.off[s];
      if ((s == 0 && x != 0) || (s == a.B && x != a.rows)) atomicOr(a.status, ERRBIT_ROWS);
      if (s < a.B) {
        const int64_t n = a.off[s + 1] - x;
        if (n < 0 || n > a.T_max) atomicOr(a.status, ERRBIT_LEN);
        if (APPEND && (a.lens[s] < n || a.lens[s] > (int64_t)a.max_pages << a.lps)) atomicOr(a.status, ERRBIT_KEYS);
      }
    }
  }
  const int64_t row0 = (int64_t)blockIdx.x * RB;
  for (int r = wave; r < RB; r += 4) {
    const int64_t row = row0 + r;
    if (row >= a.rows) continue;
    int lo = 0, hi = a.B - 1;                        // the last sequence that starts at the row or before, by 64 lanes
    while (lo < hi) {
      const int step = (hi - lo + 63) >> 6, at = lo + step * (lane + 1);
      const int n = __popcll(__ballot(at <= hi && a.off[min(at, hi)] <= row));
      lo += step * n;
      hi = min(hi, lo + step - 1);
    }
    const int64_t x = a.off[lo], y = a.off[lo + 1], i = row - x;
    Row w = {0, 0, x >= 0 && i >= 0 && row < y};
    int64_t pos = (a.first ? a.first[lo] : 0) + i;
    if constexpr (APPEND) {
      const int64_t slot = a.lens[lo] - (y - x) + i;
      pos += slot - i;
      if (w.real && slot >= 0 && slot < (int64_t)a.max_pages << a.lps) {
        const int page = a.pages[(int64_t)lo * a.max_pages + (slot >> a.lps)];
        w.write = page >= 0 && page < a.n_pages;
        if (!w.write && a.status && lane == 0) atomicOr(a.status, ERRBIT_PAGE);
        w.at = ((((int64_t)(w.write ? page : 0) * a.kv_heads) << a.lps) + (slot & ((1 << a.lps) - 1))) * a.dim;
      }
    }
    if (lane == 0) {
      info[r] = w;
      position[r] = pos;
    }
  }
  __syncthreads();
  const int rows = (int)min((int64_t)RB, a.rows - row0), pairs = a.freq ? a.rot / 2 : 0;
  for (int i = tid; i < rows * pairs; i += 256) {
    const int r = i / pairs, p = i - r * pairs;
    float2 sc = sincos_of(position[r], a.freq[p]);
    if (a.inverse) sc.x = -sc.x;
    turn[r][p] = sc;
  }
  __syncthreads();
  // a head's items: pairs of units (HALVES) or units (NEIGHBOURS) or pairs (SINGLE), then what is not turned
  const int unit = FORM == SINGLE ? 1 : V;
  const int turned = FORM == SINGLE ? pairs : FORM == HALVES ? pairs / V : 2 * pairs / V;
  const int per_head = turned + (a.dim - 2 * pairs) / unit, plain = a.dim / V;
  const int nq = a.heads * per_head, nk = APPEND ? a.kv_heads * per_head : 0, nv = APPEND ? a.kv_heads * plain : 0;
  const int items = nq + nk + nv;
  for (int i = tid; i < rows * items; i += 256) {
    const int r = i / items;
    int j = i - r * items;
    const int64_t row = row0 + r;
    const Row w = info[r];
    if (!w.real) continue;
    if (APPEND && j >= nq + nk) {
      j -= nq + nk;
      const int head = j / plain, u = j - head * plain;
      if (w.write)
        *reinterpret_cast<Unit*>(static_cast<T*>(a.v_cache) + w.at + ((int64_t)head << a.lps) * a.dim + u * V) =
            *reinterpret_cast<const Unit*>(static_cast<const T*>(a.v) + row * a.ld_v + head * a.dim + u * V);
      continue;
    }
    const bool key = APPEND && j >= nq;
    if (key) j -= nq;
    const int head = j / per_head, u = j - head * per_head;
    if (key && !w.write) continue;
    const T* src = key ? static_cast<const T*>(a.k) + row * a.ld_k + head * a.dim : static_cast<const T*>(a.q) + row * a.ld_q + head * a.dim;
    T* dst = key ? static_cast<T*>(a.k_cache) + w.at + ((int64_t)head << a.lps) * a.dim : static_cast<T*>(a.out) + row * a.ld_out + head * a.dim;
    if (u >= turned) {
      const int f = 2 * pairs + (u - turned) * unit;
      if constexpr (FORM == SINGLE) dst[f] = src[f];
      else *reinterpret_cast<Unit*>(dst + f) = *reinterpret_cast<const Unit*>(src + f);
    } else if constexpr (FORM == HALVES) {
      const Unit x = *reinterpret_cast<const Unit*>(src + u * V), y = *reinterpret_cast<const Unit*>(src + pairs + u * V);
      Unit xo, yo;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 sc = turn[r][u * V + e];
        const float p = (float)x[e], s = (float)y[e];
        xo[e] = (T)fmaf(p, sc.y, -(s * sc.x));
        yo[e] = (T)fmaf(p, sc.x, s * sc.y);
      }
      *reinterpret_cast<Unit*>(dst + u * V) = xo;
      *reinterpret_cast<Unit*>(dst + pairs + u * V) = yo;
    } else if constexpr (FORM == NEIGHBOURS) {
      const Unit x = *reinterpret_cast<const Unit*>(src + u * V);
      Unit y;
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float2 sc = turn[r][(u * V + e) / 2];
        const float p = (float)x[e], s = (float)x[e + 1];
        y[e] = (T)fmaf(p, sc.y, -(s * sc.x));
        y[e + 1] = (T)fmaf(p, sc.x, s * sc.y);
      }
      *reinterpret_cast<Unit*>(dst + u * V) = y;
    } else {
      const int f = a.interleaved ? 2 * u : u, g = a.interleaved ? 2 * u + 1 : u + pairs;
      const float2 sc = turn[r][u];
      const float p = (float)src[f], s = (float)src[g];
      dst[f] = (T)fmaf(p, sc.y, -(s * sc.x));
      dst[g] = (T)fmaf(p, sc.x, s * sc.y);
    }
  }
}

// --------------------------------------------------------------------------
// Host side.

wm_status bad(const char* m) { return set_error(WM_ERR_INVALID_ARGUMENT, m); }

bool rows_ok(int32_t dtype, const void* p, int64_t ld, int64_t rows, int64_t width) {
  const int64_t e = dtype == WM_BF16 ? 2 : 4;
  return rows == 0 || (p && (uintptr_t)p % 16 == 0 && ld >= width && ld * e % 16 == 0 && ld <= (1 << 22));
}

// Four rows per workgroup, so that a thread has several items, or one where that leaves compute units without work (rotation in bf16,
// four and one: 4095 rows of 12 heads of 64 4.8 and 6.6 us, 2048 4.0 and 4.3, 64 rows of 64 heads of 128 6.5 and 3.9, 2048 13.5 and 12.6).
constexpr int64_t MANY_ROWS = 2048;
constexpr int64_t MOST_ROWS = 4 * (((int64_t)1 << 32) / 256 - 1);          // a launch has fewer than 2^32 threads

wm_status check_rows(int32_t B, int32_t T_max, int64_t rows, const int32_t* off) {
  if (rows < 0 || rows > INT32_MAX) return bad("rows must be in [0, 2^31)");
  if (rows > MOST_ROWS) return set_error(WM_ERR_UNSUPPORTED, "more than 2^26 - 4 rows");
  if (B < 0 || T_max < 0) return bad("B and T_max must not be negative");
  if (rows > 0 && (B < 1 || T_max < 1)) return bad("rows need sequences: B and T_max at least 1");
  if (B > 0 && !off) return bad("off is NULL");
  return WM_OK;
}

template <bool APPEND>
hipError_t launch(const Args& a, int32_t dtype, hipStream_t st) {
  auto go = [&](auto tv) {
    using T = decltype(tv);
    constexpr int V = 16 / (int)sizeof(T);
    const int rot = a.freq ? a.rot : 0;
    const Form form = a.interleaved || rot == 0 ? (rot % V ? SINGLE : NEIGHBOURS) : (rot / 2 % V ? SINGLE : HALVES);
    auto rows = [&](auto f) {
      constexpr Form F = decltype(f)::value;
      if (a.rows >= MANY_ROWS) hipLaunchKernelGGL((rotate_kernel<T, F, APPEND, 4>), dim3((unsigned)((a.rows + 3) / 4)), dim3(256), 0, st, a);
      else hipLaunchKernelGGL((rotate_kernel<T, F, APPEND, 1>), dim3((unsigned)a.rows), dim3(256), 0, st, a);
    };
    if (form == HALVES) rows(std::integral_constant<Form, HALVES>{});
    else if (form == NEIGHBOURS) rows(std::integral_constant<Form, NEIGHBOURS>{});
    else rows(std::integral_constant<Form, SINGLE>{});
  };
  if (dtype == WM_BF16) go(__bf16{});
  else go(float{});
  return hipGetLastError();
}

}  // namespace cache

wm_status check_cache(const wm_cache* c) {
  using cache::bad;
  if (c->dtype != WM_FP32 && c->dtype != WM_BF16) return bad("dtype must be WM_FP32 or WM_BF16");
  if (c->kv_heads < 1 || c->kv_heads > 1024) return bad("kv_heads must be in [1, 1024]");
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return set_error(WM_ERR_UNSUPPORTED, "head_dim must be 32, 64 or 128");
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128 && c->page != 256)
    return set_error(WM_ERR_UNSUPPORTED, "a page must have 16, 32, 64, 128 or 256 slots");
  if (c->n_pages < 0 || c->B < 0 || c->max_pages < 0) return bad("n_pages, B and max_pages must not be negative");
  if ((int64_t)c->max_pages * c->page > INT32_MAX) return set_error(WM_ERR_UNSUPPORTED, "a page table covers 2^31 slots or more");
  if (c->n_pages > 0 && (!c->k || !c->v || (uintptr_t)c->k % 16 || (uintptr_t)c->v % 16)) return bad("k and v of the cache must be 16-byte aligned");
  if (c->B > 0 && (!c->lens || (c->max_pages > 0 && !c->pages))) return bad("pages or lens is NULL");
  return WM_OK;
}

}  // namespace wm

using namespace wm::cache;

#define WM_CH(K, CALL)                                                                     \
  do {                                                                                     \
    timing_begin(K, st);                                                                   \
    hipError_t e_ = (CALL);                                                                \
    timing_end(K, st);                                                                     \
    if (e_ != hipSuccess) return set_error(WM_ERR_DEVICE, std::string("kernel launch: ") + hipGetErrorString(e_)); \
  } while (0)

extern "C" {

wm_status wm_rotate(const wm_rotation* x, void* y, int64_t ld_y, void* stream) {
  if (!x) return bad("rotation arguments are NULL");
  if (x->dtype != WM_FP32 && x->dtype != WM_BF16) return bad("dtype must be WM_FP32 or WM_BF16");
  if (x->heads < 1 || x->heads > 1024) return bad("heads must be in [1, 1024]");
  if (x->head_dim < 8 || x->head_dim > MAX_DIM || x->head_dim % 8) return set_error(WM_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 up to 512");
  if (x->rot < 2 || x->rot > x->head_dim || x->rot % 2) return bad("rot must be even, in [2, head_dim]");
  if (!x->freq) return bad("freq is NULL");
  const wm_status s = check_rows(x->B, x->T_max, x->rows, x->off);
  if (s != WM_OK) return s;
  const int64_t width = (int64_t)x->heads * x->head_dim;
  if (!rows_ok(x->dtype, x->x, x->ld_x, x->rows, width) || !rows_ok(x->dtype, y, ld_y, x->rows, width))
    return bad("x and y need 16-byte aligned rows: pointer, stride at least the row's width, at most 2^22 elements");
  if (x->rows > 0 && x->x == y && x->ld_x != ld_y) return bad("y may be x with the same row stride only");
  if (x->rows == 0) return clear_error();
  hipStream_t st = static_cast<hipStream_t>(stream);
  Args a = {};
  a.off = x->off; a.first = x->first; a.freq = x->freq; a.status = x->status;
  a.rows = x->rows; a.B = x->B; a.T_max = x->T_max;
  a.q = x->x; a.ld_q = x->ld_x; a.out = y; a.ld_out = ld_y;
  a.heads = x->heads; a.dim = x->head_dim; a.rot = x->rot; a.interleaved = x->interleaved != 0; a.inverse = x->inverse != 0;
  WM_CH(TK_ROTATE, launch<false>(a, x->dtype, st));
  return clear_error();
}

wm_status wm_cache_append(const wm_append* x, void* q_out, int64_t ld_q_out, void* stream) {
  if (!x) return bad("append arguments are NULL");
  wm_status s = check_cache(&x->cache);
  if (s != WM_OK) return s;
  const wm_cache& c = x->cache;
  if (x->freq && (x->rot < 2 || x->rot > c.head_dim || x->rot % 2)) return bad("rot must be even, in [2, head_dim]");
  if (x->heads < 0 || x->heads > 1024 || (x->q != nullptr) != (x->heads > 0)) return bad("heads must be in [1, 1024] with q, 0 without");
  s = check_rows(c.B, x->T_max, x->rows, x->off);
  if (s != WM_OK) return s;
  const int64_t qw = (int64_t)x->heads * c.head_dim, kw = (int64_t)c.kv_heads * c.head_dim;
  if (!rows_ok(c.dtype, x->k, x->ld_k, x->rows, kw) || !rows_ok(c.dtype, x->v, x->ld_v, x->rows, kw))
    return bad("k and v need 16-byte aligned rows: pointer, stride at least the row's width, at most 2^22 elements");
  if (x->q && (!rows_ok(c.dtype, x->q, x->ld_q, x->rows, qw) || !rows_ok(c.dtype, q_out, ld_q_out, x->rows, qw)))
    return bad("q and q_out need 16-byte aligned rows: pointer, stride at least the row's width, at most 2^22 elements");
  if (x->rows > 0 && x->q && x->q == q_out && x->ld_q != ld_q_out) return bad("q_out may be q with the same row stride only");
  if (x->rows == 0) return clear_error();
  hipStream_t st = static_cast<hipStream_t>(stream);
  Args a = {};
  a.off = x->off; a.first = x->first; a.freq = x->freq; a.status = x->status;
  a.rows = x->rows; a.B = c.B; a.T_max = x->T_max;
  a.q = x->q; a.ld_q = x->ld_q; a.out = q_out; a.ld_out = ld_q_out;
  a.k = x->k; a.ld_k = x->ld_k; a.v = x->v; a.ld_v = x->ld_v;
  a.heads = x->heads; a.kv_heads = c.kv_heads; a.dim = c.head_dim; a.rot = x->rot; a.interleaved = x->interleaved != 0;
  a.k_cache = c.k; a.v_cache = c.v; a.pages = c.pages; a.lens = c.lens;
  a.max_pages = c.max_pages; a.n_pages = c.n_pages; a.lps = page_bits(c.page);
  WM_CH(TK_APPEND, launch<true>(a, c.dtype, st));
  return clear_error();
}

}  // extern "C"
