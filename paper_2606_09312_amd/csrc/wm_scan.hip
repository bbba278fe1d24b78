// Sequence operators over packed ragged rows: a short causal convolution and a
// selective state-space scan, forward, gradients and single steps.
//
// Sequence s has rows [off[s], off[s+1]) (device offsets; a length past T_max
// or offsets outside the rows set the error word and are clamped; offsets that
// leave rows out at either end set it too).  Every sum
// over rows, sequences or channels is in a fixed order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <type_traits>
#include <utility>

#include "wm_device.h"
#include "wm_internal.h"

using namespace wm;

namespace wm {
namespace scan {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <class T>
constexpr bool IS_BF = std::is_same<T, __bf16>::value;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_of(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float sigmoid(float x) { return rcp_of(1.0f + exp2_of(-x * LOG2E)); }

// log(1 + e) for 0 <= e <= 1 as e times a polynomial of degree 9 (Lawson-weighted least
// squares of log(1 + e) / e in float64; with its coefficients in float32 at most 3.4e-8
// of itself off, evaluated in float32 1.6e-7 at most and 2.4e-8 on average, also where e
// is small, which log2(1 + e) would lose).
__device__ __forceinline__ float log1p_unit(float e) {
  float p = fmaf(-0.0032440212089568377f, e, 0.01985144428908825f);
  p = fmaf(p, e, -0.056959498673677444f);
  p = fmaf(p, e, 0.10603651404380798f);
  p = fmaf(p, e, -0.15305590629577637f);
  p = fmaf(p, e, 0.1967593878507614f);
  p = fmaf(p, e, -0.24954134225845337f);
  p = fmaf(p, e, 0.3332996368408203f);
  p = fmaf(p, e, -0.4999990165233612f);
  p = fmaf(p, e, 1.0f);
  return p * e;
}
// softplus(x) = max(x, 0) + log(1 + exp(-|x|))
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.0f) + log1p_unit(exp2_of(-fabsf(x) * LOG2E)); }

// Rows of a sequence, clamped to what exists (`report`: what does not fit sets the error word).
struct Span {
  int64_t r0;
  int len;
};
template <class Args>
__device__ __forceinline__ Span span_of(const Args& g, int s, bool report) {
  // constant while a kernel runs: scalar loads where s is uniform, which no vector load waits for
  const __attribute__((address_space(4))) int32_t* o = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)g.off;
  const int64_t a = o[s], b = o[s + 1];
  const int64_t lo = a < 0 ? 0 : a > g.rows ? g.rows : a, hi = b < lo ? lo : b > g.rows ? g.rows : b;
  const int64_t n = hi - lo > g.T_max ? g.T_max : hi - lo;
  if (report && g.status) {
    if (lo != a || n != b - a) atomicOr(g.status, ERRBIT_LEN);
    if ((s == 0 && a != 0) || (s == g.B - 1 && b != g.rows)) atomicOr(g.status, ERRBIT_ROWS);
  }
  return {lo, (int)n};
}

template <class T, int V>
using Vec = T __attribute__((ext_vector_type(V)));

// V neighbouring values as float (V = 1: no alignment needed)
template <class T, int V>
__device__ __forceinline__ void load_vec(float (&x)[V], const T* p) {
  if constexpr (V == 1) {
    x[0] = (float)*p;
  } else {
    const Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)v[i];
  }
}
template <class T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&x)[V]) {
  if constexpr (V == 1) {
    *p = (T)x[0];
  } else {
    Vec<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)x[i];
    *reinterpret_cast<Vec<T, V>*>(p) = v;
  }
}

// --------------------------------------------------------------------------
// Convolution.  A lane takes V neighbouring channels and a run of RUN rows of a
// sequence, the taps' window in registers; the rows of SUB steps are loaded together, one
// block ahead (bytes bound it: what counts is loads in flight).  A wavefront takes 2^lp
// lanes' channels of 64 >> lp runs, so that narrow rows fill it too.  8192 sequences of
// up to 64 rows, 512 channels, bf16: 100 us, 4.0 TB/s (123 us a row at a time).
constexpr int RUN = 16, SUB = 8;

struct ConvArgs {
  const int32_t* off;
  const void *x, *state, *dy, *d_state_out;
  void *y, *state_out, *dx, *d_state;
  const float *w, *b;
  float* part;              // [groups][W + 1][D]
  int32_t* status;
  int64_t ld_x, ld_y, ld_dy, ld_dx, rows;
  int B, T_max, D, runs, silu, groups, lp;
};

// the input `t` of a sequence: before its start the carried state (zero without one)
template <class T, int V, int W>
__device__ __forceinline__ void conv_in(float (&x)[V], const ConvArgs& a, const Span& sp, int s, int t, int c) {
  if (t >= 0) {
    load_vec<T, V>(x, static_cast<const T*>(a.x) + (sp.r0 + t) * a.ld_x + c);
  } else if (a.state) {
    load_vec<T, V>(x, static_cast<const T*>(a.state) + ((int64_t)s * (W - 1) + (W - 1 + t)) * a.D + c);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.0f;
  }
}

template <int V, int W>
struct Taps {
  float w[W][V], b[V];
  __device__ __forceinline__ void load(const ConvArgs& a, int c) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][i] = a.w[(size_t)(c + i) * W + j];
      b[i] = a.b ? a.b[c + i] : 0.0f;
    }
  }
};

// This lane's slot (a run or a group of runs) of `slots` and its first channel; false past the end.
template <int V>
__device__ __forceinline__ bool conv_slot(const ConvArgs& a, uint32_t slots, uint32_t& slot, int& c) {
  const uint32_t CG = a.D / V, blocks = (CG + (1u << a.lp) - 1) >> a.lp;
  const uint32_t wave = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, row = wave / blocks;
  slot = row * (64u >> a.lp) + (lane >> a.lp);
  const uint32_t cg = ((wave - row * blocks) << a.lp) + (lane & ((1u << a.lp) - 1));
  c = (int)cg * V;
  return slot < slots && cg < CG;
}
template <class T, int V>
using Raw = std::conditional_t<V == 1, T, Vec<T, V == 1 ? 2 : V>>;
template <class T, int V>
__device__ __forceinline__ float elem(const Raw<T, V>& r, int i) {
  if constexpr (V == 1) return (float)r;
  else return (float)r[i];
}
// rows first .. first + SUB - 1 of a matrix, past `last` that one again
template <class T, int V>
__device__ __forceinline__ void load_rows(Raw<T, V> (&x)[SUB], const T* p, int64_t ld, int first, int last) {
#pragma unroll
  for (int i = 0; i < SUB; ++i) x[i] = *reinterpret_cast<const Raw<T, V>*>(p + min(first + i, last) * ld);
}

template <class T, int V, int W>
__global__ __launch_bounds__(256) void conv_kernel(const ConvArgs a) {
  uint32_t item;
  int c;
  if (!conv_slot<V>(a, (uint32_t)a.B * a.runs, item, c)) return;
  const int s = item / (uint32_t)a.runs, run = item - s * a.runs;
  const Span sp = span_of(a, s, c == 0 && run == 0);
  const int t0 = run * RUN, t1 = min(t0 + RUN, sp.len);
  if (t0 < t1) {
    const T* xp = static_cast<const T*>(a.x) + sp.r0 * a.ld_x + c;
    T* yp = static_cast<T*>(a.y) + sp.r0 * a.ld_y + c;
    Raw<T, V> next[SUB];
    load_rows<T, V>(next, xp, a.ld_x, t0, t1 - 1);
    float win[W][V];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) conv_in<T, V, W>(win[j], a, sp, s, t0 - (W - 1) + j, c);
    Taps<V, W> k;
    k.load(a, c);
#pragma unroll
    for (int tb = 0; tb < RUN; tb += SUB) {
      if (t0 + tb >= t1) break;
      Raw<T, V> x[SUB];
#pragma unroll
      for (int i = 0; i < SUB; ++i) x[i] = next[i];
      if (tb + SUB < RUN) load_rows<T, V>(next, xp, a.ld_x, t0 + tb + SUB, t1 - 1);
#pragma unroll
      for (int i = 0; i < SUB; ++i) {
        const int t = t0 + tb + i;
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          win[W - 1][e] = elem<T, V>(x[i], e);
          float v = k.b[e];
#pragma unroll
          for (int j = 0; j < W; ++j) v = fmaf(k.w[j][e], win[j][e], v);
          y[e] = a.silu ? v * sigmoid(v) : v;
        }
        if (t < t1) store_vec<T, V>(yp + t * a.ld_y, y);
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
          for (int e = 0; e < V; ++e) win[j][e] = win[j + 1][e];
      }
    }
  }
  if (a.state_out && run == 0) {          // may be the state itself: this thread alone reads and writes its channels
    float last[W - 1][V];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) conv_in<T, V, W>(last[j], a, sp, s, sp.len - (W - 1) + j, c);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) store_vec<T, V>(static_cast<T*>(a.state_out) + ((int64_t)s * (W - 1) + j) * a.D + c, last[j]);
  }
}

// dx, dstate and partial sums of dw and db.  da_t = dy_t act'(a_t) is formed again from
// the inputs; dx_t = sum_j w_j da_{t + W - 1 - j}.  A lane owns V channels and the runs
// group, group + groups, ..; each row's share of dw is counted by the run that holds it.
template <class T, int V, int W>
__global__ __launch_bounds__(256) void conv_grad_kernel(const ConvArgs a) {
  uint32_t group;
  int c;
  if (!conv_slot<V>(a, a.groups, group, c)) return;
  Taps<V, W> k;
  k.load(a, c);
  float dw[W][V] = {}, db[V] = {};
  // dL/da of a row with inputs x[0 .. W - 1] and output gradient g
  auto grad = [&](const float (&x)[W][V], int e, float g) {
    float v = k.b[e];
#pragma unroll
    for (int j = 0; j < W; ++j) v = fmaf(k.w[j][e], x[j][e], v);
    if (!a.silu) return g;
    const float sg = sigmoid(v);
    return g * sg * fmaf(v, 1.0f - sg, 1.0f);
  };
  for (uint32_t item = group; item < (uint32_t)a.B * a.runs; item += a.groups) {
    const int s = item / (uint32_t)a.runs, run = item - s * a.runs;
    const Span sp = span_of(a, s, c == 0 && run == 0);
    const int t0 = run * RUN, t1 = min(t0 + RUN, sp.len);
    // the gradient of the carried-out state reaches the last W - 1 inputs (and, in a
    // sequence shorter than that, the carried-in state)
    auto from_state = [&](int t, float (&g)[V]) {
      const int j = t - (sp.len - (W - 1));
      if (a.d_state_out && j >= 0) {
        float x[V];
        load_vec<T, V>(x, static_cast<const T*>(a.d_state_out) + ((int64_t)s * (W - 1) + j) * a.D + c);
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] += x[i];
      }
    };
    if (t0 < t1) {
      const T* xp = static_cast<const T*>(a.x) + sp.r0 * a.ld_x + c;
      const T* gp = static_cast<const T*>(a.dy) + sp.r0 * a.ld_dy + c;
      T* dp = static_cast<T*>(a.dx) + sp.r0 * a.ld_dx + c;
      // rows t0 .. t1 - 1 and the W - 1 after them; dx of row t - (W - 1) is complete at row t
      const int end = t1 + W - 1;
      Raw<T, V> xn[SUB], gn[SUB];
      load_rows<T, V>(xn, xp, a.ld_x, t0, sp.len - 1);
      load_rows<T, V>(gn, gp, a.ld_dy, t0, sp.len - 1);
      float win[W][V], da[W][V] = {};       // da[j]: of row t - (W - 1) + j
#pragma unroll
      for (int j = 0; j < W - 1; ++j) conv_in<T, V, W>(win[j], a, sp, s, t0 - (W - 1) + j, c);
      for (int tb = t0; tb < end; tb += SUB) {
        Raw<T, V> x[SUB], g[SUB];
#pragma unroll
        for (int i = 0; i < SUB; ++i) {
          x[i] = xn[i];
          g[i] = gn[i];
        }
        if (tb + SUB < end) {
          load_rows<T, V>(xn, xp, a.ld_x, tb + SUB, sp.len - 1);
          load_rows<T, V>(gn, gp, a.ld_dy, tb + SUB, sp.len - 1);
        }
#pragma unroll
        for (int i = 0; i < SUB; ++i) {
          const int t = tb + i;
          if (t >= end) break;
#pragma unroll
          for (int e = 0; e < V; ++e) win[W - 1][e] = elem<T, V>(x[i], e);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float d = t < sp.len ? grad(win, e, elem<T, V>(g[i], e)) : 0.0f, own = t < t1 ? d : 0.0f;
            da[W - 1][e] = d;
            db[e] += own;
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][e] = fmaf(own, win[j][e], dw[j][e]);
          }
          const int u = t - (W - 1);        // u's last reader of da is row t
          if (u >= t0) {
            float d[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
              d[e] = 0.0f;
#pragma unroll
              for (int j = 0; j < W; ++j) d[e] = fmaf(k.w[W - 1 - j][e], da[j][e], d[e]);
            }
            from_state(u, d);
            store_vec<T, V>(dp + u * a.ld_dx, d);
          }
#pragma unroll
          for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
              win[j][e] = win[j + 1][e];
              da[j][e] = da[j + 1][e];
            }
        }
      }
    }
    if (a.d_state && run == 0) {
      // state slot m is the input at -(W - 1) + m: rows 0 .. m read it
      float first[W - 1][V];                // da of rows 0 .. W - 2
#pragma unroll
      for (int t = 0; t < W - 1; ++t) {
#pragma unroll
        for (int i = 0; i < V; ++i) first[t][i] = 0.0f;
        if (t < sp.len) {
          float x[W][V], g[V];
#pragma unroll
          for (int j = 0; j < W; ++j) conv_in<T, V, W>(x[j], a, sp, s, t - (W - 1) + j, c);
          load_vec<T, V>(g, static_cast<const T*>(a.dy) + (sp.r0 + t) * a.ld_dy + c);
#pragma unroll
          for (int i = 0; i < V; ++i) first[t][i] = grad(x, i, g[i]);
        }
      }
#pragma unroll
      for (int m = 0; m < W - 1; ++m) {
        float d[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float v = 0.0f;
#pragma unroll
          for (int t = 0; t <= m; ++t) v = fmaf(k.w[m - t][i], first[t][i], v);
          d[i] = v;
        }
        from_state(m - (W - 1), d);
        store_vec<T, V>(static_cast<T*>(a.d_state) + ((int64_t)s * (W - 1) + m) * a.D + c, d);
      }
    }
  }
  float* out = a.part + (int64_t)group * (W + 1) * a.D + c;
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) out[(int64_t)j * a.D + i] = dw[j][i];
#pragma unroll
  for (int i = 0; i < V; ++i) out[(int64_t)W * a.D + i] = db[i];
}

// Sum over `groups` partial rows of n values each, in a fixed order: a workgroup
// takes 16 values, 16 threads each take every sixteenth group, then their sums in
// order.  put(i, sum) stores value i.
template <class Put>
__device__ __forceinline__ void sum_groups(const float* part, int groups, int64_t n, Put put) {
  __shared__ float x[16][17];
  const int v = threadIdx.x & 15, k = threadIdx.x >> 4;
  const int64_t i = (int64_t)blockIdx.x * 16 + v;
  float s = 0.0f;
  if (i < n) {
    int g = k;
    for (; g + 112 < groups; g += 128) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = part[(g + 16 * j) * n + i];
      s += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
    }
    for (; g < groups; g += 16) s += part[g * n + i];
  }
  x[k][v] = s;
  __syncthreads();
  if (k == 0 && i < n) {
#pragma unroll
    for (int j = 1; j < 16; ++j) s += x[j][v];
    put(i, s);
  }
}
__global__ __launch_bounds__(256) void conv_sum_kernel(const float* part, int groups, int W, int D, float* dw, float* db) {
  sum_groups(part, groups, (int64_t)(W + 1) * D, [&](int64_t i, float v) {
    const int j = (int)(i / D), c = (int)(i - (int64_t)j * D);
    if (j < W) dw[(int64_t)c * W + j] = v;
    else if (db) db[c] = v;
  });
}

// --------------------------------------------------------------------------
// Scan.
//   dt = softplus(delta + delta_bias), a_t[n] = exp(dt A[n]), h_t[n] = a_t[n] h_{t-1}[n] + dt B_t[n] u_t,
//   y_t = (sum_n C_t[n] h_t[n] + D u_t) silu(z_t)
// Rows of few, long sequences are also cut into chunks of `chunk` steps: every chunk's
// end state from zero and its sum of dt first, then the states that the chunks
// start from, then the chunks side by side.
constexpr int CK = 8;       // steps between kept states: what the gradient's registers hold of a block

struct ScanArgs {
  const int32_t* off;
  const void *u, *delta, *z, *Bm, *Cm, *dy;
  void *y, *du, *ddelta, *dz;
  const float *A, *Dp, *bias, *h0, *dhT;
  float *hT, *dh0, *ckpt;
  float *carry, *sdt;       // [B chunks][D][N], [B chunks][D]
  float *pbc, *pad;         // partial sums: [channel blocks][rows][2 N], [groups][D][N + 2]
  int32_t* status;
  int64_t ld_u, ld_delta, ld_z, ld_B, ld_C, ld_y, ld_dy, ld_du, ld_ddelta, ld_dz, rows;
  int B, T_max, D, chunk, chunks, groups, cblocks;
};

// First kept state of sequence s: ceil(len / CK) states each, so this leaves room for
// every sequence before it.
__device__ __forceinline__ int64_t ckpt_base(const Span& sp, int s) { return sp.r0 / CK + s; }
// Kept state i, channel c, states n ..  n + 3: quads side by side over the channels.
template <int N>
__device__ __forceinline__ float* ckpt_at(float* ckpt, int64_t i, int D, int c, int n) {
  return ckpt + ((i * (N / 4) + n / 4) * D + c) * 4 + (n & 3);
}

// A row of B or C at a uniform address, kept as the 32-bit words that it is in
// memory (scalar loads; two bf16 values a word).
template <class T, int N>
struct Row {
  static constexpr int W = N * (int)sizeof(T) / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const T* p) {
    typedef __attribute__((address_space(4))) const uint32_t cu32;
    const cu32* c = (const cu32*)(uintptr_t)p;
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = c[i];
  }
  __device__ __forceinline__ float get(int n) const {
    if constexpr (IS_BF<T>) return __uint_as_float(n & 1 ? w[n / 2] & 0xffff0000u : w[n / 2] << 16);
    else return __uint_as_float(w[n]);
  }
};

// Forward over one (sequence, chunk) and 64 channels per wavefront, one per lane, all
// N states in registers; rows of B and C are uniform (scalar loads).  LOCAL: only the
// chunk's end state from zero and its sum of dt.  What bounds it is the vector
// unit, busy 70% of the time: per step and channel 129 instructions at 16 states, 19 of
// them exponentials and reciprocals (as long as two).  8192 sequences of up to 64
// steps (184k rows), 256 channels, 16 states, gate, bf16: 255 us, 2.0 TB/s of the
// 522 MB; with rows of B and C by vector loads 349.
constexpr int SU = 8;       // steps whose rows are loaded together, one block ahead
template <class T, int N, bool LOCAL, bool Z>
__global__ __launch_bounds__(256) void scan_kernel(const ScanArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t id = blockIdx.x * 4 + wave, item = id / (uint32_t)a.cblocks;
  if (item >= (uint32_t)a.B * (uint32_t)a.chunks) return;
  const int cb = (int)(id - item * a.cblocks), s = (int)(item / (uint32_t)a.chunks), ch = (int)(item - (uint32_t)s * a.chunks);
  const Span sp = span_of(a, s, !LOCAL && cb == 0 && ch == 0 && lane == 0);
  const int t0 = ch * a.chunk, t1 = min(t0 + a.chunk, sp.len);
  if (t0 >= t1 && ch > 0) return;
  const int c = cb * 64 + lane, cc = min(c, a.D - 1);
  const bool mine = c < a.D;
  float h[N], A2[N];
#pragma unroll
  for (int n = 0; n < N; ++n) A2[n] = a.A[(int64_t)cc * N + n] * LOG2E;
  const float* h0 = LOCAL ? nullptr : a.chunks > 1 ? a.carry + ((int64_t)item * a.D + cc) * N
                                    : a.h0 ? a.h0 + ((int64_t)s * a.D + cc) * N : nullptr;
#pragma unroll
  for (int n = 0; n < N; n += 4) {
    const f32x4 v = h0 ? *reinterpret_cast<const f32x4*>(h0 + n) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) h[n + i] = v[i];
  }
  const float bias = a.bias ? a.bias[cc] : 0.0f, Dp = a.Dp ? a.Dp[cc] : 0.0f;
  // row t0 of every matrix (uniform; the lane's channel is an offset)
  const T* up = static_cast<const T*>(a.u) + (sp.r0 + t0) * a.ld_u;
  const T* dp = static_cast<const T*>(a.delta) + (sp.r0 + t0) * a.ld_delta;
  const T* zp = Z ? static_cast<const T*>(a.z) + (sp.r0 + t0) * a.ld_z : nullptr;
  const T* bp = static_cast<const T*>(a.Bm) + (sp.r0 + t0) * a.ld_B;
  const T* cp = static_cast<const T*>(a.Cm) + (sp.r0 + t0) * a.ld_C;
  T* yp = LOCAL ? nullptr : static_cast<T*>(a.y) + (sp.r0 + t0) * a.ld_y;
  float sdt = 0.0f;
  const int steps = t1 - t0;
  const int64_t ck0 = LOCAL ? 0 : ckpt_base(sp, s) + t0 / CK;
  T un[SU], dn[SU], zn[SU];
  auto load = [&](int t) {                     // rows t .. t + SU - 1, past the last one that one again
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      const int64_t r = min(t + i, steps - 1);
      un[i] = (up + r * a.ld_u)[cc];
      dn[i] = (dp + r * a.ld_delta)[cc];
      if (Z) zn[i] = (zp + r * a.ld_z)[cc];
    }
  };
  Row<T, N> Bn, Cn;
  auto load_bc = [&](int t) {
    const int64_t r = min(t, steps - 1);
    Bn.load(bp + r * a.ld_B);
    if (!LOCAL) Cn.load(cp + r * a.ld_C);
  };
  auto step = [&](int t, float u, float d, float z) {
    const Row<T, N> Br = Bn, Cr = Cn;
    load_bc(t + 1);
    const float du = d * u;
    float y = Dp * u;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      h[n] = fmaf(exp2_of(d * A2[n]), h[n], du * Br.get(n));
      if (!LOCAL) y = fmaf(Cr.get(n), h[n], y);
    }
    if (LOCAL) {
      sdt += d;
    } else {
      if (Z) y *= z * sigmoid(z);
      if (mine) (yp + (int64_t)t * a.ld_y)[cc] = (T)y;
    }
  };
  if (steps > 0) {
    load(0);
    load_bc(0);
  }
  for (int tb = 0; tb < steps; tb += SU) {
    float u[SU], d[SU], z[SU];
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      u[i] = (float)un[i];
      d[i] = softplus((float)dn[i] + bias);
      z[i] = Z ? (float)zn[i] : 0.0f;
    }
    if (tb + SU < steps) load(tb + SU);
    if (!LOCAL && a.ckpt && tb % CK == 0 && mine) {
#pragma unroll
      for (int n = 0; n < N; n += 4)
        *reinterpret_cast<f32x4*>(ckpt_at<N>(a.ckpt, ck0 + tb / CK, a.D, c, n)) = f32x4{h[n], h[n + 1], h[n + 2], h[n + 3]};
    }
    if (tb + SU <= steps) {
#pragma unroll
      for (int i = 0; i < SU; ++i) step(tb + i, u[i], d[i], z[i]);
    } else {
#pragma unroll
      for (int i = 0; i < SU - 1; ++i)
        if (tb + i < steps) step(tb + i, u[i], d[i], z[i]);
    }
  }
  if (!mine) return;
  float* out = LOCAL ? a.carry + ((int64_t)item * a.D + c) * N : a.hT && t1 == sp.len ? a.hT + ((int64_t)s * a.D + c) * N : nullptr;
  if (LOCAL) a.sdt[(int64_t)item * a.D + c] = sdt;
  if (out)
#pragma unroll
    for (int n = 0; n < N; n += 4) *reinterpret_cast<f32x4*>(out + n) = f32x4{h[n], h[n + 1], h[n + 2], h[n + 3]};
}

// The states that chunks start from, in the place of the chunks' end states.
// Forward: first to last from h0; gradient (REV): last to first from dhT.
template <int N, bool REV>
__global__ __launch_bounds__(256) void carry_kernel(const ScanArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (int64_t)a.D * N;
  if (i >= a.B * per) return;
  const int s = (int)(i / per);
  const int64_t cn = i - s * per, c = cn / N;
  const Span sp = span_of(a, s, false);
  const int used = (sp.len + a.chunk - 1) / a.chunk;
  const float A2 = a.A[cn] * LOG2E;
  const float* start = REV ? a.dhT : a.h0;
  float h = start ? start[i] : 0.0f;
  float* x = a.carry + (int64_t)s * a.chunks * per + cn;
  const float* sd = a.sdt + (int64_t)s * a.chunks * a.D + c;
  constexpr int U = 16;
  for (int k0 = 0; k0 < used; k0 += U) {
    float e[U], f[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int k = min(k0 + j, used - 1), ch = REV ? used - 1 - k : k;
      e[j] = x[ch * per];
      f[j] = sd[(int64_t)ch * a.D];
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (k0 + j >= used) break;
      x[(REV ? used - 1 - k0 - j : k0 + j) * per] = h;
      h = fmaf(exp2_of(f[j] * A2), h, e[j]);
    }
  }
  if (used == 0) x[0] = h;                   // an empty sequence's only chunk
}

// One step (T_max = 1): a workgroup takes 64 channels of a sequence, four lanes per
// channel with N / 4 states each, so that the states pass as whole 16-byte quads.
// Bytes bound it: 8 N of a channel's 8 N + 8 are its states, in and out.  2048 x 512
// x 16: 27 us, 5.2 TB/s.
template <class T, int N>
__global__ __launch_bounds__(256) void step_kernel(const ScanArgs a) {
  constexpr int L = N / 4, V = L < 4 ? L : 4;
  typedef Vec<float, V> FV;
  const uint32_t s = blockIdx.x / (uint32_t)a.cblocks, cb = blockIdx.x - s * a.cblocks;
  const int q = threadIdx.x & 3, c = cb * 64 + (threadIdx.x >> 2);
  const Span sp = span_of(a, s, cb == 0 && threadIdx.x == 0);
  if (c >= a.D) return;                      // whole quads
  FV h[L / V], A[L / V];
  const int64_t at = ((int64_t)s * a.D + c) * N + q * L;
#pragma unroll
  for (int i = 0; i < L / V; ++i) {
    h[i] = a.h0 ? *reinterpret_cast<const FV*>(a.h0 + at + i * V) : FV{};
    A[i] = *reinterpret_cast<const FV*>(a.A + (int64_t)c * N + q * L + i * V);
  }
  if (sp.len > 0) {
    const float u = (float)(static_cast<const T*>(a.u) + sp.r0 * a.ld_u)[c];
    const float d = softplus((float)(static_cast<const T*>(a.delta) + sp.r0 * a.ld_delta)[c] + (a.bias ? a.bias[c] : 0.0f));
    const T* b = static_cast<const T*>(a.Bm) + sp.r0 * a.ld_B + q * L;
    const T* cr = static_cast<const T*>(a.Cm) + sp.r0 * a.ld_C + q * L;
    float y = 0.0f;
#pragma unroll
    for (int i = 0; i < L / V; ++i) {
      const Vec<T, V> bv = *reinterpret_cast<const Vec<T, V>*>(b + i * V), cv = *reinterpret_cast<const Vec<T, V>*>(cr + i * V);
#pragma unroll
      for (int n = 0; n < V; ++n) {
        h[i][n] = fmaf(exp2_of(d * A[i][n] * LOG2E), h[i][n], d * u * (float)bv[n]);
        y = fmaf((float)cv[n], h[i][n], y);
      }
    }
    y += __shfl_xor(y, 1);
    y += __shfl_xor(y, 2);
    y = fmaf(a.Dp ? a.Dp[c] : 0.0f, u, y);
    if (q == 0) {
      if (a.z) {
        const float z = (float)(static_cast<const T*>(a.z) + sp.r0 * a.ld_z)[c];
        y *= z * sigmoid(z);
      }
      (static_cast<T*>(a.y) + sp.r0 * a.ld_y)[c] = (T)y;
    }
  }
  if (a.hT)
#pragma unroll
    for (int i = 0; i < L / V; ++i) *reinterpret_cast<FV*>(a.hT + at + i * V) = h[i];
}

// --------------------------------------------------------------------------
// Gradients.  With g_t = dL/dh_t (running back), dy = dout silu(z):
//   g += C_t dy, dC_t += dy h_t, dB_t += g dt u, w = g a_t h_{t-1},
//   du = dt sum_n g B + D dy, ddt = u sum_n g B + sum_n w A, dA += dt w, g <- g a_t
// A workgroup takes (sequence, chunk) items in turn and 16 channels per
// wavefront, four lanes per channel with N / 4 states each; blocks of CK steps are
// walked back from the kept state at their start, the steps' states and decays
// in registers.  Per-step values of a channel are computed by one of its four
// lanes (step 4 i + q by lane q) and passed around the quad.  Sums over a
// wavefront's channels are exchanges that halve the values each time; the
// wavefronts' sums meet in LDS.  The vector unit bounds it (35 instructions per
// state and step, 29 where the blocks' padding counts as steps; busy 75% of the
// time): 2048 sequences of up to 32 steps (34k rows), 512 channels, 16 states, gate,
// bf16: 386 us.  Blocks of 16 steps would keep half as many states in memory, but
// spill 50 registers and use 69% instead of 82% of these sequences' blocks.
constexpr int GW = 4, GC = 16 * GW;           // wavefronts and channels per workgroup

// f(0), f(1), .. with the index as a type (register arrays and lane patterns need constants)
template <class F, int... t>
__device__ __forceinline__ void each_step(F f, std::integer_sequence<int, t...>) {
  (f(std::integral_constant<int, t>{}), ...);
}
template <int K>
__device__ __forceinline__ float quad_get(float v) {   // lane K's value, in all four lanes of a quad
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), K * 0x55, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0xb1, 0xf, 0xf, true));   // quad_perm 1 0 3 2
  v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x4e, 0xf, 0xf, true));   // quad_perm 2 3 0 1
  return v;
}
// lanes 0..31: x summed over lane pairs (L, L ^ 32); lanes 32..63: y
__device__ __forceinline__ float fold32(float x, float y) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  const uint32_t a = r[0], b = r[1];
  return __uint_as_float(a) + __uint_as_float(b);
}
// the same over lane pairs (L, L ^ 16): even rows of 16 lanes x, odd rows y
__device__ __forceinline__ float fold16(float x, float y) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  const uint32_t a = r[0], b = r[1];
  return __uint_as_float(a) + __uint_as_float(b);
}
// sum over the lanes of a row of 16 with the same lane & 3
__device__ __forceinline__ float row_sum4(float v) {
  v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x128, 0xf, 0xf, true));  // row_ror 8
  v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x124, 0xf, 0xf, true));  // row_ror 4
  return v;
}

// Local running gradient of a chunk (the counterpart of scan_kernel<LOCAL>): one lane per channel.
template <class T, int N, bool Z>
__global__ __launch_bounds__(256) void grad_local_kernel(const ScanArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t id = blockIdx.x * 4 + wave, item = id / (uint32_t)a.cblocks;
  if (item >= (uint32_t)a.B * (uint32_t)a.chunks) return;
  const int cb = (int)(id - item * a.cblocks), s = (int)(item / (uint32_t)a.chunks), ch = (int)(item - (uint32_t)s * a.chunks);
  const Span sp = span_of(a, s, false);
  const int t0 = ch * a.chunk, t1 = min(t0 + a.chunk, sp.len), steps = t1 - t0;
  if (steps <= 0) return;
  const int c = cb * 64 + lane, cc = min(c, a.D - 1);
  float g[N], A2[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    A2[n] = a.A[(int64_t)cc * N + n] * LOG2E;
    g[n] = 0.0f;
  }
  const float bias = a.bias ? a.bias[cc] : 0.0f;
  const T* dp = static_cast<const T*>(a.delta) + (sp.r0 + t0) * a.ld_delta;
  const T* yp = static_cast<const T*>(a.dy) + (sp.r0 + t0) * a.ld_dy;
  const T* zp = Z ? static_cast<const T*>(a.z) + (sp.r0 + t0) * a.ld_z : nullptr;
  const T* cp = static_cast<const T*>(a.Cm) + (sp.r0 + t0) * a.ld_C;
  float sdt = 0.0f;
  T dn[SU], yn[SU], zn[SU];
  auto load = [&](int t) {                    // rows t, t - 1, ..
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      const int64_t r = max(t - i, 0);
      dn[i] = (dp + r * a.ld_delta)[cc];
      yn[i] = (yp + r * a.ld_dy)[cc];
      if (Z) zn[i] = (zp + r * a.ld_z)[cc];
    }
  };
  Row<T, N> Cn;
  auto step = [&](int t, float d, float dy) {
    const Row<T, N> Cr = Cn;
    Cn.load(cp + (int64_t)max(t - 1, 0) * a.ld_C);
#pragma unroll
    for (int n = 0; n < N; ++n) g[n] = fmaf(Cr.get(n), dy, g[n]) * exp2_of(d * A2[n]);
    sdt += d;
  };
  load(steps - 1);
  Cn.load(cp + (int64_t)(steps - 1) * a.ld_C);
  for (int tb = steps - 1; tb >= 0; tb -= SU) {
    float d[SU], dy[SU];
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      d[i] = softplus((float)dn[i] + bias);
      dy[i] = (float)yn[i];
      if (Z) dy[i] *= (float)zn[i] * sigmoid((float)zn[i]);
    }
    if (tb >= SU) load(tb - SU);
    if (tb >= SU - 1) {
#pragma unroll
      for (int i = 0; i < SU; ++i) step(tb - i, d[i], dy[i]);
    } else {
#pragma unroll
      for (int i = 0; i < SU - 1; ++i)
        if (tb - i >= 0) step(tb - i, d[i], dy[i]);
    }
  }
  if (c >= a.D) return;
  a.sdt[(int64_t)item * a.D + c] = sdt;
  float* out = a.carry + ((int64_t)item * a.D + c) * N;
#pragma unroll
  for (int n = 0; n < N; n += 4) *reinterpret_cast<f32x4*>(out + n) = f32x4{g[n], g[n + 1], g[n + 2], g[n + 3]};
}

template <class T, int N, bool Z>
__global__ __launch_bounds__(64 * GW, 2) void grad_kernel(const ScanArgs a) {
  constexpr int L = N / 4, K = CK, I = K / 4;      // states per lane, steps per block, steps a lane prepares
  constexpr int E = 16 / (int)sizeof(T), UN = K * N / E;               // staging of B, C: values and units of 16 bytes
  static_assert(2 * UN <= 64 * GW, "one unit per thread");
  __shared__ __attribute__((aligned(16))) float rows_buf[2][2][K][N];      // B and C of the block's steps
  __shared__ __attribute__((aligned(16))) float sums_buf[2][GW][K][2 * N]; // a wavefront's dB, dC
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = lane & 3, cb = blockIdx.x % a.cblocks, group = blockIdx.x / a.cblocks;
  const int c = cb * GC + wave * 16 + (lane >> 2), cc = min(c, a.D - 1);
  const bool mine = c < a.D;
  float A2[L], dA[L], dD = 0.0f, dbias = 0.0f;
#pragma unroll
  for (int n = 0; n < L; ++n) {
    A2[n] = a.A[(int64_t)cc * N + q * L + n] * LOG2E;
    dA[n] = 0.0f;
  }
  const float bias = a.bias ? a.bias[cc] : 0.0f, Dp = a.Dp ? a.Dp[cc] : 0.0f;
  // where this lane's sum of a step goes: lanes 0..31 dB, 32..63 dC; odd rows of 16 the
  // odd state of a pair; bit 2 the pair (with two states per lane there is one)
  const int to = (lane >> 5) * N + q * L + ((lane >> 4) & 1) + (L > 2 ? ((lane >> 2) & 1) * 2 : 0);
  const int items = a.B * a.chunks;
  // The blocks are walked one after another over the items; a block's inputs are
  // loaded while the block before it is computed.
  struct Block {
    int item, s, t0, t1, tb;
    int64_t r0;
    bool first;                                // the item's first chunk: its gradient leaves through dh0
  };
  // the block in scalar registers (what the compiler takes for divergent it would address per lane)
  auto uniform = [&](int sq, int item, int t0, int t1, int tb, int64_t r0) {
    auto u = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    Block k = {};
    k.s = u(sq);
    k.item = u(item);
    k.t0 = u(t0);
    k.t1 = u(t1);
    k.tb = u(tb);
    k.r0 = (int64_t)u((int)r0);                // rows < 2^31
    return k;
  };
  const bool have_in = a.chunks > 1 || a.dhT;
  const float* const in_base = a.chunks > 1 ? a.carry : a.dhT;
  // what reaches an item's last state from later (without any, and where not wanted,
  // some values of A, which the caller ignores: loads are unconditional, because
  // registers that are loaded on one path only are waited for there)
  auto grad_in = [&](const Block& k, bool wanted, float (&x)[L]) {
    const float* p = (wanted && have_in ? in_base + (int64_t)(a.chunks > 1 ? k.item : k.s) * a.D * N : a.A) + (uint32_t)cc * N + q * L;
    constexpr int V = L < 4 ? L : 4;
#pragma unroll
    for (int n = 0; n < L; n += V) {
      const Vec<float, V> v = *reinterpret_cast<const Vec<float, V>*>(p + n);
#pragma unroll
      for (int i = 0; i < V; ++i) x[n + i] = v[i];
    }
  };
  auto grad_out = [&](const Block& k, const float (&x)[L]) {
    if (a.dh0 && k.first && mine)
#pragma unroll
      for (int n = 0; n < L; ++n) a.dh0[((int64_t)k.s * a.D + c) * N + q * L + n] = x[n];
  };
  // the last block of the first item from `item` on that has any (item = items: none); the
  // gradient of an empty sequence's state passes through
  auto open = [&](int item) {
    Block k = {};
    for (k.item = item; k.item < items; k.item += a.groups) {
      k.s = a.chunks > 1 ? k.item / a.chunks : k.item;
      const int ch = k.item - k.s * a.chunks;
      const Span sp = span_of(a, k.s, cb == 0 && ch == 0 && tid == 0);
      k.r0 = sp.r0;
      k.first = ch == 0;
      k.t0 = ch * a.chunk;
      k.t1 = min(k.t0 + a.chunk, sp.len);
      if (k.t0 < k.t1) {
        k.tb = (k.t1 - 1) / K * K;             // chunks are whole blocks
        break;
      }
      if (k.first && a.dh0) {
        float x[L];
        grad_in(k, true, x);
#pragma unroll
        for (int n = 0; n < L; ++n) x[n] = have_in ? x[n] : 0.0f;
        grad_out(k, x);
      }
    }
    return k;
  };
  T ur[I], dr[I], yr[I], zr[I];                // this lane's steps 4 i + q; steps past the end read the last one
  float hs[L], g[L], gn[L];                    // the kept state; the running gradient, an item's first
  u32x4 row_x;                                 // 16 bytes of B or C, as they are (converting them here would wait for them)
  // this thread's 16 bytes of B or C
  const int rm = tid / UN & 1, rt = tid % UN / (N / E), rn = tid % (N / E) * E;
  const uintptr_t pb = (uintptr_t)a.Bm, pc = (uintptr_t)a.Cm;          // values: a choice of arguments would load them again
  const T* const rp = reinterpret_cast<const T*>(rm ? pc : pb) + rn;
  const int64_t lb = a.ld_B, lc = a.ld_C;
  const int64_t rl = rm ? lc : lb;
  auto load = [&](const Block& k, bool fresh, T (&u)[I], T (&d)[I], T (&y)[I], T (&z)[I], float (&h)[L], u32x4& x) {
    const int steps = min(K, k.t1 - k.tb);
    const int64_t rb = k.r0 + k.tb;
    auto row = [&](const void* p, int64_t ld) { return static_cast<const T*>(p) + rb * ld; };     // uniform
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const uint32_t t = min(4 * i + q, steps - 1);
      d[i] = row(a.delta, a.ld_delta)[t * (uint32_t)a.ld_delta + cc];
      u[i] = row(a.u, a.ld_u)[t * (uint32_t)a.ld_u + cc];
      y[i] = row(a.dy, a.ld_dy)[t * (uint32_t)a.ld_dy + cc];
      if (Z) z[i] = row(a.z, a.ld_z)[t * (uint32_t)a.ld_z + cc];
    }
    const float* kept = ckpt_at<N>(a.ckpt, ckpt_base({k.r0, 0}, k.s) + k.tb / K, a.D, 0, 0);      // uniform
    const uint32_t at = ((uint32_t)(q * L / 4) * a.D + cc) * 4 + (q * L & 3);
    constexpr int V = L < 4 ? L : 4;
#pragma unroll
    for (int n = 0; n < L; n += V) {
      const Vec<float, V> v = *reinterpret_cast<const Vec<float, V>*>(kept + at + (uint32_t)(n / 4) * a.D * 4);
#pragma unroll
      for (int i = 0; i < V; ++i) h[n + i] = v[i];
    }
    x = *reinterpret_cast<const u32x4*>(rp + (rb + min(rt, steps - 1)) * rl);      // threads past the rows: unused
    grad_in(k, fresh, gn);
  };
  Block cur = open(group);
  if (cur.item < items) {
    load(cur, true, ur, dr, yr, zr, hs, row_x);
#pragma unroll
    for (int n = 0; n < L; ++n) g[n] = have_in ? gn[n] : 0.0f;
  }
  // Results of a block are stored in the next block's turn, before its successor's loads are
  // issued: waiting for loads also waits for the stores before them, which then have
  // had a block's time.  One barrier per block: rows and sums alternate between two buffers.
  T duo[I], ddo[I], dzo[I];
  Block prev = {};
  prev.item = items;                           // none yet
  auto store = [&](const Block& k, const float (&sums)[GW][K][2 * N]) {
    const int steps = min(K, k.t1 - k.tb);
    const int64_t rb = k.r0 + k.tb;
    auto out = [&](void* p, int64_t ld) { return static_cast<T*>(p) + rb * ld; };
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const uint32_t t = 4 * i + q;
      if ((int)t >= steps || !mine) continue;
      out(a.du, a.ld_du)[t * (uint32_t)a.ld_du + c] = duo[i];
      out(a.ddelta, a.ld_ddelta)[t * (uint32_t)a.ld_ddelta + c] = ddo[i];
      if (Z) out(a.dz, a.ld_dz)[t * (uint32_t)a.ld_dz + c] = dzo[i];
    }
    float* pbc = a.pbc + ((int64_t)cb * a.rows + rb) * (2 * N);
    for (int i = tid; i < steps * 2 * N; i += 64 * GW) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < GW; ++w) v += (&sums[w][0][0])[i];
      pbc[i] = v;
    }
  };
  int buf = 0;
  for (; cur.item < items; buf ^= 1) {
    const int tb = cur.tb, steps = min(K, cur.t1 - tb);
    auto& rows = rows_buf[buf];
    auto& sums = sums_buf[buf];
    Block nxt = cur;
    nxt.tb -= K;
    const bool fresh = nxt.tb < cur.t0;
    if (fresh) nxt = open(cur.item + a.groups);
    const bool more = nxt.item < items;
    const Block ahead = uniform(more ? nxt.s : cur.s, more ? nxt.item : cur.item, more ? nxt.t0 : cur.t0, more ? nxt.t1 : cur.t1,
                                more ? nxt.tb : cur.tb, more ? nxt.r0 : cur.r0);
    if (tid < 2 * UN) {                        // rows past the end as zero
      const Vec<T, E> v = __builtin_bit_cast(Vec<T, E>, row_x);
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        f32x4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = rt < steps ? (float)v[i + j] : 0.0f;
        *reinterpret_cast<f32x4*>(&rows[rm][rt][rn + i]) = x;
      }
    }
    // steps past the end have dt = 0 and dy = 0: the state stays and the gradient passes;
    // lanes past the last channel have u = 0 and dy = 0, so that they add nothing to dB, dC
    float dt[I], du[I], dy[I], yg[I], s1[I], s2[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const bool in = 4 * i + q < steps;
      dt[i] = in ? softplus((float)dr[i] + bias) : 0.0f;
      du[i] = mine ? dt[i] * (float)ur[i] : 0.0f;
      float d = (float)yr[i];
      if (Z) d *= (float)zr[i] * sigmoid((float)zr[i]);
      dy[i] = in && mine ? d : 0.0f;
      yg[i] = s1[i] = s2[i] = 0.0f;
    }
    __syncthreads();
    if (prev.item < items) store(prev, sums_buf[buf ^ 1]);
    T un[I], dn[I], yn[I], zn[I];
    float hn[L];
    u32x4 row_n;
    load(ahead, fresh, un, dn, yn, zn, hn, row_n);
    float h[K][L], e[K][L];
    auto get_row = [&](float (&x)[L], int m, int t, int lq) {       // states lq L .. of a step's B or C
      constexpr int V = L < 4 ? L : 4;
      const Vec<float, V>* p = reinterpret_cast<const Vec<float, V>*>(&rows[m][t][0]) + lq * (L / V);
#pragma unroll
      for (int n = 0; n < L; ++n) x[n] = p[n / V][n % V];
    };
    auto forward = [&](auto tv) {
      constexpr int t = decltype(tv)::value;
      const float d = quad_get<(t & 3)>(dt[t / 4]), x = quad_get<(t & 3)>(du[t / 4]);
      float y = 0.0f, Br[L], Cr[L];
      get_row(Br, 0, t, q);
      if (Z) get_row(Cr, 1, t, q);
#pragma unroll
      for (int n = 0; n < L; ++n) {
        e[t][n] = exp2_of(d * A2[n]);
        h[t][n] = fmaf(e[t][n], t ? h[t ? t - 1 : 0][n] : hs[n], x * Br[n]);
        if (Z) y = fmaf(Cr[n], h[t][n], y);
      }
      if (Z) {
        y = quad_sum(y);
        yg[t / 4] = q == (t & 3) ? y : yg[t / 4];
      }
    };
    int at = q;
    auto backward = [&](auto tv) {
      constexpr int t = decltype(tv)::value;
      const float d = quad_get<(t & 3)>(dt[t / 4]), x = quad_get<(t & 3)>(du[t / 4]), y = quad_get<(t & 3)>(dy[t / 4]);
      float x1 = 0.0f, x2 = 0.0f, f[L], Br[L], Cr[L];
      get_row(Br, 0, t, at);
      get_row(Cr, 1, t, at);
#pragma unroll
      for (int n = 0; n < L; ++n) {
        g[n] = fmaf(Cr[n], y, g[n]);
        f[n] = fold32(g[n] * x, y * h[t][n]);
        x1 = fmaf(g[n], Br[n], x1);
        g[n] *= e[t][n];
        const float w = g[n] * (t ? h[t ? t - 1 : 0][n] : hs[n]);
        x2 = fmaf(w, A2[n], x2);
        dA[n] = fmaf(w, d, dA[n]);
      }
      x1 = quad_sum(x1);
      x2 = quad_sum(x2);
      s1[t / 4] = q == (t & 3) ? x1 : s1[t / 4];
      s2[t / 4] = q == (t & 3) ? x2 : s2[t / 4];
      float v[L / 2];
#pragma unroll
      for (int n = 0; n < L; n += 2) v[n / 2] = row_sum4(fold16(f[n], f[n + 1]));
      // lanes that hold the same sum write it to the same place
      if constexpr (L == 2) {
        sums[wave][t][to] = v[0];
      } else {
#pragma unroll
        for (int n = 0; n < L / 2; n += 2) {
          const float even = v[n], odd = v[n + 1];       // values: a choice of elements would go through memory
          sums[wave][t][to + 2 * n] = lane & 4 ? odd : even;
        }
      }
    };
    each_step(forward, std::make_integer_sequence<int, K>{});
    // values that the compiler cannot see through: the walk back reads the rows and passes
    // the steps' values again (keeping them from the walk forward takes 2 K (L + 1)
    // registers, which spill)
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int i = 0; i < I; ++i) asm volatile("" : "+v"(dt[i]), "+v"(du[i]));
    each_step([&](auto tv) { backward(std::integral_constant<int, K - 1 - decltype(tv)::value>{}); }, std::make_integer_sequence<int, K>{});
    // this lane's steps: du, ddelta, dz
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const bool in = 4 * i + q < steps;
      const float u = (float)ur[i], raw = (float)dr[i] + bias;
      duo[i] = (T)fmaf(dt[i], s1[i], Dp * dy[i]);
      const float dd = in ? fmaf(u, s1[i], s2[i] * LN2) * sigmoid(raw) : 0.0f;
      ddo[i] = (T)dd;
      dbias += dd;
      dD = fmaf(dy[i], u, dD);
      if (Z) {
        const float z = (float)zr[i], sz = sigmoid(z), yv = fmaf(Dp, u, yg[i]);
        dzo[i] = (T)((float)yr[i] * yv * sz * fmaf(z, 1.0f - sz, 1.0f));
      }
    }
    if (fresh) {
      grad_out(cur, g);
#pragma unroll
      for (int n = 0; n < L; ++n) g[n] = have_in ? gn[n] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < I; ++i) {
      ur[i] = un[i];
      dr[i] = dn[i];
      yr[i] = yn[i];
      if (Z) zr[i] = zn[i];
    }
#pragma unroll
    for (int n = 0; n < L; ++n) hs[n] = hn[n];
    row_x = row_n;
    prev = cur;
    cur = nxt;
  }
  __syncthreads();
  if (prev.item < items) store(prev, sums_buf[buf ^ 1]);
  dD = quad_sum(dD);
  dbias = quad_sum(dbias);
  if (!mine) return;
  float* out = a.pad + ((int64_t)group * a.D + c) * (N + 2);
#pragma unroll
  for (int n = 0; n < L; ++n) out[q * L + n] = dA[n];
  if (q == 0) {
    out[N] = dD;
    out[N + 1] = dbias;
  }
}

// dB and dC rows from the channel blocks' sums.
template <class T, int N>
__global__ __launch_bounds__(256) void bc_sum_kernel(const float* part, int cblocks, int64_t rows, T* dB, int64_t ld_B, T* dC,
                                                     int64_t ld_C) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = rows * 2 * N;
  if (i >= n) return;
  float s = 0.0f;
  for (int b = 0; b < cblocks; ++b) s += part[b * n + i];
  const int64_t r = i / (2 * N);
  const int k = (int)(i - r * 2 * N);
  if (k < N) dB[r * ld_B + k] = (T)s;
  else dC[r * ld_C + k - N] = (T)s;
}
template <int N>
__global__ __launch_bounds__(256) void ad_sum_kernel(const float* part, int groups, int D, float* dA, float* dD, float* dbias) {
  sum_groups(part, groups, (int64_t)D * (N + 2), [&](int64_t i, float v) {
    const int c = (int)(i / (N + 2)), k = (int)(i - (int64_t)c * (N + 2));
    if (k < N) dA[(int64_t)c * N + k] = v;
    else if (k == N) { if (dD) dD[c] = v; }
    else if (dbias) dbias[c] = v;
  });
}

// --------------------------------------------------------------------------
// Host side.
size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

wm_status bad(const char* m) { return set_error(WM_ERR_INVALID_ARGUMENT, m); }

// A launch holds fewer than 2^32 threads: workgroups of 256.
constexpr int64_t MAX_GROUPS = UINT32_MAX / 256;

wm_status check_rows(int32_t dtype, int32_t B, int32_t T_max, int64_t rows, int32_t channels, const int32_t* off) {
  if (dtype != WM_FP32 && dtype != WM_BF16) return bad("dtype must be WM_FP32 or WM_BF16");
  if (B < 0 || T_max < 0 || rows < 0 || rows > INT32_MAX) return bad("B, T_max and rows must be non-negative, rows below 2^31");
  if (channels < 1 || channels > (1 << 20)) return bad("channels must be in [1, 2^20]");
  if (B > 0 && !off) return bad("off is NULL");
  if (B == 0 && rows > 0) return bad("rows without a sequence");
  return WM_OK;
}
// row strides up to 2^24 elements: the kernels take rows of a block by 32-bit offsets
bool mat_ok(const void* p, int64_t ld, int64_t rows, int64_t width) { return rows == 0 || (p && ld >= width && ld <= (1 << 24)); }

struct ConvPlan {
  int runs, groups;
  size_t bytes;
};
wm_status check_conv(const wm_conv* a, ConvPlan* p) {
  if (!a) return bad("convolution arguments are NULL");
  const wm_status s = check_rows(a->dtype, a->B, a->T_max, a->rows, a->channels, a->off);
  if (s != WM_OK) return s;
  if (a->width < 2 || a->width > 4) return set_error(WM_ERR_UNSUPPORTED, "width must be 2, 3 or 4");
  if (!a->weight) return bad("weight is NULL");
  if (!mat_ok(a->x, a->ld_x, a->rows, a->channels)) return bad("x is NULL or its row stride is below channels");
  p->runs = std::max<int>(1, (int)cdiv(a->T_max, RUN));
  const int64_t items = (int64_t)a->B * p->runs;
  if (items > INT32_MAX / 2 || items * cdiv(a->channels, 64) > INT32_MAX / 2) return set_error(WM_ERR_UNSUPPORTED, "B x T_max is too large");
  // groups of the gradient: about eight wavefronts per SIMD when vectors can be used
  const int64_t cg = a->channels % 4 == 0 ? a->channels / 4 : a->channels;
  p->groups = (int)std::max<int64_t>(1, std::min<int64_t>(items, cdiv(256 * 4 * 4 * 64, cg)));
  p->bytes = workspace_of(al256((size_t)p->groups * (a->width + 1) * a->channels * 4));
  return WM_OK;
}
// whether V-wide accesses of rows are aligned
bool vec_ok(int v, int32_t dtype, const void* p, int64_t ld) {
  const int64_t e = dtype == WM_BF16 ? 2 : 4;
  return !p || ((uintptr_t)p % (v * e) == 0 && ld % v == 0);
}

// Lanes per run (a power of two) and workgroups of a launch over `slots` runs or groups.
int64_t conv_grid(ConvArgs& a, int vec, int64_t slots) {
  const int64_t cg = a.D / vec;
  a.lp = 0;
  while (a.lp < 6 && (1 << a.lp) < cg) ++a.lp;
  const int64_t waves = cdiv(slots, 64 >> a.lp) * cdiv(cg, 1 << a.lp);
  return cdiv(waves, 4);
}

// The gradient takes four channels per lane in both types (eight in bf16 need more
// registers than a wavefront may have twice per SIMD).
template <class T, int V, class F>
hipError_t conv_typed(int vec, int width, F f) {
  auto by_width = [&](auto vv) {
    if (width == 2) f(T{}, vv, std::integral_constant<int, 2>{});
    else if (width == 3) f(T{}, vv, std::integral_constant<int, 3>{});
    else f(T{}, vv, std::integral_constant<int, 4>{});
  };
  if (vec > 1) by_width(std::integral_constant<int, V>{});
  else by_width(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

struct ScanPlan {
  int chunk, chunks, groups, cblocks, gblocks;    // gblocks: channel blocks of the gradient
  size_t o_carry, o_sdt, o_pbc, o_pad, bytes;
};

wm_status check_scan(const wm_scan_args* a, ScanPlan* p, bool grad) {
  if (!a) return bad("scan arguments are NULL");
  const wm_status s = check_rows(a->dtype, a->B, a->T_max, a->rows, a->channels, a->off);
  if (s != WM_OK) return s;
  if (a->states != 8 && a->states != 16 && a->states != 32) return set_error(WM_ERR_UNSUPPORTED, "states must be 8, 16 or 32");
  if (!a->A) return bad("A is NULL");
  if (!mat_ok(a->u, a->ld_u, a->rows, a->channels) || !mat_ok(a->delta, a->ld_delta, a->rows, a->channels) ||
      (a->z && (a->ld_z < a->channels || a->ld_z > (1 << 24))))
    return bad("u, delta or z is NULL or its row stride is below channels");
  const int64_t e = a->dtype == WM_BF16 ? 2 : 4;
  if (!mat_ok(a->Bm, a->ld_B, a->rows, a->states) || !mat_ok(a->Cm, a->ld_C, a->rows, a->states) ||
      (uintptr_t)a->Bm % 16 || (uintptr_t)a->Cm % 16 || a->ld_B * e % 16 || a->ld_C * e % 16)
    return bad("Bm and Cm need 16-byte aligned rows of at least `states` values");
  if ((uintptr_t)a->A % 16 || (uintptr_t)a->h0 % 16) return bad("A and h0 must be 16-byte aligned");
  const int N = a->states;
  p->cblocks = (int)cdiv(a->channels, 64);
  p->gblocks = (int)cdiv(a->channels, GC);
  // Cut long sequences where whole ones leave the chip idle: a wavefront takes 64 channels
  // of one sequence, and 4096 wavefronts (four per SIMD) hide the chain of steps.  Chunks
  // cost a second pass without outputs: two sequences of 4001 steps and 768
  // channels in float32, forward, 93 us in chunks of 32 steps, 105 in chunks of 64.
  const int64_t waves = (int64_t)a->B * p->cblocks;
  p->chunk = std::max(1, a->T_max);
  p->chunks = 1;
  if (waves > 0 && waves < 1024 && a->T_max >= 128) {
    const int64_t c = std::max<int64_t>(32, cdiv(cdiv((int64_t)a->T_max * waves, 4096), 32) * 32);
    if (c < a->T_max) {
      p->chunk = (int)c;
      p->chunks = (int)cdiv(a->T_max, c);
    }
  }
  if (cdiv((int64_t)a->B * p->chunks * p->cblocks, 4) > MAX_GROUPS || (grad && cdiv(a->rows * 2 * N, 256) > MAX_GROUPS))
    return set_error(WM_ERR_UNSUPPORTED, "B x channels or rows x states is too large");
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at = al256(at + n); return o; };
  p->o_carry = p->o_sdt = p->o_pbc = p->o_pad = 0;
  const int64_t items = (int64_t)a->B * p->chunks;
  if (p->chunks > 1) {
    p->o_carry = take((size_t)items * a->channels * N * 4);
    p->o_sdt = take((size_t)items * a->channels * 4);
  }
  p->groups = 1;
  if (grad) {
    p->groups = (int)std::max<int64_t>(1, std::min<int64_t>(items, cdiv(4096, p->gblocks)));
    p->o_pbc = take((size_t)p->gblocks * a->rows * 2 * N * 4);
    p->o_pad = take((size_t)p->groups * a->channels * (N + 2) * 4);
  }
  p->bytes = workspace_of(at);
  return WM_OK;
}

template <class F>
hipError_t scan_typed(const wm_scan_args* a, F f) {
  auto by_n = [&](auto t) {
    using T = decltype(t);
    if (a->states == 8) f(T{}, std::integral_constant<int, 8>{});
    else if (a->states == 16) f(T{}, std::integral_constant<int, 16>{});
    else f(T{}, std::integral_constant<int, 32>{});
  };
  if (a->dtype == WM_BF16) by_n(__bf16{});
  else by_n(float{});
  return hipGetLastError();
}

ScanArgs scan_base(const wm_scan_args* w, const ScanPlan& p, uint8_t* w8) {
  ScanArgs a = {};
  a.off = w->off;
  a.u = w->u; a.delta = w->delta; a.z = w->z; a.Bm = w->Bm; a.Cm = w->Cm;
  a.A = w->A; a.Dp = w->D; a.bias = w->delta_bias; a.h0 = w->h0;
  a.ld_u = w->ld_u; a.ld_delta = w->ld_delta; a.ld_z = w->ld_z; a.ld_B = w->ld_B; a.ld_C = w->ld_C;
  a.rows = w->rows; a.B = w->B; a.T_max = w->T_max; a.D = w->channels;
  a.chunk = p.chunk; a.chunks = p.chunks; a.cblocks = p.cblocks; a.groups = p.groups;
  a.status = w->status;
  if (p.chunks > 1) {
    a.carry = reinterpret_cast<float*>(w8 + p.o_carry);
    a.sdt = reinterpret_cast<float*>(w8 + p.o_sdt);
  }
  return a;
}

}  // namespace scan
}  // namespace wm

using namespace wm::scan;

#define WM_ST(K, CALL)                                                                     \
  do {                                                                                     \
    timing_begin(K, st);                                                                   \
    hipError_t e_ = (CALL);                                                                \
    timing_end(K, st);                                                                     \
    if (e_ != hipSuccess) return set_error(WM_ERR_DEVICE, std::string("kernel launch: ") + hipGetErrorString(e_)); \
  } while (0)

extern "C" {

size_t wm_causal_conv_workspace_bytes(const wm_conv* w) {
  ConvPlan p;
  return check_conv(w, &p) == WM_OK ? p.bytes : 0;
}

wm_status wm_causal_conv(const wm_conv* w, void* y, int64_t ld_y, void* state_out, void* stream) {
  ConvPlan p;
  const wm_status s = check_conv(w, &p);
  if (s != WM_OK) return s;
  if (!mat_ok(y, ld_y, w->rows, w->channels)) return bad("y is NULL or its row stride is below channels");
  if (w->B == 0) return clear_error();
  hipStream_t st = static_cast<hipStream_t>(stream);
  ConvArgs a = {};
  a.off = w->off; a.x = w->x; a.state = w->state; a.y = y; a.state_out = state_out;
  a.w = w->weight; a.b = w->bias; a.status = w->status;
  a.ld_x = w->ld_x; a.ld_y = ld_y; a.rows = w->rows;
  a.B = w->B; a.T_max = w->T_max; a.D = w->channels; a.runs = p.runs; a.silu = w->silu;
  int vec = w->dtype == WM_BF16 ? 8 : 4;
  if (w->channels % vec || !vec_ok(vec, w->dtype, w->x, w->ld_x) || !vec_ok(vec, w->dtype, y, ld_y) || !vec_ok(vec, w->dtype, w->state, 0) ||
      !vec_ok(vec, w->dtype, state_out, 0))
    vec = 1;
  const int64_t grid = conv_grid(a, vec, (int64_t)w->B * p.runs);
  if (grid > MAX_GROUPS) return set_error(WM_ERR_UNSUPPORTED, "B x T_max x channels is too large");
  auto go = [&](auto t, auto v, auto wd) {
    hipLaunchKernelGGL((conv_kernel<decltype(t), decltype(v)::value, decltype(wd)::value>), dim3((unsigned)grid), dim3(256), 0, st, a);
  };
  WM_ST(TK_CONV, (w->dtype == WM_BF16 ? conv_typed<__bf16, 8>(vec, w->width, go) : conv_typed<float, 4>(vec, w->width, go)));
  return clear_error();
}

wm_status wm_causal_conv_grad(const wm_conv* w, const void* dy, int64_t ld_dy, const void* d_state_out, void* dx, int64_t ld_dx,
                              float* dweight, float* dbias, void* d_state, void* ws, size_t ws_bytes, void* stream) {
  ConvPlan p;
  const wm_status s = check_conv(w, &p);
  if (s != WM_OK) return s;
  if (!mat_ok(dy, ld_dy, w->rows, w->channels) || !mat_ok(dx, ld_dx, w->rows, w->channels))
    return bad("dy or dx is NULL or its row stride is below channels");
  if (!dweight) return bad("dweight is NULL");
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < p.bytes) return bad("workspace is NULL, not 256-byte aligned or too small");
  hipStream_t st = static_cast<hipStream_t>(stream);
  ConvArgs a = {};
  a.off = w->off; a.x = w->x; a.state = w->state; a.dy = dy; a.d_state_out = d_state_out; a.dx = dx; a.d_state = d_state;
  a.w = w->weight; a.b = w->bias; a.status = w->status;
  a.part = static_cast<float*>(ws);
  a.ld_x = w->ld_x; a.ld_dy = ld_dy; a.ld_dx = ld_dx; a.rows = w->rows;
  a.B = w->B; a.T_max = w->T_max; a.D = w->channels; a.runs = p.runs; a.silu = w->silu; a.groups = p.groups;
  int vec = w->channels % 4 ? 1 : 4;
  for (const auto& m : {std::pair<const void*, int64_t>{w->x, w->ld_x}, {dy, ld_dy}, {dx, ld_dx}, {w->state, 0}, {d_state_out, 0}, {d_state, 0}})
    if (!vec_ok(vec, w->dtype, m.first, m.second)) vec = 1;
  const int64_t grid = conv_grid(a, vec, p.groups);      // some 4096 wavefronts
  auto go = [&](auto t, auto v, auto wd) {
    hipLaunchKernelGGL((conv_grad_kernel<decltype(t), decltype(v)::value, decltype(wd)::value>), dim3((unsigned)grid), dim3(256), 0, st, a);
    hipLaunchKernelGGL(conv_sum_kernel, dim3((unsigned)cdiv((int64_t)(w->width + 1) * w->channels, 16)), dim3(256), 0, st,
                       a.part, a.groups, w->width, w->channels, dweight, dbias);
  };
  WM_ST(TK_CONV, (w->dtype == WM_BF16 ? conv_typed<__bf16, 4>(vec, w->width, go) : conv_typed<float, 4>(vec, w->width, go)));
  return clear_error();
}

size_t wm_scan_workspace_bytes(const wm_scan_args* w, int32_t grad) {
  ScanPlan p;
  return check_scan(w, &p, grad != 0) == WM_OK ? std::max(p.bytes, NO_WORKSPACE) : 0;
}

size_t wm_scan_checkpoint_bytes(const wm_scan_args* w) {
  ScanPlan p;
  if (check_scan(w, &p, false) != WM_OK) return 0;
  return al256((size_t)(w->rows / CK + w->B + 1) * w->channels * w->states * 4);
}

wm_status wm_scan(const wm_scan_args* w, void* y, int64_t ld_y, float* hT, void* checkpoints, void* ws, size_t ws_bytes,
                  void* stream) {
  ScanPlan p;
  const wm_status s = check_scan(w, &p, false);
  if (s != WM_OK) return s;
  if (!mat_ok(y, ld_y, w->rows, w->channels)) return bad("y is NULL or its row stride is below channels");
  if ((uintptr_t)hT % 16 || (uintptr_t)checkpoints % 16) return bad("hT and checkpoints must be 16-byte aligned");
  if (p.bytes && (!ws || (uintptr_t)ws % 256 || ws_bytes < p.bytes))
    return bad("workspace is NULL, not 256-byte aligned or too small");
  if (w->B == 0) return clear_error();
  hipStream_t st = static_cast<hipStream_t>(stream);
  ScanArgs a = scan_base(w, p, static_cast<uint8_t*>(ws));
  a.y = y; a.ld_y = ld_y; a.hT = hT; a.ckpt = static_cast<float*>(checkpoints);
  auto go = [&](auto t, auto nv) {
    using T = decltype(t);
    constexpr int N = decltype(nv)::value;
    if (w->T_max <= 1 && !checkpoints && (int64_t)w->B * p.cblocks <= MAX_GROUPS) {    // more: four to a workgroup below
      hipLaunchKernelGGL((step_kernel<T, N>), dim3((unsigned)(w->B * p.cblocks)), dim3(256), 0, st, a);
      return;
    }
    const dim3 grid((unsigned)cdiv((int64_t)w->B * p.chunks * p.cblocks, 4));
    if (p.chunks > 1) {
      hipLaunchKernelGGL((scan_kernel<T, N, true, false>), grid, dim3(256), 0, st, a);
      hipLaunchKernelGGL((carry_kernel<N, false>), dim3((unsigned)cdiv((int64_t)w->B * w->channels * N, 256)), dim3(256), 0, st, a);
    }
    if (a.z) hipLaunchKernelGGL((scan_kernel<T, N, false, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((scan_kernel<T, N, false, false>), grid, dim3(256), 0, st, a);
  };
  WM_ST(TK_SCAN, scan_typed(w, go));
  return clear_error();
}

wm_status wm_scan_grad(const wm_scan_args* w, const void* checkpoints, const void* dy, int64_t ld_dy, const float* dhT,
                       const wm_scan_grads* g, void* ws, size_t ws_bytes, void* stream) {
  ScanPlan p;
  const wm_status s = check_scan(w, &p, true);
  if (s != WM_OK) return s;
  if (!g) return bad("gradients are NULL");
  if (!mat_ok(dy, ld_dy, w->rows, w->channels) || !mat_ok(g->du, g->ld_du, w->rows, w->channels) ||
      !mat_ok(g->ddelta, g->ld_ddelta, w->rows, w->channels) || (w->z && !mat_ok(g->dz, g->ld_dz, w->rows, w->channels)))
    return bad("dy, du, ddelta or dz is NULL or its row stride is below channels");
  if (!mat_ok(g->dB, g->ld_dB, w->rows, w->states) || !mat_ok(g->dC, g->ld_dC, w->rows, w->states))
    return bad("dB or dC is NULL or its row stride is below states");
  if (!g->dA || !checkpoints) return bad("dA or checkpoints is NULL");
  if ((uintptr_t)dhT % 16 || (uintptr_t)checkpoints % 16) return bad("dhT and checkpoints must be 16-byte aligned");
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < p.bytes) return bad("workspace is NULL, not 256-byte aligned or too small");
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  ScanArgs a = scan_base(w, p, w8);
  a.ckpt = static_cast<float*>(const_cast<void*>(checkpoints));
  a.dy = dy; a.ld_dy = ld_dy; a.dhT = dhT; a.dh0 = g->dh0;
  a.du = g->du; a.ddelta = g->ddelta; a.dz = g->dz;
  a.ld_du = g->ld_du; a.ld_ddelta = g->ld_ddelta; a.ld_dz = g->ld_dz;
  a.pbc = reinterpret_cast<float*>(w8 + p.o_pbc);
  a.pad = reinterpret_cast<float*>(w8 + p.o_pad);
  auto go = [&](auto t, auto nv) {
    using T = decltype(t);
    constexpr int N = decltype(nv)::value;
    if (p.chunks > 1) {
      const dim3 grid((unsigned)cdiv((int64_t)w->B * p.chunks * p.cblocks, 4));
      if (a.z) hipLaunchKernelGGL((grad_local_kernel<T, N, true>), grid, dim3(256), 0, st, a);
      else hipLaunchKernelGGL((grad_local_kernel<T, N, false>), grid, dim3(256), 0, st, a);
      hipLaunchKernelGGL((carry_kernel<N, true>), dim3((unsigned)cdiv((int64_t)w->B * w->channels * N, 256)), dim3(256), 0, st, a);
    }
    ScanArgs b = a;
    b.cblocks = p.gblocks;
    if (a.z) hipLaunchKernelGGL((grad_kernel<T, N, true>), dim3(p.groups * p.gblocks), dim3(64 * GW), 0, st, b);
    else hipLaunchKernelGGL((grad_kernel<T, N, false>), dim3(p.groups * p.gblocks), dim3(64 * GW), 0, st, b);
    if (w->rows > 0)
      hipLaunchKernelGGL((bc_sum_kernel<T, N>), dim3((unsigned)cdiv(w->rows * 2 * N, 256)), dim3(256), 0, st, a.pbc, p.gblocks,
                         w->rows, static_cast<T*>(g->dB), g->ld_dB, static_cast<T*>(g->dC), g->ld_dC);
    hipLaunchKernelGGL((ad_sum_kernel<N>), dim3((unsigned)cdiv((int64_t)w->channels * (N + 2), 16)), dim3(256), 0, st, a.pad,
                       p.groups, w->channels, g->dA, g->dD, g->ddelta_bias);
  };
  WM_ST(TK_SCAN, scan_typed(w, go));
  return clear_error();
}

}  // extern "C"
