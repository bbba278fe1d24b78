// Sequence operators over packed ragged rows: a short causal convolution and a
// selective state-space scan, forward, gradients and single steps.
//
// Sequence s has rows [off[s], off[s+1]) (device offsets; a length past T_max
// or offsets outside the rows set the error word and are clamped).  Every sum
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

constexpr float LOG2E = 1.4426950408889634f;

template <class T>
constexpr bool IS_BF = std::is_same<T, __bf16>::value;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_of(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float sigmoid(float x) { return rcp_of(1.0f + exp2_of(-x * LOG2E)); }

// log(1 + e) for 0 <= e <= 1 as 2 atanh(s), s = e / (2 + e) <= 1/3: the odd series to
// s^13 (what is left out is below 2e-8 of the value).
__device__ __forceinline__ float log1p_unit(float e) {
  const float s = e * rcp_of(2.0f + e), q = s * s;
  float p = fmaf(q, 1.0f / 13.0f, 1.0f / 11.0f);
  p = fmaf(p, q, 1.0f / 9.0f);
  p = fmaf(p, q, 1.0f / 7.0f);
  p = fmaf(p, q, 1.0f / 5.0f);
  p = fmaf(p, q, 1.0f / 3.0f);
  p = fmaf(p, q, 1.0f);
  return 2.0f * s * p;
}
// softplus(x) = max(x, 0) + log(1 + exp(-|x|))
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.0f) + log1p_unit(exp2_of(-fabsf(x) * LOG2E)); }

// Rows of a sequence, clamped to what exists.
struct Span {
  int64_t r0;
  int len;
};
__device__ __forceinline__ Span span_of(const int32_t* off, int s, int64_t rows, int T_max, int32_t* status, bool report) {
  const int64_t a = off[s], b = off[s + 1];
  const int64_t lo = a < 0 ? 0 : a > rows ? rows : a, hi = b < lo ? lo : b > rows ? rows : b;
  const int64_t n = hi - lo > T_max ? T_max : hi - lo;
  if (report && status && (lo != a || n != b - a)) atomicOr(status, ERRBIT_LEN);
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
// Convolution.  A thread takes V neighbouring channels and runs of RUN rows of a
// sequence, the taps' window in registers.
constexpr int RUN = 16;

struct ConvArgs {
  const int32_t* off;
  const void *x, *state, *dy, *d_state_out;
  void *y, *state_out, *dx, *d_state;
  const float *w, *b;
  float* part;              // [groups][W + 1][D]
  int32_t* status;
  int64_t ld_x, ld_y, ld_dy, ld_dx, rows;
  int B, T_max, D, runs, silu, groups;
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

template <class T, int V, int W>
__global__ __launch_bounds__(256) void conv_kernel(const ConvArgs a) {
  const int CG = a.D / V;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t item = id / CG;
  if (item >= (int64_t)a.B * a.runs) return;
  const int c = (int)(id - item * CG) * V, s = (int)(item / a.runs), run = (int)(item - (int64_t)s * a.runs);
  const Span sp = span_of(a.off, s, a.rows, a.T_max, a.status, c == 0 && run == 0);
  const int t0 = run * RUN, t1 = min(t0 + RUN, sp.len);
  if (t0 < t1) {
    Taps<V, W> k;
    k.load(a, c);
    float win[W][V];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) conv_in<T, V, W>(win[j], a, sp, s, t0 - (W - 1) + j, c);
#pragma unroll 4
    for (int t = t0; t < t1; ++t) {
      load_vec<T, V>(win[W - 1], static_cast<const T*>(a.x) + (sp.r0 + t) * a.ld_x + c);
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float v = k.b[i];
#pragma unroll
        for (int j = 0; j < W; ++j) v = fmaf(k.w[j][i], win[j][i], v);
        y[i] = a.silu ? v * sigmoid(v) : v;
      }
      store_vec<T, V>(static_cast<T*>(a.y) + (sp.r0 + t) * a.ld_y + c, y);
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) win[j][i] = win[j + 1][i];
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
// the inputs; dx_t = sum_j w_j da_{t + W - 1 - j}.  A thread owns V channels and the items
// group, group + groups, ..; each row's share of dw is counted by the run that holds it.
template <class T, int V, int W>
__global__ __launch_bounds__(256) void conv_grad_kernel(const ConvArgs a) {
  const int CG = a.D / V;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int group = (int)(id / CG);
  if (group >= a.groups) return;
  const int c = (int)(id - (int64_t)group * CG) * V;
  Taps<V, W> k;
  k.load(a, c);
  float dw[W][V] = {}, db[V] = {};
  for (int64_t item = group; item < (int64_t)a.B * a.runs; item += a.groups) {
    const int s = (int)(item / a.runs), run = (int)(item - (int64_t)s * a.runs);
    const Span sp = span_of(a.off, s, a.rows, a.T_max, a.status, c == 0 && run == 0);
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
      float win[W][V], da[W][V];            // da[j]: of row t - (W - 1) + j
#pragma unroll
      for (int j = 0; j < W - 1; ++j) conv_in<T, V, W>(win[j], a, sp, s, t0 - (W - 1) + j, c);
#pragma unroll
      for (int j = 0; j < W; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) da[j][i] = 0.0f;
      // rows t0 .. t1 - 1 and the W - 1 after them; dx of row t - (W - 1) is complete at row t
      const int end = t1 + W - 1;
#pragma unroll 2
      for (int t = t0; t < end; ++t) {
        float g[V];
        if (t < sp.len) {
          load_vec<T, V>(win[W - 1], static_cast<const T*>(a.x) + (sp.r0 + t) * a.ld_x + c);
          load_vec<T, V>(g, static_cast<const T*>(a.dy) + (sp.r0 + t) * a.ld_dy + c);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float v = k.b[i];
#pragma unroll
            for (int j = 0; j < W; ++j) v = fmaf(k.w[j][i], win[j][i], v);
            if (a.silu) {
              const float sg = sigmoid(v);
              g[i] *= sg * fmaf(v, 1.0f - sg, 1.0f);
            }
          }
          if (t < t1) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
              db[i] += g[i];
#pragma unroll
              for (int j = 0; j < W; ++j) dw[j][i] = fmaf(g[i], win[j][i], dw[j][i]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) g[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) da[W - 1][i] = g[i];
        const int u = t - (W - 1);          // u's last reader of da is row t
        if (u >= t0) {
          float d[V];
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float v = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) v = fmaf(k.w[W - 1 - j][i], da[j][i], v);
            d[i] = v;
          }
          from_state(u, d);
          store_vec<T, V>(static_cast<T*>(a.dx) + (sp.r0 + u) * a.ld_dx + c, d);
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            win[j][i] = win[j + 1][i];
            da[j][i] = da[j + 1][i];
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
          float x[W][V];
#pragma unroll
          for (int j = 0; j < W; ++j) conv_in<T, V, W>(x[j], a, sp, s, t - (W - 1) + j, c);
          load_vec<T, V>(first[t], static_cast<const T*>(a.dy) + (sp.r0 + t) * a.ld_dy + c);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float v = k.b[i];
#pragma unroll
            for (int j = 0; j < W; ++j) v = fmaf(k.w[j][i], x[j][i], v);
            if (a.silu) {
              const float sg = sigmoid(v);
              first[t][i] *= sg * fmaf(v, 1.0f - sg, 1.0f);
            }
          }
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
template <int N>
constexpr int CK = N == 32 ? 8 : 16;          // steps between kept states (the gradient's registers hold so many)

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
template <int N>
__device__ __forceinline__ int64_t ckpt_base(const Span& sp, int s) { return sp.r0 / CK<N> + s; }
// Kept state i, channel c, states n ..  n + 3: quads side by side over the channels.
template <int N>
__device__ __forceinline__ float* ckpt_at(float* ckpt, int64_t i, int D, int c, int n) {
  return ckpt + ((i * (N / 4) + n / 4) * D + c) * 4 + (n & 3);
}

// Row t of B or C for all lanes (uniform address).
template <class T, int N>
__device__ __forceinline__ void load_row(float (&x)[N], const T* p) {
  if constexpr (IS_BF<T>) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const uint32_t v = w[i];
      x[2 * i] = __uint_as_float(v << 16);
      x[2 * i + 1] = __uint_as_float(v & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = p[i];
  }
}

// Forward over one (sequence, chunk) and 64 channels per wavefront, one per lane, all
// N states in registers; rows of B and C are uniform (scalar loads).  LOCAL: only the
// chunk's end state from zero and its sum of dt.
constexpr int SU = 8;       // steps whose rows are loaded together, one block ahead
template <class T, int N, bool LOCAL>
__global__ __launch_bounds__(256) void scan_kernel(const ScanArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  const int64_t item = id / a.cblocks;
  if (item >= (int64_t)a.B * a.chunks) return;
  const int cb = (int)(id - item * a.cblocks), s = (int)(item / a.chunks), ch = (int)(item - (int64_t)s * a.chunks);
  const Span sp = span_of(a.off, s, a.rows, a.T_max, a.status, !LOCAL && cb == 0 && ch == 0 && lane == 0);
  const int t0 = ch * a.chunk, t1 = min(t0 + a.chunk, sp.len);
  if (t0 >= t1 && ch > 0) return;
  const int c = cb * 64 + lane, cc = min(c, a.D - 1);
  const bool mine = c < a.D;
  float h[N], A2[N];
#pragma unroll
  for (int n = 0; n < N; ++n) A2[n] = a.A[(int64_t)cc * N + n] * LOG2E;
  const float* h0 = LOCAL ? nullptr : a.chunks > 1 ? a.carry + (item * a.D + cc) * N
                                    : a.h0 ? a.h0 + ((int64_t)s * a.D + cc) * N : nullptr;
#pragma unroll
  for (int n = 0; n < N; n += 4) {
    const f32x4 v = h0 ? *reinterpret_cast<const f32x4*>(h0 + n) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) h[n + i] = v[i];
  }
  const float bias = a.bias ? a.bias[cc] : 0.0f, Dp = a.Dp ? a.Dp[cc] : 0.0f;
  const T* up = static_cast<const T*>(a.u) + sp.r0 * a.ld_u + cc;
  const T* dp = static_cast<const T*>(a.delta) + sp.r0 * a.ld_delta + cc;
  const T* zp = a.z ? static_cast<const T*>(a.z) + sp.r0 * a.ld_z + cc : nullptr;
  const T* bp = static_cast<const T*>(a.Bm) + sp.r0 * a.ld_B;
  const T* cp = static_cast<const T*>(a.Cm) + sp.r0 * a.ld_C;
  T* yp = static_cast<T*>(a.y) + sp.r0 * a.ld_y + cc;
  float sdt = 0.0f;
  T un[SU], dn[SU], zn[SU];
  auto load = [&](int t) {
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      const int64_t r = min(t + i, t1 - 1);
      un[i] = up[r * a.ld_u];
      dn[i] = dp[r * a.ld_delta];
      if (!LOCAL && zp) zn[i] = zp[r * a.ld_z];
    }
  };
  if (t0 < t1) load(t0);
  const int64_t ck0 = LOCAL ? 0 : ckpt_base<N>(sp, s);
  for (int tb = t0; tb < t1; tb += SU) {
    float u[SU], d[SU], z[SU];
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      u[i] = (float)un[i];
      d[i] = softplus((float)dn[i] + bias);
      if (!LOCAL) z[i] = zp ? (float)zn[i] : 0.0f;
    }
    if (tb + SU < t1) load(tb + SU);
    if (!LOCAL && a.ckpt && tb % CK<N> == 0 && mine) {
#pragma unroll
      for (int n = 0; n < N; n += 4)
        *reinterpret_cast<f32x4*>(ckpt_at<N>(a.ckpt, ck0 + tb / CK<N>, a.D, c, n)) = f32x4{h[n], h[n + 1], h[n + 2], h[n + 3]};
    }
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      if (tb + i >= t1) break;
      float Bv[N], Cv[N];
      load_row<T, N>(Bv, bp + (int64_t)(tb + i) * a.ld_B);
      if (!LOCAL) load_row<T, N>(Cv, cp + (int64_t)(tb + i) * a.ld_C);
      const float du = d[i] * u[i];
      float y = Dp * u[i];
#pragma unroll
      for (int n = 0; n < N; ++n) {
        h[n] = fmaf(exp2_of(d[i] * A2[n]), h[n], du * Bv[n]);
        if (!LOCAL) y = fmaf(Cv[n], h[n], y);
      }
      if (LOCAL) {
        sdt += d[i];
      } else {
        if (zp) y *= z[i] * sigmoid(z[i]);
        if (mine) yp[(int64_t)(tb + i) * a.ld_y] = (T)y;
      }
    }
  }
  if (!mine) return;
  float* out = LOCAL ? a.carry + (item * a.D + c) * N : a.hT && t1 == sp.len ? a.hT + ((int64_t)s * a.D + c) * N : nullptr;
  if (LOCAL) a.sdt[item * a.D + c] = sdt;
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
  const Span sp = span_of(a.off, s, a.rows, a.T_max, nullptr, false);
  const int used = (sp.len + a.chunk - 1) / a.chunk;
  const float A2 = a.A[cn] * LOG2E;
  const float* start = REV ? a.dhT : a.h0;
  float h = start ? start[i] : 0.0f;
  float* x = a.carry + (int64_t)s * a.chunks * per + cn;
  const float* sd = a.sdt + (int64_t)s * a.chunks * a.D + c;
  constexpr int U = 8;
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

// One step (T_max = 1): four lanes per channel, N / 4 states each, so that the
// states pass as whole 16-byte quads.
template <class T, int N>
__global__ __launch_bounds__(256) void step_kernel(const ScanArgs a) {
  constexpr int L = N / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int q = (int)(id & 3);
  const int64_t sc = id >> 2;
  if (sc >= (int64_t)a.B * a.D) return;      // whole quads
  const int s = (int)(sc / a.D), c = (int)(sc - (int64_t)s * a.D);
  const Span sp = span_of(a.off, s, a.rows, a.T_max, a.status, c == 0 && q == 0);
  float h[L];
  const int64_t at = sc * N + q * L;
#pragma unroll
  for (int n = 0; n < L; ++n) h[n] = a.h0 ? a.h0[at + n] : 0.0f;
  if (sp.len > 0) {
    const float u = (float)static_cast<const T*>(a.u)[sp.r0 * a.ld_u + c];
    const float d = softplus((float)static_cast<const T*>(a.delta)[sp.r0 * a.ld_delta + c] + (a.bias ? a.bias[c] : 0.0f));
    const T* b = static_cast<const T*>(a.Bm) + sp.r0 * a.ld_B + q * L;
    const T* cr = static_cast<const T*>(a.Cm) + sp.r0 * a.ld_C + q * L;
    float y = 0.0f;
#pragma unroll
    for (int n = 0; n < L; ++n) {
      h[n] = fmaf(exp2_of(d * a.A[(int64_t)c * N + q * L + n] * LOG2E), h[n], d * u * (float)b[n]);
      y = fmaf((float)cr[n], h[n], y);
    }
    y += __shfl_xor(y, 1);
    y += __shfl_xor(y, 2);
    y = fmaf(a.Dp ? a.Dp[c] : 0.0f, u, y);
    if (q == 0) {
      if (a.z) {
        const float z = (float)static_cast<const T*>(a.z)[sp.r0 * a.ld_z + c];
        y *= z * sigmoid(z);
      }
      static_cast<T*>(a.y)[sp.r0 * a.ld_y + c] = (T)y;
    }
  }
  if (a.hT)
#pragma unroll
    for (int n = 0; n < L; ++n) a.hT[at + n] = h[n];
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
// wavefronts' sums meet in LDS.
constexpr int GW = 8, GC = 16 * GW;           // wavefronts and channels per workgroup

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

// Local running gradient of a chunk (REV counterpart of scan_kernel<LOCAL>): one lane per channel.
template <class T, int N>
__global__ __launch_bounds__(256) void grad_local_kernel(const ScanArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  const int64_t item = id / a.cblocks;
  if (item >= (int64_t)a.B * a.chunks) return;
  const int cb = (int)(id - item * a.cblocks), s = (int)(item / a.chunks), ch = (int)(item - (int64_t)s * a.chunks);
  const Span sp = span_of(a.off, s, a.rows, a.T_max, nullptr, false);
  const int t0 = ch * a.chunk, t1 = min(t0 + a.chunk, sp.len);
  if (t0 >= t1) return;
  const int c = cb * 64 + lane, cc = min(c, a.D - 1);
  float g[N], A2[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    A2[n] = a.A[(int64_t)cc * N + n] * LOG2E;
    g[n] = 0.0f;
  }
  const float bias = a.bias ? a.bias[cc] : 0.0f;
  const T* dp = static_cast<const T*>(a.delta) + sp.r0 * a.ld_delta + cc;
  const T* yp = static_cast<const T*>(a.dy) + sp.r0 * a.ld_dy + cc;
  const T* zp = a.z ? static_cast<const T*>(a.z) + sp.r0 * a.ld_z + cc : nullptr;
  const T* cp = static_cast<const T*>(a.Cm) + sp.r0 * a.ld_C;
  float sdt = 0.0f;
  T dn[SU], yn[SU], zn[SU];
  auto load = [&](int t) {                    // rows t, t - 1, ..
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      const int64_t r = max(t - i, t0);
      dn[i] = dp[r * a.ld_delta];
      yn[i] = yp[r * a.ld_dy];
      if (zp) zn[i] = zp[r * a.ld_z];
    }
  };
  load(t1 - 1);
  for (int tb = t1 - 1; tb >= t0; tb -= SU) {
    float d[SU], dy[SU];
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      d[i] = softplus((float)dn[i] + bias);
      dy[i] = (float)yn[i];
      if (zp) {
        const float z = (float)zn[i];
        dy[i] *= z * sigmoid(z);
      }
    }
    if (tb - SU >= t0) load(tb - SU);
#pragma unroll
    for (int i = 0; i < SU; ++i) {
      if (tb - i < t0) break;
      float Cv[N];
      load_row<T, N>(Cv, cp + (int64_t)(tb - i) * a.ld_C);
#pragma unroll
      for (int n = 0; n < N; ++n) g[n] = fmaf(Cv[n], dy[i], g[n]) * exp2_of(d[i] * A2[n]);
      sdt += d[i];
    }
  }
  if (c >= a.D) return;
  a.sdt[item * a.D + c] = sdt;
  float* out = a.carry + (item * a.D + c) * N;
#pragma unroll
  for (int n = 0; n < N; n += 4) *reinterpret_cast<f32x4*>(out + n) = f32x4{g[n], g[n + 1], g[n + 2], g[n + 3]};
}

template <class T, int N>
__global__ __launch_bounds__(64 * GW) void grad_kernel(const ScanArgs a) {
  constexpr int L = N / 4, K = CK<N>, I = K / 4;      // states per lane, steps per block, steps a lane prepares
  __shared__ __attribute__((aligned(16))) float rows[2][K][N];        // B and C of the block's steps
  __shared__ float sums[GW][K][2 * N];                                 // a wavefront's dB, dC
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = lane & 3, cb = blockIdx.x % a.cblocks, group = blockIdx.x / a.cblocks;
  const int c = cb * GC + wave * 16 + (lane >> 2), cc = min(c, a.D - 1);
  const bool mine = c < a.D;
  float A[L], dA[L], dD = 0.0f, dbias = 0.0f;
#pragma unroll
  for (int n = 0; n < L; ++n) {
    A[n] = a.A[(int64_t)cc * N + q * L + n];
    dA[n] = 0.0f;
  }
  const float bias = a.bias ? a.bias[cc] : 0.0f, Dp = a.Dp ? a.Dp[cc] : 0.0f;
  const int64_t items = (int64_t)a.B * a.chunks;
  for (int64_t item = group; item < items; item += a.groups) {
    const int s = (int)(item / a.chunks), ch = (int)(item - (int64_t)s * a.chunks);
    const Span sp = span_of(a.off, s, a.rows, a.T_max, a.status, cb == 0 && ch == 0 && tid == 0);
    const int t0 = ch * a.chunk, t1 = min(t0 + a.chunk, sp.len);
    float g[L];
    const float* gin = a.chunks > 1 ? a.carry + item * a.D * N : a.dhT ? a.dhT + (int64_t)s * a.D * N : nullptr;
#pragma unroll
    for (int n = 0; n < L; ++n) g[n] = gin && (t0 < t1 || ch == 0) ? gin[(int64_t)cc * N + q * L + n] : 0.0f;
    const int64_t ck0 = ckpt_base<N>(sp, s);
    const int last = (t1 - 1) / K;                     // chunks are whole blocks
    for (int blk = last; blk >= t0 / K && t0 < t1; --blk) {
      const int tb = blk * K, steps = min(K, t1 - tb);
      __syncthreads();
      for (int i = tid; i < 2 * K * N; i += 64 * GW) {
        const int m = i / (K * N), t = i / N % K, n = i % N;
        const T* p = m ? static_cast<const T*>(a.Cm) + (sp.r0 + tb + t) * a.ld_C : static_cast<const T*>(a.Bm) + (sp.r0 + tb + t) * a.ld_B;
        rows[m][t][n] = t < steps ? (float)p[n] : 0.0f;
      }
      // this lane's steps 4 i + q; steps past the end have dt = 0 and dy = 0: the
      // state stays and the gradient passes
      float dt[I], u[I], dy[I], z[I], dout[I], sg[I], yg[I], s1[I], s2[I];
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const int t = 4 * i + q;
        const int64_t r = sp.r0 + tb + min(t, steps - 1);
        const bool in = t < steps;
        u[i] = in ? (float)static_cast<const T*>(a.u)[r * a.ld_u + cc] : 0.0f;
        dout[i] = in ? (float)static_cast<const T*>(a.dy)[r * a.ld_dy + cc] : 0.0f;
        const float raw = (float)static_cast<const T*>(a.delta)[r * a.ld_delta + cc] + bias;
        z[i] = a.z ? (float)static_cast<const T*>(a.z)[r * a.ld_z + cc] : 0.0f;
        const float e = exp2_of(-fabsf(raw) * LOG2E);
        dt[i] = in ? fmaxf(raw, 0.0f) + log1p_unit(e) : 0.0f;
        sg[i] = (raw >= 0.0f ? 1.0f : e) * rcp_of(1.0f + e);
        dy[i] = a.z ? dout[i] * z[i] * sigmoid(z[i]) : dout[i];
        yg[i] = s1[i] = s2[i] = 0.0f;
      }
      float hs[L];
      {
        const float* kept = ckpt_at<N>(a.ckpt, ck0 + blk, a.D, cc, q * L);
#pragma unroll
        for (int n = 0; n < L; ++n) hs[n] = (L < 4 || n < 4) ? kept[n] : kept[(int64_t)(n / 4) * a.D * 4 + (n & 3)];
      }
      __syncthreads();
      float h[K][L], e[K][L];
      auto forward = [&](auto tv) {
        constexpr int t = decltype(tv)::value;
        const float d = quad_get<(t & 3)>(dt[t / 4]), du = d * quad_get<(t & 3)>(u[t / 4]);
        float y = 0.0f;
#pragma unroll
        for (int n = 0; n < L; ++n) {
          e[t][n] = exp2_of(d * A[n] * LOG2E);
          h[t][n] = fmaf(e[t][n], t ? h[t ? t - 1 : 0][n] : hs[n], du * rows[0][t][q * L + n]);
          if (a.z) y = fmaf(rows[1][t][q * L + n], h[t][n], y);
        }
        if (a.z) {
          y = quad_sum(y);
          if (q == (t & 3)) yg[t / 4] = y;
        }
      };
      auto backward = [&](auto tv) {
        constexpr int t = decltype(tv)::value;
        const float d = quad_get<(t & 3)>(dt[t / 4]), du = d * quad_get<(t & 3)>(u[t / 4]), y = quad_get<(t & 3)>(dy[t / 4]);
        float x1 = 0.0f, x2 = 0.0f, db[L], dc[L];
#pragma unroll
        for (int n = 0; n < L; ++n) {
          g[n] = fmaf(rows[1][t][q * L + n], y, g[n]);
          dc[n] = mine ? y * h[t][n] : 0.0f;
          db[n] = mine ? g[n] * du : 0.0f;
          x1 = fmaf(g[n], rows[0][t][q * L + n], x1);
          g[n] *= e[t][n];
          const float w = g[n] * (t ? h[t ? t - 1 : 0][n] : hs[n]);
          x2 = fmaf(w, A[n], x2);
          dA[n] = fmaf(w, d, dA[n]);
        }
        x1 = quad_sum(x1);
        x2 = quad_sum(x2);
        if (q == (t & 3)) {
          s1[t / 4] = x1;
          s2[t / 4] = x2;
        }
        // lanes 0..31 dB, lanes 32..63 dC; then rows of 16 lanes: two states each
        float f[L];
#pragma unroll
        for (int n = 0; n < L; ++n) f[n] = fold32(db[n], dc[n]);
#pragma unroll
        for (int n = 0; n < L; n += 2) {
          const float v = row_sum4(fold16(f[n], f[n + 1]));
          if ((lane & 12) == 0) sums[wave][t][(lane >> 5) * N + q * L + n + ((lane >> 4) & 1)] = v;
        }
      };
      each_step(forward, std::make_integer_sequence<int, K>{});
      each_step([&](auto tv) { backward(std::integral_constant<int, K - 1 - decltype(tv)::value>{}); }, std::make_integer_sequence<int, K>{});
      // this lane's steps: du, ddelta, dz
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const int t = 4 * i + q;
        if (t >= steps || !mine) continue;
        const int64_t r = sp.r0 + tb + t;
        static_cast<T*>(a.du)[r * a.ld_du + c] = (T)fmaf(dt[i], s1[i], Dp * dy[i]);
        const float dd = fmaf(u[i], s1[i], s2[i]) * sg[i];
        static_cast<T*>(a.ddelta)[r * a.ld_ddelta + c] = (T)dd;
        dbias += dd;
        dD = fmaf(dy[i], u[i], dD);
        if (a.z) {
          const float sz = sigmoid(z[i]), yv = fmaf(Dp, u[i], yg[i]);
          static_cast<T*>(a.dz)[r * a.ld_dz + c] = (T)(dout[i] * yv * sz * fmaf(z[i], 1.0f - sz, 1.0f));
        }
      }
      __syncthreads();
      for (int i = tid; i < steps * 2 * N; i += 64 * GW) {
        const int t = i / (2 * N), n = i % (2 * N);
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < GW; ++w) v += sums[w][t][n];
        a.pbc[((int64_t)cb * a.rows + sp.r0 + tb + t) * (2 * N) + n] = v;
      }
    }
    if (a.dh0 && ch == 0 && mine)
#pragma unroll
      for (int n = 0; n < L; ++n) a.dh0[((int64_t)s * a.D + c) * N + q * L + n] = g[n];
  }
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

wm_status check_rows(int32_t dtype, int32_t B, int32_t T_max, int64_t rows, int32_t channels, const int32_t* off) {
  if (dtype != WM_FP32 && dtype != WM_BF16) return bad("dtype must be WM_FP32 or WM_BF16");
  if (B < 0 || T_max < 0 || rows < 0 || rows > INT32_MAX) return bad("B, T_max and rows must be non-negative, rows below 2^31");
  if (channels < 1 || channels > (1 << 20)) return bad("channels must be in [1, 2^20]");
  if (B > 0 && !off) return bad("off is NULL");
  return WM_OK;
}
bool mat_ok(const void* p, int64_t ld, int64_t rows, int64_t width) { return rows == 0 || (p && ld >= width); }

struct ConvPlan {
  int runs, groups, vec;
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
  if (items > INT32_MAX || items * a->channels > ((int64_t)1 << 39)) return set_error(WM_ERR_UNSUPPORTED, "B x T_max is too large");
  // groups of the gradient: about eight wavefronts per SIMD when vectors can be used
  const int v = a->dtype == WM_BF16 ? 8 : 4;
  p->vec = a->channels % v == 0 ? v : 1;
  const int64_t cg = a->channels / p->vec;
  p->groups = (int)std::max<int64_t>(1, std::min<int64_t>(items, cdiv(256 * 4 * 4 * 64, cg)));
  p->bytes = al256((size_t)p->groups * (a->width + 1) * a->channels * 4);
  return WM_OK;
}
// whether V-wide accesses of rows are aligned
bool vec_ok(int v, int32_t dtype, const void* p, int64_t ld) {
  const int64_t e = dtype == WM_BF16 ? 2 : 4;
  return !p || ((uintptr_t)p % (v * e) == 0 && ld % v == 0);
}

template <class T, class F>
hipError_t conv_typed(int vec, int width, F f) {
  constexpr int V = IS_BF<T> ? 8 : 4;
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
int ck_of(int N) { return N == 32 ? 8 : 16; }

wm_status check_scan(const wm_scan_args* a, ScanPlan* p, bool grad) {
  if (!a) return bad("scan arguments are NULL");
  const wm_status s = check_rows(a->dtype, a->B, a->T_max, a->rows, a->channels, a->off);
  if (s != WM_OK) return s;
  if (a->states != 8 && a->states != 16 && a->states != 32) return set_error(WM_ERR_UNSUPPORTED, "states must be 8, 16 or 32");
  if (!a->A) return bad("A is NULL");
  if (!mat_ok(a->u, a->ld_u, a->rows, a->channels) || !mat_ok(a->delta, a->ld_delta, a->rows, a->channels) ||
      (a->z && a->ld_z < a->channels))
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
  // of one sequence, and 4096 wavefronts (four per SIMD) hide the chain of steps.
  const int64_t waves = (int64_t)a->B * p->cblocks;
  p->chunk = std::max(1, a->T_max);
  p->chunks = 1;
  if (waves > 0 && waves < 1024 && a->T_max >= 128) {
    const int64_t c = std::max<int64_t>(64, cdiv(cdiv((int64_t)a->T_max * waves, 4096), 32) * 32);
    if (c < a->T_max) {
      p->chunk = (int)c;
      p->chunks = (int)cdiv(a->T_max, c);
    }
  }
  if ((int64_t)a->B * p->chunks > INT32_MAX / 4) return set_error(WM_ERR_UNSUPPORTED, "B x T_max is too large");
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
    p->groups = (int)std::max<int64_t>(1, std::min<int64_t>(items, cdiv(1024, p->gblocks)));
    p->o_pbc = take((size_t)p->gblocks * a->rows * 2 * N * 4);
    p->o_pad = take((size_t)p->groups * a->channels * (N + 2) * 4);
  }
  p->bytes = at;
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
  int vec = p.vec;
  if (!vec_ok(vec, w->dtype, w->x, w->ld_x) || !vec_ok(vec, w->dtype, y, ld_y) || !vec_ok(vec, w->dtype, w->state, 0) ||
      !vec_ok(vec, w->dtype, state_out, 0))
    vec = 1;
  const int64_t threads = (int64_t)w->B * p.runs * (w->channels / vec);
  auto go = [&](auto t, auto v, auto wd) {
    hipLaunchKernelGGL((conv_kernel<decltype(t), decltype(v)::value, decltype(wd)::value>), dim3((unsigned)cdiv(threads, 256)),
                       dim3(256), 0, st, a);
  };
  WM_ST(TK_CONV, w->dtype == WM_BF16 ? conv_typed<__bf16>(vec, w->width, go) : conv_typed<float>(vec, w->width, go));
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
  int vec = p.vec;
  for (const auto& m : {std::pair<const void*, int64_t>{w->x, w->ld_x}, {dy, ld_dy}, {dx, ld_dx}, {w->state, 0}, {d_state_out, 0}, {d_state, 0}})
    if (!vec_ok(vec, w->dtype, m.first, m.second)) vec = 1;
  const int64_t threads = (int64_t)p.groups * (w->channels / vec);
  auto go = [&](auto t, auto v, auto wd) {
    hipLaunchKernelGGL((conv_grad_kernel<decltype(t), decltype(v)::value, decltype(wd)::value>), dim3((unsigned)cdiv(threads, 256)),
                       dim3(256), 0, st, a);
    hipLaunchKernelGGL(conv_sum_kernel, dim3((unsigned)cdiv((int64_t)(w->width + 1) * w->channels, 16)), dim3(256), 0, st,
                       a.part, a.groups, w->width, w->channels, dweight, dbias);
  };
  WM_ST(TK_CONV, w->dtype == WM_BF16 ? conv_typed<__bf16>(vec, w->width, go) : conv_typed<float>(vec, w->width, go));
  return clear_error();
}

size_t wm_scan_workspace_bytes(const wm_scan_args* w, int32_t grad) {
  ScanPlan p;
  return check_scan(w, &p, grad != 0) == WM_OK ? std::max<size_t>(p.bytes, 256) : 0;
}

size_t wm_scan_checkpoint_bytes(const wm_scan_args* w) {
  ScanPlan p;
  if (check_scan(w, &p, false) != WM_OK) return 0;
  return al256((size_t)(w->rows / ck_of(w->states) + w->B + 1) * w->channels * w->states * 4);
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
    if (w->T_max <= 1 && !checkpoints) {
      hipLaunchKernelGGL((step_kernel<T, N>), dim3((unsigned)cdiv((int64_t)w->B * w->channels * 4, 256)), dim3(256), 0, st, a);
      return;
    }
    const dim3 grid((unsigned)cdiv((int64_t)w->B * p.chunks * p.cblocks, 4));
    if (p.chunks > 1) {
      hipLaunchKernelGGL((scan_kernel<T, N, true>), grid, dim3(256), 0, st, a);
      hipLaunchKernelGGL((carry_kernel<N, false>), dim3((unsigned)cdiv((int64_t)w->B * w->channels * N, 256)), dim3(256), 0, st, a);
    }
    hipLaunchKernelGGL((scan_kernel<T, N, false>), grid, dim3(256), 0, st, a);
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
      hipLaunchKernelGGL((grad_local_kernel<T, N>), dim3((unsigned)cdiv((int64_t)w->B * p.chunks * p.cblocks, 4)), dim3(256), 0, st, a);
      hipLaunchKernelGGL((carry_kernel<N, true>), dim3((unsigned)cdiv((int64_t)w->B * w->channels * N, 256)), dim3(256), 0, st, a);
    }
    ScanArgs b = a;
    b.cblocks = p.gblocks;
    hipLaunchKernelGGL((grad_kernel<T, N>), dim3(p.groups * p.gblocks), dim3(64 * GW), 0, st, b);
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
