// Attention to the keys of a program and to the sequence's own keys, under one softmax: all rows of
// packed sequences at once with gradients (dense rows), and single steps or chunks over a paged cache.
//
// As in the cross attention (wm_attend.hip) the G query heads of a key head are stacked, so a
// workgroup has rows of one (program, key head) or (sequence, key head).  Its keys come in two runs,
// cut into tiles one after the other: the program's, which every row sees, and own keys, of which a
// row sees an interval [lo, hi) (its sequence's rows up to itself).  In packed rows the intervals of
// neighbouring rows are neighbours, so a workgroup's own keys are one run as well, also where it
// holds many short sequences.
#include <string>

#include "wm_attend.h"

using namespace wm;

namespace wm {
namespace prefix {

using namespace wm::attend;

struct Args {
  const void *q, *k, *v, *pk, *pv, *o, *d_o;
  int64_t ld_q, ld_k, ld_v, ld_pk, ld_pv, ld_o, ld_do;
  const uint8_t* mask;                      // of the program's keys (dense)
  const int32_t* off;                       // [B + 1] rows of the sequences
  int32_t* status;
  int64_t rows;
  int B, T_max;
  float c2, scale;                          // scale log2(e), scale
  int heads, kv_heads, G;
  int splits, chunk;                        // a loop's shares: `chunk` tiles each, the last what is left
  void *out, *out2;                         // o; dq; dk and dv
  int64_t ld_out, ld_out2;
  float* lse;                               // forward: out (may be null); gradient: in
  float* stat;                              // gradient: [rows heads][2] (lse log2 e, delta)
  float* part;                              // partial sums [parts][rows heads][DH] (dkv: [splits][2][rows kv_heads][DH])
  float* part_ml;                           // forward: [parts][rows heads][2] maximum (log2 units), sum
  int64_t part_rows;
  int part0, parts;                         // this launch's first part (cached), all parts (join)
  // cached
  const int32_t *pages, *lens, *ppages, *plens;
  int programs;                             // lengths in plens
  int max_pages, max_ppages, len_max, plen_max, n_pages, lps;      // lps: log2 of a page's slots
  int seq0, nseq, row_tiles;                // a launch by sequences, tiles of each at most; 0 row tiles: by programs
  int slots;                                // RAGGED: workgroups of a key head and split, in place of nseq row_tiles
  int joint;                                // by sequences: their programs' keys first
  int more_blocks, more_splits, more_chunk, more_part0;            // the few-row kernel: its first workgroups go by programs
  int again;                                // rows of a tile see different keys: sums that are not finite are formed again
  int32_t* counts;                          // gradient: how many parts a row (a key) of a head has
};

// Into how many shares a loop is cut, and the tiles [x, y) of a split's.
__device__ __forceinline__ int shares_of(const Args& a, int tiles) { return min(max((tiles - 1) / a.chunk + 1, 1), a.splits); }
__device__ __forceinline__ int2 share_of(const Args& a, int tiles, int split) {
  const int64_t x = (int64_t)a.chunk * split;
  return make_int2((int)min(x, (int64_t)tiles), split == a.splits - 1 ? tiles : (int)min(x + a.chunk, (int64_t)tiles));
}

// Offsets (and key counts) that do not fit are reported by the launch's threads together, once.
__device__ __forceinline__ void check_rows(const Args& a, int tid) {
  if (!a.status) return;
  for (int64_t s = (int64_t)blockIdx.x * 256 + tid; s <= a.B; s += (int64_t)gridDim.x * 256) {
    const int64_t x = a.off[s];
    if ((s == 0 && x != 0) || (s == a.B && x != a.rows)) atomicOr(a.status, ERRBIT_ROWS);
    if (s < a.B) {
      const int64_t n = a.off[s + 1] - x;
      if (n < 0 || n > a.T_max) atomicOr(a.status, ERRBIT_LEN);
      if (a.lens && (a.lens[s] < 0 || a.lens[s] > a.len_max)) atomicOr(a.status, ERRBIT_KEYS);
    }
  }
  // here and not where a workgroup reads a program: a program without sequences, or all of them where prefix_max is 0, is read by none
  for (int64_t s = (int64_t)blockIdx.x * 256 + tid; s < a.programs; s += (int64_t)gridDim.x * 256)
    if (a.plens[s] < 0 || a.plens[s] > a.plen_max) atomicOr(a.status, ERRBIT_KEYS);
}

// The last sequence of [lo, hi] that starts at `row` or before, looked for by a wavefront's lanes together (the
// search never leaves [lo, hi], whatever the offsets are).
__device__ __forceinline__ int last_start(const int32_t* off, int lo, int hi, int row, int lane) {
  while (lo < hi) {
    const int step = (hi - lo + 63) >> 6, at = lo + step * (lane + 1);
    const int n = __popcll(__ballot(at <= hi && off[min(at, hi)] <= row));
    lo += step * n;
    hi = min(hi, lo + step - 1);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Bounds of the sequence of a row, within [first, end): a wavefront's rows ascend by lane.
// `from`: a sequence that starts at the wavefront's first row or before.
__device__ __forceinline__ int2 bounds_of(const Args& a, int from, int row, int last_row, int first, int end, int lane) {
  int hi = last_start(a.off, from, a.B - 1, last_row, lane), lo = from;
  while (__any(lo < hi)) {
    const int mid = (int)(((int64_t)lo + hi + 1) >> 1);
    if (lo < hi) {
      if (a.off[mid] <= row) lo = mid; else hi = mid - 1;
    }
  }
  return make_int2(min(max(a.off[lo], first), row), max(min(a.off[lo + 1], end), row + 1));
}

// Of n rows from q0 on those that some sequence has; rows behind the last one stay as they are and add nothing.
__device__ __forceinline__ int rows_before_end(const Args& a, int64_t q0, int n) {
  return (int)min(max((int64_t)a.off[a.B] - q0, (int64_t)0), (int64_t)n);
}

__device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1; }
__device__ __forceinline__ int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// A weight of 0 does not hide a value that is not finite from a product, and in a block of own keys that only some
// of the rows see, the others' weights are 0.  So a workgroup whose sums are not finite, and some of whose rows (or keys) do not see
// values that can have made them so, does its rows (or keys) again, one by one over what they see alone, as long as that is not NaN
// anyway.  It starts from its block's number, so that nothing is kept for it meanwhile.  (As a second form
// of the loops it took the first's registers: dk and dv at a width of 128 spilled 115 of them and took 3.6 ms for 1.7.  Launches behind
// the kernels', with a flag per workgroup, took 4.6 us each.  A training step of four sequences of 1500 rows, 32 heads on 8 of 128,
// whose values are all NaN takes 5.9 ms for 0.6, with one row of v that is NaN 9.8; each doing again whatever is not finite, to its
// last key, 82 and 37.)
template <int DB>
__device__ __forceinline__ bool not_finite(const f32x16 (&acc)[DB]) {
  float z = 0.0f;
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = fmaf(acc[b][r], 0.0f, z);
  return z != 0.0f;
}
__device__ __forceinline__ int formed_anew(int x) {
  asm volatile("" : "+s"(x));
  return x;
}

// Page of a table, checked; lanes past the tile's pages have none.
__device__ __forceinline__ int page_id(const Args& a, const int32_t* table, int entry, bool used) {
  if (!used) return -1;
  const int id = table[entry];
  if (id >= 0 && id < a.n_pages) return id;
  if (a.status) atomicOr(a.status, ERRBIT_PAGE);
  return -1;
}

// Rows of a matrix (stride ld elements) into a tile: the first n of them, others read as zero.  The buffer ends with the last
// row, so that what a lane adds to its base is the same for every tile.
template <class T, int DH, int ROWS, int NT>
__device__ __forceinline__ void copy_rows(const T* base, int ld, int n, T* tile, int tid) {
  using TL = Tile<T, DH>;
  constexpr int N = ROWS * TL::UPR / NT;
  n = min(n, ROWS);
  const u32x4 buf = buffer_of(base, n > 0 ? (uint32_t)(((n - 1) * ld + DH) * sizeof(T)) : 0u);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int row = (i * NT + tid) / TL::UPR, unit = ((i * NT + tid) % TL::UPR) ^ TL::swz(row);
    copy16(buf, tile + (size_t)(i * NT + (tid & ~63)) * TL::E, (uint32_t)(row * ld * sizeof(T) + unit * 16));
  }
}

// Two matrices' rows tile after tile: where the next tile begins, bytes from one to the next and of a whole one, what a lane
// adds to a tile's beginning and what each further copy of a tile adds to that.  A whole tile costs four scalar additions
// beside its copies (with everything formed anew a tile took 169 scalar instructions, as long as its
// products).  With lg > 0 a tile's
// rows are 2^lg heads of each row of the matrix (which divide the rows of a copy).
template <class T, int DH, int ROWS>
struct Stream {
  using TL = Tile<T, DH>;
  static constexpr int N = ROWS * TL::UPR / 256, STEP = 256 / TL::UPR;
  static constexpr int K = STEP >= 16 ? 1 : 2;        // the swizzle goes by a row's last 4 bits
  static_assert(STEP >= 8, "at most two patterns");
  uint64_t x, y;
  uint32_t next_x, next_y, step_x, step_y, last_x, last_y;
  uint32_t at_x[K], at_y[K];
  __device__ __forceinline__ void start(const T* px, int64_t ldx, const T* py, int64_t ldy, int tid, int lg = 0) {
    x = (uint64_t)px;
    y = (uint64_t)py;
    const uint32_t bx = (uint32_t)ldx * sizeof(T), by = (uint32_t)ldy * sizeof(T);
    next_x = (ROWS >> lg) * bx;
    next_y = (ROWS >> lg) * by;
    step_x = (STEP >> lg) * bx;
    step_y = (STEP >> lg) * by;
    const int row = tid / TL::UPR;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t in_row = (row & ((1 << lg) - 1)) * (uint32_t)(DH * sizeof(T)) + ((tid % TL::UPR) ^ TL::swz(row + k * STEP)) * 16;
      at_x[k] = (row >> lg) * bx + in_row;
      at_y[k] = (row >> lg) * by + in_row;
    }
    last_x = bx;                                      // bytes of n rows: (n / G - 1) last + G rows' widths
    last_y = by;
  }
  // the next tile, its first n > 0 rows (whole rows of the matrix), of them those of `vis` (where `some`)
  template <int NV>
  __device__ __forceinline__ void copy(T* tx, T* ty, int n, bool some, const uint64_t (&vis)[NV], int wave, int tid, int lg = 0) {
    const uint32_t rows = ((n < ROWS ? n : ROWS) >> lg) - 1, width = (uint32_t)(DH * sizeof(T)) << lg;
    const u32x4 bx = buffer_of((const void*)x, rows * last_x + width), by = buffer_of((const void*)y, rows * last_y + width);
    if (!some) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        copy16(bx, tx + (i * 256 + wave * 64) * TL::E, at_x[i % K], i * step_x);
        copy16(by, ty + (i * 256 + wave * 64) * TL::E, at_y[i % K], i * step_y);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = (i * 256 + tid) / TL::UPR;
        const bool see = (vis[NV > 1 ? row >> 6 : 0] >> (row & 63)) & 1;
        copy16(bx, tx + (i * 256 + wave * 64) * TL::E, see ? at_x[i % K] : BAD, i * step_x);
        copy16(by, ty + (i * 256 + wave * 64) * TL::E, see ? at_y[i % K] : BAD, i * step_y);
      }
    }
    x += next_x;
    y += next_y;
  }
};

// Where a lane reads in the tiles of a workgroup (LDS bytes).  In bf16 the units of a row differ in their place by
// exclusive ors of constants, so two addresses and an instruction per read serve in place of one register each.
template <class T, int DH>
struct Reads {
  using TL = Tile<T, DH>;
  typedef __attribute__((address_space(3))) const u32x4 lds_unit;
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  uint32_t row, col;
  __device__ __forceinline__ void start(const T* lds, int lane) {
    const uint32_t base = (uint32_t)(uintptr_t)(lds_void*)const_cast<T*>(lds);
    const int h = lane >> 5, r = lane & 31, c = 4 * h + ((lane >> 2) & 3);
    row = base + r * DH * 2 + ((h ^ TL::swz(r)) * 16);
    col = base + c * DH * 2 + (((2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ TL::swz(c)) * 16) + 8 * (lane & 1);
  }
  // Tile::mm_row and mm_col of the block at byte OFF (a multiple of 32 rows) of the workgroup's tiles
  // (op: its registers, the last of which may be kept in LDS)
  template <int OFF, class Op>
  __device__ __forceinline__ f32x16 mm_row(Op op, f32x16 acc = f32x16{}) const {
#pragma unroll
    for (int i = 0; i < TL::NR; ++i) {
      const u32x4 u = *(lds_unit*)(uintptr_t)((row ^ (i * 32)) + OFF);
      acc = TL::mm_one(u, op(i), acc);
    }
    return acc;
  }
  template <int OFF>
  __device__ __forceinline__ void mm_col(const f32x16& p, f32x16 (&acc)[TL::DB]) const {
    constexpr int TURN = DH == 64 ? 16 : 32;          // row + 8: swz of its fourth bit
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      bf16x8 pf;
#pragma unroll
      for (int j = 0; j < 8; ++j) pf[j] = (__bf16)p[8 * f + j];
#pragma unroll
      for (int b = 0; b < TL::DB; ++b) {
        s16x4 half[2];
#pragma unroll
        for (int jj = 0; jj < 2; ++jj)
          half[jj] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_s16x4*)(uintptr_t)((col ^ (b * 64 ^ jj * TURN)) + (16 * f + 8 * jj) * DH * 2 + OFF));
        const s16x8 x = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), pf, acc[b], 0, 0, 0);
      }
    }
  }
};

// Keys [first, first + ROWS) of a page table, of which the first `len` exist, into a tile.  A page has at least 16
// slots and a tile starts at a multiple of its length, so the 16 or fewer rows that one
// instruction copies lie in one page, whose end (or the last key) bounds the buffer: rows past it
// read as zero.  ids: lane l has the tile's l-th page.
template <class T, int DH, int ROWS>
__device__ __forceinline__ void copy_pages(const Args& a, int hk, T* kt, T* vt, int first, int len, int ids, int wave, int lane) {
  using TL = Tile<T, DH>;
  constexpr int N = ROWS * TL::UPR / 256, RPI = 64 / TL::UPR;
  constexpr uint32_t ROW = DH * sizeof(T);
  const int slots = 1 << a.lps;
  auto place = [&](int id, int row) {
    return ((((uint64_t)(uint32_t)max(id, 0) * (uint32_t)a.kv_heads + (uint32_t)hk) << a.lps) + ((first + row) & (slots - 1))) * ROW;
  };
  const uint32_t unit_of = (uint32_t)(lane / TL::UPR) * ROW;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r0 = (i * 256 + wave * 64) / TL::UPR;                  // the instruction's first row
    const int id = lane_of(ids, r0 >> a.lps);
    const uint32_t size = id < 0 ? 0 : min(max(len - first - r0, 0), RPI) * ROW;
    const uint64_t at = place(id, r0);
    const uint32_t vo = unit_of + ((lane % TL::UPR) ^ TL::swz(r0 + lane / TL::UPR)) * 16;
    copy16(buffer_of(static_cast<const uint8_t*>(a.k) + at, size), kt + (i * 256 + wave * 64) * TL::E, vo);
    copy16(buffer_of(static_cast<const uint8_t*>(a.v) + at, size), vt + (i * 256 + wave * 64) * TL::E, vo);
  }
}

// A wavefront's own block of 32 keys (or rows): from key `first` of a run on, n of them exist.  Paged: its one or two pages;
// their numbers come through scalar loads, which the copies' count of outstanding loads does not see.
struct Block {
  int first, n, id0, id1;
};
__device__ __forceinline__ Block paged_block(const Args& a, const int32_t* table, int first, int n, int lane) {
  Block b = {__builtin_amdgcn_readfirstlane(first), __builtin_amdgcn_readfirstlane(min(max(n, 0), 32)), -1, -1};
  if (b.n > 0) {
    const __attribute__((address_space(4))) int32_t* ids = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)table;
    b.id0 = ids[b.first >> a.lps];
    b.id1 = ids[(b.first + b.n - 1) >> a.lps];
    if ((b.id0 < 0 || b.id0 >= a.n_pages || b.id1 < 0 || b.id1 >= a.n_pages) && a.status && lane == 0) atomicOr(a.status, ERRBIT_PAGE);
  }
  return b;
}
// Where the block's halves of 16 keys lie in the caches, each in one page (a block starts at a multiple of 32), and their bytes.
struct Place {
  uint64_t at[2];
  uint32_t size[2];
};
template <class T, int DH>
__device__ __forceinline__ Place place_of(const Args& a, int hk, const Block& b) {
  constexpr uint32_t ROW = DH * sizeof(T);
  Place p;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int id = half ? b.id1 : b.id0;
    const bool ok = id >= 0 && id < a.n_pages;
    const uint64_t page = (uint64_t)(uint32_t)(ok ? id : 0) * (uint32_t)a.kv_heads + (uint32_t)hk;
    p.at[half] = ((page << a.lps) + ((b.first + 16 * half) & ((1 << a.lps) - 1))) * ROW;
    p.size[half] = ok ? min(max(b.n - 16 * half, 0), 16) * ROW : 0;
  }
  return p;
}
template <class T, int DH>
__device__ __forceinline__ void copy_block(const void* cache, const Place& p, T* tile, int lane) {
  using TL = Tile<T, DH>;
  constexpr int N = 32 * TL::UPR / 64, RPI = 64 / TL::UPR;
  constexpr uint32_t ROW = DH * sizeof(T);
  static_assert(RPI <= 16, "an instruction's rows lie in one half");
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const u32x4 buf = buffer_of(static_cast<const uint8_t*>(cache) + p.at[half], p.size[half]);
#pragma unroll
    for (int i = half * N / 2; i < (half + 1) * N / 2; ++i) {
      const int r = lane / TL::UPR, unit = (lane % TL::UPR) ^ TL::swz(i * RPI + r);
      copy16(buf, tile + (size_t)i * 64 * TL::E, (uint32_t)(r * ROW + unit * 16), (uint32_t)(i * RPI % 16) * ROW);
    }
  }
}

// Scores of 32 keys to weights against the running maximum of a lane's row, with its sum and accumulators brought along.
template <class T, int DB>
__device__ __forceinline__ void weigh(f32x16& s, float& mx, float& sum, f32x16 (&acc)[DB], float c2) {
  float bm = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) bm = fmaxf(bm, s[r]);
  bm = pair_max(bm);
  const float f = bm > mx ? exp2_of(log2_units<T>(mx - bm, c2)) : 1.0f;
  mx = bm > mx ? bm : mx;
  const float mc = mx == -INFINITY ? 0.0f : log2_units<T>(mx, c2);            // only keys of weight 0 so far
  float bs = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    s[r] = weight<T>(s[r], c2, mc);
    bs += s[r];
  }
  sum = fmaf(sum, f, bs);
  if (__any(f != 1.0f)) {
#pragma unroll
    for (int b = 0; b < DB; ++b) acc[b] *= f;
  }
}
// Values of a lane's column where bit acc_row(0, r) of its half of `seen` is set, `other` elsewhere.
__device__ __forceinline__ void only(f32x16& s, uint32_t seen, float other, int h) {
  uint32_t m = seen >> (4 * h);
  asm volatile("" : "+v"(m));                 // where this is under a condition it stays a branch: 48 instructions
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = (m >> acc_row(0, r)) & 1 ? s[r] : other;
}

// RAGGED: sequences that differ so much that as many tiles for each as for the longest would be more than their rows' and one for each
// (1024 single steps with a chunk of 300 rows, 12 heads of 64: 352 us with the longest's for each, 133 so; of 4000 rows 2227 and 618).
// Sequence i of the launch has the slots from floor((off[i] - off[0]) G / rows) + i on, of which there are always enough for its tiles
// before the next one's.  (A form of its own: in the common one it cost single steps and chunks 1%.)  `sequence_of_slot`: the last
// sequence that begins at the slot or before.
__device__ __forceinline__ int first_slot(const Args& a, int rows, int i) {
  const int64_t x = (int64_t)a.off[a.seq0 + i] - a.off[a.seq0];
  return (int)min(max(x * a.G / rows, (int64_t)0), (int64_t)a.slots) + i;
}
__device__ __forceinline__ int sequence_of_slot(const Args& a, int rows, int slot, int lane) {
  int lo = 0, hi = a.nseq - 1;
  while (lo < hi) {
    const int step = (hi - lo + 63) >> 6, at = lo + step * (lane + 1);
    const int n = __popcll(__ballot(at <= hi && first_slot(a, rows, min(at, hi)) <= slot));
    lo += step * n;
    hi = min(hi, lo + step - 1);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// A workgroup's rows (stacked rows of one key head from packed row q0 on, a tile of them), the program's keys and
// own keys [o0, o1) that some row of the tile sees.  Those before `rest` come in whole tiles of KB, which the rows of the tile's
// first sequence see (the paged forms' only one); of those from there on, about as many as the tile has queries, every
// wavefront takes what its own rows see.
struct Work {
  int64_t q0, p0;                           // p0: dense, the program's first key row
  int R, hk, tile, split, P, o0, rest, o1;
  int seq;                                  // dense: the sequence of the tile's first row
  int before;                               // paged: row i of the sequence sees before + i + 1 own keys
  const int32_t *own_table, *shared_table;  // paged
};
template <bool PAGED, bool RAGGED = false>
__device__ __forceinline__ bool work_of(const Table& t, const Args& a, int block, int blocks, int rows, int KB, int lane, Work& w) {
  w.p0 = w.o0 = w.rest = w.o1 = w.seq = 0;
  w.own_table = w.shared_table = nullptr;
  if constexpr (!PAGED) {
    Prob p;
    if (!problem<false>(t, a, rows, p, block)) return false;
    w.q0 = p.q0; w.p0 = p.k0; w.hk = p.hk; w.split = p.split; w.P = p.Lk;
    w.tile = (p.R + rows - 1) / rows - 1 - p.tile;            // the longest loops first
    w.R = rows_before_end(a, p.q0, p.R / a.G) * a.G;
    if (w.tile * rows >= w.R) return false;
    const int first = p.q0 + w.tile * rows / a.G;
    w.seq = last_start(a.off, 0, a.B - 1, first, lane);
    w.o0 = min(max(a.off[w.seq], p.q0), first);
    w.rest = w.o0 + (first + 1 - w.o0) / KB * KB;
    w.o1 = p.q0 + (min((w.tile + 1) * rows, w.R) - 1) / a.G + 1;
  } else {
    int64_t n;
    int seg = -1, seen = 0;
    if (a.row_tiles) {
      int at = xcd_tile(block, blocks);
      w.split = at % a.splits; at /= a.splits;
      int s;
      if constexpr (RAGGED) {
        w.hk = at / a.slots; at -= w.hk * a.slots;
        s = sequence_of_slot(a, rows, at, lane);
        at -= first_slot(a, rows, s);
        s += a.seq0;
      } else {
        w.tile = a.row_tiles - 1 - at % a.row_tiles; at /= a.row_tiles;
        s = a.seq0 + at % a.nseq;
        w.hk = at / a.nseq;
      }
      const int64_t x = a.off[s], y = a.off[s + 1];
      w.q0 = min(max(x, (int64_t)0), a.rows);
      n = min(min(max(y, w.q0), a.rows) - w.q0, (int64_t)a.T_max);
      if constexpr (RAGGED) {
        w.tile = (int)((n * a.G + rows - 1) / rows) - 1 - at;                 // the longest loops first
        if (w.tile < 0) return false;
      }
      int g = 0, gh = t.n - 1;                                // the sequence's program
      while (g < gh) {
        const int mid = (g + gh + 1) >> 1;
        if (t.seg[mid].q0 <= s) g = mid; else gh = mid - 1;
      }
      if (a.joint) seg = t.seg[g].k0;
      w.own_table = a.pages + (int64_t)s * a.max_pages;
      seen = min(max(a.lens[s], 0), a.len_max);
    } else {
      Prob p;
      if (!problem<false>(t, a, rows, p, block)) return false;
      w.hk = p.hk; w.tile = p.tile; w.split = p.split; seg = p.k0;
      const int64_t x = a.off[p.q0], y = a.off[p.q0 + p.Lk];
      w.q0 = min(max(x, (int64_t)0), a.rows);
      n = min(min(max(y, w.q0), a.rows) - w.q0, (int64_t)(p.R / a.G));
    }
    w.R = (int)n * a.G;
    if (w.tile * rows >= w.R) return false;
    w.before = a.row_tiles ? seen - (int)n : INT32_MIN / 2;
    w.o1 = max(w.before + (min((w.tile + 1) * rows, w.R) - 1) / a.G + 1, 0);
    w.rest = max(w.before + w.tile * rows / a.G + 1, 0) / KB * KB;
    w.P = 0;
    if (seg >= 0) {
      w.P = min(max(a.plens[seg], 0), a.plen_max);
      w.shared_table = a.ppages + (int64_t)seg * a.max_ppages;
    }
  }
  return true;
}

// 128 keys of a segment (of its n from row k0 on), and the stacked rows [x0, x1) from row q0 on that see one of them: OWN, its
// own keys (each seen by the rows from its own to its sequence's last), or the program's.
struct KeyWork {
  int64_t q0, k0;
  int n, first, hk, split, seq, x0, x1, t0, t1;
};
template <bool OWN>
__device__ __forceinline__ bool key_work_of(const Table& t, const Args& a, int block, int rows, int lane, KeyWork& w) {
  Prob p;
  if (!problem<true>(t, a, 128, p, block)) return false;
  w.q0 = p.q0; w.k0 = p.k0; w.n = p.Lk; w.first = p.tile * 128; w.hk = p.hk; w.split = p.split;
  w.x0 = w.seq = 0;
  w.x1 = p.R > 0 ? rows_before_end(a, p.q0, p.R / a.G) * a.G : 0;
  if constexpr (OWN) {
    w.n = rows_before_end(a, p.q0, w.n);
    if (w.first >= w.n) return false;
    const int last = min(w.first + 128, w.n) - 1;
    w.seq = last_start(a.off, 0, a.B - 1, p.q0 + w.first, lane);
    const int s = last_start(a.off, w.seq, a.B - 1, p.q0 + last, lane);
    w.x0 = w.first * a.G;
    w.x1 = (max(min(a.off[s + 1], p.q0 + w.n), p.q0 + last + 1) - p.q0) * a.G;
  }
  const int2 tt = share_of(a, (w.x1 - w.x0 + rows - 1) / rows, w.split);
  w.t0 = tt.x;
  w.t1 = tt.y;
  return true;
}

// --------------------------------------------------------------------------
// Workgroups whose sums are not finite, again: a wavefront takes every fourth row (key) of the workgroup's and its lanes
// 64 of the keys (rows) that it sees at a time, then its features.
__device__ __forceinline__ float wave_max(float v) {
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
template <class T>
__device__ __forceinline__ float dot(const T* x, const T* y, int n) {
  float d = 0.0f;
  for (int i = 0; i < n; ++i) d = fmaf((float)x[i], (float)y[i], d);
  return d;
}
// Features lane and lane + 64 of the lanes' rows base + at, weighted by their w, one after the other.
template <class T, int DH>
__device__ __forceinline__ void add_rows(float& lower, float& upper, float w, uint64_t used, const T* base, int64_t at, int lane) {
  for (int i = 0; i < 64; ++i) {
    if (!((used >> i) & 1)) continue;
    const float wi = __shfl(w, i);
    const T* x = base + __shfl(at, i);
    if (lane < DH) lower = fmaf(wi, (float)x[lane], lower);
    if (DH > 64) upper = fmaf(wi, (float)x[lane + 64], upper);
  }
}
template <class T, int DH>
__device__ __forceinline__ void store_lane(T* row, float lower, float upper, int lane) {
  if (lane < DH) row[lane] = (T)lower;
  if (DH > 64) row[lane + 64] = (T)upper;
}
// A NaN stays one, whatever is added: a loop whose sums are all NaN can end.
template <int DH>
__device__ __forceinline__ bool all_nan(float lower, float upper, int lane) {
  return __all((lane >= DH || lower != lower) && (DH <= 64 || upper != upper));
}
// Whether one of the rows [first, end), `row` gives their addresses (null: none), holds a value that is not below `limit` (as NaN is not).
template <class T, int DH, class Row>
__device__ __forceinline__ bool any_beyond(int first, int end, float limit, int lane, Row row) {
  using TL = Tile<T, DH>;
  typedef T unit __attribute__((ext_vector_type(TL::E)));
  constexpr int RPI = 64 / TL::UPR, AHEAD = 4;
  bool beyond = false;
  for (int at = first; at < end && !__any(beyond); at += AHEAD * RPI) {
    unit x[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const T* p = row(min(at + i * RPI + lane / TL::UPR, end - 1));
      x[i] = p ? *reinterpret_cast<const unit*>(p + (lane % TL::UPR) * TL::E) : unit{};
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
      for (int e = 0; e < TL::E; ++e) beyond |= !(fabsf((float)x[i][e]) < limit);
  }
  return __any(beyond);
}
// Element of key i of a run (its program's, or own) in k or v; -1: its page does not exist, it reads as zero.
template <int DH, bool PAGED>
__device__ __forceinline__ int64_t key_at(const Args& a, const Work& w, bool own, int i, bool value) {
  if constexpr (PAGED) {
    const int id = (own ? w.own_table : w.shared_table)[i >> a.lps];
    if (id < 0 || id >= a.n_pages) return -1;
    return ((((int64_t)id * a.kv_heads + w.hk) << a.lps) + (i & ((1 << a.lps) - 1))) * DH;
  } else {
    return (own ? i * (value ? a.ld_v : a.ld_k) : (w.p0 + i) * (value ? a.ld_pv : a.ld_pk)) + w.hk * DH;
  }
}

// The part of the loop that a workgroup has, in keys of the program and own keys.
struct Span {
  int p_lo, p_hi, o_lo, o_hi;
};
__device__ __forceinline__ Span span_of(const Args& a, const Work& w, int KB) {
  const int nP = (w.P + KB - 1) / KB, tiles = nP + (w.rest - w.o0) / KB;
  const int2 tt = share_of(a, tiles, w.split);
  const int t0 = tt.x, t1 = tt.y, last = a.counts ? shares_of(a, tiles) - 1 : a.splits - 1;
  return {min(t0, nP) * KB, min(min(t1, nP) * KB, w.P), w.o0 + max(t0 - nP, 0) * KB, w.split == last ? w.o1 : w.o0 + max(t1 - nP, 0) * KB};
}
// Own keys that a row sees.
template <bool PAGED>
__device__ __forceinline__ int2 seen_by(const Args& a, const Work& w, int row, int lane) {
  if constexpr (PAGED) {
    return make_int2(0, max(w.before + row / a.G + 1, 0));
  } else {
    const int qrow = (int)w.q0 + row / a.G, s = last_start(a.off, w.seq, a.B - 1, qrow, lane);
    return make_int2(min(max(a.off[s], (int)w.q0), qrow), qrow + 1);
  }
}

template <class T, int DH, bool PAGED, bool RAGGED>
__device__ __forceinline__ void forward_again(const Table& t, const Args& a, int block, int blocks, int rows, int KB) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Work w;
  if (!work_of<PAGED, RAGGED>(t, a, formed_anew(block), blocks, rows, KB, lane, w)) return;
  if (rows == 32 && PAGED) w.rest = (w.o1 + KB - 1) / KB * KB;         // the few-row kernel's: all keys in tiles
  const Span sp = span_of(a, w, KB);
  for (int row = w.tile * rows + wave; row < min((w.tile + 1) * rows, w.R); row += 4) {
    const int head = w.hk * a.G + row % a.G;
    const int64_t qrow = w.q0 + row / a.G, orow = qrow * a.heads + head;
    const T* q = static_cast<const T*>(a.q) + qrow * a.ld_q + head * DH;
    const int2 see = seen_by<PAGED>(a, w, row, lane);
    float top = -INFINITY, sum = 0.0f, x = 0.0f, y = 0.0f;
    for (int own = 0; own < 2 && sum == sum; ++own) {
      const T* kb = static_cast<const T*>(own || PAGED ? a.k : a.pk);
      const T* vb = static_cast<const T*>(own || PAGED ? a.v : a.pv);
      const int end = own ? min(sp.o_hi, see.y) : sp.p_hi;
      for (int i0 = own ? max(sp.o_lo, see.x) : sp.p_lo; i0 < end; i0 += 64) {
        const int i = i0 + lane;
        const bool shown = i < end && (own || PAGED || !a.mask || a.mask[w.p0 + i] != 0);
        const int64_t at = shown ? key_at<DH, PAGED>(a, w, own, i, false) : -1, vat = shown ? key_at<DH, PAGED>(a, w, own, i, true) : -1;
        const float s = !shown ? -INFINITY : at < 0 ? 0.0f : dot(q, kb + at, DH) * a.c2;
        const float m = wave_max(s), f = m > top ? exp2_of(top - m) : 1.0f;
        top = m > top ? m : top;
        const float p = shown ? exp2_of(s - (top == -INFINITY ? 0.0f : top)) : 0.0f;
        sum = sum * f + wave_sum(p);
        x *= f;
        y *= f;
        if (sum != sum) break;
        if (!all_nan<DH>(x, y, lane)) add_rows<T, DH>(x, y, p, __ballot(vat >= 0), vb, vat, lane);
      }
    }
    if (a.parts > 1) {
      const int64_t prow = (int64_t)(a.part0 + w.split) * a.part_rows + orow;
      store_lane<float, DH>(a.part + prow * DH, x, y, lane);
      if (lane == 0) {
        a.part_ml[2 * prow] = top;
        a.part_ml[2 * prow + 1] = sum;
      }
    } else {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      store_lane<T, DH>(static_cast<T*>(a.out) + qrow * a.ld_out + head * DH, x * inv, y * inv, lane);
      if (a.lse && lane == 0) a.lse[orow] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
    }
  }
}

template <class T, int DH>
__device__ __forceinline__ void dq_again(const Table& t, const Args& a, const float2* stat) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Work w;
  if (!work_of<false>(t, a, formed_anew(blockIdx.x), gridDim.x, 128, TILE_ROWS<T, DH>, lane, w)) return;
  const Span sp = span_of(a, w, TILE_ROWS<T, DH>);
  for (int row = w.tile * 128 + wave; row < min((w.tile + 1) * 128, w.R); row += 4) {
    const int head = w.hk * a.G + row % a.G;
    const int64_t qrow = w.q0 + row / a.G, orow = qrow * a.heads + head;
    const T* q = static_cast<const T*>(a.q) + qrow * a.ld_q + head * DH;
    const T* g = static_cast<const T*>(a.d_o) + qrow * a.ld_do + head * DH;
    const int2 see = seen_by<false>(a, w, row, lane);
    const float l2 = stat[row - 128 * w.tile].x, delta = stat[row - 128 * w.tile].y;
    float x = 0.0f, y = 0.0f;
    for (int own = 0; own < 2; ++own) {
      const T* kb = static_cast<const T*>(own ? a.k : a.pk);
      const T* vb = static_cast<const T*>(own ? a.v : a.pv);
      const int end = own ? min(sp.o_hi, see.y) : sp.p_hi;
      for (int i0 = own ? max(sp.o_lo, see.x) : sp.p_lo; i0 < end && !all_nan<DH>(x, y, lane); i0 += 64) {
        const int i = i0 + lane;
        const bool shown = i < end && (own || !a.mask || a.mask[w.p0 + i] != 0);
        const int64_t at = shown ? key_at<DH, false>(a, w, own, i, false) : 0;
        float ds = 0.0f;
        if (shown) ds = exp2_of(fmaf(dot(q, kb + at, DH), a.c2, -l2)) * (dot(g, vb + key_at<DH, false>(a, w, own, i, true), DH) - delta);
        add_rows<T, DH>(x, y, ds, __ballot(shown), kb, at, lane);
      }
    }
    x *= a.scale;
    y *= a.scale;
    if (a.splits > 1) store_lane<float, DH>(a.part + (w.split * a.part_rows + orow) * DH, x, y, lane);
    else store_lane<T, DH>(static_cast<T*>(a.out) + qrow * a.ld_out + head * DH, x, y, lane);
  }
}

// Whether rows that only some of a wavefront's keys see, in the blocks that it took, can have spoilt its sums: values that are not
// finite, and such that a score that starts from -infinity may overflow the other way.
template <class T, int DH>
__device__ __forceinline__ bool dkv_spoilt(const Args& a, const KeyWork& w, int lo_a, int lo_z, int hi_a, int hi_z, int wave, int lane) {
  constexpr float LARGE = 0x1p56f;            // 128 products of two such stay finite
  const int key = w.first + 32 * wave, keys = min(key + 32, w.n);
  const float c2 = IS_BF<T> ? 1.0f : fmaxf(a.c2, 1.0f);                 // float32 keys are scaled
  if (any_beyond<T, DH>(key, keys, LARGE / c2, lane, [&](int i) { return static_cast<const T*>(a.k) + (w.q0 + i) * a.ld_k + w.hk * DH; }) ||
      any_beyond<T, DH>(key, keys, LARGE, lane, [&](int i) { return static_cast<const T*>(a.v) + (w.q0 + i) * a.ld_v + w.hk * DH; }))
    return true;
  auto rows = [&](int first, int end) {
    bool stat = false;
    for (int x = first + lane; __any(x < end); x += 64) {
      const float* at = a.stat + 2 * ((w.q0 + min(x, end - 1) / a.G) * a.heads + w.hk * a.G + min(x, end - 1) % a.G);
      stat |= !(fabsf(at[0]) < INFINITY) || !(fabsf(at[1]) < INFINITY);
    }
    return __any(stat) ||
           any_beyond<T, DH>(first, end, LARGE, lane, [&](int x) { return static_cast<const T*>(a.q) + (w.q0 + x / a.G) * a.ld_q + (w.hk * a.G + x % a.G) * DH; }) ||
           any_beyond<T, DH>(first, end, LARGE, lane, [&](int x) { return static_cast<const T*>(a.d_o) + (w.q0 + x / a.G) * a.ld_do + (w.hk * a.G + x % a.G) * DH; });
  };
  const int begin = w.x0 + w.t0 * TILE_ROWS<T, DH>, end = min(w.x0 + w.t1 * TILE_ROWS<T, DH>, w.x1);
  return rows(max(w.x0 + (lo_a - w.x0) / 32 * 32, begin), min(lo_z, end)) || rows(max(hi_a, begin), min(w.x0 + (hi_z - w.x0 + 31) / 32 * 32, end));
}

template <class T, int DH>
__device__ __forceinline__ void dkv_again(const Table& t, const Args& a, bool with_v) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  KeyWork w;
  if (!key_work_of<true>(t, a, formed_anew(blockIdx.x), TILE_ROWS<T, DH>, lane, w)) return;
  for (int key = w.first + wave; key < min(w.first + 128, w.n); key += 4) {
    const int64_t krow = w.q0 + key;
    const T* k = static_cast<const T*>(a.k) + krow * a.ld_k + w.hk * DH;
    const T* v = static_cast<const T*>(a.v) + krow * a.ld_v + w.hk * DH;
    const int s = last_start(a.off, w.seq, a.B - 1, (int)krow, lane);
    const int hi = (max(min(a.off[s + 1], (int)w.q0 + w.n), (int)krow + 1) - (int)w.q0) * a.G;
    const int end = min(min(w.x0 + w.t1 * TILE_ROWS<T, DH>, w.x1), hi);
    float kx = 0.0f, ky = 0.0f, vx = 0.0f, vy = 0.0f;
    for (int x0 = max(w.x0 + w.t0 * TILE_ROWS<T, DH>, key * a.G); x0 < end && !(all_nan<DH>(kx, ky, lane) && (!with_v || all_nan<DH>(vx, vy, lane))); x0 += 64) {
      const int x = min(x0 + lane, end - 1), head = w.hk * a.G + x % a.G;
      const int64_t qrow = w.q0 + x / a.G, orow = qrow * a.heads + head;
      const int64_t qat = qrow * a.ld_q + head * DH, gat = qrow * a.ld_do + head * DH;
      const T* q = static_cast<const T*>(a.q);
      const T* g = static_cast<const T*>(a.d_o);
      const float p = exp2_of(fmaf(dot(q + qat, k, DH), a.c2, -a.stat[2 * orow]));
      const float ds = p * (dot(g + gat, v, DH) - a.stat[2 * orow + 1]);
      const uint64_t used = __ballot(x0 + lane < end);
      if (with_v) add_rows<T, DH>(vx, vy, p, used, g, gat, lane);
      add_rows<T, DH>(kx, ky, ds, used, q, qat, lane);
    }
    kx *= a.scale;
    ky *= a.scale;
    if (a.splits > 1) {
      const int64_t prow = krow * a.kv_heads + w.hk;
      store_lane<float, DH>(a.part + ((2 * w.split) * a.part_rows + prow) * DH, kx, ky, lane);
      if (with_v) store_lane<float, DH>(a.part + ((2 * w.split + 1) * a.part_rows + prow) * DH, vx, vy, lane);
    } else {
      store_lane<T, DH>(static_cast<T*>(a.out) + krow * a.ld_out + w.hk * DH, kx, ky, lane);
      if (with_v) store_lane<T, DH>(static_cast<T*>(a.out2) + krow * a.ld_out2 + w.hk * DH, vx, vy, lane);
    }
  }
}

// --------------------------------------------------------------------------
// Forward: o = sum P v / sum P, P = exp(S - m), S = scale q k, m the running maximum.  A workgroup of 4 wavefronts takes 128 / WK
// rows (32 per wavefront); WK wavefronts share rows and take every WK-th block of 32 keys.  Tiles of K and V are staged two deep;
// softmax online (wm_attend.hip).  PAGED: the launch goes by programs (the rows of all its sequences, the program's keys
// only) or by sequences (row_tiles > 0: its own keys, after the program's if it has any).
// What bounds it is the vector unit, 64% busy at a width of 64 beside matrix cores at 34% (16 bits; 33324 rows on 256 to 2048 keys
// 174 us, 628 TFLOP/s; 183 with three wavefronts per SIMD for four); at 128 both, 38 and 41% (830 TFLOP/s causal).
template <class T, int DH, int WK>
constexpr int FWD_PER_CU = IS_BF<T> && DH == 64 && WK == 1 ? 4 : 4 * (WK > 1 ? 32 * WK : TILE_ROWS<T, DH>) * DH * (int)sizeof(T) <= 80 * 1024 ? 2 : 1;
template <class T, int DH, int WK, bool PAGED, bool RAGGED = false>
__global__ __launch_bounds__(256, (FWD_PER_CU<T, DH, WK>)) void forward_kernel(const Table t, const Args a) {
  using TL = Tile<T, DH>;
  constexpr int WR = 4 / WK, DB = TL::DB;
  constexpr int KB = WK > 1 ? 32 * WK : TILE_ROWS<T, DH>;     // keys per tile
  constexpr int NV = (KB + 63) / 64;                          // visibility words per tile
  constexpr int NB = KB / 32 / WK;                            // blocks of 32 keys of a wavefront in a tile
  __shared__ __attribute__((aligned(16))) T lds[4 * KB * DH];
  T* const ks = lds;                                          // [2][KB][DH]
  T* const vs = lds + 2 * KB * DH;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, wr = wave % WR, wk = wave / WR;
  if (a.part0 == 0) check_rows(a, tid);

  Work w;
  if (!work_of<PAGED, RAGGED>(t, a, blockIdx.x, gridDim.x, 32 * WR, KB, lane, w)) return;
  const int64_t q0 = w.q0, p0 = w.p0;
  const int R = w.R, hk = w.hk, tile = w.tile, split = w.split, P = w.P, o0 = w.o0, rest = w.rest, o1 = w.o1;
  const int row = tile * (32 * WR) + wr * 32 + (lane & 31);   // may pass R: computed, not stored
  const int rr = min(row, R - 1), head = hk * a.G + rr % a.G;
  const int64_t qrow = q0 + rr / a.G;
  typename TL::Op qf;
  TL::load_op(qf, static_cast<const T*>(a.q) + qrow * a.ld_q + head * DH, h);
  TL::scale_op(qf, a.c2);
  int lo = 0, hi;                                             // the own keys that the lane's row sees
  if constexpr (!PAGED) {
    lo = bounds_of(a, w.seq, (int)qrow, lane_of((int)qrow, 31), (int)q0, (int)q0 + R / a.G, lane).x;
    hi = (int)qrow + 1;
  } else {
    hi = max(w.before + rr / a.G + 1, 0);
  }
  const int lo_a = lane_of(lo, 0), lo_z = lane_of(lo, 31), hi_a = lane_of(hi, 0), hi_z = lane_of(hi, 31);

  const int nP = (P + KB - 1) / KB, tiles = nP + (rest - o0) / KB;
  const int2 tt = share_of(a, tiles, split);
  const int t0 = tt.x, t1 = tt.y;
  const uint8_t* mask = !PAGED && a.mask ? a.mask + p0 : nullptr;
  // What a tile's copy needs from memory, loaded a tile ahead: mask bytes, or page numbers (lane l: page l).
  int pre[NV];
  auto look_ahead = [&](int ti) {
    if constexpr (PAGED) {
      const bool own = ti >= nP;
      const int first = (own ? ti - nP : ti) * KB, len = own ? rest : P;
      const int entry = (first >> a.lps) + lane;
      pre[0] = page_id(a, own ? w.own_table : w.shared_table, entry, lane < max(KB >> a.lps, 1) && ((int64_t)entry << a.lps) < len);
    } else if (mask && ti < nP) {
#pragma unroll
      for (int w = 0; w < NV; ++w) {
        const int key = ti * KB + 64 * w + lane;
        pre[w] = (KB >= 64 || lane < KB) && key < P ? mask[key] : 0;
      }
    }
  };
  uint64_t vis[NV], next[NV];                                 // with a mask: the tile's keys that are shown
#pragma unroll
  for (int w = 0; w < NV; ++w) vis[w] = next[w] = 0;
  Stream<T, DH, KB> rows;
  auto copy = [&](int ti, uint64_t (&v)[NV], T* kt, T* vt) {
    const bool own = ti >= nP;
    if constexpr (PAGED) {
      copy_pages<T, DH, KB>(a, hk, kt, vt, (own ? ti - nP : ti) * KB, own ? rest : P, pre[0], wave, lane);
    } else {
      if (ti == nP || ti == t0) {
        const int64_t first = own ? (int64_t)o0 + (int64_t)(ti - nP) * KB : p0 + (int64_t)ti * KB;
        const int64_t lk = own ? a.ld_k : a.ld_pk, lv = own ? a.ld_v : a.ld_pv;
        rows.start(static_cast<const T*>(own ? a.k : a.pk) + first * lk + hk * DH, lk,
                   static_cast<const T*>(own ? a.v : a.pv) + first * lv + hk * DH, lv, tid);
      }
      if (mask && !own) {
#pragma unroll
        for (int w = 0; w < NV; ++w) v[w] = __ballot(pre[w] != 0);
      }
      rows.copy(kt, vt, own ? KB : min(P - ti * KB, KB), mask && !own, v, wave, tid);
    }
  };

  f32x16 acc[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b] = f32x16{};
  float mx = -INFINITY, sum = 0.0f;
  bool started = false;                       // every row has a maximum
  if (t0 < t1) {
    look_ahead(t0);
    copy(t0, vis, ks, vs);
    if (t0 + 1 < t1) look_ahead(t0 + 1);
  }
  // a tile; the buffer it is in is known when the kernel is compiled, so that the reads' addresses stay in registers
  auto step = [&](int ti, auto buffer) {
    constexpr int BUF = decltype(buffer)::value;
    wait_counts<0, true>();
    raw_barrier();
    if (ti + 1 < t1) {
      copy(ti + 1, next, ks + (BUF ^ 1) * KB * DH, vs + (BUF ^ 1) * KB * DH);
      if (ti + 2 < t1) look_ahead(ti + 2);
    }
    const T* kt = ks + BUF * KB * DH;
    const T* vt = vs + BUF * KB * DH;
    // All rows see all keys of the program that are shown, and an own tile is seen whole by the rows of the tile's
    // first sequence and not at all by the others.
    const bool own = ti >= nP;
    const int at = own ? o0 + (ti - nP) * KB : ti * KB;
    const bool all = own ? lo_z <= at : !mask && at + KB <= P, none = own && lo_a > at;
    if (!none) {
      f32x16 s[NB];
      float bs;
      bool look_for_max = !started || !all;
      // a second time, scores and all, with the maximum that the first lacked
      for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) s[kb] = TL::mm_row(kt, 32 * (kb * WK + wk), qf, lane);
        if (!all) {
#pragma unroll
          for (int kb = 0; kb < NB; ++kb) {
            const int base = 32 * (kb * WK + wk);
            const uint32_t seen = own ? (lo <= at ? ~0u : 0u) : mask ? (uint32_t)(vis[NV > 1 ? base >> 6 : 0] >> (base & 63)) : below(P - at - base);
            uint32_t m = seen >> (4 * h);
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
        const float mc = mx == -INFINITY ? 0.0f : log2_units<T>(mx, a.c2);    // only keys of weight 0 so far
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
    }
    if (mask) {
#pragma unroll
      for (int w = 0; w < NV; ++w) vis[w] = next[w];
    }
  };
  for (int ti = t0; ti < t1; ti += 2) {
    step(ti, std::integral_constant<int, 0>{});
    if (ti + 1 < t1) step(ti + 1, std::integral_constant<int, 1>{});
  }
  if (split == a.splits - 1 && rest < o1) {
    // What is left of the own keys, without barriers: K and V of 32 keys per wavefront (one buffer for both in turn
    // where a tile has 32 rows).
    constexpr bool TWO = KB >= 64;
    constexpr int N = 32 * TL::UPR / 64;
    __syncthreads();
    T* const kt = lds + wave * KB * DH;
    T* const vt = TWO ? kt + 32 * DH : kt;
    const int end = min(hi_z, o1);
    auto block_of = [&](int first) -> Block {
      if constexpr (PAGED) return paged_block(a, w.own_table, first, end - first, lane);
      else return {first, min(max(end - first, 0), 32), 0, 0};
    };
    Place place;
    auto copy_k = [&](const Block& b) {
      if constexpr (PAGED) {
        place = place_of<T, DH>(a, hk, b);
        copy_block<T, DH>(a.k, place, kt, lane);
      }
      else copy_rows<T, DH, 32, 64>(static_cast<const T*>(a.k) + b.first * a.ld_k + hk * DH, (int)a.ld_k, b.n, kt, lane);
    };
    auto copy_v = [&](const Block& b) {
      if constexpr (PAGED) copy_block<T, DH>(a.v, place, vt, lane);        // K's block
      else copy_rows<T, DH, 32, 64>(static_cast<const T*>(a.v) + b.first * a.ld_v + hk * DH, (int)a.ld_v, b.n, vt, lane);
    };
    Block now = block_of(max(lo_a, rest) + 32 * wk);
    if (now.n > 0) {
      copy_k(now);
      if (TWO) copy_v(now);
    }
    while (now.n > 0) {
      const Block after = block_of(now.first + 32 * WK);
      wait_counts<TWO ? N : 0, true>();                       // K is there
      f32x16 s = TL::mm_row(kt, 0, qf, lane);
      wait_counts<63, true>();
      if (!TWO) copy_v(now);
      else if (after.n > 0) copy_k(after);
      if (lo_z > now.first || hi_a < now.first + 32) only(s, below(hi - now.first) & ~below(lo - now.first), -INFINITY, h);
      weigh<T, DB>(s, mx, sum, acc, a.c2);
      if (TWO && after.n > 0) wait_counts<N, false>(); else wait_counts<0, false>();      // V is there
      TL::mm_col(vt, 0, s, acc, lane);
      wait_counts<63, true>();
      if (after.n > 0) {
        if (TWO) copy_v(after);
        else copy_k(after);
      }
      now = after;
    }
  }
  // only what some of a wavefront's rows do not see can have spoilt their sums
  auto spoilt = [&]() {
    auto row = [&](int i) -> const T* {
      const int64_t at = key_at<DH, PAGED>(a, w, true, i, true);
      return at < 0 ? nullptr : static_cast<const T*>(a.v) + at;
    };
    return any_beyond<T, DH>(lo_a, lo_z, INFINITY, lane, row) || any_beyond<T, DH>(hi_a, min(hi_z, o1), INFINITY, lane, row);
  };
  if (a.again && __syncthreads_or(__any(not_finite<DB>(acc)) && spoilt())) {
    forward_again<T, DH, PAGED, RAGGED>(t, a, blockIdx.x, gridDim.x, 32 * WR, KB);
    return;
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
    const float ref = top == -INFINITY ? 0.0f : top;
    float f = exp2_of(m2 - ref);
    sum *= f;
#pragma unroll
    for (int b = 0; b < DB; ++b) acc[b] *= f;
#pragma unroll
    for (int k = 1; k < WK; ++k) {
      const int w = (wr + WR * k) * 32 + (lane & 31);
      f = exp2_of(ml[2 * w] - ref);
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
  if (row >= R) return;
  const int64_t orow = qrow * a.heads + head;
  if (a.parts > 1) {
    const int64_t prow = (int64_t)(a.part0 + split) * a.part_rows + orow;
    if (sum != 0.0f) store_cols<float, DB>(a.part + prow * DH, acc, 1.0f, h);           // else no part
    if (h == 0) {
      a.part_ml[2 * prow] = m2;
      a.part_ml[2 * prow + 1] = sum;
    }
    return;
  }
  store_cols<T, DB>(static_cast<T*>(a.out) + qrow * a.ld_out + head * DH, acc, sum == 0.0f ? 0.0f : 1.0f / sum, h);
  if (a.lse && h == 0) a.lse[orow] = sum == 0.0f ? -INFINITY : (m2 + __builtin_amdgcn_logf(sum)) * LN2;
}

// Single steps: at most 32 rows of a key head, over pages.  Each wavefront takes every fourth block of 32 keys and stages
// K and V of its own, one block each: the next block's K is under way while the softmax and V's product run, its V
// while the next scores are formed, and no wavefront waits for another.  What bounds it is reading k and v: 16 streams over 4k to
// 16k keys, 8 key heads of 128, 16 bits, 116 us, 5.0 TB/s.
template <class T, int DH>
constexpr int FEW_LDS = 8 * 32 * DH * (int)sizeof(T);
template <class T, int DH>
constexpr int FEW_PER_CU = FEW_LDS<T, DH> > 80 * 1024 ? 1 : FEW_LDS<T, DH> > 40 * 1024 ? 2 : 4;
template <class T, int DH>
__global__ __launch_bounds__(256, (FEW_PER_CU<T, DH>)) void few_kernel(const Table t, const Args given) {
  using TL = Tile<T, DH>;
  constexpr int DB = TL::DB, KB = 128, N = 32 * TL::UPR / 64;
  __shared__ __attribute__((aligned(16))) uint8_t lds[FEW_LDS<T, DH> + 1024];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  T* const kt = reinterpret_cast<T*>(lds) + wave * 2 * 32 * DH;
  T* const vt = kt + 32 * DH;
  Args a = given;
  const bool by_program = (int)blockIdx.x < given.more_blocks;
  if (by_program) {
    a.splits = given.more_splits; a.chunk = given.more_chunk; a.part0 = given.more_part0;
    a.row_tiles = 0;
    a.again = 0;
  }
  if (given.part0 == 0) check_rows(a, tid);
  const int block = by_program ? blockIdx.x : blockIdx.x - given.more_blocks;
  Work w;
  if (!work_of<true>(t, a, block, by_program ? given.more_blocks : gridDim.x - given.more_blocks, 32, KB, lane, w)) return;
  const int row = w.tile * 32 + (lane & 31);                  // may pass R: computed, not stored
  const int rr = min(row, w.R - 1), head = w.hk * a.G + rr % a.G;
  const int64_t qrow = w.q0 + rr / a.G;
  const int hi = max(w.before + rr / a.G + 1, 0), hi_a = lane_of(hi, 0);
  const int nP = (w.P + KB - 1) / KB, tiles = nP + (w.o1 + KB - 1) / KB;
  const int2 tt = share_of(a, tiles, w.split);

  auto block_of = [&](int ti) {
    const bool own = ti >= nP;
    const int first = (own ? ti - nP : ti) * KB + 32 * wave;
    return paged_block(a, own ? w.own_table : w.shared_table, first, ti < tt.y ? (own ? w.o1 : w.P) - first : 0, lane);
  };
  Place place;
  f32x16 acc[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b] = f32x16{};
  float mx = -INFINITY, sum = 0.0f;
  Block now = block_of(tt.x);
  auto copy_both = [&]() {
    place = place_of<T, DH>(a, w.hk, now);
    copy_block<T, DH>(a.k, place, kt, lane);
    copy_block<T, DH>(a.v, place, vt, lane);
  };
  if (now.n > 0) copy_both();
  typename TL::Op qf;
  TL::load_op(qf, static_cast<const T*>(a.q) + qrow * a.ld_q + head * DH, h);
  TL::scale_op(qf, a.c2);
  int ti = tt.x;
  bool own = ti >= nP;
  // A run's blocks of a wavefront end with the first that has no keys; the program's run goes over into the own keys'.
  auto following = [&](int& tn) {
    Block b = block_of(++tn);
    if (b.n == 0 && tn <= nP && nP < tt.y) b = block_of(tn = nP);
    return b;
  };
  if (now.n == 0 && ti < nP && nP < tt.y) {
    now = block_of(ti = nP);
    if (now.n > 0) copy_both();
  }
  while (now.n > 0) {
    own = ti >= nP;
    int tn = ti;
    const Block next = following(tn);
    wait_counts<N, true>();                                   // K is there
    f32x16 s = TL::mm_row(kt, 0, qf, lane);
    wait_counts<63, true>();
    if (next.n > 0) {
      place = place_of<T, DH>(a, w.hk, next);
      copy_block<T, DH>(a.k, place, kt, lane);
    }
    if (own ? hi_a < now.first + 32 : now.n < 32) only(s, own ? below(hi - now.first) & below(now.n) : below(now.n), -INFINITY, h);
    weigh<T, DB>(s, mx, sum, acc, a.c2);
    if (next.n > 0) wait_counts<N, false>(); else wait_counts<0, false>();    // V is there
    TL::mm_col(vt, 0, s, acc, lane);
    wait_counts<63, true>();
    if (next.n > 0) copy_block<T, DH>(a.v, place, vt, lane);
    now = next;
    ti = tn;
  }
  auto spoilt = [&]() {                                       // as in the forward kernel
    return any_beyond<T, DH>(hi_a, w.o1, INFINITY, lane, [&](int i) -> const T* {
      const int64_t at = key_at<DH, true>(a, w, true, i, true);
      return at < 0 ? nullptr : static_cast<const T*>(a.v) + at;
    });
  };
  if (a.again && __syncthreads_or(tt.y > nP && __any(not_finite<DB>(acc)) && spoilt())) {
    forward_again<T, DH, true, false>(t, a, block, gridDim.x - given.more_blocks, 32, KB);
    return;
  }
  sum = pair_sum(sum);
  float m2 = mx == -INFINITY ? -INFINITY : log2_units<T>(mx, a.c2);
  // join the wavefronts
  constexpr int LW = DH + 4;
  float* x = reinterpret_cast<float*>(lds);                   // [3][32][LW]
  float* ml = x + 3 * 32 * LW;                                // [3][32][2]
  static_assert((3 * 32 * LW + 192) * 4 <= sizeof(lds), "the exchange takes the tiles' place");
  __syncthreads();
  if (wave > 0) {
    store_cols<float, DB>(x + ((wave - 1) * 32 + (lane & 31)) * LW, acc, 1.0f, h);
    if (h == 0) {
      ml[((wave - 1) * 32 + lane) * 2] = m2;
      ml[((wave - 1) * 32 + lane) * 2 + 1] = sum;
    }
  }
  __syncthreads();
  if (wave > 0) return;
  float top = m2;
#pragma unroll
  for (int k = 0; k < 3; ++k) top = fmaxf(top, ml[(32 * k + (lane & 31)) * 2]);
  const float ref = top == -INFINITY ? 0.0f : top;
  float f = exp2_of(m2 - ref);
  sum *= f;
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b] *= f;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int l = 32 * k + (lane & 31);
    f = exp2_of(ml[2 * l] - ref);
    sum = fmaf(ml[2 * l + 1], f, sum);
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      const f32x16 y = load_acc(x + l * LW + 32 * b, h);
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][r] = fmaf(y[r], f, acc[b][r]);
    }
  }
  m2 = top;
  if (row >= w.R) return;
  const int64_t orow = qrow * a.heads + head;
  if (a.parts > 1) {
    const int64_t prow = (int64_t)(a.part0 + w.split) * a.part_rows + orow;
    if (sum != 0.0f) store_cols<float, DB>(a.part + prow * DH, acc, 1.0f, h);           // else no part
    if (h == 0) {
      a.part_ml[2 * prow] = m2;
      a.part_ml[2 * prow + 1] = sum;
    }
    return;
  }
  store_cols<T, DB>(static_cast<T*>(a.out) + qrow * a.ld_out + head * DH, acc, sum == 0.0f ? 0.0f : 1.0f / sum, h);
  if (a.lse && h == 0) a.lse[orow] = sum == 0.0f ? -INFINITY : (m2 + __builtin_amdgcn_logf(sum)) * LN2;
}

// Joins the parts of every row that some sequence has, o = sum 2^(m_i - m) o_i / sum 2^(m_i - m) s_i in their order: 16-byte quads
// of a row's features, one per thread.  Reading the parts bounds it (32768 rows of 128 in up to 9 parts 27 us); eight are under way together.
template <class T, int DH>
__global__ __launch_bounds__(256) void join_kernel(const Args a, int64_t rows) {
  constexpr int Q = DH / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * Q) return;
  const int64_t r = i / Q;
  if (r / a.heads >= a.off[a.B]) return;
  const int d = (int)(i % Q) * 4;
  float top = -INFINITY, sum = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int AHEAD = 8;                                    // parts whose loads are under way together
  for (int s0 = 0; s0 < a.parts; s0 += AHEAD) {
    float2 ml[AHEAD];
    f32x4 x[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int64_t p = min(s0 + i, a.parts - 1) * a.part_rows + r;
      ml[i] = *reinterpret_cast<const float2*>(a.part_ml + 2 * p);
      if (s0 + i >= a.parts) ml[i].y = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (ml[i].y != 0.0f) x[i] = *reinterpret_cast<const f32x4*>(a.part + ((s0 + i) * a.part_rows + r) * DH + d);
    float m = top;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) m = ml[i].y != 0.0f ? fmaxf(m, ml[i].x) : m;
    const float f0 = top == m ? 1.0f : exp2_of(top - m);
    top = m;
    sum *= f0;
    acc *= f0;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (ml[i].y == 0.0f) continue;
      const float f = exp2_of(ml[i].x - top);
      sum = fmaf(ml[i].y, f, sum);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(x[i][j], f, acc[j]);
    }
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
// Gradients, as in wm_attend.hip: P = exp(S - lse) is formed again; delta = do . o; dS = P (do . v - delta).
// One kernel owns rows (dq; it also writes every row's statistics) and one keys, own ones or the programs': seven products where
// five are counted, no atomics.  dq: matrix cores 43% and vector unit 53% busy at a width of 64 (31129 rows on 1k to 2k keys 253 us,
// 16 bits), 50 and 33% at 128.

template <class T, int DH>
__global__ __launch_bounds__(256, IS_BF<T> ? DH == 64 ? 3 : 2 : 1) void dq_kernel(const Table t, const Args a) {
  using TL = Tile<T, DH>;
  constexpr int DB = TL::DB, KB = TILE_ROWS<T, DH>;
  __shared__ __attribute__((aligned(16))) T lds[4 * KB * DH];
  T* const ks = lds;
  T* const vs = lds + 2 * KB * DH;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5;
  check_rows(a, tid);
  Work w;
  if (!work_of<false>(t, a, blockIdx.x, gridDim.x, 128, KB, lane, w)) return;
  const int row = w.tile * 128 + wave * 32 + (lane & 31);
  const int rr = min(row, w.R - 1), head = w.hk * a.G + rr % a.G;
  const int64_t qrow = w.q0 + rr / a.G, orow = qrow * a.heads + head;
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
  // a row that saw only keys of weight 0 has lse = -inf: its P is 0
  const float l2 = lse == -INFINITY ? INFINITY : lse * LOG2E;
  const int split = w.split;
  const int lo = bounds_of(a, w.seq, (int)qrow, lane_of((int)qrow, 31), (int)w.q0, (int)w.q0 + w.R / a.G, lane).x, hi = (int)qrow + 1;
  const int lo_a = lane_of(lo, 0), lo_z = lane_of(lo, 31), hi_a = lane_of(hi, 0), hi_z = lane_of(hi, 31);

  const int P = w.P, o0 = w.o0, rest = w.rest, o1 = w.o1, nP = (P + KB - 1) / KB, tiles = nP + (rest - o0) / KB;
  const int2 tt = share_of(a, tiles, split);
  const int shares = shares_of(a, tiles);
  if (split >= shares) return;
  if (split == 0 && h == 0 && row < w.R) a.counts[orow] = shares;
  const int t0 = tt.x, t1 = tt.y;
  const uint8_t* mask = a.mask ? a.mask + w.p0 : nullptr;
  // Where a row sees few keys, the rounding of o in do . o would be the largest of its errors: its delta is the sum of P (do . v) instead.
  // (16 bits, width 64, dq's 2-norm in 2^-8 of it: sequences of 3 rows 0.57, with do . o 0.8; with a program of 16 keys 0.61 and 0.67;
  // of 64 keys, where do . o is taken, 0.63.)  The row alone decides, by its own keys and its program's, so that it does not matter what
  // shares its tile.
  constexpr int FEW = 64;
  if (P < FEW) {
    constexpr bool TWO = KB >= 64;
    T* const kt = lds + wave * KB * DH;
    T* const vt = TWO ? kt + 32 * DH : kt;
    const bool few = P + hi - lo <= FEW;
    const uint64_t which = __ballot(few);
    float sum = 0.0f;
    auto block = [&](const T* k, int64_t ldk, const T* v, int64_t ldv, int n, uint32_t seen) {
      copy_rows<T, DH, 32, 64>(v, (int)ldv, n, vt, lane);
      wait_counts<0, true>();
      const f32x16 dp = TL::mm_row(vt, 0, gf, lane);
      wait_counts<63, true>();
      copy_rows<T, DH, 32, 64>(k, (int)ldk, n, kt, lane);
      wait_counts<0, true>();
      f32x16 s = TL::mm_row(kt, 0, qf, lane);
      wait_counts<63, true>();
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = weight<T>(s[r], a.c2, l2) * dp[r];
      only(s, seen, 0.0f, h);
#pragma unroll
      for (int r = 0; r < 16; ++r) sum += s[r];
    };
    if (which) {
      for (int at = 0; at < P; at += 32) {
        const uint32_t seen = (uint32_t)__ballot(lane < 32 && at + lane < P && (!mask || mask[at + lane] != 0));
        block(static_cast<const T*>(a.pk) + (w.p0 + at) * a.ld_pk + w.hk * DH, a.ld_pk,
              static_cast<const T*>(a.pv) + (w.p0 + at) * a.ld_pv + w.hk * DH, a.ld_pv, P - at, seen);
      }
      // rows ascend: from the first such row's keys to the last one's
      const int end = lane_of(hi, 63 - __builtin_clzll(which));
      for (int at = lane_of(lo, __builtin_ctzll(which)); at < end; at += 32)
        block(static_cast<const T*>(a.k) + at * a.ld_k + w.hk * DH, a.ld_k, static_cast<const T*>(a.v) + at * a.ld_v + w.hk * DH, a.ld_v,
              end - at, below(hi - at) & ~below(lo - at));
      const float d = pair_sum(sum);
      delta = few ? d : delta;
    }
    __syncthreads();
  }
  uint64_t vis[1] = {0}, next[1] = {0};
  int mb = 0;
  auto mask_byte = [&](int ti) -> int {
    const int key = ti * KB + lane;
    return mask && (KB >= 64 || lane < KB) && key < P ? mask[key] : 0;
  };
  Stream<T, DH, KB> rows;
  auto copy = [&](int ti, uint64_t (&v)[1], T* kt, T* vt) {
    const bool own = ti >= nP;
    if (ti == nP || ti == t0) {
      const int64_t first = own ? (int64_t)o0 + (int64_t)(ti - nP) * KB : w.p0 + (int64_t)ti * KB;
      const int64_t lk = own ? a.ld_k : a.ld_pk, lv = own ? a.ld_v : a.ld_pv;
      rows.start(static_cast<const T*>(own ? a.k : a.pk) + first * lk + w.hk * DH, lk,
                 static_cast<const T*>(own ? a.v : a.pv) + first * lv + w.hk * DH, lv, tid);
    }
    if (mask && !own) v[0] = __ballot(mb != 0);
    rows.copy(kt, vt, own ? KB : min(P - ti * KB, KB), mask && !own, v, wave, tid);
  };
  f32x16 acc[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b] = f32x16{};
  if (t0 < t1) {
    mb = mask_byte(t0);
    copy(t0, vis, ks, vs);
    if (t0 + 1 < t1) mb = mask_byte(t0 + 1);
  }
  auto step = [&](int ti, auto buffer) {
    constexpr int BUF = decltype(buffer)::value;
    wait_counts<0, true>();
    raw_barrier();
    if (ti + 1 < t1) {
      copy(ti + 1, next, ks + (BUF ^ 1) * KB * DH, vs + (BUF ^ 1) * KB * DH);
      if (ti + 2 < t1) mb = mask_byte(ti + 2);
    }
    const T* kt = ks + BUF * KB * DH;
    const T* vt = vs + BUF * KB * DH;
    const bool own = ti >= nP;
    const int at = own ? o0 + (ti - nP) * KB : ti * KB;
    const bool all = own ? lo_z <= at : !mask && at + KB <= P, none = own && lo_a > at;
#pragma unroll
    for (int kb = 0; kb < KB / 32; ++kb) {
      if (none) break;
      f32x16 s = TL::mm_row(kt, 32 * kb, qf, lane);
      const f32x16 dp = TL::mm_row(vt, 32 * kb, gf, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = weight<T>(s[r], a.c2, l2) * (dp[r] - delta);
      if (!all) {
        const uint32_t seen = own ? (lo <= at ? ~0u : 0u) : mask ? (uint32_t)(vis[0] >> (32 * kb)) : below(P - at - 32 * kb);
        uint32_t m = seen >> (4 * h);
        asm volatile("" : "+v"(m));             // keeps this a branch: seldom taken, 48 instructions
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = (m >> acc_row(0, r)) & 1 ? s[r] : 0.0f;
      }
      TL::mm_col(kt, 32 * kb, s, acc, lane);
    }
    vis[0] = next[0];
  };
  for (int ti = t0; ti < t1; ti += 2) {
    step(ti, std::integral_constant<int, 0>{});
    if (ti + 1 < t1) step(ti + 1, std::integral_constant<int, 1>{});
  }
  if (split == shares - 1 && rest < o1) {                      // as in the forward kernel
    constexpr bool TWO = KB >= 64;
    __syncthreads();
    T* const kt = lds + wave * KB * DH;
    T* const vt = TWO ? kt + 32 * DH : kt;
    const int end = min(hi_z, o1);
    auto copy_of = [&](const void* x, int64_t ld, int first, T* tile) {
      copy_rows<T, DH, 32, 64>(static_cast<const T*>(x) + first * ld + w.hk * DH, (int)ld, end - first, tile, lane);
    };
    int first = max(lo_a, rest);
    if (first < end) copy_of(a.v, a.ld_v, first, vt);
    if (TWO && first < end) copy_of(a.k, a.ld_k, first, kt);
    for (; first < end; first += 32) {
      const bool more = first + 32 < end;
      wait_counts<0, true>();
      const f32x16 dp = TL::mm_row(vt, 0, gf, lane);
      wait_counts<63, true>();
      if (!TWO) {
        copy_of(a.k, a.ld_k, first, kt);
        wait_counts<0, true>();
      }
      f32x16 s = TL::mm_row(kt, 0, qf, lane);
      if (TWO && more) copy_of(a.v, a.ld_v, first + 32, vt);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = weight<T>(s[r], a.c2, l2) * (dp[r] - delta);
      if (lo_z > first || hi_a < first + 32) only(s, below(hi - first) & ~below(lo - first), 0.0f, h);
      TL::mm_col(kt, 0, s, acc, lane);
      wait_counts<63, true>();
      if (more) copy_of(TWO ? a.k : a.v, TWO ? a.ld_k : a.ld_v, first + 32, TWO ? kt : vt);
    }
  }
  if (split == 0 && h == 0 && row < w.R) {
    a.stat[2 * orow] = l2;
    a.stat[2 * orow + 1] = delta;
  }
  auto spoilt = [&]() {                                        // as in the forward kernel
    auto key = [&](int i) { return static_cast<const T*>(a.k) + key_at<DH, false>(a, w, true, i, false); };
    return any_beyond<T, DH>(lo_a, lo_z, INFINITY, lane, key) || any_beyond<T, DH>(hi_a, min(hi_z, o1), INFINITY, lane, key);
  };
  if (__syncthreads_or(__any(not_finite<DB>(acc)) && spoilt())) {
    float2* const stat = reinterpret_cast<float2*>(lds);     // the tile's rows'
    if (h == 0) stat[32 * wave + lane] = make_float2(l2, delta);
    __syncthreads();
    dq_again<T, DH>(t, a, stat);
    return;
  }
  if (row >= w.R) return;
  if (a.splits > 1) store_cols<float, DB>(a.part + (split * a.part_rows + orow) * DH, acc, a.scale, h);
  else store_cols<T, DB>(static_cast<T*>(a.out) + qrow * a.ld_out + head * DH, acc, a.scale, h);
}

// dk and dv of 128 keys (32 per wavefront, in registers as row operands).  EVEN: the heads of a key head divide the rows of
// a copy, so that a tile of stacked rows is the same pattern everywhere (with the other form everywhere: training at a width of 64
// 879 us for 817, causal at 128 3224 for 2280).  The programs' keys at 64: matrix cores 47%, vector unit 42% busy at two wavefronts per
// SIMD (320 us); own keys at 128: 44 and 32% (820 us, 890 TFLOP/s), where LDS is read as long as the products take.
template <class T, int DH, bool EVEN>
constexpr int KEYS_PER_CU = IS_BF<T> && EVEN && DH == 64 ? 3 : IS_BF<T> && (EVEN || DH <= 64) ? 2 : 1;
template <class T, int DH, bool OWN, bool EVEN>
__global__ __launch_bounds__(256, (KEYS_PER_CU<T, DH, EVEN>)) void dkv_kernel(const Table t, const Args a) {
  using TL = Tile<T, DH>;
  constexpr int DB = TL::DB, RB = TILE_ROWS<T, DH>;
  __shared__ __attribute__((aligned(16))) T lds[4 * RB * DH];
  __shared__ __attribute__((aligned(16))) float st[2][2 * RB];     // [buffer][row][lse log2 e, delta]
  // The sums and operands leave too few of 256 registers (168 at a width of 64): some of the operands' stay in LDS.  (Where the
  // compiler spilled three, every reload waited for the copies under way, 1.53 ms for 1.25.)
  constexpr int KEPT_K = IS_BF<T> && EVEN && (DH == 128 || (DH == 64 && OWN)) ? 1 : 0, KEPT_V = DH == 128 ? 2 * KEPT_K : 0;
  __shared__ __attribute__((aligned(16))) u32x4 kept[KEPT_K ? (KEPT_K + KEPT_V) * 256 : 1];
  T* const qs = lds;
  T* const gs = lds + 2 * RB * DH;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5;
  KeyWork w;
  if (!key_work_of<OWN>(t, a, blockIdx.x, RB, lane, w)) return;
  const int shares = shares_of(a, (w.x1 - w.x0 + RB - 1) / RB);
  if (w.split >= shares) return;
  const int kc = min(w.first + wave * 32 + (lane & 31), w.n - 1);
  const int hk = w.hk, split = w.split, x0 = w.x0, x1 = w.x1, t0 = w.t0, t1 = w.t1;
  const int64_t kclamped = w.k0 + kc;
  typename TL::Op kf, vf;
  TL::load_op(kf, static_cast<const T*>(a.k) + kclamped * a.ld_k + hk * DH, h);
  TL::load_op(vf, static_cast<const T*>(a.v) + kclamped * a.ld_v + hk * DH, h);
  TL::scale_op(kf, a.c2);
  if constexpr (KEPT_K > 0) {                                // a thread reads back its own: no barrier
    kept[tid] = kf[TL::NR - 1];
#pragma unroll
    for (int i = 1; i <= KEPT_V; ++i) kept[256 * i + tid] = vf[TL::NR - i];
  }
  auto k_op = [&](int i) -> u32x4 { return i < TL::NR - KEPT_K ? kf[i] : kept[tid]; };
  auto v_op = [&](int i) -> u32x4 { return i < TL::NR - KEPT_V ? vf[i] : kept[256 * (TL::NR - i) + tid]; };
  // stacked rows of the segment that see a lane's key: [lo, hi)
  int lo = 0, hi = x1;
  if constexpr (OWN) {
    lo = kc * a.G;
    hi = (bounds_of(a, w.seq, (int)kclamped, lane_of((int)kclamped, 31), (int)w.q0, (int)w.q0 + w.n, lane).y - (int)w.q0) * a.G;
  }
  const int lo_a = lane_of(lo, 0), lo_z = lane_of(lo, 31), hi_a = lane_of(hi, 0), hi_z = lane_of(hi, 31);
  __shared__ int2 seen_by[OWN ? 128 : 1];                    // out of the registers' way; written and read by the same wavefront
  const int mine = 32 * wave + (lane & 31);
  if constexpr (OWN) seen_by[mine] = make_int2(lo, hi);

  Stream<T, DH, RB> rows;
  const float* stats;
  const int lg = EVEN ? 31 - __builtin_clz(a.G) : 0;
  auto start = [&]() {
    const int64_t q1 = w.q0 + ((x0 + t0 * RB) >> lg);        // the first tile's first query
    rows.start(static_cast<const T*>(a.q) + q1 * a.ld_q + hk * a.G * DH, a.ld_q, static_cast<const T*>(a.d_o) + q1 * a.ld_do + hk * a.G * DH,
               a.ld_do, tid, lg);
    stats = a.stat + 2 * (q1 * a.heads + hk * a.G);
  };
  auto copy = [&](int ti, T* qt, T* gt) {
    const int r0 = x0 + ti * RB;
    if constexpr (EVEN) {
      const uint64_t every[1] = {~0ull};
      rows.copy(qt, gt, x1 - r0, false, every, wave, tid, lg);
    } else {
      const int q1 = r0 / a.G;                               // the tile's first query
      const T* const q = static_cast<const T*>(a.q) + (w.q0 + q1) * a.ld_q + hk * a.G * DH;
      const T* const g = static_cast<const T*>(a.d_o) + (w.q0 + q1) * a.ld_do + hk * a.G * DH;
      const u32x4 qb = buffer_of(q, BAD - 1), gb = buffer_of(g, BAD - 1);
      auto off = [&](int r, int64_t ld) {
        const int x = r0 + r, qi = x / a.G;
        return x < x1 ? (uint32_t)(((qi - q1) * ld + (x - qi * a.G) * DH) * sizeof(T)) : BAD;
      };
      copy_tile<T, DH, RB, 256>(qb, qt, tid, [&](int r) { return off(r, a.ld_q); });
      copy_tile<T, DH, RB, 256>(gb, gt, tid, [&](int r) { return off(r, a.ld_do); });
    }
  };
  // (lse log2 e, delta) of a tile's rows; rows past the end read as zero like q and do, and add nothing
  auto copy_stat = [&](int ti, int buffer) {
    if (wave >= RB / 32) return;
    const int r0 = x0 + ti * RB, r = 32 * wave + (lane >> 1);
    if constexpr (EVEN) {
      const int n = min(x1 - r0, RB) >> lg;
      copy4(buffer_of(stats, ((n - 1) * a.heads + a.G) * 8), &st[buffer][64 * wave], ((r >> lg) * a.heads + (r & (a.G - 1))) * 8 + (lane & 1) * 4);
      stats += 2 * (RB >> lg) * a.heads;
    } else {
      const int q1 = r0 / a.G, qi = (r0 + r) / a.G;
      copy4(buffer_of(a.stat + 2 * ((w.q0 + q1) * a.heads + hk * a.G), BAD - 1), &st[buffer][64 * wave],
            r0 + r < x1 ? ((qi - q1) * a.heads + r0 + r - qi * a.G) * 8 + (lane & 1) * 4 : BAD);
    }
  };
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) dk[i] = dv[i] = f32x16{};
  if (t0 < t1) {
    if constexpr (EVEN) start();
    copy(t0, qs, gs);
    copy_stat(t0, 0);
  }
  Reads<T, DH> at;
  at.start(lds, lane);
  auto step = [&](int ti, auto buffer) {
    constexpr int BUF = decltype(buffer)::value;
    wait_counts<0, true>();
    raw_barrier();
    if (ti + 1 < t1) {
      copy(ti + 1, qs + (BUF ^ 1) * RB * DH, gs + (BUF ^ 1) * RB * DH);
      copy_stat(ti + 1, BUF ^ 1);
    }
    if constexpr (IS_BF<T> && DH == 128) asm volatile("" : "+v"(at.row), "+v"(at.col));        // not a register per read
    auto block = [&](auto which) {
      constexpr int RBK = decltype(which)::value, QOFF = (BUF * RB + 32 * RBK) * DH * (int)sizeof(T), GOFF = QOFF + 2 * RB * DH * (int)sizeof(T);
      const int r0 = x0 + ti * RB + 32 * RBK;
      if (OWN ? lo_a >= r0 + 32 || hi_z <= r0 : r0 >= x1) return;          // no key is seen by these rows
      // Where not every key sees every row, scores start from -infinity in the others' place: weights of 0 there, at no
      // register's cost.
      f32x16 s = {}, dp;
      if (OWN && (lo_z > r0 || hi_a < r0 + 32)) {
        const int2 by = seen_by[mine];
        only(s, below(by.y - r0) & ~below(by.x - r0), -INFINITY, h);
      }
      if constexpr (IS_BF<T>) {
        s = at.template mm_row<QOFF>(k_op, s);
        dp = at.template mm_row<GOFF>(v_op);
      } else {
        const f32x16 x = TL::mm_row(qs + BUF * RB * DH, 32 * RBK, kf, lane);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] += x[r];
        dp = TL::mm_row(gs + BUF * RB * DH, 32 * RBK, vf, lane);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(&st[BUF][2 * (32 * RBK + acc_row(h, 4 * q) + i)]);
          s[4 * q + i] = weight<T>(s[4 * q + i], a.c2, x[0]);
          s[4 * q + i + 1] = weight<T>(s[4 * q + i + 1], a.c2, x[2]);
          dp[4 * q + i] -= x[1];
          dp[4 * q + i + 1] -= x[3];
        }
      }
      if constexpr (IS_BF<T>) at.template mm_col<GOFF>(s, dv);
      else TL::mm_col(gs + BUF * RB * DH, 32 * RBK, s, dv, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= dp[r];
      if constexpr (IS_BF<T>) at.template mm_col<QOFF>(s, dk);
      else TL::mm_col(qs + BUF * RB * DH, 32 * RBK, s, dk, lane);
    };
    block(std::integral_constant<int, 0>{});
    if constexpr (RB > 32) block(std::integral_constant<int, 1>{});
  };
  for (int ti = t0; ti < t1; ti += 2) {
    step(ti, std::integral_constant<int, 0>{});
    if (ti + 1 < t1) step(ti + 1, std::integral_constant<int, 1>{});
  }
  bool again = false, again_v = false;
  if constexpr (OWN) {
    if (split == 0 && h == 0 && a.splits > 1 && w.first + mine < w.n) a.counts[(w.k0 + w.first + mine) * a.kv_heads + hk] = shares;
    again = __syncthreads_or(__any(not_finite<DB>(dk) || not_finite<DB>(dv)) && dkv_spoilt<T, DH>(a, w, lo_a, lo_z, hi_a, hi_z, wave, lane));
    if (again) again_v = __syncthreads_or(not_finite<DB>(dv));
  }
  int kl = threadIdx.x & 31;                                 // formed again, as above
  asm volatile("" : "+v"(kl));
  const int key = w.first + wave * 32 + kl;
  const int64_t krow = w.k0 + key;
  if (key < w.n) {
    if (!OWN && a.mask && a.mask[krow] == 0) {               // also where such a key holds NaN
#pragma unroll
      for (int b = 0; b < DB; ++b) dk[b] = dv[b] = f32x16{};
    }
    if (a.splits > 1) {
      const int64_t prow = krow * a.kv_heads + hk;
      if (!OWN && split == 0 && h == 0) a.counts[prow] = shares;
      store_cols<float, DB>(a.part + ((2 * split) * a.part_rows + prow) * DH, dk, a.scale, h);
      store_cols<float, DB>(a.part + ((2 * split + 1) * a.part_rows + prow) * DH, dv, 1.0f, h);
    } else {
      store_cols<T, DB>(static_cast<T*>(a.out) + krow * a.ld_out + hk * DH, dk, a.scale, h);
      store_cols<T, DB>(static_cast<T*>(a.out2) + krow * a.ld_out2 + hk * DH, dv, 1.0f, h);
    }
  }
  if constexpr (OWN) {
    if (again) {                                             // over what was stored, dv only where it is not finite
      __syncthreads();
      dkv_again<T, DH>(t, a, again_v);
    }
  }
}

// out[row] = sum of its parts' rows, in order; blockIdx.y picks dk or dv.  end (may be null): rows before it have parts.
template <class T, int DH>
__global__ __launch_bounds__(256) void add_kernel(const float* part, const int32_t* counts, int64_t rows, int sets, int heads, const int32_t* end,
                                                  void* out0, int64_t ld0, void* out1, int64_t ld1) {
  constexpr int Q = DH / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * Q) return;
  const int set = blockIdx.y;
  const int64_t r = i / Q, ld = set ? ld1 : ld0;
  if (end && r / heads >= *end) return;
  const int d = (int)(i % Q) * 4;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  const int n = counts[r];
  for (int s = 0; s < n; ++s) acc += *reinterpret_cast<const f32x4*>(part + (((int64_t)s * sets + set) * rows + r) * DH + d);
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 y;
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = (T)acc[j];
  *reinterpret_cast<t4*>(static_cast<T*>(set ? out1 : out0) + (r / heads) * ld + (r % heads) * DH + d) = y;
}

// --------------------------------------------------------------------------
// Host side.

constexpr int64_t MOST_TILES = INT32_MAX / 64 / XCDS;        // 64: splits
// Rates that the kernels reach: TFLOP/s of the products, bytes of the few-row form (wm_attend.hip).
double step_us(bool bf, int products, int64_t rows, int64_t keys, int dh, int per_cu) {
  return std::max(1.0, products * 2.0 * rows * keys * dh * 256 * per_cu / (bf ? 600e6 : 90e6));
}
double few_us(bool bf, int64_t keys, int dh, int per_cu) {
  return std::max(1.0, 2.0 * keys * dh * (bf ? 2 : 4) * 256 * per_cu / 4.5e6);
}
// A tile's time beside few others, of that where a compute unit's places are taken: products hardly gain, reading does.
double alone_of(bool few, int per_cu) { return few ? 0.3 + 0.7 / per_cu : 0.7 + 0.3 / per_cu; }
double part_us(int64_t values, int dh) { return 2.0 * values * dh * 4 / 4.5e6; }

// How loops are cut into splits of `chunk` tiles (long ones into more): `blocks` loops of `avg` tiles on average and `longest` at
// most, on 256 x per_cu places.  A tile takes unit_us where all places are taken, and `alone` of that where few are.  More shares than
// places take an even part of the work and `tail` of a share on top, fewer as long as the longest share; parts have to be
// written and read.  A split of the longest loop keeps `least` tiles.  (Measured at 256 loops of 64 to 256 tiles on 512 places, a
// step over long programs: 9 splits 284 us, 3 splits 375.)
struct Cut {
  int splits, chunk;
  double us;                      // what the loops and their parts take, by this
};
Cut cut_for(int64_t blocks, double avg, int64_t longest, int64_t least, int per_cu, double alone, double unit_us, double part_us,
            double tail = 0.5) {
  Cut best = {1, (int)std::max<int64_t>(longest, 1), 0.0};
  const double places = 256.0 * per_cu, even = blocks * avg / places;
  double cost = 0.0;
  for (int s = 1; s <= 64 && (s == 1 || s <= longest / least); ++s) {
    const int64_t chunk = std::max<int64_t>(cdiv(longest, s), 1);
    const double shares = s > 1 ? avg / chunk + 0.5 : 1.0, fill = blocks * shares / places;
    const double tiles = std::max(fill <= 1.0 ? even : even + tail * std::min<double>(chunk, avg), chunk * alone);
    const double c = tiles * unit_us + (s > 1 ? shares * part_us + 4.0 : 0.0);
    if (s == 1 || c < 0.98 * cost) {
      cost = c;
      best = {(int)std::max<int64_t>(cdiv(longest, chunk), 1), (int)chunk, c};
    }
  }
  return best;
}

// Rows and keys per tile, workgroups that share a compute unit (registers, LDS).
struct Shape {
  bool bf;
  int few_rows, few_keys, tile, few_cu, fwd_cu, dq_cu, dkv_cu;
};
Shape shape_of(int dtype, int dh) {
  const bool bf = dtype == WM_BF16, wide32 = !bf && dh == 128;
  const int wi = dh == 32 ? 0 : dh == 64 ? 1 : 2;
  static const int few[2][3] = {{2, 1, 1}, {4, 2, 1}}, fwd[2][3] = {{3, 2, 2}, {4, 4, 2}};
  static const int dq[2][3] = {{2, 2, 1}, {4, 3, 2}}, dkv[2][3] = {{2, 1, 1}, {4, 3, 2}};
  return {bf, wide32 ? 64 : 32, wide32 ? 64 : 128, wide32 ? 32 : 64, few[bf][wi], fwd[bf][wi], dq[bf][wi], dkv[bf][wi]};
}

wm_status bad(const char* m) { return set_error(WM_ERR_INVALID_ARGUMENT, m); }
// the launches that join parts have a thread per 4 features, and a launch at most 2^32 threads
bool too_wide(int64_t rows_all, int dh) { return rows_all > (int64_t)UINT32_MAX / (dh / 4) - 256; }

// ---- dense rows --------------------------------------------------------------
struct Plan {
  Shared sh;
  bool few;
  Cut fwd, dq, dkv, dpkv;
  size_t o_part, o_ml, o_stat, o_counts, bytes;
};

wm_status check(const wm_prefix* a, Plan* p, bool grad) {
  if (!a) return bad("prefix attention arguments are NULL");
  const wm_attention* w = &a->shared;
  const wm_status s = check_shared(w, &p->sh);
  if (s != WM_OK) return s;
  if (a->B < 0 || a->T_max < 0) return bad("B and T_max must not be negative");
  const int64_t nq = p->sh.nq;
  if (nq > 0 && (a->B < 1 || a->T_max < 1 || !a->off)) return bad("rows need sequences: B and T_max at least 1, off not NULL");
  if (!rows_ok(w, a->k, a->ld_k, nq, w->kv_heads) || !rows_ok(w, a->v, a->ld_v, nq, w->kv_heads))
    return bad("k and v need 16-byte aligned rows: pointer, stride at least the row's width, at most 2^22 elements");
  const Shape f = shape_of(w->dtype, w->head_dim);
  const int G = w->heads / w->kv_heads, dh = w->head_dim;
  int64_t row_tiles = 0, few_tiles = 0, key_tiles = 0, shared_tiles = 0, longest = 0, longest_rows = 0;
  double row_steps = 0, few_steps = 0, key_steps = 0, shared_steps = 0;
  for (int i = 0; i < w->S; ++i) {
    const int64_t lq = (int64_t)w->q_off[i + 1] - w->q_off[i], P = (int64_t)w->k_off[i + 1] - w->k_off[i];
    shared_tiles += cdiv(P, 128);
    shared_steps += (double)cdiv(P, 128) * cdiv(lq * G, f.tile);
    if (lq == 0) continue;
    // own keys of a tile's rows: their own and those before them, half a sequence on average
    const int64_t T = std::min<int64_t>(a->T_max, lq), own = std::min(lq, 128 / G + T / 2 + 1), few_own = std::min(lq, f.few_rows / G + T / 2 + 1);
    const int64_t seen = std::min(lq, 128 + T / 2) * G;
    row_tiles += cdiv(lq * G, 128);
    few_tiles += cdiv(lq * G, f.few_rows);
    key_tiles += cdiv(lq, 128);
    row_steps += (double)cdiv(lq * G, 128) * (cdiv(P, f.tile) + cdiv(own, f.tile));
    few_steps += (double)cdiv(lq * G, f.few_rows) * (cdiv(P, f.few_keys) + cdiv(few_own, f.few_keys));
    key_steps += (double)cdiv(lq, 128) * cdiv(seen, f.tile);
    longest = std::max(longest, P + std::min(lq, 128 / G + T));
    longest_rows = std::max(longest_rows, std::min(lq, 128 + T) * G);
  }
  if (row_tiles * w->kv_heads > MOST_TILES || few_tiles * w->kv_heads > MOST_TILES || key_tiles * w->kv_heads > MOST_TILES)
    return set_error(WM_ERR_UNSUPPORTED, "too many row or key tiles");
  const int64_t rows_all = nq * w->heads, kv_all = nq * w->kv_heads;
  auto avg = [](double steps, int64_t tiles) { return tiles ? steps / tiles : 0.0; };
  // Where loops differ (causal ones), shares do too, and the last ones leave more places empty: up to a whole share (training of four
  // causal sequences of 2583 to 3990 rows, 32 heads on 8 of 128: 1911 us, with half a share 2258).
  auto tail = [&](int64_t longest, double steps, int64_t tiles) { return 0.5 * std::min(2.0, longest / std::max(avg(steps, tiles), 1.0)); };
  // Few rows: a program's keys by four wavefronts (two), not by one after the other.  16-bit, width 64, 32 rows over 500, 8000 keys: 13 us
  // (22 in tiles of 128 rows), 42 (56); float32, width 128, 35 (48), 128 (205).  16-bit at 128 one workgroup fits a compute unit, and
  // tiles are no slower: 18.0 (18.5), 70 us (83) with 64 programs of 2000.
  p->few = !(f.bf && dh == 128) && p->sh.max_r <= f.few_rows;
  const int64_t few_loop = cdiv(longest, f.few_keys), loop = cdiv(longest, f.tile), key_loop = cdiv(longest_rows, f.tile),
                shared_loop = cdiv(p->sh.max_r, f.tile);
  if (p->few)
    p->fwd = cut_for(few_tiles * w->kv_heads, avg(few_steps, few_tiles), few_loop, 2, f.few_cu, alone_of(true, f.few_cu),
                     few_us(f.bf, f.few_keys, dh, f.few_cu), part_us(rows_all, dh), tail(few_loop, few_steps, few_tiles));
  else
    p->fwd = cut_for(row_tiles * w->kv_heads, avg(row_steps, row_tiles), loop, 2, f.fwd_cu, alone_of(false, f.fwd_cu),
                     step_us(f.bf, 2, 128, f.tile, dh, f.fwd_cu), part_us(rows_all, dh), tail(loop, row_steps, row_tiles));
  p->dq = cut_for(row_tiles * w->kv_heads, avg(row_steps, row_tiles), loop, 2, f.dq_cu, alone_of(false, f.dq_cu),
                  step_us(f.bf, 3, 128, f.tile, dh, f.dq_cu), part_us(rows_all, dh), tail(loop, row_steps, row_tiles));
  p->dkv = cut_for(key_tiles * w->kv_heads, avg(key_steps, key_tiles), key_loop, 2, f.dkv_cu, alone_of(false, f.dkv_cu),
                   step_us(f.bf, 4, 128, f.tile, dh, f.dkv_cu), part_us(2 * kv_all, dh), tail(key_loop, key_steps, key_tiles));
  p->dpkv = cut_for(shared_tiles * w->kv_heads, avg(shared_steps, shared_tiles), shared_loop, 2, f.dkv_cu, alone_of(false, f.dkv_cu),
                    step_us(f.bf, 4, 128, f.tile, dh, f.dkv_cu), part_us(2 * p->sh.nk * w->kv_heads, dh),
                    tail(shared_loop, shared_steps, shared_tiles));
  if (too_wide(rows_all, dh) || too_wide(p->sh.nk * w->kv_heads, dh)) return set_error(WM_ERR_UNSUPPORTED, "rows x heads x head_dim is too large");
  size_t at = 0;
  p->o_part = p->o_ml = p->o_stat = p->o_counts = 0;
  auto take = [&](size_t n) { const size_t o = at; at = al256(at + n); return o; };
  if (!grad) {
    if (p->fwd.splits > 1) {
      p->o_part = take((size_t)p->fwd.splits * rows_all * dh * 4);
      p->o_ml = take((size_t)p->fwd.splits * rows_all * 8);
    }
  } else {
    p->o_stat = take((size_t)rows_all * 8);
    size_t part = 0;                             // dq's, own keys' and the programs' keys', one after the other on the stream
    if (p->dq.splits > 1) part = std::max(part, (size_t)p->dq.splits * rows_all * dh * 4);
    if (p->dkv.splits > 1) part = std::max(part, (size_t)p->dkv.splits * 2 * kv_all * dh * 4);
    if (p->dpkv.splits > 1) part = std::max(part, (size_t)p->dpkv.splits * 2 * p->sh.nk * w->kv_heads * dh * 4);
    if (part) p->o_part = take(part);
    p->o_counts = take((size_t)std::max({rows_all, kv_all, p->sh.nk * w->kv_heads}) * 4);
  }
  p->bytes = workspace_of(at);
  return WM_OK;
}

Args base_args(const wm_prefix* x, const Plan& p) {
  const wm_attention* w = &x->shared;
  Args a = {};
  a.q = w->q; a.pk = w->k; a.pv = w->v; a.k = x->k; a.v = x->v;
  a.ld_q = w->ld_q; a.ld_pk = w->ld_k; a.ld_pv = w->ld_v; a.ld_k = x->ld_k; a.ld_v = x->ld_v;
  a.mask = w->kv_mask;
  a.off = x->off; a.status = x->status; a.rows = p.sh.nq; a.B = x->B; a.T_max = x->T_max;
  a.scale = w->scale;
  a.c2 = w->scale * LOG2E;
  a.heads = w->heads; a.kv_heads = w->kv_heads; a.G = w->heads / w->kv_heads;
  return a;
}

template <class T, int DH>
hipError_t join(const Args& a, int64_t n, hipStream_t st) {
  hipLaunchKernelGGL((join_kernel<T, DH>), dim3((unsigned)cdiv(n * (DH / 4), 256)), dim3(256), 0, st, a, n);
  return hipGetLastError();
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
                              if constexpr (!IS_BF<T> || DH < 128) {
                                if (p.few) hipLaunchKernelGGL((forward_kernel<T, DH, WK, false>), grid, dim3(256), 0, st, t, a);
                              }
                              if (!p.few) hipLaunchKernelGGL((forward_kernel<T, DH, 1, false>), grid, dim3(256), 0, st, t, a);
                            });
    if (e != hipSuccess || a.parts == 1) return e;
    return join<T, DH>(a, p.sh.nq * a.heads, st);
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
    const int64_t n = p.sh.nq * a.heads;
    hipLaunchKernelGGL((add_kernel<T, DH>), dim3((unsigned)cdiv(n * (DH / 4), 256), 1), dim3(256), 0, st, a.part, a.counts, n,
                       1, a.heads, a.off + a.B, a.out, a.ld_out, nullptr, (int64_t)0);
    return hipGetLastError();
  });
}

// dk and dv of own keys (OWN: they are the rows themselves) or of the programs' keys.
template <bool OWN>
hipError_t grad_keys(const wm_attention* w, int64_t keys, const Args& a, hipStream_t st) {
  wm_attention own = *w;
  own.k_off = OWN ? w->q_off : w->k_off;
  return typed(w, [&](auto tv, auto dh) {
    using T = decltype(tv);
    constexpr int DH = decltype(dh)::value;
    const bool even = Stream<T, DH, TILE_ROWS<T, DH>>::STEP % a.G == 0;
    hipError_t e = each_run(&own, true, a.splits, [&](int64_t, int64_t lk) { return cdiv(lk, 128); },
                            [&](const Table& t, int blocks) {
                              if (even) hipLaunchKernelGGL((dkv_kernel<T, DH, OWN, true>), dim3(blocks), dim3(256), 0, st, t, a);
                              else hipLaunchKernelGGL((dkv_kernel<T, DH, OWN, false>), dim3(blocks), dim3(256), 0, st, t, a);
                            });
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t n = keys * a.kv_heads;
    hipLaunchKernelGGL((add_kernel<T, DH>), dim3((unsigned)cdiv(n * (DH / 4), 256), 2), dim3(256), 0, st, a.part, a.counts, n,
                       2, a.kv_heads, OWN ? a.off + a.B : nullptr, a.out, a.ld_out, a.out2, a.ld_out2);
    return hipGetLastError();
  });
}

// ---- paged cache -----------------------------------------------------------------
struct CachedPlan {
  wm_attention w;                 // types and widths
  bool joint;                     // one launch by sequences (their program's keys among them), no launch by programs
  bool few, shared_few;           // rows of 32 per workgroup, its wavefronts sharing them
  Cut own, shared;                // of the launch by sequences, by programs
  int64_t most_rows;              // stacked rows of a program, at most
  size_t o_part, o_ml, bytes;
};

// Workgroups of a key head and split for the tiles of `seqs` sequences: as many for each as the longest needs, or, where that is more,
// their rows' and one for each (first_slot).
int64_t tiles_of_longest(const wm_cached* a, int G, int tile) { return cdiv(std::min<int64_t>(a->T_max, a->rows) * G, tile); }
int64_t slots_of(const wm_cached* a, int64_t seqs, int G, int tile) {
  return std::min(seqs * tiles_of_longest(a, G, tile), a->rows * G / tile + seqs);
}
// Rows of n sequences of one program, at most.
int64_t rows_of(const wm_cached* a, int64_t n) { return std::min(n * a->T_max, a->rows); }

wm_status check(const wm_cached* a, CachedPlan* p) {
  if (!a) return bad("cached attention arguments are NULL");
  const wm_status s = check_cache(&a->cache);
  if (s != WM_OK) return s;
  const wm_cache& c = a->cache;
  if (a->heads < 1 || a->heads % c.kv_heads) return bad("heads must be a positive multiple of kv_heads");
  if (a->heads > 1024) return set_error(WM_ERR_UNSUPPORTED, "more than 1024 heads");
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale * LOG2E)) return bad("scale must be positive and below 2e38");
  if (a->rows < 0 || a->rows > INT32_MAX || a->T_max < 0) return bad("rows must be in [0, 2^31), T_max not negative");
  if (a->rows > 0 && (c.B < 1 || a->T_max < 1)) return bad("rows need sequences: B and T_max at least 1");
  if (c.B > 0 && !a->off) return bad("off is NULL");
  if (a->len_max < 0 || a->len_max > (int64_t)c.max_pages * c.page) return bad("len_max must be in [0, max_pages page]");
  p->w = {};
  p->w.dtype = c.dtype; p->w.heads = a->heads; p->w.kv_heads = c.kv_heads; p->w.head_dim = c.head_dim;
  if (!rows_ok(&p->w, a->q, a->ld_q, a->rows, a->heads))
    return bad("q needs 16-byte aligned rows: pointer, stride at least the row's width, at most 2^22 elements");
  if (a->S < 0 || a->S > WM_MAX_SEGMENTS) return bad("S must be in [0, WM_MAX_SEGMENTS]");
  const int G = a->heads / c.kv_heads, dh = c.head_dim;
  const int64_t seq_rows = std::min<int64_t>(a->T_max, std::max<int64_t>(a->rows, 1)) * G;
  int64_t most_seqs = 0, shared_few_tiles = 0;
  const Shape f = shape_of(c.dtype, dh);
  constexpr int FEW_ROWS = 32, FEW_KEYS = 128;
  const int few_cu = c.dtype == WM_BF16 ? (dh == 128 ? 2 : 4) : (dh == 128 ? 1 : dh == 64 ? 2 : 4);
  if (a->S > 0) {
    if (!a->seg_off || a->seg_off[0] != 0 || a->seg_off[a->S] != c.B) return bad("seg_off must run from 0 to B");
    for (int i = 0; i < a->S; ++i) {
      const int64_t n = (int64_t)a->seg_off[i + 1] - a->seg_off[i];
      if (n < 0) return bad("seg_off must not decrease");
      most_seqs = std::max(most_seqs, n);
      shared_few_tiles += cdiv(rows_of(a, n) * G, FEW_ROWS);
    }
    if (a->prefix_max < 0 || a->prefix_max > (int64_t)a->prefix_max_pages * c.page) return bad("prefix_max must be in [0, prefix_max_pages page]");
    if (!a->prefix_lens || (a->prefix_max_pages > 0 && !a->prefix_pages)) return bad("prefix_lens/prefix_pages is NULL");
  }
  if (rows_of(a, most_seqs) * G > INT32_MAX) return set_error(WM_ERR_UNSUPPORTED, "a program has more than 2^31 rows of one key head");
  const int P = a->S > 0 ? a->prefix_max : 0;
  p->few = seq_rows <= FEW_ROWS;
  p->most_rows = rows_of(a, most_seqs) * G;
  // Tiles of 32 rows of a program in the launch by sequences, or of 128 in a launch of their own.  The former read the keys as often
  // as there are tiles, from L2; they win while that is little.  16-bit, width 64, of 120 rows, 16 programs: of 300 keys 47 us (53
  // in two launches), of 4096 106 (104), of 48 rows 71 (81); width 128, 16 of 4096: 48 rows 95 (122), 96 rows 150 (130).
  const int64_t few_tiles = cdiv(p->most_rows, FEW_ROWS);
  p->shared_few = p->few && (few_tiles <= 2 || (few_tiles <= 8 && few_tiles * P <= 4096));
  const int64_t rows_all = a->rows * a->heads;
  const bool full = shared_few_tiles * c.kv_heads > MOST_TILES;            // no launch by programs
  if (slots_of(a, c.B, G, p->few ? FEW_ROWS : 128) * c.kv_heads > MOST_TILES || (full && p->few))
    return set_error(WM_ERR_UNSUPPORTED, "too many row tiles");
  // lengths are known to the device alone: loops of 0.6 of the longest on average
  auto cut = [&](bool few, int64_t blocks, int64_t longest) {
    const int keys = few ? FEW_KEYS : f.tile, cu = few ? few_cu : f.fwd_cu;
    const int64_t steps = cdiv(longest, keys);
    const double unit_us = few ? few_us(f.bf, keys, dh, cu) : step_us(f.bf, 2, 128, keys, dh, cu);
    return cut_for(blocks, 0.6 * steps, steps, 2, cu, alone_of(few, cu), unit_us, part_us(rows_all, dh));
  };
  // Sequences of many rows may read the program's keys along with their own, in tiles that the last rows of each do not fill, or leave
  // them to a launch by programs, whose tiles are full; the latter's parts have to be written and read, and where the estimates are close
  // it is the slower.  (16-bit, width 64, 64 sequences of two programs of up to 2048 keys, in one and in two launches: 32 to 64 rows
  // each 90 and 69 us, 64 to 128 rows 75 and 89; float32, four key heads: 188 and 102, 145 and 132.)
  const int64_t avg_rows = cdiv(a->rows, std::max(c.B, 1)) * G, program_rows = a->S > 0 ? cdiv(a->rows, a->S) * G : 0;
  const int64_t own_tiles = c.B * cdiv(avg_rows, p->few ? FEW_ROWS : 128) * c.kv_heads;
  p->own = cut(p->few, own_tiles, (int64_t)a->len_max + P);
  p->shared = {0, 0, 0.0};
  p->joint = true;
  if (P > 0 && most_seqs > 1) {
    const int64_t program_tiles = a->S * cdiv(program_rows, p->shared_few ? FEW_ROWS : 128) * c.kv_heads;
    const Cut own = cut(p->few, own_tiles, a->len_max), shared = cut(p->shared_few, program_tiles, P);
    p->joint = !p->few && (full || own.us + shared.us + 8.0 >= 0.8 * p->own.us);
    if (!p->joint) {
      p->own = own;
      p->shared = shared;
    }
  }
  if (too_wide(rows_all, dh)) return set_error(WM_ERR_UNSUPPORTED, "rows x heads x head_dim is too large");
  size_t at = 0;
  p->o_part = p->o_ml = 0;
  auto take = [&](size_t n) { const size_t o = at; at = al256(at + n); return o; };
  const int parts = p->own.splits + p->shared.splits;
  if (parts > 1) {
    p->o_part = take((size_t)parts * rows_all * dh * 4);
    p->o_ml = take((size_t)parts * rows_all * 8);
  }
  p->bytes = workspace_of(at);
  return WM_OK;
}

hipError_t cached(const wm_cached* x, const CachedPlan& p, Args a, hipStream_t st) {
  return typed(&p.w, [&](auto tv, auto dh) {
    using T = decltype(tv);
    constexpr int DH = decltype(dh)::value;
    hipError_t e = hipSuccess;
    const int tile = p.few ? 32 : 128, shared_tile = p.shared_few ? 32 : 128;
    a.row_tiles = (int)tiles_of_longest(x, a.G, tile);
    a.splits = p.own.splits;
    a.chunk = p.own.chunk;
    a.joint = p.joint && x->S > 0 && x->prefix_max > 0;
    a.more_splits = p.shared.splits;
    a.more_chunk = p.shared.chunk;
    a.more_part0 = p.own.splits;
    // a launch by sequences, its first workgroups by programs
    auto by_sequences = [&](const Table& t) {
      a.slots = (int)slots_of(x, a.nseq, a.G, tile);
      const int64_t own = (int64_t)a.slots * a.kv_heads * a.splits;
      if (own + a.more_blocks == 0 || e != hipSuccess) return;
      if (p.few) hipLaunchKernelGGL((few_kernel<T, DH>), dim3((unsigned)(own + a.more_blocks)), dim3(256), 0, st, t, a);
      else if (a.slots < (int64_t)a.nseq * a.row_tiles) hipLaunchKernelGGL((forward_kernel<T, DH, 1, true, true>), dim3((unsigned)own), dim3(256), 0, st, t, a);
      else hipLaunchKernelGGL((forward_kernel<T, DH, 1, true>), dim3((unsigned)own), dim3(256), 0, st, t, a);
      e = hipGetLastError();
    };
    const bool programs = x->S > 0 && x->prefix_max > 0;
    if (!programs) {
      a.nseq = x->cache.B;
      by_sequences(Table{});
    }
    for (int s0 = 0; programs && s0 < x->S; s0 += MAX_SEGS) {
      Table t = {};
      for (int i = s0; i < std::min(x->S, s0 + MAX_SEGS); ++i) {
        const int n = x->seg_off[i + 1] - x->seg_off[i];
        const int64_t rows = rows_of(x, n);
        t.seg[t.n] = {x->seg_off[i], (int32_t)rows, i, n};
        t.off[t.n + 1] = t.off[t.n] + (int32_t)cdiv(cdiv(rows * a.G, shared_tile) * a.kv_heads * p.shared.splits, XCDS);
        ++t.n;
      }
      a.seq0 = x->seg_off[s0];
      a.nseq = x->seg_off[s0 + t.n] - a.seq0;
      a.more_blocks = p.shared_few && p.few ? t.off[t.n] * XCDS : 0;
      by_sequences(t);
      if (p.joint || a.more_blocks || t.off[t.n] == 0 || e != hipSuccess) continue;
      Args b = a;                   // by programs: all their rows see all their keys
      b.row_tiles = 0;
      b.again = 0;
      b.part0 = a.more_part0;
      b.splits = a.more_splits;
      b.chunk = a.more_chunk;
      hipLaunchKernelGGL((forward_kernel<T, DH, 1, true>), dim3((unsigned)t.off[t.n] * XCDS), dim3(256), 0, st, t, b);
      e = hipGetLastError();
    }
    if (e != hipSuccess || a.parts == 1) return e;
    return join<T, DH>(a, x->rows * a.heads, st);
  });
}

}  // namespace prefix
}  // namespace wm

using namespace wm::prefix;

#define WM_PF(K, CALL)                                                                     \
  do {                                                                                     \
    timing_begin(K, st);                                                                   \
    hipError_t e_ = (CALL);                                                                \
    timing_end(K, st);                                                                     \
    if (e_ != hipSuccess) return set_error(WM_ERR_DEVICE, std::string("kernel launch: ") + hipGetErrorString(e_)); \
  } while (0)

extern "C" {

size_t wm_prefix_attention_workspace_bytes(const wm_prefix* a, int32_t grad) {
  Plan p;
  return check(a, &p, grad != 0) == WM_OK ? std::max(p.bytes, NO_WORKSPACE) : 0;
}

wm_status wm_prefix_attention(const wm_prefix* x, void* o, int64_t ld_o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  Plan p;
  const wm_status s = check(x, &p, false);
  if (s != WM_OK) return s;
  const wm_attention* w = &x->shared;
  if (!rows_ok(w, o, ld_o, p.sh.nq, w->heads)) return bad("o needs 16-byte aligned rows");
  if (p.bytes && (!ws || (uintptr_t)ws % 256 || ws_bytes < p.bytes)) return bad("workspace is NULL, not 256-byte aligned or too small");
  if (p.sh.nq == 0) return clear_error();
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  Args a = base_args(x, p);
  a.out = o;
  a.ld_out = ld_o;
  a.lse = lse;
  a.splits = a.parts = p.fwd.splits;
  a.chunk = p.fwd.chunk;
  a.part = reinterpret_cast<float*>(w8 + p.o_part);
  a.part_ml = reinterpret_cast<float*>(w8 + p.o_ml);
  a.again = 1;
  a.part_rows = p.sh.nq * w->heads;
  WM_PF(TK_PREFIX, forward(w, p, a, st));
  return clear_error();
}

wm_status wm_prefix_attention_grad(const wm_prefix* x, const void* o, int64_t ld_o, const float* lse, const void* d_o, int64_t ld_do,
                                   const wm_prefix_grads* g, void* ws, size_t ws_bytes, void* stream) {
  Plan p;
  const wm_status s = check(x, &p, true);
  if (s != WM_OK) return s;
  const wm_attention* w = &x->shared;
  const int64_t nq = p.sh.nq, nk = p.sh.nk;
  if (!g) return bad("gradient outputs are NULL");
  if (!rows_ok(w, o, ld_o, nq, w->heads) || !rows_ok(w, d_o, ld_do, nq, w->heads) || !rows_ok(w, g->dq, g->ld_dq, nq, w->heads) ||
      !rows_ok(w, g->dk, g->ld_dk, nq, w->kv_heads) || !rows_ok(w, g->dv, g->ld_dv, nq, w->kv_heads) ||
      !rows_ok(w, g->dpk, g->ld_dpk, nk, w->kv_heads) || !rows_ok(w, g->dpv, g->ld_dpv, nk, w->kv_heads))
    return bad("o, d_o, dq, dk, dv, dpk and dpv need 16-byte aligned rows");
  if (nq > 0 && !lse) return bad("lse is NULL");
  if (p.bytes && (!ws || (uintptr_t)ws % 256 || ws_bytes < p.bytes)) return bad("workspace is NULL, not 256-byte aligned or too small");
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  Args a = base_args(x, p);
  a.o = o; a.ld_o = ld_o;
  a.d_o = d_o; a.ld_do = ld_do;
  a.lse = const_cast<float*>(lse);
  a.stat = reinterpret_cast<float*>(w8 + p.o_stat);
  a.part = reinterpret_cast<float*>(w8 + p.o_part);
  a.counts = reinterpret_cast<int32_t*>(w8 + p.o_counts);
  if (nq > 0) {
    a.out = g->dq; a.ld_out = g->ld_dq;
    a.splits = p.dq.splits;
    a.chunk = p.dq.chunk;
    a.part_rows = nq * w->heads;
    WM_PF(TK_PREFIX, grad_rows(w, p, a, st));
    a.out = g->dk; a.ld_out = g->ld_dk;
    a.out2 = g->dv; a.ld_out2 = g->ld_dv;
    a.splits = p.dkv.splits;
    a.chunk = p.dkv.chunk;
    a.part_rows = nq * w->kv_heads;
    WM_PF(TK_PREFIX, grad_keys<true>(w, nq, a, st));
  }
  if (nk > 0) {
    a.k = w->k; a.ld_k = w->ld_k;
    a.v = w->v; a.ld_v = w->ld_v;
    a.out = g->dpk; a.ld_out = g->ld_dpk;
    a.out2 = g->dpv; a.ld_out2 = g->ld_dpv;
    a.splits = p.dpkv.splits;
    a.chunk = p.dpkv.chunk;
    a.part_rows = nk * w->kv_heads;
    WM_PF(TK_PREFIX, grad_keys<false>(w, nk, a, st));
  }
  return clear_error();
}

size_t wm_cached_attention_workspace_bytes(const wm_cached* a) {
  CachedPlan p;
  return check(a, &p) == WM_OK ? std::max(p.bytes, NO_WORKSPACE) : 0;
}

wm_status wm_cached_attention(const wm_cached* x, void* o, int64_t ld_o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  CachedPlan p;
  const wm_status s = check(x, &p);
  if (s != WM_OK) return s;
  if (!rows_ok(&p.w, o, ld_o, x->rows, x->heads)) return bad("o needs 16-byte aligned rows");
  if (p.bytes && (!ws || (uintptr_t)ws % 256 || ws_bytes < p.bytes)) return bad("workspace is NULL, not 256-byte aligned or too small");
  if (x->rows == 0) return clear_error();
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint8_t* w8 = static_cast<uint8_t*>(ws);
  const wm_cache& c = x->cache;
  Args a = {};
  a.q = x->q; a.ld_q = x->ld_q;
  a.k = c.k; a.v = c.v;
  a.off = x->off; a.status = x->status; a.rows = x->rows; a.B = c.B; a.T_max = x->T_max;
  a.scale = x->scale;
  a.c2 = x->scale * LOG2E;
  a.heads = x->heads; a.kv_heads = c.kv_heads; a.G = x->heads / c.kv_heads;
  a.pages = c.pages; a.lens = c.lens; a.ppages = x->prefix_pages; a.plens = x->prefix_lens;
  a.programs = x->S;
  a.max_pages = c.max_pages; a.max_ppages = x->prefix_max_pages; a.len_max = x->len_max; a.plen_max = x->prefix_max;
  a.n_pages = c.n_pages; a.lps = page_bits(c.page);
  a.out = o;
  a.ld_out = ld_o;
  a.lse = lse;
  a.parts = p.own.splits + p.shared.splits;
  a.part = reinterpret_cast<float*>(w8 + p.o_part);
  a.part_ml = reinterpret_cast<float*>(w8 + p.o_ml);
  // one row per sequence: the rows of a tile see the same keys
  a.again = x->T_max > 1;
  a.part_rows = x->rows * x->heads;
  WM_PF(TK_CACHED, cached(x, p, a, st));
  return clear_error();
}

}  // extern "C"
