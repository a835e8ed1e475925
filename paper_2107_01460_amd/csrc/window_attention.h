// Attention over a window of the last steps and the first steps of an episode, on the matrix cores.
//
// Row i (a query) sees column j (a key) where j is a step of i's episode up to i and i - j < window or j is among the episode's first `sinks` steps:
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  P_ij = exp(s_ij - lse_i),  out_i = sum_j P_ij v_j
//   delta_i = dout_i . out_i,  dS_ij = P_ij (dout_i . v_j - delta_i),  dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij dout_i
//
// All three passes (output; dq; dk and dv) are one scheme.  A wavefront owns 32 rows of two arrays ("own": queries, or keys and values), whose
// rows stay in registers as the second operand, one row a lane; tiles of 32 rows of two other arrays ("streamed") go through LDS.  For output and dq the workgroup's
// wavefronts share them, two on their way while one is at work; for dk and dv each wavefront streams through LDS of its own, with as many on their way as its registers
// allow (tiles_ahead), and waits for no other.  The first product S^T = Y own^T leaves a lane 16 of the 32 streamed rows of its own column; that layout is the second operand
// of the next product, acc^T += Y^T P, as it is, once the contraction runs over the streamed rows in the order in which the registers hold them.
// So scores and weights never leave the registers; softmax statistics are one number a lane, joined between the two halves of a wavefront.
// Y^T comes from the same row-major tile: transposed reads of 4 x 16 for bf16, single elements for fp32.
//
// bf16: inputs are exact operands, sums are fp32.  P and dS are rounded once to bf16 as operands (2^-8 of each term at most; the statistics lse and the row
// sums come from the fp32 values): about what the output's own rounding is, and half the matrix products of keeping two parts (outputs 0.0020 to 0.0022 off, relative to 64
// bits, gradients 0.0024, where the output's rounding alone makes it 0.0016).  fp32: fp32 products.
// Exponents are to base two in here and lse, which the caller keeps, to base e: a product on either side, 2^-24 of lse each, so some 2^-23 |lse| of a gradient's weights.
//
// Zero times infinity: a product of tiles multiplies masked places by zero.  The loop runs without care for it; a workgroup that finds
// an infinity or a NaN in its sums runs once more, adding the streamed rows one by one to the columns that see them only.
#pragma once
#include <type_traits>

#include "common.h"

namespace marl {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;

struct WindowArray {
  char* data;
  int64_t step, seq, head;  // bytes
};
struct WindowArgs {
  WindowArray q, k, v, out, dout, dq, dk, dv;
  const char *cache_k, *cache_v;  // [B][Hk][slots][dim], null: none
  const int32_t* positions;       // null: first + t
  int32_t first;
  uint32_t n_flags, seqs_per_flag;
  float *lse, *delta;  // [B][H][T]
  int* places;         // [n_flags][T]: the rows' positions, each environment's side by side
  int2* reach;         // [n_flags][tiles]: of a tile's rows, the earliest and the latest beginning of an episode
  int32_t T;
  uint32_t B, H, Hk, group;
  int32_t dk_dim, dv_dim, window, sinks;
  float scale, c;      // c = |scale| log2(e)
  uint32_t flip;       // the sign of a negative scale, for the elements of an own array (two of bf16, one of fp32)
  uint32_t heads_each; // query heads of a key head that a workgroup takes
  uint32_t blocks_t;   // workgroups along time
  int32_t fast;        // rows as Fetch's FAST wants them
  // first steps seen from beyond the window (far): chunks of far_tiles tiles of rows, far_slots tiles of columns each (none: 0), their numbers and sums
  uint32_t far_chunks, far_slots;
  int32_t far_tiles;
  int* far_numbers;    // [B][Hk][chunk][slot], -1: none
  float* far_parts;    // the same places, registers of dk and dv each
};

// Workgroups go round-robin to the eight XCDs.  Where there are many sequences, `run` workgroups next to each other in logical order stay on one XCD, and all XCDs work
// on neighbouring sequences: their rows of a step lie side by side (777 steps of 111 sequences, heads of 40 and 72 in bf16: 132 us against 142 with an eighth of the
// sequences for each XCD, as in xcd_remap; 128 x 4096 steps of 8 heads of 64: 1166 against 1186).  With few sequences an XCD walks along time, its neighbours' keys in
// its L2.  (Steps a power of two of bytes apart are slow however workgroups are laid out: 128 x 4096 steps of 8 heads of 64 in bf16 take 701 to 753 us without a cache when
// steps are 4 MB apart, 516 to 540 when a few lines lie between them, about what the memory gives.)
__device__ __forceinline__ uint32_t xcd_order(uint32_t at, uint32_t total, uint32_t run, uint32_t sequences) {
  if (sequences < 64) return xcd_remap(at, total);
  const uint32_t turn = 8 * run, whole = total / turn * turn;
  if (at >= whole) return at;
  const uint32_t in = at / 8;
  return in / run * turn + at % 8 * run + in % run;
}

// What a row sees.  Rows that hold no step see nothing.
struct Row {
  int i, start, lo;       // steps from `lo` to i
  uint32_t span, n_sinks; // i - lo; first steps from `start` on
  int position;           // negative: no step
  __device__ __forceinline__ bool valid() const { return position >= 0; }
};
__device__ __forceinline__ Row row_with(const WindowArgs& a, int i, int position) {
  Row r;
  r.i = i;
  r.position = position;
  if (r.position < 0) {
    r.position = -1;
    r.start = r.lo = 0x7fffffff;
    r.span = r.n_sinks = 0;
    return r;
  }
  r.start = i - r.position;
  r.lo = max(r.start, i - a.window + 1);
  r.span = (uint32_t)(i - r.lo);
  r.n_sinks = (uint32_t)(min(a.sinks - 1, r.position) + 1);
  return r;
}

// What a rare branch computes from a value that never changes goes through here: the compiler otherwise keeps it in registers across the loop.
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}


template <int CONTROL>
__device__ __forceinline__ int from_lane(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CONTROL, 0xf, 0xf, true);
}
template <class F>
__device__ __forceinline__ int wave_reduce(int v, F f) {
  v = f(v, from_lane<0xB1>(v));   // the neighbour
  v = f(v, from_lane<0x4E>(v));   // the other pair
  v = f(v, from_lane<0x141>(v));  // mirrored in eight
  v = f(v, from_lane<0x140>(v));  // mirrored in sixteen
  return f(f(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)), f(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}
// A value and the other half's, the same in both
struct Halves {
  float lo, hi;
};
__device__ __forceinline__ Halves halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ int wave_min(int v) { return wave_reduce(v, [](int a, int b) { return min(a, b); }); }
__device__ __forceinline__ int wave_max(int v) { return wave_reduce(v, [](int a, int b) { return max(a, b); }); }

// ---- 16 bytes of a row ---------------------------------------------------------------------------------------------------------------
// Elements from `col` on, zeros behind the row's `dim`; nothing behind the row is read.
template <class T>
__device__ __forceinline__ uint4 load_unit(const char* row, int col, int dim) {
  constexpr int E = 16 / sizeof(T), kBits = 8 * sizeof(T);
  const T* p = reinterpret_cast<const T*>(row);
  unsigned __int128 w = 0;
  if (dim >= E) {  // at any alignment; at the row's end its last 16 bytes, moved into place
    const int base = min(col, dim - E);
    __builtin_memcpy(&w, p + base, 16);
    if (dim % E != 0) w = col - base < E ? w >> kBits * (col - base) : 0;
    else if (col != base) w = 0;
  } else if (col == 0) {
#pragma unroll 1
    for (int e = 0; e < dim; ++e) {
      uint32_t u = 0;
      __builtin_memcpy(&u, p + e, sizeof(T));
      w |= (unsigned __int128)u << kBits * e;
    }
  }
  uint4 r;
  __builtin_memcpy(&r, &w, 16);
  return r;
}

// ---- tiles in LDS -------------------------------------------------------------------------------------------------------------------
// Read in two ways: 16 bytes of 16 rows at once (a product's first operand), and, in bf16, pieces of four rows' 64 bytes (the transposed reads).  bf16: a row's pieces
// are exchanged by bits of the row's number, so that both touch every bank once (rows padded to 272 bytes: 2.7e7 cycles of conflicts in a long sequence of 8 heads of 128,
// exchanged: 8e5; 266 us and 242, with the sums in ordinary registers).  fp32: padded by 16 bytes; its second reads are of single elements.
template <class T, int DP>
struct TileShape {
  static constexpr bool kExchanged = sizeof(T) == 2;
  static constexpr int kStride = kExchanged ? (DP <= 32 ? 64 : DP <= 64 ? 128 : 256) : DP * (int)sizeof(T) + 16;
  static constexpr int kBytes = kTile * kStride;
  static constexpr int kUnits = DP * (int)sizeof(T) / 16;  // of a row
  // what a row's pieces are exchanged by: rows next to each other by the higher bits, which the transposed reads of four rows need
  __device__ __forceinline__ static int mix(int row) {
    return kStride == 64 ? row >> 2 & 3 : kStride == 128 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
  }
  __device__ __forceinline__ static int at(int row, int unit) { return row * kStride + 16 * (kExchanged ? unit ^ mix(row) : unit); }
};

// Memory that a tile lies in, for loads that give zeros outside it.  (Workgroups hold the same: in scalar registers.)
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
struct Window {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ Window(const char* p, int64_t bytes) : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, (int)bytes, 0x00020000)) {}
  __device__ __forceinline__ uint4 load(uint32_t at) const {
    const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
};
constexpr uint32_t kOutside = 0x80000000u;  // of any window

// A fetch of a tile of 32 rows by WAVES wavefronts (one: each by itself), held in registers until the tile's place is free.  FAST: rows are whole 16-byte pieces, four-byte aligned, and 32 of them
// span less than 2 GB; every load is then issued unconditionally, so that the wait for one tile leaves the next one's on their way.
template <class T, int DP, int WAVES, bool FAST>
struct Fetch {
  static constexpr int kUnits = TileShape<T, DP>::kUnits, kThreads = 64 * WAVES, kAll = kTile * kUnits, kEach = (kAll + kThreads - 1) / kThreads;
  static constexpr bool kEven = kThreads % kUnits == 0;  // a thread's units lie in one column, the same number of rows apart
  static constexpr int kPlaces = kEven ? 1 : kEach;
  __device__ __forceinline__ static int tid() { return threadIdx.x % kThreads; }
  // where a thread's units lie in a tile of rows `step` bytes apart
  struct Places {
    uint32_t at[FAST ? kPlaces : 1];
    uint32_t more;
    __device__ __forceinline__ void set(int64_t step, int dim) {
      if constexpr (FAST) {
        more = (uint32_t)(kThreads / kUnits) * (uint32_t)step;
#pragma unroll
        for (int u = 0; u < kPlaces; ++u) at[u] = unit_at(tid(), u) * 16 < dim * (int)sizeof(T) && row_at(tid(), u) < kTile ? row_at(tid(), u) * (uint32_t)step + 16 * unit_at(tid(), u) : kOutside;
      }
    }
  };
  uint4 v[kEach];
  __device__ __forceinline__ static int row_at(int tid, int u) { return (tid + u * kThreads) / kUnits; }
  __device__ __forceinline__ static int unit_at(int tid, int u) { return (tid + u * kThreads) % kUnits; }
  // Of rows `step` bytes apart: tile number `tile`, `count` rows of it; the others zero (or, where rows share memory, any value of theirs)
  __device__ __forceinline__ void request(const Places& p, const char* array, int64_t step, int tile, int count, int dim) {
    if constexpr (FAST) {
      const char* rows = array + (uint64_t)(uint32_t)tile * (uint32_t)(kTile * (uint32_t)step);
      const uint32_t last = (uint32_t)(count < kTile ? count - 1 : kTile - 1);
      const Window w(rows, count > 0 ? (int)(last * (uint32_t)step + dim * (uint32_t)sizeof(T)) : 0);
#pragma unroll
      for (int u = 0; u < kEach; ++u) v[u] = w.load(kEven ? p.at[0] + u * p.more : p.at[kEven ? 0 : u]);
    } else {
      const char* rows = array + tile * (kTile * step);
      const int tid = fresh(threadIdx.x % kThreads);
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        v[u] = make_uint4(0, 0, 0, 0);
        if (row_at(tid, u) < count) v[u] = load_unit<T>(rows + row_at(tid, u) * step, unit_at(tid, u) * (16 / (int)sizeof(T)), dim);
      }
    }
  }
  __device__ __forceinline__ void store(char* tile) const {
#pragma unroll
    for (int u = 0; u < kEach; ++u)
      if (kAll % kThreads == 0 || tid() + u * kThreads < kAll)
        *reinterpret_cast<uint4*>(tile + TileShape<T, DP>::at(row_at(tid(), u), unit_at(tid(), u))) = v[u];
  }
};

// A wavefront's own 32 rows, fetched like any tile, whole rows at a time, and handed to their lanes through a place in LDS of the wavefront's own: lanes that each read
// their row piece by piece ask for every line once for each piece, while it is on its way (128 x 4096 steps of 8 heads of 64 in bf16: 950 us against 828; gradient of 4
// heads of 32 in fp32: 1330 against 1136).
template <class T, int DP, bool FAST>
struct OwnRows : Fetch<T, DP, 1, FAST> {
  typedef Fetch<T, DP, 1, FAST> Base;
  __device__ __forceinline__ void request_own(const char* array, int64_t step, int tile, int count, int dim) {
    typename Base::Places p;
    p.set(step, dim);
    this->request(p, array, step, tile, count, dim);
  }
  // one wavefront's LDS accesses are done in order; the fences keep the compiler from changing it
  template <class P>
  __device__ __forceinline__ void take(typename P::Own& own, char* place, uint32_t flip) const {
    this->store(place);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    P::load_own(own, place, flip);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
};

// ---- products ----------------------------------------------------------------------------------------------------------------------
// The row among 32 that register r of a 32 x 32 result holds in half h of a wavefront
__device__ __forceinline__ constexpr int result_row(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

template <class T, int DP>
struct Products;

template <int DP>
struct Products<bf16_t, DP> {
  typedef TileShape<bf16_t, DP> Shape;
  struct Own {
    bf16x8_t v[DP / 16];
  };
  // unit s of a lane's row: elements 2 E s + E half on
  static __device__ __forceinline__ void load_own(Own& own, const char* tile, uint32_t flip) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      uint4 u = *reinterpret_cast<const uint4*>(tile + Shape::at(lane % 32, 2 * s + lane / 32));
      u.x ^= flip; u.y ^= flip; u.z ^= flip; u.w ^= flip;
      __builtin_memcpy(&own.v[s], &u, 16);
    }
  }
  static __device__ __forceinline__ float dot(const Own& a, const Own& b) {  // of this half's elements
    float s = 0.f;
#pragma unroll
    for (int n = 0; n < DP / 16; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += (float)a.v[n][e] * (float)b.v[n][e];
    return s;
  }
  // (a piece's place is the row's beginning and the exchanged number of the piece: one exclusive or from one piece to another)
  static __device__ __forceinline__ f32x16_t score(const char* tile, const Own& own) {
    const int lane = threadIdx.x & 63, first = Shape::at(lane % 32, lane / 32);
    f32x16_t s = {0.f};
#pragma unroll
    for (int n = 0; n < DP / 16; ++n) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_t*>(tile + (first ^ 32 * n)), own.v[n], s, 0, 0, 0);
    return s;
  }
  typedef short s16x8_t __attribute__((ext_vector_type(8)));
  // Four streamed rows of sixteen columns, transposed, for rows 16 g of columns 32 t
  static __device__ __forceinline__ s16x8_t turned(const char* tile, int t, int g) {
    const int lane = threadIdx.x & 63, row = 4 * (lane / 32) + lane % 16 / 4, unit = 2 * (lane / 16 % 2) + lane % 4 / 2, in = 8 * (lane % 2);
    const int first = (Shape::at(row, unit) + in) ^ 64 * t, second = (Shape::at(row + 8, unit) + in) ^ 64 * t;  // (rows 16 on are exchanged alike)
    typedef __attribute__((address_space(3))) i16x4_t* Lds;
    const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(tile + first + 16 * g * Shape::kStride));
    const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(tile + second + 16 * g * Shape::kStride));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ bf16x8_t pack(const float* p) {
    uint4 u = make_uint4(pack2_bf16(p[0], p[1]), pack2_bf16(p[2], p[3]), pack2_bf16(p[4], p[5]), pack2_bf16(p[6], p[7]));
    bf16x8_t r;
    __builtin_memcpy(&r, &u, 16);
    return r;
  }
  template <int N>
  static __device__ __forceinline__ void add(f32x16_t (&acc)[N], const char* tile, const float (&p)[16]) {
    const bf16x8_t w[2] = {pack(p), pack(p + 8)};
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int t = 0; t < N; ++t)
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, turned(tile, t, g)), w[g], acc[t], 0, 0, 0);
  }
};

template <int DP>
struct Products<float, DP> {
  typedef TileShape<float, DP> Shape;
  struct Own {
    float4 v[DP / 8];
  };
  // unit s of a lane's row: elements 2 E s + E half on
  static __device__ __forceinline__ void load_own(Own& own, const char* tile, uint32_t flip) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < DP / 8; ++s) {
      uint4 u = *reinterpret_cast<const uint4*>(tile + Shape::at(lane % 32, 2 * s + lane / 32));
      u.x ^= flip; u.y ^= flip; u.z ^= flip; u.w ^= flip;
      __builtin_memcpy(&own.v[s], &u, 16);
    }
  }
  static __device__ __forceinline__ float dot(const Own& a, const Own& b) {
    float s = 0.f;
#pragma unroll
    for (int n = 0; n < DP / 8; ++n) s += a.v[n].x * b.v[n].x + a.v[n].y * b.v[n].y + a.v[n].z * b.v[n].z + a.v[n].w * b.v[n].w;
    return s;
  }
  static __device__ __forceinline__ f32x16_t score(const char* tile, const Own& own) {
    const int lane = threadIdx.x & 63;
    const char* p = tile + (lane % 32) * Shape::kStride + 16 * (lane / 32);
    f32x16_t s = {0.f};
#pragma unroll
    for (int n = 0; n < DP / 8; ++n) {
      const float4 y = *reinterpret_cast<const float4*>(p + 32 * n);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(y.x, own.v[n].x, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(y.y, own.v[n].y, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(y.z, own.v[n].z, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(y.w, own.v[n].w, s, 0, 0, 0);
    }
    return s;
  }
  template <int N>
  static __device__ __forceinline__ void add(f32x16_t (&acc)[N], const char* tile, const float (&p)[16]) {
    const int lane = threadIdx.x & 63;
    const char* y = tile + 4 * (lane / 32) * Shape::kStride + 4 * (lane % 32);
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int t = 0; t < N; ++t)
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(y + result_row(r, 0) * Shape::kStride + 128 * t), p[r], acc[t], 0, 0, 0);
  }
};

// Where a row's four elements 32 t + result_row(r, half) on lie
template <class T, int DP>
__device__ __forceinline__ int four_at(int row, int t, int r, int half) {
  return sizeof(T) == 4 ? TileShape<T, DP>::at(row, 8 * t + r / 2 + half) : TileShape<T, DP>::at(row, 4 * t + r / 4) + 8 * half;
}

// acc^T += Y^T P one streamed row after another (weights of rows that a column does not see are zero), for tiles that hold infinities or NaNs: a column takes the rows that it sees (bit r of `seen` for the row
// of register r) and nothing else.  On the vector units, few registers at a time: this must not cost the loop around it any.
template <class T, int DP>
__device__ __forceinline__ void add_with_care(f32x16_t (&acc)[DP / 32], const char* tile, const float (&p)[16], uint32_t seen) {
  const int lane = fresh(threadIdx.x & 63), half = lane / 32;
#pragma unroll 1
  for (int row = 0; row < kTile; ++row) {
    const int from = row / 4 % 2, at = row / 8 * 4 + row % 4;  // the half and the register that hold the row's weights
    float w = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) w = r == at ? p[r] : w;
    w = __shfl(w, lane % 32 + 32 * from);
    const bool on = __shfl((int)seen, lane % 32 + 32 * from) >> at & 1;
    // (a bit mask, not a choice: the compiler makes branches of choices here, with half of the registers inside them)
    const uint32_t mask = on ? 0xffffffffu : 0u;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const T* y = reinterpret_cast<const T*>(tile + four_at<T, DP>(row, t, r, half));
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][r + e] = __builtin_fmaf(w, __uint_as_float(__float_as_uint(load_act(y, e)) & mask), acc[t][r + e]);
        __builtin_amdgcn_sched_barrier(0);
      }
  }
}

template <int N>
__device__ __forceinline__ bool not_finite(const f32x16_t (&acc)[N]) {
  float x = 0.f;  // zero times an infinity or a NaN stays a NaN
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) x = __builtin_fmaf(acc[t][r], 0.f, x);
  return !(x == 0.f);
}

template <class T>
__device__ __forceinline__ void store4(char* p, float a, float b, float c, float d) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
  else *reinterpret_cast<uint2*>(p) = make_uint2(pack2_bf16(a, b), pack2_bf16(c, d));
}

// 32 own rows out: through a place in LDS of the wavefront's own, so that rows are stored in runs of 16 bytes a lane.  acc^T holds an own row a lane.
template <class T, int DP>
__device__ __forceinline__ void store_rows(char* place, const f32x16_t (&acc)[DP / 32], float factor, bool zero, char* rows, int64_t step, int count, int dim) {
  typedef TileShape<T, DP> Shape;
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, h = lane / 32;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = zero ? 0.f : acc[t][r + e] * factor;
      store4<T>(place + four_at<T, DP>(lane % 32, t, r, h), o[0], o[1], o[2], o[3]);
    }
  // (one wavefront's LDS accesses are done in order; the fence keeps the compiler from moving the reads up)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (dim % E == 0) {  // no unit ends inside
#pragma unroll
    for (int u = 0; u < kTile * Shape::kUnits / 64; ++u) {
      const int at = lane + 64 * u, row = at / Shape::kUnits, c = at % Shape::kUnits * E;
      const uint4 v = *reinterpret_cast<const uint4*>(place + Shape::at(row, at % Shape::kUnits));
      if (row < count && c < dim) __builtin_memcpy(rows + row * step + (int)sizeof(T) * c, &v, 16);
    }
  } else {
#pragma unroll 1
    for (int at = lane; at < kTile * DP; at += 64) {
      const int row = at / DP, c = at % DP;
      if (row < count && c < dim) reinterpret_cast<T*>(rows + row * step)[c] = *reinterpret_cast<const T*>(place + Shape::at(row, c / E) + (int)sizeof(T) * (c % E));
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- which tiles a workgroup's rows see ------------------------------------------------------------------------------------------------
// The window's tiles first, backwards in time: the first of them is known before the rows' positions are.  Then tiles of cached slots, then of first steps.
enum { TILE_WINDOW, TILE_CACHE, TILE_SINK, TILE_NONE };
struct Tile {
  int kind, at;
};
struct Tiles {
  // of the workgroup's rows (up to 128, two a lane)
  Row r0, r1;
  int first_window;               // tile
  int cached;                     // slots that hold a step
  int newest_slot, newest;        // the slot of the cache's last step, and that step
  int least;                      // the least position of a row whose episode began before step 0
  int all_from, all_to;           // tiles that every row sees whole
  bool any_sinks;

  __device__ __forceinline__ void set(const WindowArgs& a, const Row& x, const Row& y, int first_position) {
    r0 = x;
    r1 = y;
    first_window = max(wave_min(min(r0.lo, r1.lo)), 0) / kTile;  // (of no row: behind every tile)
    const int most = wave_max(max(r0.valid() ? r0.lo : -0x7fffffff, r1.valid() ? r1.lo : -0x7fffffff));
    all_from = max(most, 0) / kTile + (max(most, 0) % kTile != 0);
    all_to = (wave_min(min(r0.valid() ? r0.i : 0x7ffffffe, r1.valid() ? r1.i : 0x7ffffffe)) + 1) / kTile - 1;
    any_sinks = a.sinks > 0 && __ballot(r0.valid() || r1.valid()) != 0;
    cached = 0;
    newest_slot = newest = 0;
    least = 0x7fffffff;
    if (a.cache_k != nullptr) {
      const int n = __builtin_amdgcn_readfirstlane(first_position);
      least = wave_min(min(r0.valid() && r0.start < 0 ? r0.position : 0x7fffffff, r1.valid() && r1.start < 0 ? r1.position : 0x7fffffff));
      if (n > 0 && least != 0x7fffffff) {
        cached = min(n, a.sinks + a.window);
        newest = n - 1;
        newest_slot = newest < a.sinks ? newest : a.sinks + (newest - a.sinks) % a.window;
      }
    }
  }
  // the step that a slot below `cached` holds
  __device__ __forceinline__ int step_of(const WindowArgs& a, int slot) const {
    if (newest < a.sinks + a.window || slot < a.sinks) return slot;  // (not yet gone round)
    return newest - newest_slot + slot - (slot <= newest_slot ? 0 : a.window);
  }
  __device__ __forceinline__ int sink_tile(const Row& r, int from) const {
    if (r.n_sinks == 0) return 0x7fffffff;
    const int last = r.start + (int)r.n_sinks - 1;
    if (last < 0 || last / kTile < from) return 0x7fffffff;
    return max(max(r.start, 0) / kTile, from);
  }
  // the one behind t
  __device__ __forceinline__ Tile next(const WindowArgs& a, Tile t) const {
    if (t.kind == TILE_WINDOW) {
      if (--t.at >= first_window) return t;
      t.kind = TILE_CACHE;
      t.at = -1;
    }
    if (t.kind == TILE_CACHE) {
      while (++t.at * kTile < cached) {
        const int slot = t.at * kTile + (threadIdx.x & 31);
        bool needed = false;
        if (slot < cached) needed = slot < a.sinks || least - step_of(a, slot) < a.window;
        if (__ballot(needed) != 0) return t;
      }
      t.kind = TILE_SINK;
      t.at = -1;
    }
    if (t.kind == TILE_SINK) {
      if (any_sinks) {
        const int n = wave_min(min(sink_tile(r0, t.at + 1), sink_tile(r1, t.at + 1)));
        if (n < first_window) return {TILE_SINK, n};
      }
      t.kind = TILE_NONE;
    }
    return t;
  }
};

// Wavefronts a SIMD that the registers are shared out for: as many as spill none to memory, but for dq of bf16 heads wider than 64 (1 to 36 registers).  (dq of fp32 heads
// wider than 96 puts 2 to 6 into accumulation registers, which it has to spare.)
template <class T, int DP, int WAVES, bool GRADIENT>
constexpr int rows_waves() { return sizeof(T) == 4 ? (DP > 64 ? 1 : DP > 32 || WAVES == 1 ? 2 : 3) : DP <= 32 || (DP <= 64 && WAVES > 1 && !GRADIENT) ? 3 : 2; }
template <class T, int DP>
constexpr int columns_waves() { return DP > (sizeof(T) == 4 ? 32 : 64) ? 1 : 2; }

// ---- output, and dq ------------------------------------------------------------------------------------------------------------------
// A workgroup: `heads_each` query heads of one key head, WAVES / heads_each tiles of 32 rows each.
template <class T, int DP, int WAVES, bool GRADIENT, bool FAST>
__global__ void __launch_bounds__(64 * WAVES, (rows_waves<T, DP, WAVES, GRADIENT>())) window_rows_kernel(const WindowArgs a) {
  typedef Products<T, DP> P;
  typedef TileShape<T, DP> Shape;
  __shared__ __attribute__((aligned(16))) char lds[4 * Shape::kBytes];  // two tiles of both arrays; a place for each wavefront's own rows before and after
  auto tile_at = [&](int buffer, int which) __attribute__((always_inline)) { return lds + (2 * buffer + which) * Shape::kBytes; };
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
  // neighbouring heads, then stretches of time, then sequences: next to each other on one XCD
  const uint32_t teams = a.group / a.heads_each;
  uint32_t at = xcd_order(blockIdx.x, gridDim.x, a.Hk * teams * a.blocks_t, a.B);
  const uint32_t head_team = at % (a.Hk * teams);
  at /= a.Hk * teams;
  const uint32_t block_t = at % a.blocks_t, b = at / a.blocks_t;
  const uint32_t hk = head_team / teams, env = b / a.seqs_per_flag;
  const uint32_t h = hk * a.group + head_team % teams * a.heads_each + wave % a.heads_each;
  const int tiles_each = WAVES / a.heads_each, row0 = (int)block_t * tiles_each * kTile, my0 = row0 + (int)(wave / a.heads_each) * kTile;
  const int i = my0 + lane % 32;
  // positions first, then rows and the first tile: all on their way together
  const int rows = tiles_each * kTile;
  const int i0 = lane < rows ? row0 + lane : a.T, i1 = 64 + lane < rows ? row0 + 64 + lane : a.T;
  int position = a.first + i, position0 = a.first + i0, position1 = a.first + i1, first_position = a.first;
  if (a.positions != nullptr) {
    const int32_t* p = a.positions + env;
    position = p[(int64_t)min(i, a.T - 1) * a.n_flags];
    position0 = p[(int64_t)min(i0, a.T - 1) * a.n_flags];
    position1 = p[(int64_t)min(i1, a.T - 1) * a.n_flags];
    first_position = p[0];
  }
  const char *kp = a.k.data + b * a.k.seq + hk * a.k.head, *vp = a.v.data + b * a.v.seq + hk * a.v.head;
  const int64_t cached_at = ((int64_t)b * a.Hk + hk) * (a.sinks + a.window);
  const char *ck = a.cache_k + cached_at * a.dk_dim * (int)sizeof(T), *cv = a.cache_v + cached_at * a.dv_dim * (int)sizeof(T);
  typedef OwnRows<T, DP, FAST> Rows;
  const int count = a.T - my0, own_tile = my0 / kTile;
  Rows own_q, own_d, own_o;
  own_q.request_own(a.q.data + b * a.q.seq + h * a.q.head, a.q.step, own_tile, a.scale != 0.f ? count : 0, a.dk_dim);
  float lse2 = 0.f, delta = 0.f;
  const int64_t stat = ((int64_t)b * a.H + h) * a.T + i;
  if constexpr (GRADIENT) {
    lse2 = a.lse[stat - i + min(i, a.T - 1)] * 1.44269504088896341f;
    own_d.request_own(a.dout.data + b * a.dout.seq + h * a.dout.head, a.dout.step, own_tile, count, a.dv_dim);
    own_o.request_own(a.out.data + b * a.out.seq + h * a.out.head, a.out.step, own_tile, count, a.dv_dim);
  }
  typedef Fetch<T, DP, WAVES, FAST> F;
  const int64_t ck_step = a.dk_dim * (int)sizeof(T), cv_step = a.dv_dim * (int)sizeof(T);
  typename F::Places pk, pv, pck, pcv;
  pk.set(a.k.step, a.dk_dim);
  pv.set(a.v.step, a.dv_dim);
  pck.set(ck_step, a.dk_dim);
  pcv.set(cv_step, a.dv_dim);
  // two tiles on their way
  F fk[2], fv[2];
  Tiles tiles;
  tiles.cached = 0;
  auto request = [&](F& k, F& v, const Tile& t) __attribute__((always_inline)) {
    const bool cache = t.kind == TILE_CACHE;
    const int n = t.kind == TILE_NONE ? 0 : (cache ? tiles.cached : a.T) - t.at * kTile;
    const int at = t.kind == TILE_NONE ? 0 : t.at;
    k.request(cache ? pck : pk, cache ? ck : kp, cache ? ck_step : a.k.step, at, n, a.dk_dim);
    v.request(cache ? pcv : pv, cache ? cv : vp, cache ? cv_step : a.v.step, at, n, a.dv_dim);
  };
  const Tile first_tile = {TILE_WINDOW, min(row0 / kTile + tiles_each, (a.T + kTile - 1) / kTile) - 1};
  request(fk[0], fv[0], first_tile);
  tiles.set(a, row_with(a, i0, i0 < a.T ? position0 : -1), row_with(a, i1, i1 < a.T ? position1 : -1), first_position);
  const Row row = row_with(a, i, i < a.T ? position : -1);
  if constexpr (GRADIENT) {  // for dk and dv: the positions (far apart in their own array), and where the episodes of each tile's rows began
    if (h == 0 && b % a.seqs_per_flag == 0 && my0 < a.T) {
      if (half == 0 && i < a.T) a.places[(int64_t)env * a.T + i] = row.position;
      const int lo = wave_min(row.valid() ? row.start : 0x7fffffff), hi = wave_max(row.valid() ? row.start : -0x7fffffff);
      if (lane == 0) a.reach[(int64_t)env * ((a.T + kTile - 1) / kTile) + my0 / kTile] = make_int2(lo, hi);
    }
  }
  char* place = lds + wave * Shape::kBytes;
  typename P::Own q, d;
  own_q.template take<P>(q, place, a.flip);
  if constexpr (GRADIENT) {
    typename P::Own o;
    own_d.template take<P>(d, place, 0);
    own_o.template take<P>(o, place, 0);
    delta = P::dot(d, o);
    const Halves both = halves(delta);
    delta = both.lo + both.hi;
    if (half == 0 && i < a.T) a.delta[stat] = delta;
  }
  __syncthreads();
  f32x16_t acc[DP / 32];
  float top = 0.f, sum = 0.f;  // output: the largest exponent (of two) so far, the sum of this half's weights
  auto pass = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) acc[t] = (f32x16_t){0.f};
    top = -__builtin_inff();
    sum = 0.f;
    Tile ahead[2];
    ahead[0] = first_tile;
    if constexpr (decltype(careful)::value) request(fk[0], fv[0], first_tile);
    ahead[1] = tiles.next(a, ahead[0]);
    request(fk[1], fv[1], ahead[1]);
    // One tile: into LDS, the one after the next requested, the products.  (The loop ends between pairs of turns only, the last turn without a tile where their number is
    // odd: with a way out between the two, or a request on some ways only, the compiler waits for both tiles at each.)
    // Within the window, where every row sees whole tiles, nothing is looked at on the way (inside).
    auto turn = [&](auto which, auto within) __attribute__((always_inline)) {
      constexpr int buffer = decltype(which)::value;
      constexpr bool inside = decltype(within)::value;
      const Tile now = ahead[buffer];
      fk[buffer].store(tile_at(buffer, 0));
      fv[buffer].store(tile_at(buffer, 1));
      if constexpr (inside) {
        ahead[buffer].at -= 2;
        fk[buffer].request(pk, kp, a.k.step, ahead[buffer].at, kTile, a.dk_dim);
        fv[buffer].request(pv, vp, a.v.step, ahead[buffer].at, kTile, a.dv_dim);
      } else {
        ahead[buffer] = tiles.next(a, ahead[buffer ^ 1]);
        request(fk[buffer], fv[buffer], ahead[buffer]);
      }
      __syncthreads();
      // What each lane's row sees of the tile, as simply as all rows allow: all of it, the steps from one on to another, or more
      enum { SEE_ALL, SEE_BAND, SEE_MORE, SEE_CACHE };
      const int j0 = now.at * kTile;
      int sight = SEE_CACHE;
      if constexpr (inside) {
        sight = SEE_ALL;
      } else if (now.kind == TILE_CACHE) {
        if (__ballot(row.valid() && row.start < 0) == 0) return;
      } else {
        const int j1 = j0 + kTile - 1;
        const bool band = j1 >= row.lo && j0 <= row.i, sinks = row.start <= j1 && row.start + (int)row.n_sinks > j0 && j0 < row.lo;
        if (now.kind == TILE_NONE || __ballot(row.valid() && (band || sinks)) == 0) return;
        sight = __ballot(row.valid() && sinks) != 0 ? SEE_MORE : __ballot(row.valid() && !(j0 >= row.lo && j1 <= row.i)) != 0 ? SEE_BAND : SEE_ALL;
      }
      // (register r's column is result_row(r, half) behind the tile's first)
      auto for_seen = [&](auto f) __attribute__((always_inline)) {  // f(register, whether it is seen)
        const int first = j0 + 4 * fresh(half);
        if (sight == SEE_BAND) {
          const uint32_t from = (uint32_t)(first - row.lo);
#pragma unroll
          for (int r = 0; r < 16; ++r) f(r, from + result_row(r, 0) <= row.span);
        } else if (sight == SEE_MORE) {
          const uint32_t from = (uint32_t)(first - row.lo), begun = (uint32_t)(first - row.start);
#pragma unroll
          for (int r = 0; r < 16; ++r) f(r, from + result_row(r, 0) <= row.span || begun + result_row(r, 0) < row.n_sinks);
        } else {
          // slots of first steps; of the ring, whose steps from `from` on are seen, up to the newest step's slot, and from where it goes round
          const bool goes_on = row.valid() && row.start < 0;
          const int from = row.position - a.window + 1;
          const bool round = tiles.newest >= a.sinks + a.window;
          const int turned = tiles.newest - tiles.newest_slot;  // a slot's step, up to the newest; a window less behind it
          const int x = round ? max(from - turned, a.sinks) : max(from, a.sinks), y = round ? max(from - turned + a.window, tiles.newest_slot + 1) : 0x7fffffff;
          const int end = goes_on ? tiles.cached : 0, last = goes_on ? (round ? tiles.newest_slot : tiles.cached - 1) : -1, heads = goes_on ? min(a.sinks, tiles.cached) : 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int slot = first + result_row(r, 0);
            f(r, (slot < heads) | ((slot >= x) & (slot <= last)) | ((slot >= y) & (slot < end)));
          }
        }
      };
      f32x16_t s = P::score(tile_at(buffer, 0), q);
      float p[16];
      if constexpr (!GRADIENT) {
        if (sight != SEE_ALL) for_seen([&](int r, bool on) __attribute__((always_inline)) { s[r] = on ? s[r] : -__builtin_inff(); });
        float most = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) most = fmaxf(most, s[r]);
        const Halves both = halves(most);
        // The sums are kept relative to the largest exponent within a factor of 2^8: nearly every tile holds a new largest score of one of 32 rows, few a much larger one.
        // (A long sequence of 8 heads of 128, window 1024: 219 us against 243 with every new one.)
        const float new_top = fmaxf(top, fmaxf(both.lo, both.hi) * a.c);
        if (__ballot(new_top > top + 8.f) != 0) {
          const float shrink = __builtin_amdgcn_exp2f(top - (new_top == -__builtin_inff() ? 0.f : new_top));
          sum *= shrink;
#pragma unroll
          for (int t = 0; t < DP / 32; ++t) acc[t] *= shrink;
          top = new_top;
        }
        const float base = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c, -base));
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += p[r];
      } else {
        const f32x16_t e = P::score(tile_at(buffer, 1), d);
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c, -lse2)) * (e[r] - delta);
        if (sight != SEE_ALL) for_seen([&](int r, bool on) __attribute__((always_inline)) { p[r] = on ? p[r] : 0.f; });
      }
      const char* y = tile_at(buffer, GRADIENT ? 0 : 1);
      if constexpr (!decltype(careful)::value) {
        P::add(acc, y, p);
      } else {
        uint32_t seen = 0xffffu;
        if (sight != SEE_ALL) {
          seen = 0;
          for_seen([&](int r, bool on) __attribute__((always_inline)) { seen |= on ? 1u << r : 0u; });
        }
        add_with_care<T, DP>(acc, y, p, seen);
      }
    };
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    do {
      if constexpr (!decltype(careful)::value && !GRADIENT) {
        // (the two tiles on their way, and the two that follow them)
        while (ahead[0].kind == TILE_WINDOW && ahead[0].at <= tiles.all_to && ahead[0].at - 1 >= tiles.all_from && ahead[0].at - 3 >= tiles.first_window) {
          turn(even, std::true_type());
          turn(odd, std::true_type());
        }
      }
      turn(even, std::false_type());
      turn(odd, std::false_type());
    } while (ahead[0].kind != TILE_NONE);
  };
  pass(std::false_type());
  if (__syncthreads_or(row.valid() && not_finite(acc))) pass(std::true_type());
  __syncthreads();
  if constexpr (!GRADIENT) {
    const Halves both = halves(sum);
    sum = both.lo + both.hi;
    if (half == 0 && a.lse != nullptr && row.i < a.T) a.lse[stat] = row.valid() ? (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : -__builtin_inff();
    store_rows<T, DP>(place, acc, 1.f / sum, !row.valid(), a.out.data + my0 * a.out.step + b * a.out.seq + h * a.out.head, a.out.step, count, a.dv_dim);
  } else {
    store_rows<T, DP>(place, acc, a.scale, !row.valid(), a.dq.data + my0 * a.dq.step + b * a.dq.seq + h * a.dq.head, a.dq.step, count, a.dk_dim);
  }
}

// ---- dk, dv ----------------------------------------------------------------------------------------------------------------------------
// A wavefront takes 32 columns of one key head and, of the query heads that share it, every `heads_each`-th; it streams the rows that see them through a place in LDS of
// its own, so that wavefronts never wait for each other (four that share tiles of rows wait at every tile for the one that has work: the gradient of 128 x 4096 steps of
// 4 heads of 32 in fp32, window 32: 1735 us against 1527).  The heads_each wavefronts of the same columns add up their sums at the end, in order.
//
// First steps are seen by every later row of their episode: in a long sequence far more tiles of rows than any other column, one wavefront's work.  There the pairs
// of tiles beyond the window are cut along the rows (far): every so many tiles of rows a wavefront takes the first `far_slots` tiles of first steps that they see, into
// fp32 parts with the tile's number beside them (8192 steps, 4 first steps: 411 us of gradient against 2881); the columns' own wavefronts add the parts with their number, in order, and take what was beyond the slots themselves.
// Tiles of rows on their way: two where a wavefront has a SIMD's registers to itself anyway (8192 steps of 8 heads of 128 in bf16, window 512: 119 us against 124 with one),
// none beside the one at work for fp32 heads wider than 64, whose registers are full without (heads of 65 to 96 put 96 of them into accumulation registers even so).
template <class T, int DP>
constexpr int tiles_ahead() { return sizeof(T) == 2 ? (DP > 64 ? 2 : 1) : DP <= 64 ? 1 : 0; }

template <class T, int DP, bool FAST>
__global__ void __launch_bounds__(256, (columns_waves<T, DP>())) window_columns_kernel(const WindowArgs a, const int far) {
  typedef Products<T, DP> P;
  typedef TileShape<T, DP> Shape;
  __shared__ __attribute__((aligned(16))) char lds[4][2 * Shape::kBytes];
  __shared__ __attribute__((aligned(16))) float all_stats[4][2][kTile];  // lse (exponent of two), delta
  __shared__ int4 all_sight[4][kTile];                                   // lo, span, start, first steps
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
  char *tile_q = lds[wave], *tile_d = lds[wave] + Shape::kBytes;
  auto& stats = all_stats[wave];
  int4* sight = all_sight[wave];
  const uint32_t heads = a.heads_each, units_each = 4 / heads, team = wave % heads;
  const int n_tiles = (a.T + kTile - 1) / kTile;
  const uint32_t per_head = far ? a.far_chunks * a.far_slots : (uint32_t)n_tiles;  // units of a key head
  // neighbouring heads, then sequences, 64 of them where there are as many, then tiles: wavefronts at work together read along a step's sequences more than along time
  // (128 x 4096 steps of 4 heads of 32 in fp32, steps 2 MB apart: 692 us against 766 with a sequence's tiles next to each other)
  const int64_t unit = (int64_t)xcd_order(blockIdx.x, gridDim.x, (a.Hk + units_each - 1) / units_each, a.B) * units_each + wave / heads;
  const bool on = unit < (int64_t)a.B * a.Hk * per_head;
  const uint32_t hk = on ? (uint32_t)(unit % a.Hk) : 0;
  const uint32_t together = a.B < 64 ? 1 : 64;
  const int64_t pair = on ? unit / a.Hk : 0, turn_of = pair / ((int64_t)together * per_head);
  const uint32_t in_turn = (uint32_t)(pair - turn_of * together * per_head), seqs = min(together, a.B - (uint32_t)turn_of * together);
  const uint32_t which = in_turn / seqs, b = (uint32_t)turn_of * together + in_turn % seqs;
  const uint32_t env = b / a.seqs_per_flag;
  const int2* reach = a.reach + (int64_t)env * n_tiles;
  const int* places = a.places + (int64_t)env * a.T;
  const int64_t slots = (int64_t)a.far_chunks * a.far_slots, head_slots = ((int64_t)b * a.Hk + hk) * slots;
  int* numbers = a.far_numbers + head_slots;
  int col_tile = on ? (int)which : -1, first_tile = 0, end_tile = n_tiles;
  if (far) {  // the columns: the chunk's slot-th tile of first steps that its rows see from beyond the window
    const int chunk = which / a.far_slots;
    first_tile = chunk * a.far_tiles;
    end_tile = min(first_tile + a.far_tiles, n_tiles);
    int from = 0;
    col_tile = -1;
    for (int n = (int)(which % a.far_slots); on && n >= 0; --n) {
      int least = 0x7fffffff;
      for (int i = first_tile * kTile + lane; i < end_tile * kTile; i += 64) {
        const Row r = row_with(a, i, i < a.T ? places[i] : -1);
        const int t = i / kTile, most = t * kTile >= a.window + kTile - 1 ? (t * kTile - a.window - kTile + 1) / kTile : -1;
        if (r.n_sinks == 0) continue;
        const int last = r.start + (int)r.n_sinks - 1, c = max(max(r.start, 0) / kTile, from);
        if (last >= 0 && c <= min(last / kTile, most)) least = min(least, c);
      }
      least = wave_min(least);
      col_tile = least == 0x7fffffff ? -1 : least;
      if (col_tile < 0) break;
      from = col_tile + 1;
    }
    if (on && team == 0 && lane == 0) numbers[which] = col_tile;
  }
  const int my0 = max(col_tile, 0) * kTile, my1 = min(my0 + kTile, a.T) - 1, j = my0 + lane % 32;
  OwnRows<T, DP, FAST> own_k, own_v;
  own_k.request_own(a.k.data + b * a.k.seq + hk * a.k.head, a.k.step, max(col_tile, 0), a.scale != 0.f ? a.T - my0 : 0, a.dk_dim);
  own_v.request_own(a.v.data + b * a.v.seq + hk * a.v.head, a.v.step, max(col_tile, 0), a.T - my0, a.dv_dim);
  // The tiles of rows that see any of the columns, 64 looked at at a time
  struct Cursor {
    int base;
    uint64_t left;
    int tile;  // -1: none yet, -2: no more
    uint32_t g;
  };
  uint64_t taken = 0;  // chunks (at most 64) whose rows beyond the window are in parts
  auto look = [&](int base) __attribute__((always_inline)) {
    const int t = base + lane;
    bool needed = false;
    if (t < end_tile) {
      const int2 r = reach[t];
      const bool beyond = t * kTile - my1 >= a.window;
      needed = r.x <= my1 && (!beyond || (a.sinks > 0 && (int64_t)r.y + a.sinks > my0)) && (far ? beyond : t >= col_tile);
      if (beyond && !far && taken != 0 && (taken >> (t / a.far_tiles) & 1)) needed = false;
    }
    return (uint64_t)__ballot(needed);
  };
  auto next = [&](Cursor c) __attribute__((always_inline)) {
    if (c.tile == -2) return c;
    if (c.tile >= 0 && (c.g += heads) < a.group) return c;
    c.g = team;
    while (c.left == 0) {
      c.base += 64;
      if (c.base >= end_tile) {
        c.tile = -2;
        return c;
      }
      c.left = look(c.base);
    }
    const int bit = __builtin_ctzll(c.left);
    c.left &= c.left - 1;
    c.tile = c.base + bit;
    return c;
  };
  typedef Fetch<T, DP, 1, FAST> F;
  typename F::Places pq, pd;
  pq.set(a.q.step, a.dk_dim);
  pd.set(a.dout.step, a.dv_dim);
  const char *qp = a.q.data + b * a.q.seq, *dp = a.dout.data + b * a.dout.seq;
  constexpr int kSets = tiles_ahead<T, DP>() > 1 ? 2 : 1;
  struct Set {
    F q, d;
    float lse, delta;
    int position;
  } sets[kSets];
  auto request = [&](Set& set, const Cursor& c) __attribute__((always_inline)) {
    const uint32_t h = hk * a.group + c.g;
    const int i0 = c.tile < 0 ? 0 : c.tile * kTile, n = c.tile < 0 ? 0 : a.T - i0;
    set.q.request(pq, qp + h * a.q.head, a.q.step, i0 / kTile, n, a.dk_dim);
    set.d.request(pd, dp + h * a.dout.head, a.dout.step, i0 / kTile, n, a.dv_dim);
    const int i = min(i0 + lane % kTile, a.T - 1);
    const int64_t stat = ((int64_t)b * a.H + h) * a.T + i;
    set.lse = a.lse[stat];
    set.delta = a.delta[stat];
    set.position = places[i];
  };
  // (the rows next to the columns are always looked at: on their way before anything else is known)
  const bool near = !far && tiles_ahead<T, DP>() > 0;
  const Cursor beside = {col_tile, 0, col_tile < 0 ? -2 : col_tile, team};
  if (near) request(sets[0], beside);
  if (!far && on) {
    for (int s0 = 0; s0 < (int)slots; s0 += 64)
      for (uint64_t left = __ballot(s0 + lane < (int)slots && numbers[min(s0 + lane, (int)slots - 1)] == col_tile); left != 0; left &= left - 1)
        taken |= 1ull << ((s0 + __builtin_ctzll(left)) / a.far_slots);
  }
  typename P::Own k, v;
  own_k.template take<P>(k, tile_q, a.flip);
  own_v.template take<P>(v, tile_d, 0);
  f32x16_t dk[DP / 32], dv[DP / 32];
  auto pass = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) dk[t] = dv[t] = (f32x16_t){0.f};
    if (col_tile < 0) return;
    Cursor ahead[kSets];
    ahead[0] = beside;
    if (far) ahead[0] = next({first_tile, look(first_tile), -1, team});
    else ahead[0].left = look(col_tile) & ~1ull;
    if (tiles_ahead<T, DP>() > 0 && (!near || decltype(careful)::value)) request(sets[0], ahead[0]);
    if constexpr (kSets > 1) {
      ahead[1] = next(ahead[0]);
      request(sets[1], ahead[1]);
    }
    auto turn = [&](auto which) __attribute__((always_inline)) {
      constexpr int at = decltype(which)::value;
      Set& set = sets[at];
      const Cursor now = ahead[at];
      if constexpr (tiles_ahead<T, DP>() == 0) request(set, now);
      __builtin_amdgcn_wave_barrier();
      set.q.store(tile_q);
      set.d.store(tile_d);
      if (lane < kTile) {
        const int i = now.tile * kTile + lane;
        const Row seer = row_with(a, i, now.tile >= 0 && i < a.T ? set.position : -1);
        stats[0][lane] = seer.valid() ? set.lse * 1.44269504088896341f : 0.f;
        stats[1][lane] = seer.valid() ? set.delta : 0.f;
        sight[lane] = make_int4(seer.lo, (int)seer.span, seer.start, (int)seer.n_sinks);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      ahead[at] = next(ahead[(at + kSets - 1) % kSets]);
      if constexpr (tiles_ahead<T, DP>() > 0) request(set, ahead[at]);
      // (a row's last step is lo + span; rows that hold no step see nothing: lo above every column)
      const int4 w = sight[lane % 32];
      const int last = w.x == 0x7fffffff ? -1 : w.x + w.y;
      const bool whole = w.x <= my0 && my1 <= last, band = w.x <= my1 && my0 <= last, sinks = (int64_t)w.z + w.w > my0 && w.z <= my1;
      if (__ballot(band || sinks) == 0) return;
      const bool masked = __ballot(!whole) != 0, more = __ballot(sinks) != 0;
      auto for_seen = [&](auto f) __attribute__((always_inline)) {  // f(register, whether its row sees the lane's column)
        const int4* from = sight + 4 * fresh(half);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int4 x = from[result_row(r, 0)];
          f(r, (uint32_t)(j - x.x) <= (uint32_t)x.y || (more && (uint32_t)(j - x.z) < (uint32_t)x.w));
          if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
      };
      const f32x16_t s = P::score(tile_q, k), e = P::score(tile_d, v);
      float p[16], ds[16];
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const float4 l = *reinterpret_cast<const float4*>(&stats[0][result_row(r, half)]);
        const float4 m = *reinterpret_cast<const float4*>(&stats[1][result_row(r, half)]);
        const float ls[4] = {l.x, l.y, l.z, l.w}, ms[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          p[r + u] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + u], a.c, -ls[u]));
          ds[r + u] = p[r + u] * (e[r + u] - ms[u]);
        }
      }
      if (masked) {
        for_seen([&](int r, bool on) __attribute__((always_inline)) {
          p[r] = on ? p[r] : 0.f;
          ds[r] = on ? ds[r] : 0.f;
        });
      }
      if constexpr (!decltype(careful)::value) {
        P::add(dv, tile_d, p);
        P::add(dk, tile_q, ds);
      } else {
        uint32_t seen = 0xffffu;
        if (masked) {
          seen = 0;
          for_seen([&](int r, bool on) __attribute__((always_inline)) { seen |= on ? 1u << r : 0u; });
        }
        add_with_care<T, DP>(dv, tile_d, p, seen);
        add_with_care<T, DP>(dk, tile_q, ds, seen);
      }
    };
    while (ahead[0].tile >= 0) {
      turn(std::integral_constant<int, 0>());
      if constexpr (kSets > 1) turn(std::integral_constant<int, 1>());
    }
  };
  pass(std::false_type());
  if (__ballot(j < a.T && (not_finite(dk) || not_finite(dv))) != 0) pass(std::true_type());
  // (a part: four registers a lane, lanes next to each other; dk, then dv)
  constexpr int kPart = 64 * 16 * (DP / 32);
  if (taken != 0) {  // the chunks' parts, every heads-th to a wavefront
    uint32_t n = 0;
    for (int s0 = 0; s0 < (int)slots; s0 += 64)
      for (uint64_t left = __ballot(s0 + lane < (int)slots && numbers[min(s0 + lane, (int)slots - 1)] == col_tile); left != 0; left &= left - 1, ++n) {
        if (n % heads != team) continue;
        const float4* part = reinterpret_cast<const float4*>(a.far_parts + (head_slots + s0 + __builtin_ctzll(left)) * (2 * kPart)) + lane;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const float4 x = part[64 * (4 * t + r / 4)], y = part[kPart / 4 + 64 * (4 * t + r / 4)];
            dk[t][r] += x.x; dk[t][r + 1] += x.y; dk[t][r + 2] += x.z; dk[t][r + 3] += x.w;
            dv[t][r] += y.x; dv[t][r + 1] += y.y; dv[t][r + 2] += y.z; dv[t][r + 3] += y.w;
          }
      }
  }
  // the heads' sums, in order
  if (heads > 1) {
    float4* mine = reinterpret_cast<float4*>(lds[wave]) + lane;
    auto gather = [&](f32x16_t (&acc)[DP / 32]) __attribute__((always_inline)) {
      __syncthreads();
      if (team != 0) {
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
          for (int r = 0; r < 16; r += 4) mine[64 * (4 * t + r / 4)] = make_float4(acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]);
      }
      __syncthreads();
      if (team == 0) {
        for (uint32_t n = 1; n < heads; ++n) {
          const float4* other = reinterpret_cast<const float4*>(lds[wave + n]) + lane;
#pragma unroll
          for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
              const float4 x = other[64 * (4 * t + r / 4)];
              acc[t][r] += x.x; acc[t][r + 1] += x.y; acc[t][r + 2] += x.z; acc[t][r + 3] += x.w;
            }
        }
      }
    };
    gather(dk);
    gather(dv);
    __syncthreads();
  }
  if (team != 0 || col_tile < 0) return;
  if (far) {
    float4* part = reinterpret_cast<float4*>(a.far_parts + (head_slots + which) * (2 * kPart)) + lane;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        part[64 * (4 * t + r / 4)] = make_float4(dk[t][r], dk[t][r + 1], dk[t][r + 2], dk[t][r + 3]);
        part[kPart / 4 + 64 * (4 * t + r / 4)] = make_float4(dv[t][r], dv[t][r + 1], dv[t][r + 2], dv[t][r + 3]);
      }
    return;
  }
  store_rows<T, DP>(lds[wave], dk, a.scale, false, a.dk.data + my0 * a.dk.step + b * a.dk.seq + hk * a.dk.head, a.dk.step, a.T - my0, a.dk_dim);
  store_rows<T, DP>(lds[wave], dv, 1.f, false, a.dv.data + my0 * a.dv.step + b * a.dv.seq + hk * a.dv.head, a.dv.step, a.T - my0, a.dv_dim);
}

// The wavefronts that fetch a tile, at the least: a wavefront that fetches one of wide fp32 heads alone holds 128 registers of it and spills.
constexpr int least_waves(size_t elem, int dim) { return elem == 4 && dim > 64 ? 4 : 1; }

// ---- launches --------------------------------------------------------------------------------------------------------------------------
enum { WINDOW_OUTPUT, WINDOW_DQ, WINDOW_DKV, WINDOW_FAR };

template <class T, int DP, int WAVES, bool FAST>
void launch_window(const WindowArgs& a, int pass, unsigned blocks, hipStream_t s) {
  if (pass == WINDOW_OUTPUT) hipLaunchKernelGGL((window_rows_kernel<T, DP, WAVES, false, FAST>), dim3(blocks), dim3(64 * WAVES), 0, s, a);
  if (pass == WINDOW_DQ) hipLaunchKernelGGL((window_rows_kernel<T, DP, WAVES, true, FAST>), dim3(blocks), dim3(64 * WAVES), 0, s, a);
}
template <class T, int DP>
void launch_window(const WindowArgs& a, int pass, int waves, unsigned blocks, hipStream_t s) {
  if (pass == WINDOW_DKV || pass == WINDOW_FAR) {
    if (a.fast) hipLaunchKernelGGL((window_columns_kernel<T, DP, true>), dim3(blocks), dim3(256), 0, s, a, pass == WINDOW_FAR);
    else hipLaunchKernelGGL((window_columns_kernel<T, DP, false>), dim3(blocks), dim3(256), 0, s, a, pass == WINDOW_FAR);
    return;
  }
  if (!a.fast) return launch_window<T, DP, 4, false>(a, pass, blocks, s);
  if constexpr (least_waves(sizeof(T), DP) <= 1) {
    if (waves == 1) return launch_window<T, DP, 1, true>(a, pass, blocks, s);
  }
  if constexpr (least_waves(sizeof(T), DP) <= 2) {
    if (waves == 2) return launch_window<T, DP, 2, true>(a, pass, blocks, s);
  }
  launch_window<T, DP, 4, true>(a, pass, blocks, s);
}
// Heads as wide as the wider of keys and values, in steps of 32
template <class T>
void launch_window(const WindowArgs& a, int pass, int waves, unsigned blocks, hipStream_t s) {
  const int d = a.dk_dim > a.dv_dim ? a.dk_dim : a.dv_dim;
  if (d <= 32) launch_window<T, 32>(a, pass, waves, blocks, s);
  else if (d <= 64) launch_window<T, 64>(a, pass, waves, blocks, s);
  else if (d <= 96) launch_window<T, 96>(a, pass, waves, blocks, s);
  else launch_window<T, 128>(a, pass, waves, blocks, s);
}
void launch_window_f32(const WindowArgs& a, int pass, int waves, unsigned blocks, hipStream_t s);
void launch_window_bf16(const WindowArgs& a, int pass, int waves, unsigned blocks, hipStream_t s);

}  // namespace marl
