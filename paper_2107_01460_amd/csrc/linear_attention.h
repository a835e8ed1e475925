// Linear attention with a decay for each head, its gradient, and the states between stretches of time: one scan.
//
// With x, y, z arrays of rows over time and g the head's decay, a scan forms
//     out_i = inner sum_j g^|i-j| (x_i . y_j) z_j + inter g^(..) S^T x_i        S <- g^n S + update sum_j g^(..) y_j z_j^T
// over the steps j up to i (a reverse scan: from i on) in i's episode, S being the state that came in.  Everything is that:
//     out: (x, y, z) = (q, k, v);   dq: (dout, v, k), the state transposed;   dv: (k, q, dout) and dk: (v, dout, q) in reverse,
// because dq_i = scale S_i dout_i with the same S, and R_j = scale q_j dout_j^T + g R_{j+1} gives dv_j = R_j^T k_j, dk_j = R_j v_j.
//
// A wavefront takes up to 32 z columns of one head of one sequence through time, a tile of 16 (fp32) or 32 steps (bf16) at once, on the matrix
// cores, with its columns of S in accumulator registers: four small products a tile, scores y x^T, x S, scores z and y^T z.  Transposed
// throughout (out^T = z^T scores^T), the accumulator layout of a product -- lane = column, four rows in registers -- is the operand layout of
// the next, so that neither scores nor S go through LDS.
// A workgroup of up to four wavefronts takes neighbouring heads (and all slices of their columns): a step's rows of neighbouring heads are one run of
// memory, and steps are far apart in it (megabytes, when there are many sequences), so its wavefronts fetch and store whole runs together and hand
// them to each other through LDS; the next tile is on its way in registers meanwhile.
//
// Measured (MI355X): output of 128 x 4096 steps of 8 heads of 64 in bf16 with states 697 us, 4.6 TB/s, 94 % of a copy's rate, bound by memory (a wavefront a
// head with its own loads: 1070); gradient of 128 x 4096 steps of 4 heads of 32 in fp32 599 us, 1.84 GB read and 0.87 written beyond the L2, 4.5 TB/s, where every
// array once is 1.2 and 0.87 (dk and dv share their arrays in the L2, dq, which walks the other way, reads its own again); 32 768 steps of one sequence with 8 query
// heads of 128 on 2 in bf16 81 us for the scan, 0.30 GB beyond the L2, 3.7 TB/s (each query head reads the shared keys and values anew: every array once is 0.20),
// vector ALUs busy 50 %, matrix cores 27 %: none of them full, two wavefronts a SIMD.
#pragma once
#include "split_bf16.h"

namespace marl {

constexpr int kMaxRoles = 3;

struct ScanArray {
  const char* data;
  int64_t step, seq, head;  // bytes
  uint32_t share;           // query heads per head of this array
  int32_t dim;
};

// A state [rows][columns] fp32 of (sequence, query head) u and stretch of time p at data + (u * stretches + p) * size, element (r, c) at r * row + c * col
struct ScanState {
  float* data;
  int32_t stretches, row, col;
};

struct ScanRole {
  ScanArray x, y, z, out;
  int32_t out_f32;  // out: a share in fp32, of a gradient that query heads share
  int32_t reverse;
  float inner, inter, update;
  ScanState from, to;
};

struct ScanArgs {
  ScanRole role[kMaxRoles];
  const float* decay;
  const uint8_t* done;
  float* carry;          // states only: [sequence, head][stretch] factor from a stretch's first state to its last, or kCarryEnded
  int32_t T, B;
  uint32_t n_roles, H, seqs_per_flag, n_stretches;
  int32_t stretch;       // steps of a stretch, whole tiles
  uint32_t pairs;        // B * H
};

// A carry that is no factor (a decay is none below 0): an episode ended in the stretch, so that nothing of what came in is left.  A power of a decay above 0 that
// 32 bits do not hold is rounded up to the least number that they do, not down to 0: an infinity that came in stays one, as step by step.
constexpr float kCarryEnded = -2.f, kCarryLeast = 0x1p-149f;

template <class T>
struct ScanTraits;
template <>
struct ScanTraits<float> {
  typedef floatx4 Frag;                     // four elements along a contraction
  static constexpr int kSub = 1;            // blocks of sixteen steps in a tile: the fewest products
};
template <>
struct ScanTraits<bf16_t> {
  typedef shortx4 Frag;
  static constexpr int kSub = 2;            // products contract over 32 steps, and S is split into parts once for 32
};
// Feature of element e of lane group g in tile a of N tiles of sixteen x and y features.  bf16: two tiles deal a lane eight consecutive ones, 16 bytes;
// the last of an odd number stands alone.
template <class T, int N>
__host__ __device__ constexpr bool in_pair(int a) { return sizeof(T) == 2 && a < N / 2 * 2; }
template <class T, int N>
__device__ __forceinline__ int feat(int a, int g, int e) {
  return in_pair<T, N>(a) ? 32 * (a / 2) + 8 * g + 4 * (a & 1) + e : 16 * a + 4 * g + e;
}

__device__ __forceinline__ double ipow(float base, int m) {  // base^m, 0^0 = 1
  double r = 1.0, g = base;
  for (; m != 0; m >>= 1, g *= g)
    if (m & 1) r *= g;
  return r;
}

// ---- products of 16 x 16 outputs; the contraction index of element e of lane group g is the same on both sides -----------------------
// bf16: one instruction, of 32 along the contraction, half of it zeros where there is one tile.  It takes no longer than the one of 16, and the two must not meet: a
// product that adds to the result of one of the other length, a few instructions behind it, gets half of that result or none of it, and the compiler puts no wait
// between them (back to back, half of all values were wrong; of one length, none).
__device__ __forceinline__ floatx4 mma(floatx4 a, floatx4 b, floatx4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ shortx8 both(shortx4 a, shortx4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
// over two tiles' contraction: one instruction of twice the length in bf16
__device__ __forceinline__ floatx4 mma2(floatx4 a0, floatx4 a1, floatx4 b0, floatx4 b1, floatx4 c) { return mma(a1, b1, mma(a0, b0, c)); }
__device__ __forceinline__ floatx4 mma2(shortx4 a0, shortx4 a1, shortx4 b0, shortx4 b1, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, both(a0, a1)), __builtin_bit_cast(bf16x8, both(b0, b1)), c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mma(shortx4 a, shortx4 b, floatx4 c) { return mma2(a, shortx4{}, b, shortx4{}, c); }

__device__ __forceinline__ shortx4 pack4(floatx4 v) {
  const uint2 u = make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]));
  return __builtin_bit_cast(shortx4, u);
}
__device__ __forceinline__ floatx4 unpack4(shortx4 s) {
  const uint2 u = __builtin_bit_cast(uint2, s);
  return floatx4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u)};
}
// fp32 values as operands beside exact ones.  bf16: as a sum of two parts (relative error 2^-16 of a term: scores and S, where the result is an output of eight bits
// or a share of one) or of three (2^-24: what enters a state that goes on).  Three for the outputs too: 3e-5 instead of 1e-4 of them rounded to another neighbour (the
// error against 64 bits, that of rounding, is 0.0017 either way), at 728 us instead of 697 for the rollout of the header, 146 instead of 130 for 32 768 steps.
template <class T, int P>
struct Parts {
  typename ScanTraits<T>::Frag p[sizeof(T) == 4 ? 1 : P];
};
template <class T, int P>
__device__ __forceinline__ Parts<T, P> parts_of(floatx4 v) {
  Parts<T, P> r;
  if constexpr (sizeof(T) == 4) {
    r.p[0] = v;
  } else {
#pragma unroll
    for (int k = 0; k < P; ++k) {
      r.p[k] = pack4(v);
      if (k + 1 < P) v -= unpack4(r.p[k]);
    }
  }
  return r;
}
__device__ __forceinline__ floatx4 widen4(floatx4 v) { return v; }
__device__ __forceinline__ floatx4 widen4(shortx4 v) { return unpack4(v); }

// One step after another from memory, where there are infinities or NaNs: a matrix product multiplies masked places by zero, which makes a NaN of
// them, and would carry them into other steps' and other episodes' outputs.  n steps from t0 on, S before them (reverse: behind them) on entry.
template <class T, int NK, int NV, bool STATE_ONLY>
__device__ void scan_slow(floatx4 (&S)[NK][NV], const ScanRole& r, const char* xb, const char* yb, const char* zb, char* ob, int t0, int n, int slice0,
                          float decay, const uint8_t* done, int64_t n_flags, int i, int g) {
  for (int s = 0; s < n; ++s) {
    const int64_t t = t0 + (r.reverse ? n - 1 - s : s);
    const bool end = done != nullptr && done[t * n_flags] != 0;
    const T* y = reinterpret_cast<const T*>(yb + t * r.y.step);
    const T* z = reinterpret_cast<const T*>(zb + t * r.z.step);
    const T* x = STATE_ONLY ? nullptr : reinterpret_cast<const T*>(xb + t * r.x.step);
    float zv[NV], o[NV];
#pragma unroll
    for (int b = 0; b < NV; ++b) {
      const int c = slice0 + 16 * b + i;
      zv[b] = c < r.z.dim ? r.update * load_act(z, c) : 0.f;
      o[b] = 0.f;
    }
    const float before = r.reverse ? 1.f : decay, after = r.reverse ? decay : 1.f;
#pragma unroll
    for (int a = 0; a < NK; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int f = feat<T, NK>(a, g, e);
        const bool in = f < r.y.dim;
        const float yv = in ? load_act(y, f) : 0.f, xv = STATE_ONLY || !in ? 0.f : load_act(x, f);
#pragma unroll
        for (int b = 0; b < NV; ++b) {
          float v = S[a][b][e];
          if (r.reverse && end) v = 0.f;
          v = v * before + yv * zv[b];
          if (!in) v = 0.f;
          if (in) o[b] += xv * v;
          S[a][b][e] = !r.reverse && end ? 0.f : v * after;
        }
      }
    if constexpr (!STATE_ONLY) {
#pragma unroll
      for (int b = 0; b < NV; ++b) {
        float v = o[b];
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
        const int c = slice0 + 16 * b + i;
        if (g == 0 && c < r.z.dim) {
          char* p = ob + t * r.out.step;
          v *= r.inter;
          if (r.out_f32 || sizeof(T) == 4)
            reinterpret_cast<float*>(p)[c] = v;
          else
            reinterpret_cast<bf16_t*>(p)[c] = to_bf16(v);
        }
      }
    }
  }
}

// Between LDS writes and reads of one wavefront's own part: its LDS accesses take effect in order, the compiler has to keep it.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A copy that the compiler takes for a new value: what a rare branch works out from it is worked out there, not kept in registers across the loop
// (a hundred of them in all, and spilled).
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// ---- tiles in LDS: [sequence, head][step][pieces of 16 bytes], a row's pieces exchanged so that sixteen rows' equal pieces lie in different banks --------
template <int PIECES>
__device__ __forceinline__ int swizzle(int row) {
  return PIECES % 16 == 0 ? row & 15 : PIECES % 8 == 0 ? row >> 1 & 7 : PIECES % 4 == 0 ? row >> 2 & 3 : row >> 3 & 1;
}
// Rows: lane (i, g) gets features feat(a, g, 0..3) of step `row`
template <class T, int N>
struct Rows {
  typename ScanTraits<T>::Frag f[N];
};
template <class T, int N>
__device__ __forceinline__ void rows_of(Rows<T, N>& r, const char* tile, int row, int g) {
  constexpr int kPieces = N * (int)sizeof(T);
  const char* p = tile + row * kPieces * 16;
  const int swz = swizzle<kPieces>(row);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int t = 0; t < N; ++t) r.f[t] = *reinterpret_cast<const floatx4*>(p + ((4 * t + g) ^ swz) * 16);
  } else {
#pragma unroll
    for (int t = 0; t + 1 < N; t += 2) {
      const shortx8 v = *reinterpret_cast<const shortx8*>(p + ((2 * t + g) ^ swz) * 16);
      r.f[t] = __builtin_shufflevector(v, v, 0, 1, 2, 3);
      r.f[t + 1] = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    }
    if constexpr (N % 2 == 1) r.f[N - 1] = *reinterpret_cast<const shortx4*>(p + ((2 * (N - 1) + (g >> 1)) ^ swz) * 16 + 8 * (g & 1));
  }
}
// Columns: lane (i, g) gets one feature at steps 4 g .. 4 g + 3 of the block of sixteen steps that begins at `row`.  first: of the sixteen features,
// run: how far apart fours of them lie (lanes i = 4 c .. 4 c + 3 take first + run c .. + 3)
template <class T, int PIECES>
__device__ __forceinline__ floatx4 column(const float* tile, int row, int first, int run, int i, int g) {
  const int f = first + run * (i >> 2) + (i & 3);
  floatx4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int at = row + 4 * g + e;
    v[e] = tile[at * PIECES * 4 + (((f >> 2) ^ swizzle<PIECES>(at)) << 2) + (f & 3)];
  }
  return v;
}
template <class T, int PIECES>
__device__ __forceinline__ shortx4 column(const bf16_t* tile, int row, int first, int run, int i, int g) {
  typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
  const int at = row + 4 * g + (i >> 2), f = first + run * (i & 3);  // (the transposing read: a lane names four features of one step)
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(tile + at * PIECES * 8 + (((f >> 3) ^ swizzle<PIECES>(at)) << 3) + (f & 7)));
}

// ---- a workgroup's share of an array's tile: SLOTS pieces a thread, piece fastest, then head, then step ------------------------------------
// Sixteen bytes at any element's address (the accesses of this target need no alignment)
template <class P>
__device__ __forceinline__ uint4 load16(const P* p) {
  uint4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
template <class P>
__device__ __forceinline__ void store16(P* p, uint4 v) { __builtin_memcpy(p, &v, 16); }
__device__ __forceinline__ uint4 shift_right(uint4 v, int bytes) {  // 1 .. 15
  uint64_t lo = v.x | (uint64_t)v.y << 32, hi = v.z | (uint64_t)v.w << 32;
  if (bytes < 8) {
    lo = lo >> 8 * bytes | hi << (64 - 8 * bytes);
    hi >>= 8 * bytes;
  } else {
    lo = hi >> (8 * bytes - 64);
    hi = 0;
  }
  return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

// WHOLE: the arrays' rows are whole pieces.
template <class T, int PIECES, int P, int TILE, int THREADS, bool WHOLE>
struct Stage {
  static constexpr int E = 16 / sizeof(T), kAll = PIECES * P * TILE, kSlots = (kAll + THREADS - 1) / THREADS;
  static constexpr bool kShort = !WHOLE && PIECES * E <= 16;  // rows may be shorter than sixteen bytes
  const char* from[kSlots];  // of the piece in the tile that is fetched next
  uint4 v[kSlots];
  uint32_t past = 0;         // slots whose pieces lie past the array's columns: their loads go to column 0, zeros go to LDS
  uint32_t last = 0;         // slots whose pieces are a row's last columns and fewer than sixteen bytes: the sixteen bytes that end with the row are loaded
  static __device__ __forceinline__ int index(int s, int tid) { return min(s * THREADS + tid, kAll - 1); }
  static __device__ __forceinline__ int piece(int q) { return q % PIECES; }
  static __device__ __forceinline__ int pair(int q) { return q / PIECES % P; }
  static __device__ __forceinline__ int row(int q) { return q / (PIECES * P); }
  template <class Base>
  __device__ __forceinline__ void begin(const ScanArray& a, int t0, int tid, Base base) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int q = index(s, tid), in = a.dim - piece(q) * E;  // elements of the piece that there are
      int first = piece(q) * E;
      if (in <= 0) {
        past |= 1u << s;
        first = 0;
      } else if (in < E) {
        last |= 1u << s;
        first = max(a.dim - E, 0);
      }
      from[s] = base(a, pair(q)) + (int64_t)(t0 + row(q)) * a.step + first * (int)sizeof(T);
    }
  }
  __device__ __forceinline__ void request(const ScanArray& a, int n, int64_t next, int tid) {  // n: steps in the tile; next: bytes to the tile after
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const char* p = from[s];
      if (n < TILE) {
        const int at = row(index(s, fresh(tid)));
        p -= at < n ? 0 : (at - n + 1) * a.step;
      }
      if (!kShort || a.dim >= E) {
        v[s] = load16(p);
      } else {  // a row shorter than sixteen bytes, element by element
        uint64_t lo = 0, hi = 0;
#pragma unroll 1
        for (int k = 0; k < a.dim; ++k) {
          const T e = reinterpret_cast<const T*>(p)[k];
          uint64_t bits = 0;
          __builtin_memcpy(&bits, &e, sizeof(T));
          const int at = 8 * (int)sizeof(T) * k;
          if (at < 64) lo |= bits << at;
          else hi |= bits << (at - 64);
        }
        v[s] = make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
      }
      from[s] += next;
    }
  }
  __device__ __forceinline__ void to_lds(char* tile, const ScanArray& a, int n, int tid) {
    const bool padded = PIECES * E > a.dim;
    const int over = a.dim > E && a.dim % E != 0 ? (E - a.dim % E) * (int)sizeof(T) : 0;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int q = index(s, tid), at = row(q);
      if (!WHOLE && over != 0) {
        const uint4 rest = shift_right(v[s], over);
        if (last >> s & 1u) v[s] = rest;
      }
      if (padded && (past >> s & 1u)) v[s] = make_uint4(0, 0, 0, 0);
      if (n < TILE && row(index(s, fresh(tid))) >= n) v[s] = make_uint4(0, 0, 0, 0);
      if (kAll % THREADS == 0 || s * THREADS + tid < kAll)
        *reinterpret_cast<uint4*>(tile + ((pair(q) * TILE + at) * PIECES + (piece(q) ^ swizzle<PIECES>(at))) * 16) = v[s];
    }
  }
};

// The state's element (feat(a, g, e), first + 16 c + i) for every a, c, e of a lane: f(element's place in the lane's registers, its address or nullptr).
// Addresses are a uniform part and an offset of the lane.
template <class T, int NK, int NV, class F>
__device__ __forceinline__ void each_state_element(float* s, int row, int col, int Dx, int Dz, int first, int i, int g, F f) {
  const bool whole = Dx == 16 * NK && first + 16 * NV <= Dz;
#pragma unroll
  for (int a = 0; a < NK; ++a) {
    const int f0 = in_pair<T, NK>(a) ? 8 * g : 4 * g;
    const uint32_t lane = (uint32_t)(f0 * row + (first + i) * col);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        float* p = s + (feat<T, NK>(a, 0, e) * row + 16 * c * col);
        if (whole) f(a, c, e, p + lane);
        else f(a, c, e, f0 + feat<T, NK>(a, 0, e) < Dx && first + 16 * c + i < Dz ? p + lane : nullptr);
      }
  }
}

// Wavefronts a SIMD that the registers are dealt out for: three up to 48 features (48 with one slice: two), two above, because a spilled register costs more than a
// wavefront: its reload waits for every load and store on its way (64 features, rollout of the header: three with 7 registers spilled 732 us, two with none 698;
// 128 features, 32 768 steps: three with 100 spilled 355, two 126).
// Of the 280 instances 23 spill all the same, by the compiler's account: 48 features with two slices in bf16 7 to 9 registers; 96 features with one slice 3 to 4 in fp32,
// 19 to 25 in bf16; 128 features with fewer than four slices 1 to 27 in fp32 (with four 1 to 2), 4 to 22 in bf16, where the output with one slice and rows that are no whole
// pieces keeps 1 KB of its staged pieces in scratch and runs one wavefront a SIMD.  (The pairs of a workgroup go by its slices alone: four pairs of 128 features
// are eight pieces a thread of x and of y each.)
// Slices of 32 columns: of 48 they spilled as much, and halved the wavefronts (gradient with heads of 40 and 72: 466 -> 890 us).
template <int SL>
constexpr int scan_pairs() { return SL == 1 ? 4 : SL == 2 ? 2 : 1; }  // (sequence, head) pairs of a workgroup

template <class T, int NK, int NV, int SL, bool STATE_ONLY, bool WHOLE>
__global__ void __launch_bounds__(64 * SL * scan_pairs<SL>(), NK >= 4 || (NK == 3 && SL == 1) ? 2 : 3) scan_kernel(const ScanArgs args) {
  typedef ScanTraits<T> Tr;
  typedef typename Tr::Frag Frag;
  constexpr int U = Tr::kSub, kTile = 16 * U, P = scan_pairs<SL>(), kThreads = 64 * SL * P, E = 16 / sizeof(T);
  constexpr int kPiecesX = NK * (int)sizeof(T), kPiecesZ = SL * NV * (int)sizeof(T);
  typedef Stage<T, kPiecesX, P, kTile, kThreads, WHOLE> StageX;
  typedef Stage<T, kPiecesZ, P, kTile, kThreads, WHOLE> StageZ;
  constexpr int kBytesX = StageX::kAll * 16, kBytesZ = StageZ::kAll * 16;
  __shared__ __align__(16) char lds_x[STATE_ONLY ? 16 : kBytesX];
  __shared__ __align__(16) char lds_y[kBytesX];
  __shared__ __align__(16) char lds_z[kBytesZ];
  __shared__ __align__(16) char lds_o[STATE_ONLY ? 16 : kBytesZ];
  __shared__ uint32_t lds_left[SL * P];  // wavefronts that have left the common way
  __shared__ float powers[SL * P][kTile + 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  // neighbours in a contiguous run on one XCD: first the roles, which read the same arrays, then the stretches, then the pairs
  uint32_t at = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t role_index = at % args.n_roles;
  at /= args.n_roles;
  const int stretch = (int)(at % args.n_stretches);
  const uint32_t pair0 = at / args.n_stretches * P;
  const ScanRole& r = args.role[role_index];
  const int local = wave / SL, slice0 = wave % SL * 16 * NV;
  const bool active = pair0 + local < args.pairs;
  const int64_t pair = min(pair0 + local, args.pairs - 1);  // (sequence, query head)
  const int64_t b = (uint32_t)pair / args.H;
  const int h = (int)((uint32_t)pair % args.H);
  const int t_begin = stretch * args.stretch, t_end = min(args.T, t_begin + args.stretch);
  const bool reverse = r.reverse != 0;
  auto base = [&](const ScanArray& a, int which) {
    const uint32_t p = min(pair0 + which, args.pairs - 1);
    return a.data + (int64_t)(p / args.H) * a.seq + (int64_t)(p % args.H / a.share) * a.head;
  };
  const float decay = args.decay[h];
  const uint8_t* done = args.done == nullptr ? nullptr : args.done + (uint32_t)b / args.seqs_per_flag;
  const int64_t n_flags = (uint32_t)args.B / args.seqs_per_flag;
  const int Dx = r.y.dim, Dz = r.z.dim;

  floatx4 S[NK][NV];  // rows feat(a, g, e), columns slice0 + 16 c + i
  if (!STATE_ONLY && r.from.data != nullptr) {
    float* s = r.from.data + (pair * r.from.stretches + (r.from.stretches > 1 ? stretch : 0)) * Dx * Dz;
    each_state_element<T, NK, NV>(s, r.from.row, r.from.col, Dx, Dz, slice0, i, g,
                                  [&](int a, int c, int e, const float* p) { S[a][c][e] = p != nullptr ? *p : 0.f; });
  } else {
#pragma unroll
    for (int a = 0; a < NK; ++a)
#pragma unroll
      for (int c = 0; c < NV; ++c) S[a][c] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // Blocks of a tile are numbered in the order of the scan: block u of a reverse scan is the tile's block U - 1 - u in time.
  // Powers of the decay between a row of x (lane i) and rows of y (4 g + e): in one block, and from the block before; from the state that
  // came in to a row; from a row of y of the last block to the state that goes on.  Times the scan's factors.
  if (lane <= kTile) powers[wave][lane] = (float)ipow(decay, lane);
  const float* power = powers[wave];
  wave_lds_order();
  floatx4 near, far, from_j;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int j = 4 * g + e, d = reverse ? j - i : i - j;
    near[e] = d < 0 ? 0.f : r.inner * power[abs(d)];
    far[e] = U > 1 ? r.inner * power[16 + d] : 0.f;
    from_j[e] = r.update * power[reverse ? j + 1 : 15 - j];
  }
  const float to_i = r.inter * power[reverse ? 15 - i : i + 1], block = power[16], whole = power[kTile];
  const float lost = (float)(1.0 - ipow(decay, kTile));   // whole > 0.5: S -= lost S, so that no tile adds whole's own rounding to a long memory
  auto block_at = [&](int u) { return 16 * (reverse ? U - 1 - u : u); };

  const int n_tiles = (t_end - t_begin + kTile - 1) / kTile;
  int t0 = reverse ? t_begin + kTile * (n_tiles - 1) : t_begin;
  StageX sx, sy;
  StageZ sz;
  const int tile_way = reverse ? -kTile : kTile;
  if constexpr (!STATE_ONLY) sx.begin(r.x, t0, tid, base);
  sy.begin(r.y, t0, tid, base);
  sz.begin(r.z, t0, tid, base);
  char* to_out[StageZ::kSlots];  // of a thread's pieces of the output's tile
  uint32_t out_on = 0;
  if constexpr (!STATE_ONLY) {
#pragma unroll
    for (int s = 0; s < StageZ::kSlots; ++s) {
      const int q = StageZ::index(s, tid);
      to_out[s] = const_cast<char*>(base(r.out, StageZ::pair(q))) + (int64_t)(t0 + StageZ::row(q)) * r.out.step + StageZ::piece(q) * 16;
      if ((StageZ::kAll % kThreads == 0 || s * kThreads + tid < StageZ::kAll) && StageZ::piece(q) * E < Dz) out_on |= 1u << s;
    }
  }
  const int64_t out_way = tile_way * r.out.step;
  uint8_t flag = 0;
  auto request = [&](int t) {
    const int n = min(kTile, t_end - t);
    if constexpr (!STATE_ONLY) sx.request(r.x, n, tile_way * r.x.step, tid);
    sy.request(r.y, n, tile_way * r.y.step, tid);
    sz.request(r.z, n, tile_way * r.z.step, tid);
    if (done != nullptr) flag = done[(int64_t)(t + min(lane, n - 1)) * n_flags];
  };
  request(t0);
  if (lane == 0) lds_left[wave] = active ? 0 : 1;
  const char* x_tile = lds_x + local * kTile * kPiecesX * 16;
  const char* y_tile = lds_y + local * kTile * kPiecesX * 16;
  const char* z_tile = lds_z + local * kTile * kPiecesZ * 16;
  auto y_column = [&](int u, int a) {
    const bool runs = in_pair<T, NK>(a);
    return column<T, kPiecesX>(reinterpret_cast<const T*>(y_tile), block_at(u), runs ? 32 * (a / 2) + 4 * (a & 1) : 16 * a, runs ? 8 : 4, i, g);
  };
  auto z_column = [&](int u, int c) {
    return column<T, kPiecesZ>(reinterpret_cast<const T*>(z_tile), block_at(u), slice0 + 16 * c, 4, i, g);
  };
  constexpr int kParts = sizeof(T) == 4 ? 1 : 2;
  bool any_end = false;
  int left_at = -1;  // the tile's first step from which on this wavefront does its work the slow way

  for (int k = 0; k < n_tiles; ++k, t0 += tile_way) {
    const int n = min(kTile, t_end - t0);
    const uint32_t ends = (uint32_t)__builtin_amdgcn_ballot_w64(flag != 0 && lane < n);  // episodes that end in the tile, by step
    if constexpr (!STATE_ONLY) sx.to_lds(lds_x, r.x, n, tid);
    sy.to_lds(lds_y, r.y, n, tid);
    sz.to_lds(lds_z, r.z, n, tid);
    lds_barrier();
    if (k + 1 < n_tiles) request(t0 + tile_way);

    if (left_at < 0) {
      Frag zt[U][NV];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int c = 0; c < NV; ++c) zt[u][c] = z_column(u, c);
      if constexpr (!STATE_ONLY) {
        // scores: block u of x with the blocks v <= u of y; lane i of x, rows 4 g + e of y
        floatx4 score[U][U];
        Rows<T, NK> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) rows_of<T, NK>(x[u], x_tile, block_at(u) + i, g);
#pragma unroll
        for (int v = 0; v < U; ++v) {
          Rows<T, NK> y;
          rows_of<T, NK>(y, y_tile, block_at(v) + i, g);
#pragma unroll
          for (int u = v; u < U; ++u) {
            floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int a = 0; a + 1 < NK; a += 2) acc = mma2(y.f[a], y.f[a + 1], x[u].f[a], x[u].f[a + 1], acc);
            if constexpr (NK % 2 == 1) acc = mma(y.f[NK - 1], x[u].f[NK - 1], acc);
            score[u][v] = acc;
          }
        }
        floatx4 o[U][NV];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int c = 0; c < NV; ++c) o[u][c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NV; ++c) {
#pragma unroll
          for (int a = 0; a < NK; a += 2) {
            const Parts<T, 2> s0 = parts_of<T, 2>(S[a][c]), s1 = parts_of<T, 2>(S[min(a + 1, NK - 1)][c]);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
              for (int p = kParts - 1; p >= 0; --p) {
                if (a + 1 < NK) o[u][c] = mma2(s0.p[p], s1.p[p], x[u].f[a], x[u].f[min(a + 1, NK - 1)], o[u][c]);
                else o[u][c] = mma(s0.p[p], x[u].f[a], o[u][c]);
              }
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float to = to_i;
          if (u > 0) to *= block;
          if (reverse && n < kTile) {  // the tile's last step is n - 1
            const int ti = block_at(u) + fresh(i);
            to = ti < n ? r.inter * power[n - 1 - ti] : 0.f;
          }
          if (ends == 0) {
#pragma unroll
            for (int c = 0; c < NV; ++c) o[u][c] *= to;
#pragma unroll
            for (int v = 0; v <= u; ++v) score[u][v] *= u == v ? near : far;
          } else {
            // step ti sees the steps from the last end before it on; in a reverse scan up to the first end from it on
            const int ti = block_at(u) + fresh(i);
            const uint32_t between = reverse ? ends >> ti : ends & ((1u << ti) - 1u);
            const int edge = (reverse ? ti + __builtin_ctz(between | 0x80000000u) : 32 - __clz(between)) - 4 * g;
            const bool clear = between == 0;
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[u][c][e] = clear ? o[u][c][e] * to : 0.f;
#pragma unroll
            for (int v = 0; v <= u; ++v)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const bool seen = reverse ? clear || block_at(v) + e <= edge : block_at(v) + e >= edge;
                score[u][v][e] = seen ? score[u][v][e] * (u == v ? near[e] : far[e]) : 0.f;
              }
          }
        }
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          Parts<T, 2> w[U];
#pragma unroll
          for (int v = 0; v <= u; ++v) w[v] = parts_of<T, 2>(score[u][v]);
#pragma unroll
          for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int p = kParts - 1; p >= 0; --p) {
              if constexpr (U == 1) o[u][c] = mma(zt[0][c], w[0].p[p], o[u][c]);
              else o[u][c] = mma2(zt[0][c], zt[1][c], w[0].p[p], u == 0 ? Frag{} : w[1].p[p], o[u][c]);
            }
#pragma unroll
          for (int c = 0; c < NV; ++c) sum += (o[u][c][0] + o[u][c][1]) + (o[u][c][2] + o[u][c][3]);
        }
        // an infinity or a NaN in a row of y or z shows in that step's own output: the rest of the sequence is done the slow way then
        if (__builtin_amdgcn_ballot_w64(!(fabsf(sum) < __builtin_inff())) != 0) {
          left_at = t0;
          if (lane == 0) lds_left[wave] = 1;
        } else if (sizeof(T) == 4 || !r.out_f32) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int row = block_at(u) + i, swz = swizzle<kPiecesZ>(row);
            char* p = lds_o + (local * kTile + row) * kPiecesZ * 16;
#pragma unroll
            for (int c = 0; c < NV; ++c) {
              const int f = slice0 + 16 * c + 4 * g;
              if constexpr (sizeof(T) == 4) *reinterpret_cast<floatx4*>(p + ((f / 4) ^ swz) * 16) = o[u][c];
              else *reinterpret_cast<shortx4*>(p + ((f / 8) ^ swz) * 16 + (f & 4) * 2) = pack4(o[u][c]);
            }
          }
        } else if (active) {  // shares in fp32
          char* ob = const_cast<char*>(base(r.out, local));
          const int i0 = fresh(i), f0 = slice0 + 4 * fresh(g);
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (block_at(u) + i0 < n) {
              char* row = ob + (int64_t)(t0 + block_at(u) + i0) * r.out.step;
#pragma unroll
              for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int f = f0 + 16 * c + e;
                  if (f >= Dz) continue;
                  reinterpret_cast<float*>(row)[f] = o[u][c][e];
                }
            }
        }
      }
      if (left_at < 0) {
        floatx4 w[U];  // what a row of y adds to the state that goes on
#pragma unroll
        for (int u = 0; u < U; ++u) {
          w[u] = from_j;
          if (u + 1 < U) w[u] *= block;
        }
        if (n < kTile || ends != 0) {
          const int g4 = 4 * fresh(g);
          // steps that reach the state that goes on: those behind the last end; in a reverse scan those up to the first
          const int from = reverse || ends == 0 ? 0 : 32 - __builtin_clz(ends), to = reverse && ends != 0 ? __builtin_ctz(ends) : kTile;
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int tj = block_at(u) + g4 + e;
              if (!reverse && n < kTile) w[u][e] = tj < n ? r.update * power[n - 1 - tj] : 0.f;
              if (tj < from || tj > to) w[u][e] = 0.f;
            }
        }
        if (ends != 0) {
          any_end = true;
#pragma unroll
          for (int a = 0; a < NK; ++a)
#pragma unroll
            for (int c = 0; c < NV; ++c) S[a][c] = floatx4{0.f, 0.f, 0.f, 0.f};
        } else if (whole > 0.5f && n == kTile) {
#pragma unroll
          for (int a = 0; a < NK; ++a)
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) S[a][c][e] = fmaf(-lost, S[a][c][e], S[a][c][e]);
        } else {
          const float f = n == kTile ? whole : power[n];
#pragma unroll
          for (int a = 0; a < NK; ++a)
#pragma unroll
            for (int c = 0; c < NV; ++c) S[a][c] *= f;
        }
        // the weights go to the side with fewer fragments
        constexpr int Q = sizeof(T) == 4 ? 1 : 3;
        Parts<T, 3> zw[U][NV];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int c = 0; c < NV; ++c) zw[u][c] = parts_of<T, 3>(widen4(zt[u][c]) * w[u]);
#pragma unroll
        for (int a = 0; a < NK; ++a) {
          Frag yt[U];
#pragma unroll
          for (int u = 0; u < U; ++u) yt[u] = y_column(u, a);
#pragma unroll
          for (int p = Q - 1; p >= 0; --p)
#pragma unroll
            for (int c = 0; c < NV; ++c) {
              if constexpr (U == 2) S[a][c] = mma2(yt[0], yt[1], zw[0][c].p[p], zw[1][c].p[p], S[a][c]);
              else S[a][c] = mma(yt[0], zw[0][c].p[p], S[a][c]);
            }
        }
      }
    }
    lds_barrier();
    if constexpr (!STATE_ONLY) {
      if (sizeof(T) == 4 || !r.out_f32) {
#pragma unroll
        for (int s = 0; s < StageZ::kSlots; ++s) {
          const int q = StageZ::index(s, tid), row = StageZ::row(q), piece = StageZ::piece(q), which = StageZ::pair(q);
          if ((out_on >> s & 1u) && row < n && lds_left[which * SL + piece * E / (16 * NV)] == 0) {
            const uint4 v = *reinterpret_cast<const uint4*>(lds_o + ((which * kTile + row) * kPiecesZ + (piece ^ swizzle<kPiecesZ>(row))) * 16);
            if (WHOLE || piece * E + E <= Dz) {
              store16(to_out[s], v);
            } else {
              T e[E];
              __builtin_memcpy(e, &v, 16);
#pragma unroll
              for (int k = 0; k < E - 1; ++k)
                if (piece * E + k < Dz) reinterpret_cast<T*>(to_out[s])[k] = e[k];
            }
          }
          to_out[s] += out_way;
        }
      }
    }
  }

  if (!active) return;
  auto own = [&](const ScanArray& a) { return const_cast<char*>(base(a, local)); };
  if constexpr (STATE_ONLY) {  // nothing shows on the way: look at the end, and start again the slow way
    float sum = 0.f;
#pragma unroll
    for (int a = 0; a < NK; ++a)
#pragma unroll
      for (int c = 0; c < NV; ++c) sum += (S[a][c][0] + S[a][c][1]) + (S[a][c][2] + S[a][c][3]);
    if (__builtin_amdgcn_ballot_w64(!(fabsf(sum) < __builtin_inff())) != 0) {
#pragma unroll
      for (int a = 0; a < NK; ++a)
#pragma unroll
        for (int c = 0; c < NV; ++c) S[a][c] = floatx4{0.f, 0.f, 0.f, 0.f};
      scan_slow<T, NK, NV, STATE_ONLY>(S, r, nullptr, own(r.y), own(r.z), nullptr, t_begin, t_end - t_begin, slice0, decay, done, n_flags, i, g);
    }
  } else if (left_at >= 0) {
    const int from = reverse ? t_begin : left_at, to = reverse ? min(left_at + kTile, t_end) : t_end;
    scan_slow<T, NK, NV, STATE_ONLY>(S, r, own(r.x), own(r.y), own(r.z), own(r.out), from, to - from, slice0, decay, done, n_flags, i, g);
  }

  if (r.to.data != nullptr) {
    float* s = r.to.data + (pair * r.to.stretches + (r.to.stretches > 1 ? stretch : 0)) * Dx * Dz;
    each_state_element<T, NK, NV>(s, r.to.row, r.to.col, Dx, Dz, slice0, i, g, [&](int a, int c, int e, float* p) {
      if (p != nullptr) *p = S[a][c][e];
    });
  }
  if (STATE_ONLY && role_index == 0 && slice0 == 0 && lane == 0) {
    const float factor = (float)ipow(decay, t_end - t_begin);
    args.carry[pair * args.n_stretches + stretch] = any_end ? kCarryEnded : factor == 0.f && decay != 0.f ? kCarryLeast : factor;
  }
}

// ---- launch: the instance by (padded) widths -------------------------------------------------------------------------------------------
inline int scan_nk(int dim) { return dim <= 96 ? (dim + 15) / 16 : 8; }
inline int scan_nv(int dim) { return dim <= 16 ? 1 : 2; }
inline int scan_slices(int dim) { return dim <= 32 ? 1 : (dim + 31) / 32; }

// A scan of no steps has no valid row to point at: the caller never launches one.
void launch_scan_f32(const ScanArgs& a, int dx, int dz, bool state_only, hipStream_t s);
void launch_scan_bf16(const ScanArgs& a, int dx, int dz, bool state_only, hipStream_t s);

template <class T>
inline void launch_scan(const ScanArgs& a, int dx, int dz, bool state_only, hipStream_t s) {
  const int nk = scan_nk(dx), nv = scan_nv(dz), slices = scan_slices(dz);
  const bool whole = dx * sizeof(T) % 16 == 0 && dz * sizeof(T) % 16 == 0;
#define MARL_SCAN(K, V, SL)                                                                                               \
  if (nk == K && nv == V && slices == SL) {                                                                               \
    constexpr uint32_t P = scan_pairs<SL>();                                                                              \
    const dim3 grid((a.pairs + P - 1) / P * a.n_stretches * a.n_roles), block(64 * SL * P);                               \
    if (state_only && whole) hipLaunchKernelGGL((scan_kernel<T, K, V, SL, true, true>), grid, block, 0, s, a);           \
    else if (state_only) hipLaunchKernelGGL((scan_kernel<T, K, V, SL, true, false>), grid, block, 0, s, a);              \
    else if (whole) hipLaunchKernelGGL((scan_kernel<T, K, V, SL, false, true>), grid, block, 0, s, a);                   \
    else hipLaunchKernelGGL((scan_kernel<T, K, V, SL, false, false>), grid, block, 0, s, a);                             \
    return;                                                                                                               \
  }
#define MARL_SCAN_ALL(K) MARL_SCAN(K, 1, 1) MARL_SCAN(K, 2, 1) MARL_SCAN(K, 2, 2) MARL_SCAN(K, 2, 3) MARL_SCAN(K, 2, 4)
  MARL_SCAN_ALL(1) MARL_SCAN_ALL(2) MARL_SCAN_ALL(3) MARL_SCAN_ALL(4) MARL_SCAN_ALL(5) MARL_SCAN_ALL(6) MARL_SCAN_ALL(8)
#undef MARL_SCAN_ALL
#undef MARL_SCAN
}

}  // namespace marl
