// Linear attention with a decay for each head, its gradient, and the states between stretches of time: one scan.
//
// With x, y, z arrays of rows over time and g the head's decay, a scan forms
//     out_i = inner sum_j g^|i-j| (x_i . y_j) z_j + inter g^(..) S^T x_i        S <- g^n S + update sum_j g^(..) y_j z_j^T
// over the steps j up to i (a reverse scan: from i on) in i's episode, S being the state that came in.  Everything is that:
//     out: (x, y, z) = (q, k, v);   dq: (dout, v, k), the state transposed;   dv: (k, q, dout) and dk: (v, dout, q) in reverse,
// because dq_i = scale S_i dout_i with the same S, and R_j = scale q_j dout_j^T + g R_{j+1} gives dv_j = R_j^T k_j, dk_j = R_j v_j.
//
// One wavefront takes one head of one sequence (or a slice of its z columns) through time, sixteen steps at once, on the matrix cores, with S
// in accumulator registers: per 16 steps four small products, scores y x^T, x S, scores z and y^T z.  Transposed throughout (out^T = z^T
// scores^T), the accumulator layout of a product -- lane = column, four rows in registers -- is the operand layout of the next, so that neither
// scores nor S go through LDS; y and z do, because the last two products contract over time.
#pragma once
#include "split_bf16.h"

namespace marl {

constexpr int kTile = 16;          // steps that a wavefront takes at once
constexpr int kMaxWaves = 4;       // of a workgroup; they share nothing
constexpr int kMaxRoles = 3;

struct ScanArray {
  const char* data;
  int64_t step, seq, head;  // bytes
  uint32_t share;           // query heads per head of this array
  int32_t dim;
  int32_t wide;             // 16-byte accesses
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
  float* carry;          // states only: [sequence, head][stretch] factor from a stretch's first state to its last
  int32_t T, B;
  uint32_t n_roles, H, seqs_per_flag;
  uint32_t slices;       // of the z columns, one wavefront each
  uint32_t n_stretches;
  int32_t stretch;       // steps of a stretch, a multiple of kTile
  uint32_t units;        // B * H * slices
};

template <class T>
struct ScanTraits;
template <>
struct ScanTraits<float> {
  typedef floatx4 Frag;                     // four elements along a contraction
  static constexpr int kPad = 4;            // of an LDS row, elements
};
template <>
struct ScanTraits<bf16_t> {
  typedef shortx4 Frag;
  static constexpr int kPad = 8;
};
// Feature of element e of lane group g in tile a of N tiles of sixteen features.  bf16: two tiles deal a lane eight consecutive ones, 16 bytes.
template <class T, int N>
__device__ __forceinline__ int feat(int a, int g, int e) {
  return sizeof(T) == 2 && N % 2 == 0 ? 32 * (a / 2) + 8 * g + 4 * (a & 1) + e : 16 * a + 4 * g + e;
}

__device__ __forceinline__ float ipow(float g, int m) {  // g^m, 0^0 = 1
  float r = 1.f;
  while (m != 0) {
    if (m & 1) r *= g;
    g *= g;
    m >>= 1;
  }
  return r;
}

// ---- products of 16 x 16 outputs; the contraction index of element e of lane group g is the same on both sides -----------------------
__device__ __forceinline__ floatx4 mma(floatx4 a, floatx4 b, floatx4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ floatx4 mma(shortx4 a, shortx4 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0); }

__device__ __forceinline__ shortx4 pack4(floatx4 v) {
  const uint2 u = make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]));
  return __builtin_bit_cast(shortx4, u);
}
__device__ __forceinline__ floatx4 unpack4(shortx4 s) {
  const uint2 u = __builtin_bit_cast(uint2, s);
  return floatx4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u)};
}
// fp32 values times exact operands.  bf16: the values in two parts (relative error 2^-16: what the scores and the state are rounded to where
// the result is an output of eight bits) or in three (2^-24: where it is a state that goes on).
__device__ __forceinline__ floatx4 mma_two(floatx4 v, floatx4 b, floatx4 c) { return mma(v, b, c); }
__device__ __forceinline__ floatx4 mma_two(floatx4 v, shortx4 b, floatx4 c) {
  const shortx4 h = pack4(v);
  c = mma(pack4(v - unpack4(h)), b, c);
  return mma(h, b, c);
}
struct Weighed {
  shortx4 h, m, l;
};
__device__ __forceinline__ floatx4 weigh_parts(floatx4 y, floatx4 w) { return y * w; }
__device__ __forceinline__ Weighed weigh_parts(shortx4 y, floatx4 w) {
  floatx4 v = unpack4(y) * w;
  Weighed p;
  p.h = pack4(v);
  v -= unpack4(p.h);
  p.m = pack4(v);
  v -= unpack4(p.m);
  p.l = pack4(v);
  return p;
}
__device__ __forceinline__ floatx4 mma(const Weighed& a, shortx4 b, floatx4 c) {
  c = mma(a.l, b, c);
  c = mma(a.m, b, c);
  return mma(a.h, b, c);
}

// ---- rows of sixteen steps: lane (i = lane % 16, g = lane / 16) holds features feat(a, g, 0..3) of step i --------------------------------
template <class T, int N>
struct Rows {
  typename ScanTraits<T>::Frag f[N];
};
__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ short load_one(const bf16_t* p) { return (short)*p; }

// row: of the lane's step (clamped to a valid one), n: valid steps; column 0 of the slice at `first`
template <class T, int N>
__device__ __forceinline__ void load_rows(Rows<T, N>& r, const ScanArray& a, const char* row, int first, bool valid, int g) {
  constexpr int kRun = (sizeof(T) == 2 && N % 2 == 0) ? 2 : 1;  // tiles a 16-byte access covers
  if (a.wide) {
#pragma unroll
    for (int t = 0; t < N; t += kRun) {
      const int col = first + feat<T, N>(t, g, 0);
      const bool in = valid && col < a.dim;
      const char* p = row + (in ? col * (int)sizeof(T) : 0);
      if constexpr (sizeof(T) == 4) {
        const floatx4 v = *reinterpret_cast<const floatx4*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) r.f[t][e] = in ? v[e] : 0.f;
      } else if constexpr (kRun == 2) {
        uint4 v = *reinterpret_cast<const uint4*>(p);
        v.x = in ? v.x : 0u; v.y = in ? v.y : 0u; v.z = in ? v.z : 0u; v.w = in ? v.w : 0u;
        r.f[t] = __builtin_bit_cast(shortx4, make_uint2(v.x, v.y));
        r.f[t + 1] = __builtin_bit_cast(shortx4, make_uint2(v.z, v.w));
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        r.f[t] = __builtin_bit_cast(shortx4, make_uint2(in ? v.x : 0u, in ? v.y : 0u));
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int col = first + feat<T, N>(t, g, e);
        const bool in = valid && col < a.dim;
        const auto v = load_one(reinterpret_cast<const T*>(row) + (in ? col : 0));
        r.f[t][e] = in ? v : 0;
      }
  }
}
// Is there an infinity or a NaN among them?  (exponents of ones; bit 31 or 15 of the result)
__device__ __forceinline__ uint32_t not_finite(floatx4 v) {
  uint32_t r = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) r |= (__float_as_uint(v[e]) & 0x7f800000u) + 0x00800000u;
  return r;
}
__device__ __forceinline__ uint32_t not_finite(shortx4 v) {
  const uint2 u = __builtin_bit_cast(uint2, v);
  return ((u.x & 0x7f807f80u) + 0x00800080u) | ((u.y & 0x7f807f80u) + 0x00800080u);
}

template <class T, int N>
__device__ __forceinline__ void rows_to_lds(T* lds, const Rows<T, N>& r, int i, int g) {
  constexpr int kPitch = 16 * N + ScanTraits<T>::kPad;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int t = 0; t < N; ++t) *reinterpret_cast<floatx4*>(lds + i * kPitch + feat<T, N>(t, g, 0)) = r.f[t];
  } else if constexpr (N % 2 == 0) {
#pragma unroll
    for (int t = 0; t < N; t += 2) {
      const shortx8 v = __builtin_shufflevector(r.f[t], r.f[t + 1], 0, 1, 2, 3, 4, 5, 6, 7);
      *reinterpret_cast<shortx8*>(lds + i * kPitch + feat<T, N>(t, g, 0)) = v;
    }
  } else {
#pragma unroll
    for (int t = 0; t < N; ++t) *reinterpret_cast<shortx4*>(lds + i * kPitch + feat<T, N>(t, g, 0)) = r.f[t];
  }
}
// Columns: lane m = lane % 16 of tile t gets feature feat(t, m / 4, m % 4) at steps 4 g .. 4 g + 3
template <int N>
__device__ __forceinline__ floatx4 column(const float* lds, int t, int i, int g) {
  constexpr int kPitch = 16 * N + ScanTraits<float>::kPad;
  floatx4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = lds[(4 * g + e) * kPitch + 16 * t + i];
  return v;
}
template <int N>
__device__ __forceinline__ shortx4 column(const bf16_t* lds, int t, int i, int g) {
  constexpr int kPitch = 16 * N + ScanTraits<bf16_t>::kPad;
  typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
  const int at = feat<bf16_t, N>(t, i & 3, 0);
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(lds + (4 * g + (i >> 2)) * kPitch + at));
}

// Between LDS writes and reads of one wavefront's own part: its LDS accesses take effect in order, the compiler has to keep it.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Powers of the decay that a tile of n steps needs, as lane (i, g) uses them: row i on the x side, rows 4 g + e on the y side
struct TilePowers {
  float to_i;        // from the tile's first state to step i: g^(i+1); reverse: from its last, g^(n-1-i)
  float whole;       // g^n
  floatx4 from_j;    // from step j to the tile's other end: g^(n-1-j), reverse g^(j+1)
};
__device__ __forceinline__ TilePowers tile_powers(float decay, int n, bool reverse, int i, int g) {
  TilePowers p;
  p.to_i = reverse ? (i < n ? ipow(decay, n - 1 - i) : 0.f) : ipow(decay, i + 1);
  p.whole = ipow(decay, n);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int j = 4 * g + e;
    p.from_j[e] = j >= n ? 0.f : reverse ? ipow(decay, j + 1) : ipow(decay, n - 1 - j);
  }
  return p;
}

// One tile the slow way, step by step from memory, where it holds infinities or NaNs: a matrix product multiplies masked places by zero, which
// makes a NaN of them, and would carry them into other steps' and other episodes' outputs.  (noinline would put S into memory.)
template <class T, int NK, int NV, bool STATE_ONLY>
__device__ void scan_tile_slow(floatx4 (&S)[NK][NV], const ScanRole& r, const char* xb, const char* yb, const char* zb, char* ob, int t0, int n,
                               int slice0, float decay, uint32_t ends, int i, int g) {
  for (int s = 0; s < n; ++s) {
    const int at = r.reverse ? n - 1 - s : s, t = t0 + at;
    const bool end = (ends >> at) & 1u;
    const T* y = reinterpret_cast<const T*>(yb + (int64_t)t * r.y.step);
    const T* z = reinterpret_cast<const T*>(zb + (int64_t)t * r.z.step);
    const T* x = STATE_ONLY ? nullptr : reinterpret_cast<const T*>(xb + (int64_t)t * r.x.step);
    float zv[NV], o[NV];
#pragma unroll
    for (int b = 0; b < NV; ++b) {
      const int c = slice0 + feat<T, NV>(b, i >> 2, i & 3);
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
        const int c = slice0 + feat<T, NV>(b, i >> 2, i & 3);
        if (g == 0 && c < r.z.dim) {
          char* p = ob + (int64_t)t * r.out.step;
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

template <class T, int NK, int NV, bool STATE_ONLY>
__global__ void __launch_bounds__(64 * kMaxWaves, 2) scan_kernel(const ScanArgs args) {
  typedef ScanTraits<T> Tr;
  typedef typename Tr::Frag Frag;
  constexpr int kPitchY = 16 * NK + Tr::kPad, kPitchZ = 16 * NV + Tr::kPad;
  constexpr int kWaveLds = kTile * (kPitchY + kPitchZ);
  __shared__ __align__(16) T lds_all[kMaxWaves * kWaveLds];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  // neighbours in a contiguous run on one XCD: first the roles, which read the same arrays, then the stretches, then the units
  uint32_t at = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t role_index = at % args.n_roles;
  at /= args.n_roles;
  const int stretch = (int)(at % args.n_stretches);
  const uint32_t unit = at / args.n_stretches * (blockDim.x >> 6) + wave;
  if (unit >= args.units) return;
  const ScanRole& r = args.role[role_index];
  const int slice0 = (int)(unit % args.slices) * 16 * NV;
  const int64_t pair = unit / args.slices;  // (sequence, query head)
  const int64_t b = (uint32_t)pair / args.H;
  const int h = (int)((uint32_t)pair % args.H);
  T* lds_y = lds_all + wave * kWaveLds;
  T* lds_z = lds_y + kTile * kPitchY;
  const int t_begin = stretch * args.stretch, t_end = min(args.T, t_begin + args.stretch);
  const bool reverse = r.reverse != 0;
  auto base = [&](const ScanArray& a) { return const_cast<char*>(a.data) + b * a.seq + (int64_t)((uint32_t)h / a.share) * a.head; };
  const char *xb = STATE_ONLY ? nullptr : base(r.x), *yb = base(r.y), *zb = base(r.z);
  char* ob = STATE_ONLY ? nullptr : base(r.out);
  const float decay = args.decay[h];
  const uint8_t* done = args.done == nullptr ? nullptr : args.done + (uint32_t)b / args.seqs_per_flag;
  const int64_t n_flags = (uint32_t)args.B / args.seqs_per_flag;

  // features of the state's elements: rows feat_x(a, g, e), columns feat_z(c, i / 4, i % 4)
  auto feat_x = [&](int a, int e) { return feat<T, NK>(a, g, e); };
  auto feat_z = [&](int c) { return slice0 + feat<T, NV>(c, i >> 2, i & 3); };
  const int Dx = r.y.dim, Dz = r.z.dim;
  floatx4 S[NK][NV];
  {
    const float* s = nullptr;
    if (!STATE_ONLY && r.from.data != nullptr) s = r.from.data + (pair * r.from.stretches + (r.from.stretches > 1 ? stretch : 0)) * Dx * Dz;
#pragma unroll
    for (int a = 0; a < NK; ++a)
#pragma unroll
      for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int f = feat_x(a, e), z = feat_z(c);
          S[a][c][e] = s != nullptr && f < Dx && z < Dz ? s[f * r.from.row + z * r.from.col] : 0.f;
        }
  }

  floatx4 near;  // g^|i-j|
#pragma unroll
  for (int e = 0; e < 4; ++e) near[e] = ipow(decay, abs(i - (4 * g + e)));
  const TilePowers full = tile_powers(decay, kTile, reverse, i, g);
  float carried = 1.f;

  const int n_tiles = (t_end - t_begin + kTile - 1) / kTile;
  Rows<T, NK> x, y, x_next, y_next;
  Rows<T, NV> z, z_next;
  uint8_t flag = 0, flag_next = 0;
  auto tile_start = [&](int k) { return t_begin + kTile * (reverse ? n_tiles - 1 - k : k); };
  auto request = [&](int k) {
    const int t0 = tile_start(k), n = min(kTile, t_end - t0);
    const int64_t t = t0 + min(i, n - 1);
    const bool valid = i < n;
    if constexpr (!STATE_ONLY) load_rows<T, NK>(x_next, r.x, xb + t * r.x.step, 0, valid, g);
    load_rows<T, NK>(y_next, r.y, yb + t * r.y.step, 0, valid, g);
    load_rows<T, NV>(z_next, r.z, zb + t * r.z.step, slice0, valid, g);
    if (done != nullptr) flag_next = valid ? done[t * n_flags] : (uint8_t)0;
  };
  request(0);
  for (int k = 0; k < n_tiles; ++k) {
    x = x_next; y = y_next; z = z_next; flag = flag_next;
    const int t0 = tile_start(k), n = min(kTile, t_end - t0);
    if (k + 1 < n_tiles) request(k + 1);
    const uint32_t ends = (uint32_t)__builtin_amdgcn_ballot_w64(flag != 0) & 0xffffu;  // episodes that end in the tile, by step
    TilePowers p = full;
    if (n < kTile) p = tile_powers(decay, n, reverse, i, g);

    rows_to_lds<T, NK>(lds_y, y, i, g);
    rows_to_lds<T, NV>(lds_z, z, i, g);
    wave_lds_order();
    uint32_t bad = 0;
#pragma unroll
    for (int a = 0; a < NK; ++a) bad |= not_finite(y.f[a]);
#pragma unroll
    for (int c = 0; c < NV; ++c) bad |= not_finite(z.f[c]);
    bad &= sizeof(T) == 4 ? 0x80000000u : 0x80008000u;

    Frag zt[NV];
#pragma unroll
    for (int c = 0; c < NV; ++c) zt[c] = column<NV>(lds_z, c, i, g);

    floatx4 o[NV];
    if constexpr (!STATE_ONLY) {
      const uint32_t to_here = reverse ? ends >> i : ends & ((1u << i) - 1u);  // ends between the state that came in and step i
      const float w_in = to_here == 0 ? p.to_i * r.inter : 0.f;
      floatx4 score = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int a = 0; a < NK; ++a) score = mma(y.f[a], x.f[a], score);
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int a = 0; a < NK; ++a) acc = mma_two(S[a][c], x.f[a], acc);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[c][e] = to_here == 0 ? acc[e] * w_in : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = 4 * g + e, lo = min(i, j), hi = max(i, j);
        const bool seen = (reverse ? j >= i : j <= i) && ((ends & ((1u << hi) - 1u)) >> lo) == 0;
        score[e] = seen ? score[e] * near[e] * r.inner : 0.f;
      }
      // (scores as the second operand: the two parts of a bf16 score are formed once)
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int c = 0; c < NV; ++c) o[c] = mma(zt[c], score, o[c]);
      } else {
        const shortx4 hi = pack4(score), lo = pack4(score - unpack4(hi));
#pragma unroll
        for (int c = 0; c < NV; ++c) o[c] = mma(zt[c], hi, mma(zt[c], lo, o[c]));
      }
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < NV; ++c) sum += (o[c][0] + o[c][1]) + (o[c][2] + o[c][3]);
      if (!(fabsf(sum) < __builtin_inff())) bad = 1;
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(bad != 0) != 0, 0)) {
      scan_tile_slow<T, NK, NV, STATE_ONLY>(S, r, xb, yb, zb, ob, t0, n, slice0, decay, ends, i, g);
      carried = ends == 0 ? carried * p.whole : 0.f;
      continue;
    }
    if constexpr (!STATE_ONLY) {
      if (i < n) {
        char* row = ob + (int64_t)(t0 + i) * r.out.step;
        if (r.out_f32 || sizeof(T) == 4) {
#pragma unroll
          for (int c = 0; c < NV; ++c) {
            const int f0 = slice0 + feat<T, NV>(c, g, 0);
            if (r.out.wide && f0 < Dz)
              *reinterpret_cast<floatx4*>(reinterpret_cast<float*>(row) + f0) = o[c];
            else if (!r.out.wide)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (f0 + e < Dz) reinterpret_cast<float*>(row)[f0 + e] = o[c][e];
          }
        } else if (NV % 2 == 0 && r.out.wide) {
#pragma unroll
          for (int c = 0; c + 1 < NV; c += 2) {
            const int f0 = slice0 + feat<T, NV>(c, g, 0);
            if (f0 < Dz) {
              const shortx8 v = __builtin_shufflevector(pack4(o[c]), pack4(o[c + 1]), 0, 1, 2, 3, 4, 5, 6, 7);
              *reinterpret_cast<shortx8*>(reinterpret_cast<bf16_t*>(row) + f0) = v;
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < NV; ++c) {
            const int f0 = slice0 + feat<T, NV>(c, g, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (f0 + e < Dz) reinterpret_cast<bf16_t*>(row)[f0 + e] = to_bf16(o[c][e]);
          }
        }
      }
    }
    floatx4 w;  // what step j adds to the state that goes on
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = 4 * g + e;
      const uint32_t after = reverse ? ends & ((1u << j) - 1u) : ends >> j;
      w[e] = after == 0 ? p.from_j[e] * r.update : 0.f;
    }
#pragma unroll
    for (int a = 0; a < NK; ++a) {
      const auto yw = weigh_parts(column<NK>(lds_y, a, i, g), w);
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        floatx4 s = S[a][c];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = ends == 0 ? s[e] * p.whole : 0.f;
        S[a][c] = mma(yw, zt[c], s);
      }
    }
    carried = ends == 0 ? carried * p.whole : 0.f;
    wave_lds_order();
  }

  if (r.to.data != nullptr) {
    float* s = r.to.data + (pair * r.to.stretches + (r.to.stretches > 1 ? stretch : 0)) * Dx * Dz;
#pragma unroll
    for (int a = 0; a < NK; ++a)
#pragma unroll
      for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int f = feat_x(a, e), zc = feat_z(c);
          if (f < Dx && zc < Dz) s[f * r.to.row + zc * r.to.col] = S[a][c][e];
        }
  }
  if (STATE_ONLY && role_index == 0 && slice0 == 0 && lane == 0) args.carry[pair * args.n_stretches + stretch] = carried;
}

// ---- launch: the instance by (padded) widths -------------------------------------------------------------------------------------------
// Columns of the state that one wavefront holds: at most 64 accumulator registers a lane
inline int scan_nk(int dim) { return dim <= 16 ? 1 : dim <= 32 ? 2 : dim <= 64 ? 4 : 8; }
inline int scan_nv(int nk, int dim) { return dim <= 16 ? 1 : dim <= 32 || nk == 8 ? 2 : 4; }
inline int scan_slices(int nk, int dim) {
  const int w = 16 * scan_nv(nk, dim);
  return (dim + w - 1) / w;
}

// A stretch of no steps has no valid row to point at: the caller never launches one.
void launch_scan_f32(const ScanArgs& a, int nk, int nv, bool state_only, dim3 grid, dim3 block, hipStream_t s);
void launch_scan_bf16(const ScanArgs& a, int nk, int nv, bool state_only, dim3 grid, dim3 block, hipStream_t s);

template <class T>
inline void launch_scan(const ScanArgs& a, int nk, int nv, bool state_only, dim3 grid, dim3 block, hipStream_t s) {
#define MARL_SCAN(K, V)                                                                                 \
  if (nk == K && nv == V) {                                                                             \
    if (state_only) hipLaunchKernelGGL((scan_kernel<T, K, V, true>), grid, block, 0, s, a);            \
    else hipLaunchKernelGGL((scan_kernel<T, K, V, false>), grid, block, 0, s, a);                      \
    return;                                                                                             \
  }
  MARL_SCAN(1, 1) MARL_SCAN(1, 2) MARL_SCAN(1, 4)
  MARL_SCAN(2, 1) MARL_SCAN(2, 2) MARL_SCAN(2, 4)
  MARL_SCAN(4, 1) MARL_SCAN(4, 2) MARL_SCAN(4, 4)
  MARL_SCAN(8, 1) MARL_SCAN(8, 2)
#undef MARL_SCAN
}

}  // namespace marl
