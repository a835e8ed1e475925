// Rotary positions: the table of cosines and sines, and the rotation of queries and keys in one launch.  Bound by memory: every element in and
// out once; a step's table row is shared by its heads and comes from a cache.  Measured: 128 x 4096 steps, 8 + 8 heads of 64 in bf16, half of each rotated:
// 389 us, 5.5 TB/s (one item a thread, division by division, table rows element by element: 616).  Rows that are no whole vectors go pair by pair: in bf16, as many
// steps with heads of 40, all of each rotated: 758 us in halves (floor 272), 266 interleaved, where a row is whole vectors; of 32 with 8 rotated 948 and 207 (218).
#include "common.h"

namespace marl {
namespace {

// ---- table -----------------------------------------------------------------------------------------------------------------------
// In 64 bits: an angle of p radians has an error of p * 2^-24 in 32.
__global__ void __launch_bounds__(256) rotary_table_kernel(marl_rotary_dims d, float* __restrict__ table) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int half = d.rotary_dim / 2;
  if (at >= (int64_t)d.n_positions * half) return;
  const int64_t position = at / half;
  const int i = (int)(at % half);
  const double R = d.rotary_dim;
  double base = d.base;
  if (d.scaling == 2) base *= pow((double)d.factor, R / (R - 2.0));
  double f = pow(base, -2.0 * i / R);
  if (d.scaling == 1) f /= d.factor;
  if (d.scaling == 3) {
    const double turns = d.trained_length * f / 6.283185307179586476925;
    double m = (turns - d.slow) / ((double)d.fast - d.slow);
    m = m < 0.0 ? 0.0 : m > 1.0 ? 1.0 : m;
    f = m * f + (1.0 - m) * f / d.factor;
  }
  double sine, cosine;
  sincos((double)position * f, &sine, &cosine);
  table[position * d.rotary_dim + i] = (float)(cosine * d.amplitude);
  table[position * d.rotary_dim + half + i] = (float)(sine * d.amplitude);
}

// Division of n < 2^31 by a number fixed at launch: a product and a shift.  (magic d = 2^shift + e with 0 < e <= 2^(shift - 31), so n magic / 2^shift
// is less than n / d + 1 / d.)
struct Divisor {
  uint32_t d = 1, magic = 0;
  int shift = 0;
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return __umulhi(2 * n, magic) >> (shift - 31); }
};
Divisor divisor(uint32_t d) {
  Divisor r;
  r.d = d;
  int lg = 0;
  while ((1u << lg) < d) ++lg;
  r.shift = 31 + lg;
  r.magic = (uint32_t)(((uint64_t)1 << r.shift) / d + 1);
  return r;
}

// ---- rotation ----------------------------------------------------------------------------------------------------------------------
struct RotaryArray {
  const char* in;
  char* out;
  int64_t in_step, in_seq, in_head, out_step, out_seq, out_head;  // elements
};
struct RotaryArgs {
  RotaryArray a[2];     // q, k
  const float* table;
  const int32_t* positions;
  int32_t n_positions, rotary, first, inverse;
  uint32_t heads[2], n_flags, dim;
  uint32_t pair_items;  // items of a head: rotated ones, then ones that are copied
  Divisor B, seqs_per_flag, items, per_token;
  int32_t table_wide;   // 16-byte accesses to table rows
  int64_t tokens;
};

// One item: E elements and their partners E (half layout), or E consecutive ones that hold E / 2 pairs (interleaved, E > 1); E = 1: one pair, or one
// element that is copied.
template <class T, int E>
struct Piece {
  T v[E];
};
template <class T, int E>
__device__ __forceinline__ Piece<T, E> get(const T* p) {
  Piece<T, E> r;
  if constexpr (E == 1) {
    r.v[0] = *p;
  } else {
    __builtin_memcpy(&r, p, 16);  // (at any alignment)
  }
  return r;
}
template <class T, int E>
__device__ __forceinline__ void put(T* p, const Piece<T, E>& r) {
  if constexpr (E == 1) {
    *p = r.v[0];
  } else {
    __builtin_memcpy(p, &r, 16);
  }
}
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return from_bf16(v); }
template <class T>
__device__ __forceinline__ T narrow(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else return to_bf16(v);
}

// N consecutive values of a table row's half from `first` on, those that there are
template <int N>
__device__ __forceinline__ void load_row(float (&v)[N], const float* half_row, int first, int half, int wide) {
  if (N % 4 == 0 && wide) {  // (half is a multiple of four, and so of a run of four)
#pragma unroll
    for (int k = 0; k + 3 < N; k += 4) {
      const float4 f = *reinterpret_cast<const float4*>(half_row + (first + k < half ? first + k : 0));
      v[k] = f.x; v[k + 1] = f.y; v[k + 2] = f.z; v[k + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = half_row[min(first + k, half - 1)];
  }
}

// A thread takes kItems items, each 256 after the last, so that the chains of loads (position, table row) of several are on their way together.
constexpr int kItems = 4;

template <class T, int E, bool INTERLEAVED>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs args) {
  constexpr bool kPairsInside = INTERLEAVED && E > 1;
  constexpr int kPairs = kPairsInside ? E / 2 : E;  // pairs of an item
  // items in order: token, head (of q, then of k), item of the head; a workgroup's first token and the rest by 32-bit division
  const int64_t first = (int64_t)blockIdx.x * (256 * kItems);
  const int64_t token0 = first / args.per_token.d;
  const uint32_t in0 = (uint32_t)(first - token0 * args.per_token.d) + threadIdx.x;
  const int64_t t00 = token0 / args.B.d;
  const uint32_t b0 = (uint32_t)(token0 - t00 * args.B.d);
  const int R = args.rotary, half = R / 2;
  struct Item {
    T* out;
    Piece<T, E> p1, p2;
    int first_pair;  // -1: copied
    uint32_t c1, c2;
    const float* row;
    bool on, known;
  } it[kItems];
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    Item& x = it[u];
    const uint32_t at = in0 + 256 * u, more = args.per_token(at), in_token = at - more * args.per_token.d;
    x.on = token0 + more < args.tokens;
    if (!x.on) continue;
    uint32_t b = b0 + more;
    const uint32_t over = args.B(b);
    b -= over * args.B.d;
    const int64_t t = t00 + over;
    uint32_t head = args.items(in_token);
    const uint32_t item = in_token - head * args.items.d;
    const bool second = head >= args.heads[0];
    if (second) head -= args.heads[0];
    const RotaryArray& a = args.a[second];
    const T* in = reinterpret_cast<const T*>(a.in) + t * a.in_step + b * a.in_seq + head * a.in_head;
    x.out = reinterpret_cast<T*>(a.out) + t * a.out_step + b * a.out_seq + head * a.out_head;
    if (item >= args.pair_items) {  // behind the rotated part
      x.first_pair = -1;
      x.c1 = kPairsInside ? item * E : R + (item - args.pair_items) * E;
    } else {
      x.first_pair = (int)item * kPairs;
      x.c1 = kPairsInside ? item * E : INTERLEAVED ? 2 * item : item * E;
      x.c2 = INTERLEAVED ? x.c1 + 1 : x.c1 + half;
    }
    x.p1 = get<T, E>(in + x.c1);
    if (!kPairsInside && x.first_pair >= 0) x.p2 = get<T, E>(in + x.c2);
    if (x.first_pair >= 0) {
      const int64_t position = args.positions != nullptr ? args.positions[t * args.n_flags + args.seqs_per_flag(b)] : args.first + t;
      x.known = position >= 0 && position < args.n_positions;
      x.row = args.table + (x.known ? position : 0) * R;
    }
  }
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    Item& x = it[u];
    if (!x.on) continue;
    if (x.first_pair >= 0) {
      float cosine[kPairs], sine[kPairs];
      load_row<kPairs>(cosine, x.row, x.first_pair, half, args.table_wide);
      load_row<kPairs>(sine, x.row + half, x.first_pair, half, args.table_wide);
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        if (kPairsInside && x.first_pair + k >= half) break;
        float c = cosine[k], s = sine[k];
        if (args.inverse) s = -s;
        if (!x.known) c = s = __builtin_nanf("");
        T& v1 = kPairsInside ? x.p1.v[2 * k] : x.p1.v[k];
        T& v2 = kPairsInside ? x.p1.v[2 * k + 1] : x.p2.v[k];
        const float x1 = widen(v1), x2 = widen(v2);
        v1 = narrow<T>(x1 * c - x2 * s);
        v2 = narrow<T>(x1 * s + x2 * c);
      }
      if (!kPairsInside) put<T, E>(x.out + x.c2, x.p2);
    }
    put<T, E>(x.out + x.c1, x.p1);
  }
}

// The items of a head and of a token, and the workgroups for all tokens: 0 where no launch has so many
int64_t lay_out(RotaryArgs& a, int E, bool interleaved) {
  const bool inside = interleaved && E > 1;
  a.pair_items = inside ? ((uint32_t)a.rotary + E - 1) / E : (uint32_t)a.rotary / 2 / E;
  const uint32_t items = inside ? a.dim / E : a.pair_items + (a.dim - a.rotary) / E, per_token = (a.heads[0] + a.heads[1]) * items;
  if (a.tokens > ((int64_t)1 << 40) / per_token) return 0;  // (the product below)
  a.items = divisor(items);
  a.per_token = divisor(per_token);
  const int64_t blocks = (a.tokens * per_token + 256 * kItems - 1) / (256 * kItems);
  return launchable(blocks, 256) ? blocks : 0;
}

template <class T, int E>
int32_t rotate(const RotaryArgs& a, int64_t blocks, bool interleaved, hipStream_t s) {
  if (interleaved) hipLaunchKernelGGL((rotary_kernel<T, E, true>), dim3((unsigned)blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((rotary_kernel<T, E, false>), dim3((unsigned)blocks), dim3(256), 0, s, a);
  return launch_status();
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int32_t marl_rotary_table(const marl_rotary_dims* dims, float* table, void* stream) {
  if (dims == nullptr) return MARL_E_NULL;
  const marl_rotary_dims& d = *dims;
  if (d.n_positions < 1 || d.rotary_dim < 2) return MARL_E_SIZE;
  if (d.rotary_dim % 2 != 0 || d.scaling < 0 || d.scaling > 3) return MARL_E_CONFIG;
  if (!(d.base > 0.f) || (d.scaling != 0 && !(d.factor > 0.f)) || (d.scaling == 2 && d.rotary_dim < 4)) return MARL_E_CONFIG;
  if (d.scaling == 3 && (!(d.trained_length > 0.f) || !(d.fast > d.slow))) return MARL_E_CONFIG;
  MARL_REQUIRE_PTR(table);
  const int64_t blocks = ((int64_t)d.n_positions * (d.rotary_dim / 2) + 255) / 256;
  if (!launchable(blocks, 256)) return MARL_E_SIZE;
  hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, d, table);
  return launch_status();
}

int32_t marl_rotary(const marl_attention_dims* dims, marl_view q, marl_view k, const float* table, int32_t n_positions,
                    int32_t rotary_dim, const int32_t* positions, int32_t first_position, int32_t interleaved,
                    int32_t inverse, marl_view q_out, marl_view k_out, void* stream) {
  if (dims == nullptr) return MARL_E_NULL;
  const marl_attention_dims& d = *dims;
  if (d.precision != 0 && d.precision != 1) return MARL_E_CONFIG;
  if (d.n_steps < 0 || d.n_seqs < 0 || d.n_seqs > (1 << 30) || n_positions < 1) return MARL_E_SIZE;
  if (d.dim_k < 1 || d.dim_k > 1024 || rotary_dim < 2 || rotary_dim > d.dim_k) return MARL_E_SIZE;
  if (rotary_dim % 2 != 0 || interleaved < 0 || interleaved > 1 || inverse < 0 || inverse > 1) return MARL_E_CONFIG;
  if (d.n_heads < 1 || d.n_heads > (1 << 14) || (k.data != nullptr && (d.n_kv_heads < 1 || d.n_kv_heads > (1 << 14)))) return MARL_E_CONFIG;
  if (d.seqs_per_flag < 1 || d.n_seqs % d.seqs_per_flag != 0) return MARL_E_CONFIG;
  RotaryArgs a{};
  a.tokens = (int64_t)d.n_steps * d.n_seqs;
  if (a.tokens == 0) return MARL_OK;
  const uintptr_t odd = d.precision == 0 ? 3u : 1u;
  const int elem = d.precision == 0 ? 4 : 2;
  const int n = k.data != nullptr ? 2 : 1;
  const marl_view in[2] = {q, k}, out[2] = {q_out, k_out};
  for (int u = 0; u < n; ++u) {
    if (in[u].data == nullptr || out[u].data == nullptr) return MARL_E_NULL;
    const uintptr_t pi = reinterpret_cast<uintptr_t>(in[u].data), po = reinterpret_cast<uintptr_t>(out[u].data);
    if (((pi | po) & odd) != 0) return MARL_E_ALIGN;
    if ((out[u].step == 0 && d.n_steps > 1) || (out[u].seq == 0 && d.n_seqs > 1) || (out[u].head == 0 && (u == 0 ? d.n_heads : d.n_kv_heads) > 1))
      return MARL_E_CONFIG;  // an output's elements are places of their own
    if (out[u].data == in[u].data && ((out[u].step != in[u].step && d.n_steps > 1) || (out[u].seq != in[u].seq && d.n_seqs > 1) ||
                                      (out[u].head != in[u].head && (u == 0 ? d.n_heads : d.n_kv_heads) > 1)))
      return MARL_E_CONFIG;  // in place: the strides agree
    a.a[u] = {static_cast<const char*>(in[u].data), static_cast<char*>(out[u].data), in[u].step, in[u].seq, in[u].head, out[u].step, out[u].seq,
              out[u].head};
  }
  MARL_REQUIRE_PTR(table);
  if ((reinterpret_cast<uintptr_t>(positions) & 3u) != 0) return MARL_E_ALIGN;
  a.table = table;
  a.positions = positions;
  a.n_positions = n_positions;
  a.rotary = rotary_dim;
  a.first = first_position;
  a.inverse = inverse;
  a.B = divisor((uint32_t)d.n_seqs);
  a.heads[0] = (uint32_t)d.n_heads;
  a.heads[1] = n == 2 ? (uint32_t)d.n_kv_heads : 0;
  a.seqs_per_flag = divisor((uint32_t)d.seqs_per_flag);
  a.n_flags = (uint32_t)(d.n_seqs / d.seqs_per_flag);
  a.dim = (uint32_t)d.dim_k;
  a.table_wide = rotary_dim % 8 == 0;
  const int E = 16 / elem;
  const bool wide = d.dim_k % E == 0 && (interleaved || rotary_dim / 2 % E == 0);
  const int64_t blocks = lay_out(a, wide ? E : 1, interleaved != 0);
  if (blocks == 0) return MARL_E_SIZE;
  if (n == 2 && (q_out.data == k_out.data || q_out.data == k.data || k_out.data == q.data)) return MARL_E_CONFIG;
  hipStream_t s = (hipStream_t)stream;
  if (d.precision == 0) return wide ? rotate<float, 4>(a, blocks, interleaved != 0, s) : rotate<float, 1>(a, blocks, interleaved != 0, s);
  return wide ? rotate<bf16_t, 8>(a, blocks, interleaved != 0, s) : rotate<bf16_t, 1>(a, blocks, interleaved != 0, s);
}

}  // extern "C"
