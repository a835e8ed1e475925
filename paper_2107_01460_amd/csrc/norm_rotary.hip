// The norm of each head of queries and keys with the rotation by position in the same pass, and its gradient.
//   u = x r w,  r = 1 / sqrt(mean(x^2) + eps),  y = turn(u);   with du = turn back(dy) and g = du w:  dx = r g - x r^3 mean(g x),  dw = sum over rows of du x r
// dw is summed in fp32 (a lane's rows, then a workgroup's lanes, then the workgroups): 2.7e-7 off, relative to 64 bits, over 128 x 4096 steps of 4 heads in fp32.
// Bound by memory: every element in and out once; table rows, weights and the partners of a rotation come from caches.  128 x 4096 steps of 8 + 8 heads of 64 in bf16: 427 us
// for 2.1 GB; gradient of 4 + 2 heads of 32 in fp32: 237 us for 1.2 GB, and 8 for the sums of the weights' gradients: what a copy reaches.
#include "attention_checks.h"
#include "divisor.h"
#include "lane_sums.h"

namespace marl {
namespace {

constexpr int kMaxNormDim = 256;

struct NormArray {
  const char *x, *dy;
  char* out;  // y, or dx
  int64_t x_step, x_seq, x_head, dy_step, dy_seq, dy_head, out_step, out_seq, out_head;  // bytes
  const float* weight;
  float* part;  // [workgroups][dim]: a workgroup's share of dw
  uint32_t heads;
  Divisor chunks;  // of kHeads heads: of a token
  int64_t units;   // tokens times chunks
};
struct NormArgs {
  NormArray a[2];  // q, k
  const float* table;
  const int32_t* positions;
  int32_t n_positions, first, rotary, dim, inter;
  float eps;
  uint32_t n_flags;
  Divisor B, seqs_per_flag;
  uint32_t blocks_q;  // workgroups of q; those of k follow
};

// E elements of a row from `col` on, which may begin before the row or end behind it: zeros there, and nothing outside the row is read.
template <class T, bool WHOLE>
__device__ __forceinline__ void get(float (&f)[16 / sizeof(T)], const char* row, int col, int dim) {
  constexpr int E = 16 / sizeof(T);
  const T* p = reinterpret_cast<const T*>(row);
  T v[E];
  if constexpr (WHOLE) {
    __builtin_memcpy(v, p + col, 16);  // (at any alignment)
  } else if (dim >= E) {
    const int base = min(max(col, 0), dim - E), by = col - base;  // moved down by `by` elements
    unsigned __int128 w;
    __builtin_memcpy(&w, p + base, 16);
    if (by > 0) w = by < E ? w >> 8 * (int)sizeof(T) * by : 0;
    if (by < 0) w = by > -E ? w << 8 * (int)sizeof(T) * -by : 0;
    __builtin_memcpy(v, &w, 16);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = col + e >= 0 && col + e < dim ? p[col + e] : (T)0;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = load_act(v, e);
}
template <class T, bool WHOLE>
__device__ __forceinline__ void put(char* row, int col, int dim, const float (&f)[16 / sizeof(T)]) {
  constexpr int E = 16 / sizeof(T);
  T v[E];
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = f[e];
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const uint32_t u = pack2_bf16(f[e], f[e + 1]);
      __builtin_memcpy(v + e, &u, 4);
    }
  }
  T* p = reinterpret_cast<T*>(row) + col;
  if (WHOLE || col + E <= dim) {
    __builtin_memcpy(p, v, 16);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (col + e < dim) p[e] = v[e];
  }
}
// What a lane's E columns are to the rotation
template <class T, bool INTER, bool WHOLE>
struct Columns {
  static constexpr int E = 16 / sizeof(T);
  int col, half, rotary;
  // the table's cosines and sines for a position's row, 1 and 0 behind the rotated part; sine with the sign of an element's partner
  __device__ __forceinline__ void angles(const float* row, bool known, float (&c)[E], float (&s)[E]) const {
    const float none = __builtin_nanf("");
    if constexpr (WHOLE && !INTER) {
      const bool on = col < rotary;
      const int at = on ? (col < half ? col : col - half) : 0;
      const float sign = col < half ? -1.f : 1.f;
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        float a[4], b[4];
        __builtin_memcpy(a, row + at + e, 16);
        __builtin_memcpy(b, row + half + at + e, 16);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          c[e + x] = on ? known ? a[x] : none : 1.f;
          s[e + x] = on ? known ? sign * b[x] : none : 0.f;
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = col + e;
        const bool on = i < rotary;
        const int at = !on ? 0 : INTER ? i / 2 : i < half ? i : i - half;
        const float sign = INTER ? (e % 2 == 0 ? -1.f : 1.f) : i < half ? -1.f : 1.f;
        c[e] = on ? known ? row[at] : none : 1.f;
        s[e] = on ? known ? sign * row[half + at] : none : 0.f;
      }
    }
  }
  // each element's partner: inside the vector (taken from there where it is used), or half the rotated part away; zero behind the rotated part, since a neighbour's infinity
  // times the sine of 0 is a NaN
  __device__ __forceinline__ float partner(const float (&own)[E], const float (&p)[E], int e) const {
    if constexpr (INTER) return col + (e & ~1) < rotary ? own[e ^ 1] : 0.f;
    else return p[e];
  }
  template <class F>
  __device__ __forceinline__ void partners(float (&p)[E], F load) const {
    if constexpr (INTER) {
      (void)load;
    } else if constexpr (WHOLE) {
      if (col < rotary) load(p, col < half ? col + half : col - half);
      else {
#pragma unroll
        for (int e = 0; e < E; ++e) p[e] = 0.f;
      }
    } else {
      float up[E], down[E];
#pragma unroll
      for (int e = 0; e < E; ++e) up[e] = down[e] = 0.f;
      if (col < half) load(up, col + half);
      if (col + E > half && col < rotary) load(down, col - half);
#pragma unroll
      for (int e = 0; e < E; ++e) p[e] = col + e < half ? up[e] : col + e < rotary ? down[e] : 0.f;
    }
  }
};

constexpr int kHeads = 4;  // of a token, one after another: position, table row and places are worked out once for them (one by one: 790 us for those 427, 293 for the 235)

// L lanes take a token's heads, kHeads of them; a workgroup every so many of one array's units.
template <class T, int L, bool INTER, bool WHOLE, bool GRADIENT>
__global__ void __launch_bounds__(256) norm_rotary_kernel(const NormArgs args) {
  constexpr int E = 16 / sizeof(T), kAtOnce = 256 / L;
  const bool second = blockIdx.x >= args.blocks_q;
  const NormArray a = second ? args.a[1] : args.a[0];
  const uint32_t block = second ? blockIdx.x - args.blocks_q : blockIdx.x, blocks = second ? gridDim.x - args.blocks_q : args.blocks_q;
  const int dim = args.dim, lane = threadIdx.x % L;
  Columns<T, INTER, WHOLE> cols{lane * E, args.rotary / 2, args.rotary};
  const int col = cols.col;
  const bool on = col < dim;
  float w[E], wp[E];  // weights, and the partners'
  auto weights = [&](float (&f)[E], int from) {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = from + e >= 0 && from + e < dim ? a.weight[from + e] : 0.f;
  };
  if (a.weight == nullptr || !on) {
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = wp[e] = 1.f;
  } else {
    weights(w, col);
    if constexpr (!GRADIENT) cols.partners(wp, weights);
  }
  float dw[E];
#pragma unroll
  for (int e = 0; e < E; ++e) dw[e] = 0.f;
  const float each = 1.f / (float)dim;
  const bool small = a.units < 0x7fffffff;
  for (int64_t unit = (int64_t)block * kAtOnce + threadIdx.x / L; unit < a.units; unit += (int64_t)blocks * kAtOnce) {
    uint32_t chunk, b;
    int64_t t;
    if (small) {
      const uint32_t token = a.chunks((uint32_t)unit), row = args.B(token);
      chunk = (uint32_t)unit - token * a.chunks.d;
      t = row;
      b = token - row * args.B.d;
    } else {
      const int64_t token = unit / a.chunks.d;
      chunk = (uint32_t)(unit - token * a.chunks.d);
      t = token / args.B.d;
      b = (uint32_t)(token - t * args.B.d);
    }
    const int position = args.positions != nullptr ? args.positions[t * args.n_flags + args.seqs_per_flag(b)] : args.first + (int)t;
    const uint32_t head0 = chunk * kHeads;
    const int n = min((int)(a.heads - head0), kHeads);
    const char* x = a.x + t * a.x_step + b * a.x_seq + head0 * a.x_head;
    const char* dy = GRADIENT ? a.dy + t * a.dy_step + b * a.dy_seq + head0 * a.dy_head : nullptr;
    char* out = a.out + t * a.out_step + b * a.out_seq + head0 * a.out_head;
    float v[kHeads][E], z[kHeads][E], zp[kHeads][E];  // x; what is turned (x, or dy) and its partners
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[u][e] = z[u][e] = zp[u][e] = 0.f;
      if (u >= n || !on) continue;
      get<T, WHOLE>(v[u], x + u * a.x_head, col, dim);
      if constexpr (!GRADIENT) {
        cols.partners(zp[u], [&](float (&f)[E], int from) { get<T, WHOLE>(f, x + u * a.x_head, from, dim); });
      } else {
        get<T, WHOLE>(z[u], dy + u * a.dy_head, col, dim);
        cols.partners(zp[u], [&](float (&f)[E], int from) { get<T, WHOLE>(f, dy + u * a.dy_head, from, dim); });
      }
    }
    const bool known = position < args.n_positions;
    float c[E], s[E];
    cols.angles(args.table + (int64_t)(known ? max(position, 0) : 0) * args.rotary, known, c, s);
    if constexpr (!GRADIENT) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        c[e] *= w[e];
        s[e] *= cols.partner(w, wp, e);
      }
    }
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      if (u >= n) break;
      float squares = 0.f, y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) squares = __builtin_fmaf(v[u][e], v[u][e], squares);
      squares = sum_lanes<L>(squares);
      const float rstd = 1.f / __builtin_sqrtf(squares * each + args.eps);
      if constexpr (!GRADIENT) {
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = rstd * (v[u][e] * c[e] + cols.partner(v[u], zp[u], e) * s[e]);
      } else {
        float g[E], du[E], dot = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          du[e] = z[u][e] * c[e] - cols.partner(z[u], zp[u], e) * s[e];
          g[e] = du[e] * w[e];
          if (on) dot = __builtin_fmaf(g[e], v[u][e], dot);
        }
        dot = sum_lanes<L>(dot);
        const float back = rstd * rstd * (dot * each);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          y[e] = rstd * (g[e] - v[u][e] * back);
          if (position >= 0 && on) dw[e] = __builtin_fmaf(du[e], v[u][e] * rstd, dw[e]);
        }
      }
      if (position < 0) {  // no step: zeros
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = 0.f;
      }
      if (on) put<T, WHOLE>(out + u * a.out_head, col, dim, y);
    }
  }
  if constexpr (GRADIENT) {
    if (a.part == nullptr) return;
    // the lanes that took the same columns, in the order of the threads
    __shared__ float sums[256 / L][L * E];
#pragma unroll
    for (int e = 0; e < E; ++e) sums[threadIdx.x / L][lane * E + e] = dw[e];
    __syncthreads();
    for (int i = threadIdx.x; i < dim; i += 256) {
      float sum = 0.f;
      for (int r = 0; r < 256 / L; ++r) sum += sums[r][i];
      a.part[(int64_t)block * dim + i] = sum;
    }
  }
}

// dw: the workgroups' shares, 32 columns a workgroup, in a fixed order
struct WeightArgs {
  const float* part[2];
  float* out[2];
  int32_t n[2], dim;
};
__global__ void __launch_bounds__(1024) norm_weight_kernel(const WeightArgs a) {
  __shared__ float sums[32][33];
  const int which = blockIdx.y, c = threadIdx.x % 32, r = threadIdx.x / 32, col = blockIdx.x * 32 + c;
  if (a.out[which] == nullptr) return;
  float sum = 0.f;
  if (col < a.dim) {
#pragma unroll 8
    for (int i = r; i < a.n[which]; i += 32) sum += a.part[which][(int64_t)i * a.dim + col];
  }
  sums[r][c] = sum;
  __syncthreads();
  if (r == 0 && col < a.dim) {
    float all = 0.f;
    for (int i = 0; i < 32; ++i) all += sums[i][c];
    a.out[which][col] = all;
  }
}

int lanes_of(int precision, int dim) {
  const int units = (dim + (precision == 0 ? 3 : 7)) / (precision == 0 ? 4 : 8);
  int L = 1;
  while (L < units) L *= 2;
  return L;
}
// Workgroups of an array: as many as fill the chip, so that weights are read once
constexpr int64_t kMaxBlocks = 2048;
int64_t blocks_of(int64_t units, int L) {
  const int64_t run = 256 / L, n = (units + run - 1) / run;
  return n > kMaxBlocks ? kMaxBlocks : n;
}
// Of the workspace: the shares of dw of one array's workgroups
int64_t share_bytes(const marl_attention_dims& d) { return (kMaxBlocks * d.dim_k * 4 + 255) / 256 * 256; }

template <class T, int L, bool GRADIENT>
void launch_lanes(const NormArgs& a, unsigned blocks, bool inter, bool whole, hipStream_t s) {
  if (inter && whole) hipLaunchKernelGGL((norm_rotary_kernel<T, L, true, true, GRADIENT>), dim3(blocks), dim3(256), 0, s, a);
  else if (inter) hipLaunchKernelGGL((norm_rotary_kernel<T, L, true, false, GRADIENT>), dim3(blocks), dim3(256), 0, s, a);
  else if (whole) hipLaunchKernelGGL((norm_rotary_kernel<T, L, false, true, GRADIENT>), dim3(blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((norm_rotary_kernel<T, L, false, false, GRADIENT>), dim3(blocks), dim3(256), 0, s, a);
}
template <class T, bool GRADIENT>
void launch_norm(const NormArgs& a, int L, unsigned blocks, bool inter, bool whole, hipStream_t s) {
  if (L == 1) launch_lanes<T, 1, GRADIENT>(a, blocks, inter, whole, s);
  else if (L == 2) launch_lanes<T, 2, GRADIENT>(a, blocks, inter, whole, s);
  else if (L == 4) launch_lanes<T, 4, GRADIENT>(a, blocks, inter, whole, s);
  else if (L == 8) launch_lanes<T, 8, GRADIENT>(a, blocks, inter, whole, s);
  else if (L == 16) launch_lanes<T, 16, GRADIENT>(a, blocks, inter, whole, s);
  else if (L == 32) launch_lanes<T, 32, GRADIENT>(a, blocks, inter, whole, s);
  else if constexpr (sizeof(T) == 4) launch_lanes<T, 64, GRADIENT>(a, blocks, inter, whole, s);
}

int32_t check_norm(const marl_attention_dims* dims, bool k) {
  if (dims == nullptr) return MARL_E_NULL;
  const marl_attention_dims& d = *dims;
  if (d.precision != 0 && d.precision != 1) return MARL_E_CONFIG;
  if (d.n_steps < 0 || d.n_steps > (1 << 30) || d.n_seqs < 0 || d.n_seqs > (1 << 30) || d.dim_k < 1 || d.dim_k > kMaxNormDim) return MARL_E_SIZE;
  if (d.n_heads < 1 || d.n_heads > (1 << 14) || (k && (d.n_kv_heads < 1 || d.n_kv_heads > (1 << 14)))) return MARL_E_CONFIG;
  if (d.seqs_per_flag < 1 || d.n_seqs % d.seqs_per_flag != 0) return MARL_E_CONFIG;
  const int64_t tokens = (int64_t)d.n_steps * d.n_seqs;
  if (tokens > ((int64_t)1 << 48) / (1 << 15)) return MARL_E_SIZE;
  return MARL_OK;
}
int32_t check_turn(const marl_attention_dims& d, float eps, const float* table, int32_t n_positions, int32_t rotary_dim, const int32_t* positions,
                   int32_t first, int32_t interleaved) {
  if (n_positions < 1 || rotary_dim < 2 || rotary_dim > d.dim_k) return MARL_E_SIZE;
  if (rotary_dim % 2 != 0 || interleaved < 0 || interleaved > 1 || !(eps >= 0.f) || !(eps < __builtin_inff())) return MARL_E_CONFIG;
  if (positions == nullptr && (int64_t)first + d.n_steps > 0x7fffffff) return MARL_E_SIZE;
  MARL_REQUIRE_PTR(table);
  return (reinterpret_cast<uintptr_t>(positions) & 3u) != 0 ? MARL_E_ALIGN : MARL_OK;
}
int32_t check_vector(const float* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0 ? MARL_E_ALIGN : MARL_OK; }
// An output in the place of an input has its strides
int32_t check_in_place(const marl_view& out, const marl_view& in, const marl_attention_dims& d, int heads) {
  if (out.data != in.data) return MARL_OK;
  return (out.step != in.step && d.n_steps > 1) || (out.seq != in.seq && d.n_seqs > 1) || (out.head != in.head && heads > 1) ? MARL_E_CONFIG : MARL_OK;
}

NormArray array_of(const marl_attention_dims& d, const marl_view& x, const marl_view* dy, const marl_view& out, int heads, const float* weight) {
  const int elem = d.precision == 0 ? 4 : 2;
  NormArray a{};
  a.x = static_cast<const char*>(x.data);
  a.x_step = x.step * elem;
  a.x_seq = x.seq * elem;
  a.x_head = x.head * elem;
  if (dy != nullptr) {
    a.dy = static_cast<const char*>(dy->data);
    a.dy_step = dy->step * elem;
    a.dy_seq = dy->seq * elem;
    a.dy_head = dy->head * elem;
  }
  a.out = static_cast<char*>(out.data);
  a.out_step = out.step * elem;
  a.out_seq = out.seq * elem;
  a.out_head = out.head * elem;
  a.weight = weight;
  a.heads = (uint32_t)heads;
  a.chunks = divisor((uint32_t)(heads + kHeads - 1) / kHeads);
  a.units = (int64_t)d.n_steps * d.n_seqs * a.chunks.d;
  return a;
}
NormArgs args_of(const marl_attention_dims& d, float eps, const float* table, int32_t n_positions, int32_t rotary_dim, const int32_t* positions,
                 int32_t first, int32_t interleaved) {
  NormArgs a{};
  a.table = table;
  a.positions = positions;
  a.n_positions = n_positions;
  a.first = first;
  a.rotary = rotary_dim;
  a.dim = d.dim_k;
  a.inter = interleaved;
  a.eps = eps;
  a.n_flags = (uint32_t)(d.n_seqs / d.seqs_per_flag);
  a.B = divisor((uint32_t)d.n_seqs);
  a.seqs_per_flag = divisor((uint32_t)d.seqs_per_flag);
  return a;
}
int32_t run(NormArgs& a, const marl_attention_dims& d, bool gradient, bool k, hipStream_t s) {
  const int L = lanes_of(d.precision, d.dim_k), E = d.precision == 0 ? 4 : 8;
  const bool whole = d.dim_k % E == 0 && (a.inter || a.rotary / 2 % E == 0);
  a.blocks_q = (uint32_t)blocks_of(a.a[0].units, L);
  const unsigned blocks = a.blocks_q + (k ? (unsigned)blocks_of(a.a[1].units, L) : 0);
  if (d.precision == 0) (gradient ? launch_norm<float, true> : launch_norm<float, false>)(a, L, blocks, a.inter != 0, whole, s);
  else (gradient ? launch_norm<bf16_t, true> : launch_norm<bf16_t, false>)(a, L, blocks, a.inter != 0, whole, s);
  return launch_status();
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int32_t marl_norm_rotary(const marl_attention_dims* dims, marl_view q, marl_view k, const float* q_weight, const float* k_weight, float eps,
                         const float* table, int32_t n_positions, int32_t rotary_dim, const int32_t* positions, int32_t first_position,
                         int32_t interleaved, marl_view q_out, marl_view k_out, void* stream) {
  const bool two = k.data != nullptr;
  MARL_CHECK(check_norm(dims, two));
  const marl_attention_dims& d = *dims;
  const bool used = d.n_steps > 0 && d.n_seqs > 0;
  if (!used) return MARL_OK;
  MARL_CHECK(check_turn(d, eps, table, n_positions, rotary_dim, positions, first_position, interleaved));
  MARL_CHECK(check_vector(q_weight));
  MARL_CHECK(check_vector(k_weight));
  const marl_view in[2] = {q, k}, out[2] = {q_out, k_out};
  for (int u = 0; u < (two ? 2 : 1); ++u) {
    const int heads = u == 0 ? d.n_heads : d.n_kv_heads;
    MARL_CHECK(check_view(in[u], d.precision, true));
    MARL_CHECK(check_view(out[u], d.precision, true));
    MARL_CHECK(check_output(out[u], d, heads, true));
    MARL_CHECK(check_in_place(out[u], in[u], d, heads));
  }
  if (two && (q_out.data == k_out.data || q_out.data == k.data || k_out.data == q.data)) return MARL_E_CONFIG;
  for (int u = 0; u < (two ? 2 : 1); ++u)
    if (touches(out[u], d, u == 0 ? d.n_heads : d.n_kv_heads, d.dim_k,
                {extent(table, (int64_t)n_positions * rotary_dim * 4), places_of(d, positions), extent(q_weight, d.dim_k * 4), extent(k_weight, d.dim_k * 4)}))
      return MARL_E_CONFIG;
  NormArgs a = args_of(d, eps, table, n_positions, rotary_dim, positions, first_position, interleaved);
  a.a[0] = array_of(d, q, nullptr, q_out, d.n_heads, q_weight);
  if (two) a.a[1] = array_of(d, k, nullptr, k_out, d.n_kv_heads, k_weight);
  return run(a, d, false, two, (hipStream_t)stream);
}

int32_t marl_norm_rotary_workspace(const marl_attention_dims* dims, int64_t* bytes) {
  MARL_CHECK(check_norm(dims, true));
  if (bytes == nullptr) return MARL_E_NULL;
  *bytes = 2 * share_bytes(*dims);
  return MARL_OK;
}

int32_t marl_norm_rotary_backward(const marl_attention_dims* dims, marl_view dq_out, marl_view dk_out, marl_view q, marl_view k, const float* q_weight,
                                  const float* k_weight, float eps, const float* table, int32_t n_positions, int32_t rotary_dim,
                                  const int32_t* positions, int32_t first_position, int32_t interleaved, marl_view dq, marl_view dk,
                                  float* dq_weight, float* dk_weight, void* workspace, void* stream) {
  const bool two = k.data != nullptr;
  MARL_CHECK(check_norm(dims, two));
  const marl_attention_dims& d = *dims;
  const bool used = d.n_steps > 0 && d.n_seqs > 0;
  MARL_CHECK(check_vector(q_weight));
  MARL_CHECK(check_vector(k_weight));
  MARL_CHECK(check_vector(dq_weight));
  MARL_CHECK(check_vector(dk_weight));
  const Extent wq = extent(q_weight, d.dim_k * 4), wk = extent(k_weight, d.dim_k * 4), gq = extent(dq_weight, d.dim_k * 4), gk = extent(dk_weight, d.dim_k * 4);
  if (gq.meets(gk)) return MARL_E_CONFIG;
  const bool weights = dq_weight != nullptr || ((two || !used) && dk_weight != nullptr);
  const marl_view in[2] = {q, k}, grad[2] = {dq_out, dk_out}, out[2] = {dq, dk};
  if (used) {
    MARL_CHECK(check_turn(d, eps, table, n_positions, rotary_dim, positions, first_position, interleaved));
    if (weights) MARL_REQUIRE_PTR(workspace);
    for (int u = 0; u < (two ? 2 : 1); ++u) {
      const int heads = u == 0 ? d.n_heads : d.n_kv_heads;
      MARL_CHECK(check_view(in[u], d.precision, true));
      MARL_CHECK(check_view(grad[u], d.precision, true));
      MARL_CHECK(check_view(out[u], d.precision, true));
      MARL_CHECK(check_output(out[u], d, heads, true));
      MARL_CHECK(check_in_place(out[u], in[u], d, heads));
      MARL_CHECK(check_in_place(out[u], grad[u], d, heads));
    }
    if (two) {
      MARL_CHECK(check_places(dq, {k, dk_out, dk}, true));
      MARL_CHECK(check_places(dk, {q, dq_out}, true));
    }
    const Extent angles = extent(table, (int64_t)n_positions * rotary_dim * 4), ps = places_of(d, positions), ws = extent(workspace, weights ? 2 * share_bytes(d) : 0);
    for (int u = 0; u < (two ? 2 : 1); ++u) {
      const int heads = u == 0 ? d.n_heads : d.n_kv_heads;
      if (touches(out[u], d, heads, d.dim_k, {angles, ps, wq, wk, gq, gk, ws}) || touches(in[u], d, heads, d.dim_k, {gq, gk, ws}) ||
          touches(grad[u], d, heads, d.dim_k, {gq, gk, ws}))
        return MARL_E_CONFIG;
    }
    for (const Extent& x : {angles, ps, wq, wk, gq, gk})
      if (ws.meets(x)) return MARL_E_CONFIG;
  }
  hipStream_t s = (hipStream_t)stream;
  WeightArgs w{};
  w.dim = d.dim_k;
  if (used) {
    NormArgs a = args_of(d, eps, table, n_positions, rotary_dim, positions, first_position, interleaved);
    a.a[0] = array_of(d, q, &dq_out, dq, d.n_heads, q_weight);
    if (two) a.a[1] = array_of(d, k, &dk_out, dk, d.n_kv_heads, k_weight);
    if (dq_weight != nullptr) a.a[0].part = static_cast<float*>(workspace);
    if (two && dk_weight != nullptr) a.a[1].part = reinterpret_cast<float*>(static_cast<char*>(workspace) + share_bytes(d));
    MARL_CHECK(run(a, d, true, two, s));
    const int L = lanes_of(d.precision, d.dim_k);
    w.part[0] = a.a[0].part;
    w.part[1] = a.a[1].part;
    w.n[0] = (int32_t)blocks_of(a.a[0].units, L);
    w.n[1] = two ? (int32_t)blocks_of(a.a[1].units, L) : 0;
  }
  if (!weights) return MARL_OK;
  w.out[0] = dq_weight;
  w.out[1] = two || !used ? dk_weight : nullptr;  // (an array of no elements has no address)
  hipLaunchKernelGGL(norm_weight_kernel, dim3((d.dim_k + 31) / 32, 2), dim3(1024), 0, s, w);
  return launch_status();
}

}  // extern "C"
