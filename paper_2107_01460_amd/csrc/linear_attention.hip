// Linear attention: the calls, the join of the stretches of a long sequence, the sum over shared heads, the single step.
#include <initializer_list>
#include <type_traits>

#include "linear_attention.h"

namespace marl {
namespace {

constexpr int kMaxDim = 128;

// ---- how a call is laid out ----------------------------------------------------------------------------------------------------
struct Plan {
  int64_t pairs;         // sequences * query heads
  int group;             // query heads per key / value head
  uint32_t n_stretches;
  int32_t stretch;
  int64_t states, carry, reverse_states, dk, dv, bytes;  // offsets into the workspace
};

// A call with few sequences is cut over time into stretches: their own states first, joined along time, then every stretch with the state that
// comes in.  The states cost a second reading of k and v and half the matrix products again, so only while there are fewer wavefronts than
// the chip holds: 8 for each of the 256 compute units.  (32 768 steps of 8 query heads of 128, with a state, when this was chosen: 147 us; aiming at 1024, 1536 or
// 4096 wavefronts 183, 171, 174.  Gradient of 8192 steps of 8 heads of 64: 59; 68, 60, 55.  Now 151 and 57.)  A gradient counts three times the slices of dim_v, its
// wavefronts where the widths agree; where they do not, it launches twice those of dim_k, then once those of dim_v.  No stretch is shorter than 64 steps.
Plan plan_of(const marl_attention_dims& d, bool backward) {
  constexpr int64_t kWaves = 2048;
  Plan p{};
  p.pairs = (int64_t)d.n_seqs * d.n_heads;
  p.group = d.n_heads / d.n_kv_heads;
  const int64_t units = p.pairs * scan_slices(d.dim_v) * (backward ? 3 : 1);
  const int tile = 16 * (d.precision == 0 ? ScanTraits<float>::kSub : ScanTraits<bf16_t>::kSub), least = 64 / tile;
  const int64_t tiles = ((int64_t)d.n_steps + tile - 1) / tile;
  int64_t n = units > 0 ? kWaves / units : 1;
  n = n < tiles / least ? n : tiles / least;
  if (n < 2) n = 1;
  const int64_t per = tiles > 0 ? (tiles + n - 1) / n : 1;
  p.stretch = (int32_t)(per * tile);
  p.n_stretches = (uint32_t)(tiles > 0 ? (tiles + per - 1) / per : 1);
  if (p.n_stretches == 1) p.stretch = tiles > 0 ? (int32_t)(tiles * tile) : tile;
  int64_t at = 0;
  auto take = [&](int64_t floats) {
    const int64_t here = at;
    at += (floats * 4 + 255) / 256 * 256;
    return here;
  };
  if (p.n_stretches > 1) {
    p.states = take(p.pairs * p.n_stretches * d.dim_k * d.dim_v);
    p.carry = take(p.pairs * p.n_stretches);
    if (backward) p.reverse_states = take(p.pairs * p.n_stretches * d.dim_k * d.dim_v);
  }
  if (backward && p.group > 1) {
    p.dk = take((int64_t)d.n_steps * p.pairs * d.dim_k);
    p.dv = take((int64_t)d.n_steps * p.pairs * d.dim_v);
  }
  p.bytes = at;
  return p;
}

// ---- the states along the stretches: one thread per element ------------------------------------------------------------------------
// Bound by memory: every stretch's state in and out (64 stretches of 8 states of 128 x 128: 67 MB, 15 us), 32 loads of a thread on their way together.
// in: states each stretch forms by itself; out: the state that comes into it.  Behind a stretch in which an episode ended nothing of what came in is left,
// infinities and NaNs included; without an end these go on whatever the decay's power is.
struct JoinArgs {
  float* states;
  const float *carry, *first;
  float* last;
  int32_t n;
  int32_t reverse;
};
__global__ void __launch_bounds__(256) join_kernel(JoinArgs a0, JoinArgs a1, uint32_t size, int64_t total) {
  const JoinArgs a = blockIdx.y == 0 ? a0 : a1;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= total) return;
  const int64_t pair = at / size, e = at % size;
  float run = a.first == nullptr ? 0.f : a.first[at];
  constexpr int kBatch = 32;  // loads on their way together
  for (int p0 = 0; p0 < a.n; p0 += kBatch) {
    float v[kBatch], c[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int q = min(p0 + u, a.n - 1), p = a.reverse ? a.n - 1 - q : q;
      v[u] = a.states[(pair * a.n + p) * size + e];
      c[u] = a.carry[pair * a.n + p];
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (p0 + u >= a.n) break;
      const int p = a.reverse ? a.n - 1 - (p0 + u) : p0 + u;
      a.states[(pair * a.n + p) * size + e] = run;
      run = c[u] == kCarryEnded ? v[u] : c[u] * run + v[u];
    }
  }
  if (a.last != nullptr) a.last[at] = run;
}

// ---- the gradient of a shared head: the sum over its query heads -------------------------------------------------------------------
// In a fixed order.  Bound by memory (777 x 111 steps, 6 heads of 40 on 2: 83 MB of shares in, 14 out, 23 us).
template <class T, int V>
__global__ void __launch_bounds__(256) sum_heads_kernel(const float* __restrict__ part, T* __restrict__ out, int64_t step, int64_t seq, int64_t head,
                                                        uint32_t B, uint32_t heads, uint32_t group, uint32_t dim) {
  const uint32_t t = blockIdx.y, per_step = B * heads * (dim / V);
  for (uint32_t at = blockIdx.x * 256 + threadIdx.x; at < per_step; at += gridDim.x * 256) {
    const uint32_t row = at / (dim / V), d = (at - row * (dim / V)) * V;  // row: (sequence, kv head)
    const uint32_t b = row / heads, h = row - b * heads;
    const float* p = part + ((int64_t)t * B * heads + row) * group * dim + d;
    float s[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = 0.f;
    for (uint32_t u = 0; u < group; ++u, p += dim) {
      if constexpr (V == 4) {
        const float4 f = *reinterpret_cast<const float4*>(p);
        s[0] += f.x; s[1] += f.y; s[2] += f.z; s[3] += f.w;
      } else {
        s[0] += *p;
      }
    }
    T* o = out + (int64_t)t * step + b * seq + h * head + d;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if constexpr (sizeof(T) == 4) o[k] = s[k];
      else o[k] = to_bf16(s[k]);
    }
  }
}

// ---- one step ------------------------------------------------------------------------------------------------------------------------
// A team of threads takes one head of one sequence: every thread its V columns of every so many rows of the state, read once, written once.  Bound by memory:
// 16 384 states of 4 heads of 32 x 32 take 99 us, 5.8 TB/s; where the columns are no multiple of four, 4-byte accesses, 2.9 TB/s (31 x 31).
template <class T, int V, int TEAM>
__global__ void __launch_bounds__(256) step_kernel(const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, T* __restrict__ out,
                                                   int64_t qs, int64_t qh, int64_t ks, int64_t kh, int64_t vs, int64_t vh, int64_t os, int64_t oh,
                                                   const float* __restrict__ decay, const float* state, const uint8_t* __restrict__ fresh,
                                                   float* next, uint32_t pairs, uint32_t H, uint32_t group, uint32_t seqs_per_flag, int Dk,
                                                   int Dv, float scale) {
  constexpr int kTeams = 256 / TEAM;
  __shared__ float sum[kTeams][TEAM * V];
  const int team = threadIdx.x / TEAM, lane = threadIdx.x % TEAM;
  const uint32_t pair = blockIdx.x * kTeams + team;
  const bool on = pair < pairs;
  const uint32_t b = on ? pair / H : 0, h = on ? pair % H : 0;
  const int Q = (Dv + V - 1) / V, R = TEAM / Q;   // column groups, rows at once
  const int c = lane % Q, r0 = lane / Q;
  float o[V];
#pragma unroll
  for (int u = 0; u < V; ++u) o[u] = 0.f;
  if (on && r0 < R) {
    const float keep = fresh != nullptr && fresh[b / seqs_per_flag] ? 0.f : decay[h];
    const bool cleared = fresh != nullptr && fresh[b / seqs_per_flag];
    const T* qp = q + b * qs + h * qh;
    const T* kp = k + b * ks + (int64_t)(h / group) * kh;
    const T* vp = v + b * vs + (int64_t)(h / group) * vh + c * V;
    float vv[V];
#pragma unroll
    for (int u = 0; u < V; ++u) vv[u] = load_act(vp, u);
    const int64_t base = (int64_t)pair * Dk * Dv + c * V;
#pragma unroll 4
    for (int r = r0; r < Dk; r += R) {
      const int64_t at = base + (int64_t)r * Dv;
      float s[V];
      if constexpr (V == 4) {
        const float4 f = *reinterpret_cast<const float4*>(state + at);
        s[0] = f.x; s[1] = f.y; s[2] = f.z; s[3] = f.w;
      } else {
#pragma unroll
        for (int u = 0; u < V; ++u) s[u] = state[at + u];
      }
      const float kr = load_act(kp, r), qr = load_act(qp, r);
#pragma unroll
      for (int u = 0; u < V; ++u) {
        s[u] = (cleared ? 0.f : keep * s[u]) + kr * vv[u];
        o[u] += qr * s[u];
      }
      if constexpr (V == 4) {
        *reinterpret_cast<float4*>(next + at) = make_float4(s[0], s[1], s[2], s[3]);
      } else {
#pragma unroll
        for (int u = 0; u < V; ++u) next[at + u] = s[u];
      }
    }
#pragma unroll
    for (int u = 0; u < V; ++u) sum[team][(r0 * Q + c) * V + u] = o[u];
  }
  __syncthreads();
  if (on) {
    T* op = out + b * os + h * oh;
    for (int col = lane; col < Dv; col += TEAM) {
      float s = 0.f;
      for (int r = 0; r < R; ++r) s += sum[team][(r * Q + col / V) * V + col % V];
      s *= scale;
      if constexpr (sizeof(T) == 4) op[col] = s;
      else op[col] = to_bf16(s);
    }
  }
}

// ---- checks ----------------------------------------------------------------------------------------------------------------------
int32_t check_dims(const marl_attention_dims* d) {
  if (d == nullptr) return MARL_E_NULL;
  if (d->precision != 0 && d->precision != 1) return MARL_E_CONFIG;
  if (d->n_steps < 0 || d->n_steps > (1 << 30) || d->n_seqs < 0) return MARL_E_SIZE;
  if (d->n_heads < 1 || d->n_kv_heads < 1 || d->n_heads % d->n_kv_heads != 0) return MARL_E_CONFIG;
  if (d->dim_k < 1 || d->dim_k > kMaxDim || d->dim_v < 1 || d->dim_v > kMaxDim) return MARL_E_CONFIG;
  if (d->seqs_per_flag < 1 || d->n_seqs % d->seqs_per_flag != 0) return MARL_E_CONFIG;
  const int64_t pairs = (int64_t)d->n_seqs * d->n_heads;
  if (pairs > ((int64_t)1 << 26) || pairs * d->n_steps > ((int64_t)1 << 48)) return MARL_E_SIZE;  // (workspaces of 64-bit sizes)
  return MARL_OK;
}
// Every launch of a call within what a grid can be, before the first of them.  (The gradient's scans have two work-items or more for each element of a step
// of dk or dv, two heads sharing one at least, so that sum_heads_kernel's 32-bit places fit too.)
int32_t check_launches(const marl_attention_dims& d, const Plan& p, bool backward) {
  auto scan = [&](int roles, int dz) {
    const int slices = scan_slices(dz), group = slices == 1 ? scan_pairs<1>() : slices == 2 ? scan_pairs<2>() : scan_pairs<4>();
    return launchable((p.pairs + group - 1) / group * p.n_stretches * roles, 64 * slices * group);
  };
  bool fits = true;
  if (d.n_steps == 0 || p.n_stretches > 1) fits = launchable((p.pairs * d.dim_k * d.dim_v + 255) / 256, 256);  // join
  if (d.n_steps > 0) {
    if (p.n_stretches > 1) fits = fits && scan(backward ? 2 : 1, d.dim_v);
    if (!backward) fits = fits && scan(1, d.dim_v);
    else if (d.dim_k == d.dim_v) fits = fits && scan(3, d.dim_k);
    else fits = fits && scan(2, d.dim_k) && scan(1, d.dim_v);
  }
  return fits ? MARL_OK : MARL_E_SIZE;
}
int32_t check_view(const marl_view& v, int precision, bool used) {
  if (!used) return MARL_OK;
  if (v.data == nullptr) return MARL_E_NULL;
  return (reinterpret_cast<uintptr_t>(v.data) & (precision == 0 ? 3u : 1u)) != 0 ? MARL_E_ALIGN : MARL_OK;
}
// An output's elements are places of their own: no stride of zero along a dimension that there is
int32_t check_output(const marl_view& v, const marl_attention_dims& d, int heads, bool used) {
  if (!used) return MARL_OK;
  const bool overlaps = (v.step == 0 && d.n_steps > 1) || (v.seq == 0 && d.n_seqs > 1) || (v.head == 0 && heads > 1);
  return overlaps ? MARL_E_CONFIG : MARL_OK;
}
// An output that begins where one of the others does
int32_t check_places(const marl_view& out, std::initializer_list<marl_view> others, bool used) {
  if (used)
    for (const marl_view& x : others)
      if (x.data == out.data) return MARL_E_CONFIG;
  return MARL_OK;
}
// Two arrays of states share memory
bool overlapping(const marl_attention_dims& d, const float* a, const float* b) {
  if (a == nullptr || b == nullptr) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return (x < y ? y - x : x - y) < (uintptr_t)d.n_seqs * d.n_heads * d.dim_k * d.dim_v * 4;
}
#define MARL_CHECK(x)                                        \
  do {                                                       \
    const int32_t rc_ = (x);                                 \
    if (rc_ != MARL_OK) return rc_;                          \
  } while (0)

ScanArray array_of(const marl_view& v, int elem, int dim, int share) {
  ScanArray a;
  a.data = static_cast<const char*>(v.data);
  a.step = v.step * elem;
  a.seq = v.seq * elem;
  a.head = v.head * elem;
  a.share = (uint32_t)share;
  a.dim = dim;
  return a;
}
ScanState state_of(const float* p, uint32_t stretches, int row, int col) { return {const_cast<float*>(p), (int32_t)stretches, row, col}; }

// Launch over roles of one shape: widths dx (x, y) and dz (z, out)
int32_t scan(ScanArgs a, const marl_attention_dims& d, const Plan& p, int dx, int dz, bool state_only, hipStream_t s) {
  a.T = d.n_steps;
  a.B = d.n_seqs;
  a.H = (uint32_t)d.n_heads;
  a.seqs_per_flag = (uint32_t)d.seqs_per_flag;
  a.n_stretches = p.n_stretches;
  a.stretch = p.stretch;
  a.pairs = (uint32_t)p.pairs;
  (d.precision == 0 ? launch_scan_f32 : launch_scan_bf16)(a, dx, dz, state_only, s);
  return launch_status();
}

int32_t join(JoinArgs a0, JoinArgs a1, int n_args, const marl_attention_dims& d, const Plan& p, hipStream_t s) {
  const int64_t total = p.pairs * d.dim_k * d.dim_v, blocks = (total + 255) / 256;
  hipLaunchKernelGGL(join_kernel, dim3((unsigned)blocks, n_args), dim3(256), 0, s, a0, a1, (uint32_t)(d.dim_k * d.dim_v), total);
  return launch_status();
}

int32_t sum_heads(const marl_attention_dims& d, const Plan& p, const float* part, const marl_view& out, int dim, hipStream_t s) {
  const int64_t per_step = (int64_t)d.n_seqs * d.n_kv_heads * dim;
  auto launch = [&](auto zero, auto v) {
    typedef decltype(zero) T;
    constexpr int V = decltype(v)::value;
    const int64_t want = (per_step / V + 255) / 256;
    for (int32_t t = 0; t < d.n_steps; t += 65535) {  // (grid y)
      const int32_t n = d.n_steps - t < 65535 ? d.n_steps - t : 65535;
      hipLaunchKernelGGL((sum_heads_kernel<T, V>), dim3((unsigned)(want < 4096 ? want : 4096), (unsigned)n), dim3(256), 0, s,
                         part + (int64_t)t * p.pairs * dim, (T*)out.data + t * out.step, out.step, out.seq, out.head, (uint32_t)d.n_seqs,
                         (uint32_t)d.n_kv_heads, (uint32_t)p.group, (uint32_t)dim);
    }
  };
  if (dim % 4 == 0) d.precision == 0 ? launch(0.f, std::integral_constant<int, 4>()) : launch((bf16_t)0, std::integral_constant<int, 4>());
  else d.precision == 0 ? launch(0.f, std::integral_constant<int, 1>()) : launch((bf16_t)0, std::integral_constant<int, 1>());
  return launch_status();
}

// Threads that take a state: a wavefront, or a workgroup from more than 32 x 32 on, with its loads on their way together (16 384 states of 32 x 32: 99 against
// 120 us; of 32 x 64 199 against 186, 8192 of 64 x 64 210 against 192; columns one by one: the same to 2 %, and a thread for each of them).
int step_team(const marl_attention_dims& d) { return d.dim_k * d.dim_v <= 1024 && (d.dim_v % 4 == 0 || d.dim_v <= 64) ? 64 : 256; }
int64_t step_blocks(const marl_attention_dims& d) {
  const int64_t pairs = (int64_t)d.n_seqs * d.n_heads, teams = 256 / step_team(d);
  return (pairs + teams - 1) / teams;
}

template <class T>
int32_t step(const marl_attention_dims& d, const marl_view& q, const marl_view& k, const marl_view& v, const float* decay, const float* state,
             const uint8_t* fresh, const marl_view& out, float* next, hipStream_t s) {
  const uint32_t pairs = (uint32_t)d.n_seqs * (uint32_t)d.n_heads;
#define MARL_STEP(V, TEAM)                                                                                                              \
  hipLaunchKernelGGL((step_kernel<T, V, TEAM>), dim3((unsigned)step_blocks(d)), dim3(256), 0, s, (const T*)q.data, (const T*)k.data,    \
                     (const T*)v.data, (T*)out.data, q.seq, q.head, k.seq, k.head, v.seq, v.head, out.seq, out.head, decay, state, fresh, \
                     next, pairs, (uint32_t)d.n_heads, (uint32_t)(d.n_heads / d.n_kv_heads), (uint32_t)d.seqs_per_flag, d.dim_k,        \
                     d.dim_v, d.scale)
  if (d.dim_v % 4 == 0) {
    if (step_team(d) == 64) MARL_STEP(4, 64);
    else MARL_STEP(4, 256);
  } else if (step_team(d) == 64) {
    MARL_STEP(1, 64);
  } else {
    MARL_STEP(1, 256);
  }
#undef MARL_STEP
  return launch_status();
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int32_t marl_linear_attention_workspace(const marl_attention_dims* dims, int32_t backward, int64_t* bytes) {
  MARL_CHECK(check_dims(dims));
  if (bytes == nullptr) return MARL_E_NULL;
  const Plan p = plan_of(*dims, backward != 0);
  MARL_CHECK(check_launches(*dims, p, backward != 0));
  *bytes = p.bytes;
  return MARL_OK;
}

int32_t marl_linear_attention(const marl_attention_dims* dims, marl_view q, marl_view k, marl_view v, const float* decay,
                              const float* state, const uint8_t* done, marl_view out, float* next_state, void* workspace,
                              void* stream) {
  MARL_CHECK(check_dims(dims));
  const marl_attention_dims& d = *dims;
  const Plan p = plan_of(d, false);
  MARL_CHECK(check_launches(d, p, false));
  const bool used = d.n_steps > 0 && d.n_seqs > 0;
  for (const marl_view& x : {q, k, v, out}) MARL_CHECK(check_view(x, d.precision, used));
  MARL_CHECK(check_output(out, d, d.n_heads, used));
  MARL_OPTIONAL_PTR(state); MARL_OPTIONAL_PTR(next_state);
  if (next_state != state && overlapping(d, next_state, state)) return MARL_E_CONFIG;
  if (p.bytes > 0 && used) MARL_REQUIRE_PTR(workspace);
  if (decay == nullptr) return MARL_E_NULL;
  if ((reinterpret_cast<uintptr_t>(decay) & 3u) != 0) return MARL_E_ALIGN;
  MARL_CHECK(check_places(out, {q, k, v}, used));
  if (d.n_seqs == 0) return MARL_OK;
  hipStream_t s = (hipStream_t)stream;
  if (d.n_steps == 0) return next_state == nullptr ? MARL_OK : join({nullptr, nullptr, state, next_state, 0, 0}, {}, 1, d, p, s);
  char* ws = static_cast<char*>(workspace);
  float *states = reinterpret_cast<float*>(ws + p.states), *carry = reinterpret_cast<float*>(ws + p.carry);
  const int elem = d.precision == 0 ? 4 : 2;
  ScanArgs a{};
  a.decay = decay;
  a.done = done;
  a.n_roles = 1;
  ScanRole& r = a.role[0];
  r.x = array_of(q, elem, d.dim_k, 1);
  r.y = array_of(k, elem, d.dim_k, p.group);
  r.z = array_of(v, elem, d.dim_v, p.group);
  r.out = array_of(out, elem, d.dim_v, 1);
  r.inner = r.inter = d.scale;
  r.update = 1.f;
  if (p.n_stretches > 1) {
    a.carry = carry;
    r.to = state_of(states, p.n_stretches, d.dim_v, 1);
    MARL_CHECK(scan(a, d, p, d.dim_k, d.dim_v, true, s));
    MARL_CHECK(join({states, carry, state, next_state, (int32_t)p.n_stretches, 0}, {}, 1, d, p, s));
    r.to.data = nullptr;
    r.from = state_of(states, p.n_stretches, d.dim_v, 1);
  } else {
    r.from = state_of(state, 1, d.dim_v, 1);
    r.to = state_of(next_state, 1, d.dim_v, 1);
  }
  return scan(a, d, p, d.dim_k, d.dim_v, false, s);
}

int32_t marl_linear_attention_backward(const marl_attention_dims* dims, marl_view q, marl_view k, marl_view v,
                                       const float* decay, const float* state, const uint8_t* done, marl_view dout,
                                       const float* dnext_state, marl_view dq, marl_view dk, marl_view dv, float* dstate,
                                       void* workspace, void* stream) {
  MARL_CHECK(check_dims(dims));
  const marl_attention_dims& d = *dims;
  const Plan p = plan_of(d, true);
  MARL_CHECK(check_launches(d, p, true));
  const bool used = d.n_steps > 0 && d.n_seqs > 0;
  for (const marl_view& x : {q, k, v, dout, dq, dk, dv}) MARL_CHECK(check_view(x, d.precision, used));
  MARL_CHECK(check_output(dq, d, d.n_heads, used));
  MARL_CHECK(check_output(dk, d, d.n_kv_heads, used));
  MARL_CHECK(check_output(dv, d, d.n_kv_heads, used));
  MARL_OPTIONAL_PTR(state); MARL_OPTIONAL_PTR(dnext_state); MARL_OPTIONAL_PTR(dstate);
  if (overlapping(d, dstate, state) || overlapping(d, dstate, dnext_state)) return MARL_E_CONFIG;
  if (p.bytes > 0 && used) MARL_REQUIRE_PTR(workspace);
  if (decay == nullptr) return MARL_E_NULL;
  if ((reinterpret_cast<uintptr_t>(decay) & 3u) != 0) return MARL_E_ALIGN;
  MARL_CHECK(check_places(dq, {q, k, v, dout, dk, dv}, used));
  MARL_CHECK(check_places(dk, {q, k, v, dout, dv}, used));
  MARL_CHECK(check_places(dv, {q, k, v, dout}, used));
  if (d.n_seqs == 0) return MARL_OK;
  hipStream_t s = (hipStream_t)stream;
  if (d.n_steps == 0) return dstate == nullptr ? MARL_OK : join({nullptr, nullptr, dnext_state, dstate, 0, 1}, {}, 1, d, p, s);
  char* ws = static_cast<char*>(workspace);
  float *states = reinterpret_cast<float*>(ws + p.states), *carry = reinterpret_cast<float*>(ws + p.carry),
        *reverse_states = reinterpret_cast<float*>(ws + p.reverse_states);
  const int elem = d.precision == 0 ? 4 : 2;
  const ScanArray qa = array_of(q, elem, d.dim_k, 1), ka = array_of(k, elem, d.dim_k, p.group), va = array_of(v, elem, d.dim_v, p.group),
                  da = array_of(dout, elem, d.dim_v, 1);
  ScanArgs a{};
  a.decay = decay;
  a.done = done;
  const bool joined = p.n_stretches > 1;
  if (joined) {
    a.n_roles = 2;
    a.carry = carry;
    a.role[0].y = ka;
    a.role[0].z = va;
    a.role[0].update = 1.f;
    a.role[0].to = state_of(states, p.n_stretches, d.dim_v, 1);
    a.role[1].y = qa;
    a.role[1].z = da;
    a.role[1].update = d.scale;
    a.role[1].reverse = 1;
    a.role[1].to = state_of(reverse_states, p.n_stretches, d.dim_v, 1);
    MARL_CHECK(scan(a, d, p, d.dim_k, d.dim_v, true, s));
    MARL_CHECK(join({states, carry, state, nullptr, (int32_t)p.n_stretches, 0}, {reverse_states, carry, dnext_state, dstate, (int32_t)p.n_stretches, 1},
                    2, d, p, s));
  }
  auto share_out = [&](const marl_view& g, int64_t offset, int dim) {  // of a shared head: in fp32 per query head first
    if (p.group == 1) return array_of(g, elem, dim, 1);
    return array_of({ws + offset, p.pairs * dim, (int64_t)d.n_heads * dim, dim}, 4, dim, 1);
  };
  const float *s0 = joined ? states : state, *r0 = joined ? reverse_states : dnext_state;
  ScanRole rq{}, rk{}, rv{};
  rq.x = da; rq.y = va; rq.z = ka;
  rq.out = array_of(dq, elem, d.dim_k, 1);
  rq.inner = rq.inter = d.scale;
  rq.update = 1.f;
  rq.from = state_of(s0, p.n_stretches, 1, d.dim_v);
  rk.x = va; rk.y = da; rk.z = qa;
  rk.out = share_out(dk, p.dk, d.dim_k);
  rk.out_f32 = p.group > 1;
  rk.reverse = 1;
  rk.inner = rk.update = d.scale;
  rk.inter = 1.f;
  rk.from = state_of(r0, p.n_stretches, 1, d.dim_v);
  rv.x = ka; rv.y = qa; rv.z = da;
  rv.out = share_out(dv, p.dv, d.dim_v);
  rv.out_f32 = p.group > 1;
  rv.reverse = 1;
  rv.inner = rv.update = d.scale;
  rv.inter = 1.f;
  rv.from = state_of(r0, p.n_stretches, d.dim_v, 1);
  if (!joined) rv.to = state_of(dstate, 1, d.dim_v, 1);
  a.carry = nullptr;
  const bool one = d.dim_k == d.dim_v;  // one launch for all three
  a.n_roles = one ? 3 : 2;
  a.role[0] = rq;
  a.role[1] = rk;
  a.role[2] = rv;
  MARL_CHECK(scan(a, d, p, d.dim_v, d.dim_k, false, s));
  if (!one) {
    a.n_roles = 1;
    a.role[0] = rv;
    MARL_CHECK(scan(a, d, p, d.dim_k, d.dim_v, false, s));
  }
  if (p.group > 1) {
    MARL_CHECK(sum_heads(d, p, reinterpret_cast<const float*>(ws + p.dk), dk, d.dim_k, s));
    MARL_CHECK(sum_heads(d, p, reinterpret_cast<const float*>(ws + p.dv), dv, d.dim_v, s));
  }
  return MARL_OK;
}

int32_t marl_linear_attention_step(const marl_attention_dims* dims, marl_view q, marl_view k, marl_view v,
                                   const float* decay, const float* state, const uint8_t* fresh, marl_view out,
                                   float* next_state, void* stream) {
  MARL_CHECK(check_dims(dims));
  const marl_attention_dims& d = *dims;
  if (d.n_steps != 1 || !launchable(step_blocks(d), 256)) return MARL_E_SIZE;
  if (d.n_seqs == 0) return MARL_OK;
  for (const marl_view& x : {q, k, v, out}) MARL_CHECK(check_view(x, d.precision, true));
  MARL_CHECK(check_output(out, d, d.n_heads, true));
  if (decay == nullptr) return MARL_E_NULL;
  if ((reinterpret_cast<uintptr_t>(decay) & 3u) != 0) return MARL_E_ALIGN;
  MARL_REQUIRE_PTR(state); MARL_REQUIRE_PTR(next_state);
  if (next_state != state && overlapping(d, next_state, state)) return MARL_E_CONFIG;
  MARL_CHECK(check_places(out, {q, k, v}, true));
  return (d.precision == 0 ? step<float> : step<bf16_t>)(d, q, k, v, decay, state, fresh, out, next_state, (hipStream_t)stream);
}

}  // extern "C"
