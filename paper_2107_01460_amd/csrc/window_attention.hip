// Window attention: the calls, the cache behind a call, the single step on a cache.
#include <type_traits>

#include "attention_checks.h"
#include "lane_sums.h"
#include "window_attention.h"

namespace marl {
namespace {

// ---- how a call is laid out ----------------------------------------------------------------------------------------------------
struct Plan {
  int tiles;                  // of 32 steps
  int heads_each, rows_waves; // query heads of a workgroup; wavefronts of one that takes rows
  int64_t rows_t;             // workgroups along time
  int64_t rows, cols, far;    // workgroups
  int far_tiles;
  uint32_t far_chunks, far_slots;
  int64_t delta, places, reach, numbers, parts, bytes;
};
int padded(const marl_attention_dims& d) { return ((d.dim_k > d.dim_v ? d.dim_k : d.dim_v) + 31) / 32 * 32; }
// A workgroup's wavefronts share the streamed tiles: query heads of one key head first, then tiles next to each other in time.
Plan plan_of(const marl_attention_dims& d, int window, int sinks, bool fast, bool gradient) {
  Plan p{};
  p.tiles = (int)(((int64_t)d.n_steps + kTile - 1) / kTile);
  const int group = d.n_heads / d.n_kv_heads, pairs = d.n_seqs * d.n_kv_heads;
  p.heads_each = group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1;
  // (Two tiles of one head where the window is short: four wait for each other more than they share.  128 x 4096 steps of 8 heads of 64 in bf16, window 64: 696 against
  // 747 us, gradient of 4 heads of 32 in fp32, window 32: 1409 against 1535; 1024 x 520 steps of 4 heads of 32 in fp32, window 1024: 1484 against 1413; 1024 x 64 steps of
  // 4 heads of 128 in bf16, window 150: 82 against 88, window 511: 118 against 112, and its gradient, whose two wavefronts would spill: 481 against 395.)
  const int most = p.heads_each == 1 && window < (padded(d) <= 64 ? 512 : gradient ? 0 : 256) ? 2 : 4;
  int along = p.tiles < 2 ? 1 : p.tiles == 2 ? 2 : 4;
  if (along > most) along = most;
  const int least = fast ? least_waves(d.precision == 0 ? 4 : 2, padded(d)) : 4;
  if (along < least) along = least;
  p.rows_waves = p.heads_each * along < 4 ? p.heads_each * along : 4;
  const int each = p.rows_waves / p.heads_each;
  p.rows_t = (p.tiles + each - 1) / each;
  p.rows = (int64_t)d.n_seqs * (d.n_heads / p.heads_each) * p.rows_t;
  auto workgroups = [&](int64_t units) { return (units * p.heads_each + 3) / 4; };
  p.cols = workgroups((int64_t)pairs * p.tiles);
  // First steps seen from afar are cut along the rows where column tiles are few (else others keep the chip busy meanwhile) and some ten tiles or more lie beyond the window
  // (fewer do not pay for a launch).  The whole gradient, without and with the cut, window 64 and 4 first steps in one episode.  1024 steps of 4 heads, 4096, 8192 and 16 384
  // column tiles: of 64 in bf16 140 and 96, 148 and 151, 259 and 297 us; of 128 in bf16 221 and 189, 286 and 342, 544 and 652; of 32 in fp32 259 and 149, 241 and 236, 410 and
  // 437.  Four sequences, 6, 8, 10 and 18 tiles beyond the window: of 64 in bf16 36 and 41, 41 and 42, 46 and 42, 67 and 44; of 32 in fp32 52 and 56, 60 and 56, 68 and 57, 99 and
  // 58.  Sequences of 8192 steps would gain on the far side of the line too (16 of them, 16 384 column tiles of heads of 64 in bf16: 824 and 350).
  if (sinks > 0 && (int64_t)pairs * p.tiles <= 8192 && p.tiles > window / kTile + 10) {
    p.far_tiles = p.tiles > 256 ? (p.tiles + 63) / 64 : 4;
    p.far_chunks = (uint32_t)((p.tiles + p.far_tiles - 1) / p.far_tiles);
    p.far_slots = (uint32_t)(sinks / kTile + 3 < 8 ? sinks / kTile + 3 : 8);
    p.far = workgroups((int64_t)pairs * p.far_chunks * p.far_slots);
  }
  auto take = [&](int64_t bytes) {
    const int64_t here = p.bytes;
    p.bytes += (bytes + 255) / 256 * 256;
    return here;
  };
  const int64_t slots = (int64_t)pairs * p.far_chunks * p.far_slots;
  p.delta = take((int64_t)d.n_seqs * d.n_heads * d.n_steps * 4);
  p.places = take((int64_t)(d.n_seqs / d.seqs_per_flag) * d.n_steps * 4);
  p.reach = take((int64_t)(d.n_seqs / d.seqs_per_flag) * p.tiles * 8);
  p.numbers = take(slots * 4);
  p.parts = take(slots * 2 * kTile * padded(d) * 4);
  return p;
}

// Rows that Fetch takes with unconditional loads: whole 16-byte pieces, four-byte aligned, 32 of them within 2 GB, so less than 64 MB from one step to the next.  One array
// whose rows are not like that takes the whole call to loads with branches, whose tiles wait for each other: 128 steps of 32 768 sequences of 8 heads of 64 in bf16, window 64,
// 4.7 ms with steps 34 MB apart, 6.3 where the values' are 101 MB apart (a view of a product of queries, keys and values), the gradient 14.1 and 23.3; of 4096 sequences heads of 50
// take 0.85 ms and 3.4, of 48 0.44 and 1.40, of 56 0.48 and 1.50; of 36 0.82 and 3.3, of 40 0.41 and 1.31; fp32 heads of 30 (4 of them, window 32) 0.53 and 1.76, of 32 0.33 and 1.04.
bool fast_rows(const marl_attention_dims& d, const marl_view& v, int dim) {
  const int elem = d.precision == 0 ? 4 : 2;
  const int64_t step = v.step * elem;
  return dim * elem % 16 == 0 && (reinterpret_cast<uintptr_t>(v.data) & 3u) == 0 && step % 4 == 0 && v.seq * elem % 4 == 0 && v.head * elem % 4 == 0 &&
         step >= 0 && step < (1 << 26) - 16;
}

// ---- the cache behind a call ---------------------------------------------------------------------------------------------------------
// A row of the next cache comes from the call's steps or, where its step is older, from the cache before; a step's slot is the same in both.  Bound by memory: 4096
// sequences of 8 heads of 64 in bf16, 68 slots: 177 us for the 0.83 GB in and out.
struct CacheArgs {
  WindowArray in[2];  // k, v
  const char* old[2];
  char* next[2];
  const int32_t* positions;
  int32_t first;
  uint32_t n_flags, seqs_per_flag, Hk;
  int32_t T, dim[2], window, sinks;
  uint32_t chunks;  // of kCacheRows slots
  int32_t in_place;
};
constexpr int kCacheRows = 128;  // slots of a workgroup (of 64, a second workgroup for the few behind them begins anew: 278 us; of 32: 220)

template <class T>
__device__ __forceinline__ void put_unit(T* p, const uint4& u, int left) {  // `left` elements, at most 16 bytes
  constexpr int E = 16 / sizeof(T);
  if (left >= E) {
    __builtin_memcpy(p, &u, 16);
  } else {
    T e[E];
    __builtin_memcpy(e, &u, 16);
#pragma unroll
    for (int x = 0; x < E; ++x)
      if (x < left) p[x] = e[x];
  }
}

template <class T>
__global__ void __launch_bounds__(256) window_cache_kernel(const CacheArgs a) {
  constexpr int E = 16 / sizeof(T);
  uint32_t at = xcd_order(blockIdx.x, gridDim.x, a.Hk * a.chunks, a.n_flags * a.seqs_per_flag);
  const uint32_t chunk = at % a.chunks;
  at /= a.chunks;
  const uint32_t hk = at % a.Hk, b = at / a.Hk, env = b / a.seqs_per_flag;
  // the last row that holds a step
  int last = -1, newest = -1;
  for (int t0 = a.T - 1; t0 >= 0 && last < 0; t0 -= 64) {
    const int t = t0 - (int)(threadIdx.x & 63);
    const int p = t < 0 ? -1 : a.positions != nullptr ? a.positions[(int64_t)t * a.n_flags + env] : a.first + t;
    const uint64_t on = __ballot(p >= 0);
    if (on != 0) {
      const int lane = __builtin_ctzll(on);
      last = t0 - lane;
      newest = __shfl(p, lane);
    }
  }
  const int slots = a.sinks + a.window;
  const int newest_slot = newest < a.sinks ? newest : a.sinks + (newest - a.sinks) % a.window;
  const int units[2] = {(a.dim[0] + E - 1) / E, (a.dim[1] + E - 1) / E}, per = units[0] + units[1];
  const int64_t base = ((int64_t)b * a.Hk + hk) * slots;
  const int slot0 = (int)chunk * kCacheRows, n = min(kCacheRows, slots - slot0) * per;
  const char *in_k = a.in[0].data + b * a.in[0].seq + hk * a.in[0].head, *in_v = a.in[1].data + b * a.in[1].seq + hk * a.in[1].head;
  constexpr int kBatch = 4;  // loads on their way together
  for (int u0 = threadIdx.x; u0 < n; u0 += 256 * kBatch) {
    uint4 v[kBatch];
    char* to[kBatch];
    int left[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int u = u0 + 256 * k;
      to[k] = nullptr;
      if (u >= n) continue;
      const int slot = slot0 + u / per, x = u % per, c = (x >= units[0] ? x - units[0] : x) * E;
      const bool values = x >= units[0];
      int64_t t = -1;
      if (last >= 0) {
        if (slot > newest && newest < slots) continue;  // holds no step
        const int step = newest < slots || slot < a.sinks ? slot : newest - newest_slot + slot - (slot <= newest_slot ? 0 : a.window);
        t = (int64_t)last - ((int64_t)newest - step);
      }
      const int dim = values ? a.dim[1] : a.dim[0];
      const char* old = values ? a.old[1] : a.old[0];
      const int64_t place = (base + slot) * dim;
      if (t < 0 && (old == nullptr || a.in_place)) continue;
      v[k] = load_unit<T>(t >= 0 ? (values ? in_v + t * a.in[1].step : in_k + t * a.in[0].step) : old + place * (int)sizeof(T), c, dim);
      to[k] = (values ? a.next[1] : a.next[0]) + (place + c) * (int)sizeof(T);
      left[k] = dim - c;
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (to[k] != nullptr) put_unit(reinterpret_cast<T*>(to[k]), v[k], left[k]);
  }
}

// ---- one step ------------------------------------------------------------------------------------------------------------------------
// A wavefront takes up to G query heads of one key head of one sequence, over a part of the cache's slots: L lanes hold a row of keys and the
// same row of values, 64 / L rows at a time, and a softmax of their own, joined at the end.  All slots that hold a step are seen, so nothing is masked.  Bound by
// memory: the cache is read once for up to four heads that share it.  4096 sequences of 8 heads of 64 in bf16, 68 slots: 86 us, 4.6 TB/s; with 8 query heads on 2 of 128 and
// 16 388 slots of four sequences, cut into parts, 23 us and 3 TB/s, and 5 us for joining them (one batch of rows at a time, none ahead: 49 us in all).
struct StepArgs {
  const char *q, *k, *v;
  char* out;
  int64_t q_seq, q_head, k_seq, k_head, v_seq, v_head, out_seq, out_head;  // bytes
  char *cache_k, *cache_v;
  const int32_t* positions;
  uint32_t seqs_per_flag, H, Hk, group, chunks, splits;
  int64_t units;  // wavefronts
  int32_t dk, dv, window, sinks;
  float c;  // scale log2(e)
  uint32_t parts;  // splits / 4: a workgroup's wavefronts take four next to each other and join them
  float* part;     // [B][H][parts][dv]
  float2* stat;    // [B][H][parts]: largest exponent of two, sum
};

template <class T>
__device__ __forceinline__ void widen(const uint4& u, float (&f)[16 / sizeof(T)]) {
  if constexpr (sizeof(T) == 4) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
  } else {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
template <class T>
__device__ __forceinline__ uint4 narrow(const float (&f)[16 / sizeof(T)]) {
  if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  else return make_uint4(pack2_bf16(f[0], f[1]), pack2_bf16(f[2], f[3]), pack2_bf16(f[4], f[5]), pack2_bf16(f[6], f[7]));
}

constexpr int kStepRows = 4;  // rows of a lane on their way together

template <class T, int L, int G>
__global__ void __launch_bounds__(256) window_step_kernel(const StepArgs a) {
  constexpr int E = 16 / sizeof(T), R = 64 / L;
  __shared__ float2 stats[4][G];
  __shared__ float accs[4][G][L * E];
  const int64_t unit = (int64_t)xcd_remap(blockIdx.x, gridDim.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (unit >= a.units) return;
  const int lane = threadIdx.x & 63, r = lane / L, c = lane % L * E;
  const uint32_t split = (uint32_t)(unit % a.splits);
  const int64_t rest = unit / a.splits;
  const uint32_t chunk = (uint32_t)(rest % a.chunks);
  const int64_t pair = rest / a.chunks;  // sequence and key head
  const uint32_t b = (uint32_t)(pair / a.Hk), hk = (uint32_t)(pair % a.Hk);
  const uint32_t h0 = hk * a.group + chunk * G, heads = min((uint32_t)G, a.group - chunk * G);
  const int position = a.positions[b / a.seqs_per_flag];
  const int slots = a.sinks + a.window;
  float q[G][E], acc[G][E], top[G], sum[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const uint4 u = load_unit<T>(a.q + b * a.q_seq + (h0 + min((uint32_t)g, heads - 1)) * a.q_head, c, a.dk);
    widen<T>(u, q[g]);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[g][e] *= a.c;
      acc[g][e] = 0.f;
    }
    top[g] = -__builtin_inff();
    sum[g] = 0.f;
  }
  if (position >= 0) {
    const int n = min(position, slots - 1) + 1, per = ((n - 1) / (int)a.splits / R + 1) * R;  // (a multiple of R that is no less than n / splits)
    const int64_t begin = (int64_t)split * per;
    const int end = (int)min((int64_t)n, begin + per);
    const int here = position < a.sinks ? position : a.sinks + (position - a.sinks) % a.window;  // this step's slot
    char *ck = a.cache_k + pair * slots * a.dk * (int64_t)sizeof(T), *cv = a.cache_v + pair * slots * a.dv * (int64_t)sizeof(T);
    const char *kp = a.k + b * a.k_seq + hk * a.k_head, *vp = a.v + b * a.v_seq + hk * a.v_head;
    const bool whole_k = a.dk % E == 0, whole_v = a.dv % E == 0;  // no 16 bytes end inside
    uint4 next_k[kStepRows], next_v[kStepRows];
    auto request = [&](int64_t base) __attribute__((always_inline)) {  // a batch of rows, one batch ahead
#pragma unroll
      for (int u = 0; u < kStepRows; ++u) {
        const int64_t slot = base + u * R + r;
        next_k[u] = next_v[u] = make_uint4(0, 0, 0, 0);
        if (slot >= end) continue;
        const char *pk = slot == here ? kp : ck + slot * a.dk * (int)sizeof(T), *pv = slot == here ? vp : cv + slot * a.dv * (int)sizeof(T);
        if (whole_k && c < a.dk) __builtin_memcpy(&next_k[u], pk + c * (int)sizeof(T), 16);
        if (whole_v && c < a.dv) __builtin_memcpy(&next_v[u], pv + c * (int)sizeof(T), 16);
        if (!whole_k) next_k[u] = load_unit<T>(pk, c, a.dk);
        if (!whole_v) next_v[u] = load_unit<T>(pv, c, a.dv);
      }
    };
    if (begin < end) request(begin);
    for (int64_t base = begin; base < end; base += R * kStepRows) {
      uint4 k[kStepRows], v[kStepRows];
#pragma unroll
      for (int u = 0; u < kStepRows; ++u) {
        k[u] = next_k[u];
        v[u] = next_v[u];
      }
      if (base + R * kStepRows < end) request(base + R * kStepRows);
      float s[G][kStepRows];
#pragma unroll
      for (int u = 0; u < kStepRows; ++u) {
        const int64_t slot = base + u * R + r;
        if (slot == here && slot < end && chunk == 0) {
          if (c < a.dk) put_unit(reinterpret_cast<T*>(ck) + slot * a.dk + c, k[u], a.dk - c);
          if (c < a.dv) put_unit(reinterpret_cast<T*>(cv) + slot * a.dv + c, v[u], a.dv - c);
        }
        float f[E];
        widen<T>(k[u], f);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float x = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) x = __builtin_fmaf(q[g][e], f[e], x);
          x = sum_lanes<L>(x);
          s[g][u] = slot < end ? x : -__builtin_inff();
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float now = top[g];
#pragma unroll
        for (int u = 0; u < kStepRows; ++u) now = fmaxf(now, s[g][u]);
        const float from = now == -__builtin_inff() ? 0.f : now, shrink = __builtin_amdgcn_exp2f(top[g] - from);
        top[g] = now;
        sum[g] *= shrink;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[g][e] *= shrink;
#pragma unroll
        for (int u = 0; u < kStepRows; ++u) {
          s[g][u] = base + u * R + r < end ? __builtin_amdgcn_exp2f(s[g][u] - from) : 0.f;
          sum[g] += s[g][u];
        }
      }
#pragma unroll
      for (int u = 0; u < kStepRows; ++u) {
        float f[E];
        widen<T>(v[u], f);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int e = 0; e < E; ++e) acc[g][e] = __builtin_fmaf(s[g][u], f[e], acc[g][e]);
      }
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    float most = top[g];
#pragma unroll
    for (int m = L; m < 64; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
    const float factor = __builtin_amdgcn_exp2f(top[g] - (most == -__builtin_inff() ? 0.f : most));
    sum[g] *= factor;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[g][e] *= factor;
#pragma unroll
    for (int m = L; m < 64; m *= 2) {
      sum[g] += __shfl_xor(sum[g], m);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[g][e] += __shfl_xor(acc[g][e], m);
    }
    if (a.splits == 1) {
      if (r != 0 || (uint32_t)g >= heads || c >= a.dv) continue;
      float o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = position < 0 ? 0.f : acc[g][e] / sum[g];
      put_unit(reinterpret_cast<T*>(a.out + b * a.out_seq + (h0 + g) * a.out_head) + c, narrow<T>(o), a.dv - c);
    } else if (r == 0) {
      const int wave = threadIdx.x / 64;
      if (lane == 0) stats[wave][g] = make_float2(most, sum[g]);
#pragma unroll
      for (int e = 0; e < E; ++e) accs[wave][g][c + e] = acc[g][e];
    }
  }
  if (a.splits == 1) return;
  __syncthreads();
  for (int at = threadIdx.x; at < (int)heads * L * E; at += 256) {
    const int g = at / (L * E), d = at % (L * E);
    const float most = fmaxf(fmaxf(stats[0][g].x, stats[1][g].x), fmaxf(stats[2][g].x, stats[3][g].x)), from = most == -__builtin_inff() ? 0.f : most;
    float all = 0.f, o = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float factor = __builtin_amdgcn_exp2f(stats[u][g].x - from);
      all = __builtin_fmaf(factor, stats[u][g].y, all);
      o = __builtin_fmaf(factor, accs[u][g][d], o);
    }
    const int64_t place = ((int64_t)b * a.H + h0 + g) * a.parts + split / 4;
    if (d == 0) a.stat[place] = make_float2(most, all);
    if (d < a.dv) a.part[place * a.dv + d] = o;
  }
}

// The parts of a cut step, one workgroup a query head, in a fixed order: eight teams of 128 threads take every eighth part.
constexpr int kMaxParts = 128;
template <class T>
__global__ void __launch_bounds__(1024) window_step_join_kernel(const StepArgs a) {
  __shared__ float2 stats[kMaxParts];
  __shared__ float sums[8], accs[8][128];
  const int64_t pair = blockIdx.x;
  const uint32_t b = (uint32_t)(pair / a.H), h = (uint32_t)(pair % a.H);
  const int d = threadIdx.x % 128, team = threadIdx.x / 128;
  const int position = a.positions[b / a.seqs_per_flag];
  for (uint32_t s = threadIdx.x; s < a.parts; s += 1024) stats[s] = a.stat[pair * a.parts + s];
  __syncthreads();
  float top = -__builtin_inff();
  for (uint32_t s = threadIdx.x & 63; s < a.parts; s += 64) top = fmaxf(top, stats[s].x);
#pragma unroll
  for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
  const float from = top == -__builtin_inff() ? 0.f : top;
  float sum = 0.f, acc = 0.f;
  const float* part = a.part + pair * a.parts * a.dv + d;
  const bool on = d < a.dv;
#pragma unroll 8
  for (uint32_t s = team; s < a.parts; s += 8) {
    const float2 x = stats[s];
    const float factor = __builtin_amdgcn_exp2f(x.x - from);
    sum = __builtin_fmaf(factor, x.y, sum);
    if (on) acc = __builtin_fmaf(factor, part[(int64_t)s * a.dv], acc);
  }
  if (d == 0) sums[team] = sum;
  accs[team][d] = acc;
  __syncthreads();
  if (team != 0 || !on) return;
  sum = acc = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    sum += sums[u];
    acc += accs[u][d];
  }
  const float o = position < 0 ? 0.f : acc / sum;
  T* out = reinterpret_cast<T*>(a.out + b * a.out_seq + h * a.out_head) + d;
  if constexpr (sizeof(T) == 4) *out = o;
  else *out = to_bf16(o);
}

struct StepPlan {
  int lanes, heads;  // of a row; of a wavefront
  uint32_t chunks, splits;
  int64_t units, part, stat, bytes;
};
// The slots are cut into parts while the wavefronts would not fill the chip, each of them two rounds of loads at least.  (Four sequences, 8 heads on 2 of 128 in bf16,
// 16 388 slots, with the call: 2048 wavefronts 28.7 us, 4096 37.3, 1536 30.0, 1024 29.1; eight rows of a lane on their way in place of four 39.3, and 4096 sequences of
// 68 slots 120 for 89.)
StepPlan step_plan(const marl_attention_dims& d, int window, int sinks) {
  constexpr int64_t kWaves = 2048;
  StepPlan p{};
  const int elements = d.precision == 0 ? 4 : 8, dim = d.dim_k > d.dim_v ? d.dim_k : d.dim_v, group = d.n_heads / d.n_kv_heads;
  p.lanes = 4;
  while (p.lanes * elements < dim) p.lanes *= 2;
  p.heads = group == 1 ? 1 : group == 2 ? 2 : 4;
  p.chunks = (uint32_t)((group + p.heads - 1) / p.heads);
  const int64_t whole = (int64_t)d.n_seqs * d.n_kv_heads * p.chunks, slots = (int64_t)window + sinks, least = 64 / p.lanes * kStepRows * 2;
  int64_t n = whole > 0 ? kWaves / whole : 1;
  n = n < slots / least ? n : slots / least;
  n = n < 4 * kMaxParts ? n / 4 * 4 : 4 * kMaxParts;
  p.splits = (uint32_t)(n < 2 ? 1 : n);
  p.units = whole * p.splits;
  auto take = [&](int64_t bytes) {
    const int64_t here = p.bytes;
    p.bytes += (bytes + 255) / 256 * 256;
    return here;
  };
  if (p.splits > 1) {
    const int64_t parts = (int64_t)d.n_seqs * d.n_heads * (p.splits / 4);
    p.part = take(parts * d.dim_v * 4);
    p.stat = take(parts * 8);
  }
  return p;
}

template <class T>
int32_t launch_step(const StepArgs& a, const StepPlan& p, int64_t pairs, hipStream_t s) {
  const dim3 grid((unsigned)((p.units + 3) / 4)), block(256);
#define MARL_STEP(L, G) hipLaunchKernelGGL((window_step_kernel<T, L, G>), grid, block, 0, s, a)
#define MARL_STEP_HEADS(L)               \
  do {                                   \
    if (p.heads == 1) MARL_STEP(L, 1);   \
    else if (p.heads == 2) MARL_STEP(L, 2); \
    else MARL_STEP(L, 4);                \
  } while (0)
  if (p.lanes == 4) MARL_STEP_HEADS(4);
  else if (p.lanes == 8) MARL_STEP_HEADS(8);
  else if (p.lanes == 16) MARL_STEP_HEADS(16);
  else if constexpr (sizeof(T) == 4) MARL_STEP_HEADS(32);
#undef MARL_STEP_HEADS
#undef MARL_STEP
  if (p.splits > 1) hipLaunchKernelGGL((window_step_join_kernel<T>), dim3((unsigned)pairs), dim3(1024), 0, s, a);
  return launch_status();
}

// ---- checks ----------------------------------------------------------------------------------------------------------------------
int32_t check_window(const marl_attention_dims* d, int32_t window, int32_t sinks) {
  MARL_CHECK(check_dims(d));
  if (window < 1 || sinks < 0 || (int64_t)window + sinks > ((int64_t)1 << 30)) return MARL_E_CONFIG;
  if ((int64_t)d->n_seqs * d->n_kv_heads > ((int64_t)1 << 48) / (window + sinks)) return MARL_E_SIZE;  // (caches of 64-bit sizes)
  return MARL_OK;
}
int32_t check_positions(const marl_attention_dims& d, const int32_t* positions, int32_t first) {
  if ((reinterpret_cast<uintptr_t>(positions) & 3u) != 0) return MARL_E_ALIGN;
  if (positions == nullptr && (int64_t)first + d.n_steps > 0x7fffffff) return MARL_E_SIZE;
  return MARL_OK;
}
Extent cached(const marl_attention_dims& d, const void* p, int64_t slots, int dim) {
  return extent(p, (int64_t)d.n_seqs * d.n_kv_heads * slots * dim * (d.precision == 0 ? 4 : 2));
}
Extent statistics(const marl_attention_dims& d, const float* lse) { return extent(lse, (int64_t)d.n_seqs * d.n_heads * d.n_steps * 4); }
// Both arrays or neither, aligned
int32_t check_cache(const marl_window_cache& c, bool needed) {
  if ((c.keys == nullptr) != (c.values == nullptr) || (needed && c.keys == nullptr)) return MARL_E_NULL;
  return misaligned(c.keys) || misaligned(c.values) ? MARL_E_ALIGN : MARL_OK;
}
int32_t check_floats(const float* p, bool needed) {
  if (p == nullptr) return needed ? MARL_E_NULL : MARL_OK;
  return (reinterpret_cast<uintptr_t>(p) & 3u) != 0 ? MARL_E_ALIGN : MARL_OK;
}

WindowArray array_of(const marl_view& v, int elem) { return {static_cast<char*>(v.data), v.step * elem, v.seq * elem, v.head * elem}; }

WindowArgs args_of(const marl_attention_dims& d, int32_t window, int32_t sinks, const int32_t* positions, int32_t first, const marl_window_cache& cache) {
  WindowArgs a{};
  a.cache_k = static_cast<const char*>(cache.keys);
  a.cache_v = static_cast<const char*>(cache.values);
  a.positions = positions;
  a.first = first;
  a.n_flags = (uint32_t)(d.n_seqs / d.seqs_per_flag);
  a.seqs_per_flag = (uint32_t)d.seqs_per_flag;
  a.T = d.n_steps;
  a.B = (uint32_t)d.n_seqs;
  a.H = (uint32_t)d.n_heads;
  a.Hk = (uint32_t)d.n_kv_heads;
  a.group = a.H / a.Hk;
  a.dk_dim = d.dim_k;
  a.dv_dim = d.dim_v;
  a.window = window;
  a.sinks = sinks;
  a.scale = d.scale;
  a.c = d.scale == 0.f ? 1.f : __builtin_fabsf(d.scale) * 1.44269504088896341f;  // (above zero, so that minus infinity stays that; the scores are zero then)
  a.flip = d.scale < 0.f ? (d.precision == 0 ? 0x80000000u : 0x80008000u) : 0u;
  return a;
}
int32_t launch(WindowArgs& a, const marl_attention_dims& d, const Plan& p, int pass, hipStream_t s) {
  a.heads_each = (uint32_t)p.heads_each;
  a.blocks_t = (uint32_t)p.rows_t;
  const int64_t blocks = pass == WINDOW_DKV ? p.cols : pass == WINDOW_FAR ? p.far : p.rows;
  (d.precision == 0 ? launch_window_f32 : launch_window_bf16)(a, pass, p.rows_waves, (unsigned)blocks, s);
  return launch_status();
}
int64_t cache_blocks(const marl_attention_dims& d, int64_t slots) { return (int64_t)d.n_seqs * d.n_kv_heads * ((slots + kCacheRows - 1) / kCacheRows); }

enum { CALL_FORWARD, CALL_BACKWARD, CALL_STEP };
// Every launch of a call within what a grid can be, before the first of them
int32_t check_launches(const marl_attention_dims& d, int32_t window, int32_t sinks, int call, bool next_cache) {
  bool fits = true;
  if (call == CALL_STEP) {
    const StepPlan p = step_plan(d, window, sinks);
    fits = launchable((p.units + 3) / 4, 256) && (p.splits == 1 || launchable((int64_t)d.n_seqs * d.n_heads, 1024));
  } else {
    for (bool fast : {false, true}) {  // (whichever the arrays' strides lead to)
      const Plan p = plan_of(d, window, sinks, fast, call == CALL_BACKWARD);
      fits = fits && launchable(p.rows, 64 * p.rows_waves) && (call == CALL_FORWARD || (launchable(p.cols, 256) && launchable(p.far, 256)));
    }
    if (next_cache) fits = fits && launchable(cache_blocks(d, (int64_t)window + sinks), 256);
  }
  return fits ? MARL_OK : MARL_E_SIZE;
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int32_t marl_window_attention_workspace(const marl_attention_dims* dims, int32_t window, int32_t sinks, int32_t call, int64_t* bytes) {
  MARL_CHECK(check_window(dims, window, sinks));
  if (call < CALL_FORWARD || call > CALL_STEP) return MARL_E_CONFIG;
  if (bytes == nullptr) return MARL_E_NULL;
  MARL_CHECK(check_launches(*dims, window, sinks, call, false));
  *bytes = call == CALL_FORWARD ? 0 : call == CALL_BACKWARD ? plan_of(*dims, window, sinks, true, true).bytes : step_plan(*dims, window, sinks).bytes;
  return MARL_OK;
}

int32_t marl_window_attention(const marl_attention_dims* dims, int32_t window, int32_t sinks, marl_view q, marl_view k, marl_view v,
                              const int32_t* positions, int32_t first_position, marl_window_cache cache, marl_view out, float* lse,
                              marl_window_cache next_cache, void* workspace, void* stream) {
  (void)workspace;  // (of no bytes)
  MARL_CHECK(check_window(dims, window, sinks));
  const marl_attention_dims& d = *dims;
  MARL_CHECK(check_launches(d, window, sinks, CALL_FORWARD, next_cache.keys != nullptr));
  const bool used = d.n_steps > 0 && d.n_seqs > 0;
  for (const marl_view& x : {q, k, v, out}) MARL_CHECK(check_view(x, d.precision, used));
  MARL_CHECK(check_output(out, d, d.n_heads, used));
  MARL_CHECK(check_positions(d, positions, first_position));
  MARL_CHECK(check_floats(lse, false));
  MARL_CHECK(check_cache(cache, false));
  MARL_CHECK(check_cache(next_cache, false));
  MARL_CHECK(check_places(out, {q, k, v}, used));
  const int64_t slots = (int64_t)window + sinks;
  const Extent ck = cached(d, cache.keys, slots, d.dim_k), cv = cached(d, cache.values, slots, d.dim_v), nk = cached(d, next_cache.keys, slots, d.dim_k),
               nv = cached(d, next_cache.values, slots, d.dim_v);
  const bool in_place = next_cache.keys != nullptr && next_cache.keys == cache.keys && next_cache.values == cache.values;
  if (nk.meets(nv) || nk.meets(cv) || nv.meets(ck) || (!in_place && (nk.meets(ck) || nv.meets(cv)))) return MARL_E_CONFIG;
  if (used) {
    const Extent ps = places_of(d, positions), ls = statistics(d, lse);
    if (touches(out, d, d.n_heads, d.dim_v, {ck, cv, nk, nv, ps, ls}) || touches(q, d, d.n_heads, d.dim_k, {nk, nv, ls}) ||
        touches(k, d, d.n_kv_heads, d.dim_k, {nk, nv, ls}) || touches(v, d, d.n_kv_heads, d.dim_v, {nk, nv, ls}))
      return MARL_E_CONFIG;
    for (const Extent& x : {ck, cv, nk, nv, ps})
      if (ls.meets(x)) return MARL_E_CONFIG;
    if (ps.meets(nk) || ps.meets(nv)) return MARL_E_CONFIG;
  }
  if (d.n_seqs == 0) return MARL_OK;
  hipStream_t s = (hipStream_t)stream;
  const int elem = d.precision == 0 ? 4 : 2;
  if (d.n_steps > 0) {
    WindowArgs a = args_of(d, window, sinks, positions, first_position, cache);
    a.q = array_of(q, elem);
    a.k = array_of(k, elem);
    a.v = array_of(v, elem);
    a.out = array_of(out, elem);
    a.lse = lse;
    a.fast = fast_rows(d, q, d.dim_k) && fast_rows(d, k, d.dim_k) && fast_rows(d, v, d.dim_v);
    MARL_CHECK(launch(a, d, plan_of(d, window, sinks, a.fast, false), WINDOW_OUTPUT, s));
  }
  if (next_cache.keys == nullptr) return MARL_OK;
  CacheArgs c{};
  c.in[0] = array_of(k, elem);
  c.in[1] = array_of(v, elem);
  c.old[0] = static_cast<const char*>(cache.keys);
  c.old[1] = static_cast<const char*>(cache.values);
  c.next[0] = static_cast<char*>(next_cache.keys);
  c.next[1] = static_cast<char*>(next_cache.values);
  c.positions = positions;
  c.first = first_position;
  c.n_flags = (uint32_t)(d.n_seqs / d.seqs_per_flag);
  c.seqs_per_flag = (uint32_t)d.seqs_per_flag;
  c.Hk = (uint32_t)d.n_kv_heads;
  c.T = d.n_steps;
  c.dim[0] = d.dim_k;
  c.dim[1] = d.dim_v;
  c.window = window;
  c.sinks = sinks;
  c.chunks = (uint32_t)((slots + kCacheRows - 1) / kCacheRows);
  c.in_place = in_place;
  const unsigned blocks = (unsigned)cache_blocks(d, slots);
  if (d.precision == 0) hipLaunchKernelGGL((window_cache_kernel<float>), dim3(blocks), dim3(256), 0, s, c);
  else hipLaunchKernelGGL((window_cache_kernel<bf16_t>), dim3(blocks), dim3(256), 0, s, c);
  return launch_status();
}

int32_t marl_window_attention_backward(const marl_attention_dims* dims, int32_t window, int32_t sinks, marl_view q, marl_view k, marl_view v,
                                       const int32_t* positions, int32_t first_position, marl_window_cache cache, marl_view out,
                                       const float* lse, marl_view dout, marl_view dq, marl_view dk, marl_view dv, void* workspace,
                                       void* stream) {
  MARL_CHECK(check_window(dims, window, sinks));
  const marl_attention_dims& d = *dims;
  MARL_CHECK(check_launches(d, window, sinks, CALL_BACKWARD, false));
  const bool used = d.n_steps > 0 && d.n_seqs > 0;
  for (const marl_view& x : {q, k, v, out, dout, dq, dk, dv}) MARL_CHECK(check_view(x, d.precision, used));
  MARL_CHECK(check_output(dq, d, d.n_heads, used));
  MARL_CHECK(check_output(dk, d, d.n_kv_heads, used));
  MARL_CHECK(check_output(dv, d, d.n_kv_heads, used));
  MARL_CHECK(check_positions(d, positions, first_position));
  MARL_CHECK(check_floats(lse, used));
  MARL_CHECK(check_cache(cache, false));
  if (used) MARL_REQUIRE_PTR(workspace);
  MARL_CHECK(check_places(dq, {q, k, v, out, dout, dk, dv}, used));
  MARL_CHECK(check_places(dk, {q, k, v, out, dout, dv}, used));
  MARL_CHECK(check_places(dv, {q, k, v, out, dout}, used));
  if (!used) return MARL_OK;
  const int64_t slots = (int64_t)window + sinks;
  const Extent ck = cached(d, cache.keys, slots, d.dim_k), cv = cached(d, cache.values, slots, d.dim_v);
  const int elem = d.precision == 0 ? 4 : 2;
  const bool fast = fast_rows(d, q, d.dim_k) && fast_rows(d, k, d.dim_k) && fast_rows(d, v, d.dim_v) && fast_rows(d, out, d.dim_v) && fast_rows(d, dout, d.dim_v);
  const Plan p = plan_of(d, window, sinks, fast, true);
  const Extent ps = places_of(d, positions), ls = statistics(d, lse), ws = extent(workspace, p.bytes);
  if (touches(dq, d, d.n_heads, d.dim_k, {ck, cv, ps, ls, ws}) || touches(dk, d, d.n_kv_heads, d.dim_k, {ck, cv, ps, ls, ws}) ||
      touches(dv, d, d.n_kv_heads, d.dim_v, {ck, cv, ps, ls, ws}) || touches(q, d, d.n_heads, d.dim_k, ws) || touches(k, d, d.n_kv_heads, d.dim_k, ws) ||
      touches(v, d, d.n_kv_heads, d.dim_v, ws) || touches(out, d, d.n_heads, d.dim_v, ws) || touches(dout, d, d.n_heads, d.dim_v, ws))
    return MARL_E_CONFIG;
  for (const Extent& x : {ck, cv, ps, ls})
    if (ws.meets(x)) return MARL_E_CONFIG;
  hipStream_t s = (hipStream_t)stream;
  WindowArgs a = args_of(d, window, sinks, positions, first_position, cache);
  a.fast = fast;
  a.q = array_of(q, elem);
  a.k = array_of(k, elem);
  a.v = array_of(v, elem);
  a.out = array_of(out, elem);
  a.dout = array_of(dout, elem);
  a.dq = array_of(dq, elem);
  a.dk = array_of(dk, elem);
  a.dv = array_of(dv, elem);
  a.lse = const_cast<float*>(lse);
  a.delta = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.delta);
  a.places = reinterpret_cast<int*>(static_cast<char*>(workspace) + p.places);
  a.reach = reinterpret_cast<int2*>(static_cast<char*>(workspace) + p.reach);
  a.far_chunks = p.far_chunks;
  a.far_slots = p.far_slots;
  a.far_tiles = p.far_tiles;
  a.far_numbers = reinterpret_cast<int*>(static_cast<char*>(workspace) + p.numbers);
  a.far_parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.parts);
  MARL_CHECK(launch(a, d, p, WINDOW_DQ, s));
  if (p.far > 0) MARL_CHECK(launch(a, d, p, WINDOW_FAR, s));
  return launch(a, d, p, WINDOW_DKV, s);
}

int32_t marl_window_attention_step(const marl_attention_dims* dims, int32_t window, int32_t sinks, marl_view q, marl_view k, marl_view v,
                                   const int32_t* positions, marl_window_cache cache, marl_view out, void* workspace, void* stream) {
  MARL_CHECK(check_window(dims, window, sinks));
  const marl_attention_dims& d = *dims;
  if (d.n_steps != 1) return MARL_E_SIZE;
  MARL_CHECK(check_launches(d, window, sinks, CALL_STEP, false));
  if (d.n_seqs == 0) return MARL_OK;
  for (const marl_view& x : {q, k, v, out}) MARL_CHECK(check_view(x, d.precision, true));
  MARL_CHECK(check_output(out, d, d.n_heads, true));
  MARL_CHECK(check_cache(cache, true));
  if (positions == nullptr) return MARL_E_NULL;
  MARL_CHECK(check_positions(d, positions, 0));
  const StepPlan p = step_plan(d, window, sinks);
  if (p.bytes > 0) MARL_REQUIRE_PTR(workspace);
  MARL_CHECK(check_places(out, {q, k, v}, true));
  const int64_t slots = (int64_t)window + sinks;
  const Extent ck = cached(d, cache.keys, slots, d.dim_k), cv = cached(d, cache.values, slots, d.dim_v), ps = places_of(d, positions), ws = extent(workspace, p.bytes);
  if (touches(out, d, d.n_heads, d.dim_v, {ck, cv, ps, ws}) || touches(q, d, d.n_heads, d.dim_k, {ck, cv, ws}) || touches(k, d, d.n_kv_heads, d.dim_k, {ck, cv, ws}) ||
      touches(v, d, d.n_kv_heads, d.dim_v, {ck, cv, ws}))
    return MARL_E_CONFIG;
  if (ck.meets(cv) || ps.meets(ck) || ps.meets(cv) || ws.meets(ck) || ws.meets(cv) || ws.meets(ps)) return MARL_E_CONFIG;
  const int elem = d.precision == 0 ? 4 : 2;
  StepArgs a{};
  a.q = static_cast<const char*>(q.data);
  a.k = static_cast<const char*>(k.data);
  a.v = static_cast<const char*>(v.data);
  a.out = static_cast<char*>(out.data);
  a.q_seq = q.seq * elem;
  a.q_head = q.head * elem;
  a.k_seq = k.seq * elem;
  a.k_head = k.head * elem;
  a.v_seq = v.seq * elem;
  a.v_head = v.head * elem;
  a.out_seq = out.seq * elem;
  a.out_head = out.head * elem;
  a.cache_k = static_cast<char*>(cache.keys);
  a.cache_v = static_cast<char*>(cache.values);
  a.positions = positions;
  a.seqs_per_flag = (uint32_t)d.seqs_per_flag;
  a.H = (uint32_t)d.n_heads;
  a.Hk = (uint32_t)d.n_kv_heads;
  a.group = a.H / a.Hk;
  a.chunks = p.chunks;
  a.splits = p.splits;
  a.parts = p.splits / 4;
  a.units = p.units;
  a.dk = d.dim_k;
  a.dv = d.dim_v;
  a.window = window;
  a.sinks = sinks;
  a.c = d.scale * 1.44269504088896341f;
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.part);
  a.stat = reinterpret_cast<float2*>(static_cast<char*>(workspace) + p.stat);
  const int64_t pairs = (int64_t)d.n_seqs * d.n_heads;
  return d.precision == 0 ? launch_step<float>(a, p, pairs, (hipStream_t)stream) : launch_step<bf16_t>(a, p, pairs, (hipStream_t)stream);
}

}  // extern "C"
