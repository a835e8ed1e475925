// Layer norm over rows, and its gradient.
//
// A team of lanes holds a row in registers (up to sixteen values a lane), so that every value is read once: mean, then the squares of
// the centred values, both summed in fp32 across the team.  Bound by memory: a row in, a row out.  Measured: 128 x 4096 rows of 512 bf16 209 us, 5.2 TB/s;
// gradient of as many rows of 128 fp32 156 us, 5.2 TB/s (a copy of 2 GiB: 4.9); of 10 007 rows of 147 bf16 10 us and 5 for the column sums.
#include "common.h"

namespace marl {
namespace {

// Values of a row that a lane holds at most.  (Eight, with twice the lanes a row: 10 007 rows of 147 6.7 instead of 10 us, large calls 3 to 4 % slower.)
constexpr int kLane = 16;
constexpr int kMaxWidth = 16384;
constexpr int kThreads = 256;

// Columns of a lane: vectors of E consecutive values (sixteen bytes, at any alignment; E = 1 for rows shorter than that), vector u of lane l at
// ((u * TEAM) + l) * E.  A last vector that would pass the row's end is moved back to end with it: its first `skip` values are its neighbour's too, they
// are computed and stored twice alike and counted once.
template <int E>
struct Columns {
  int at, skip;  // first column; values to pass over in sums: E where there is nothing
  __device__ __forceinline__ Columns(int vector, int width) {
    const int c = vector * E;
    at = c < width ? min(c, width - E) : 0;
    skip = c < width ? c - at : E;
  }
};
template <class T, int E>
__device__ __forceinline__ void load_vec(float (&v)[E], const T* p) {
  if constexpr (E == 1) {
    v[0] = load_act(p, 0);
  } else if constexpr (sizeof(T) == 4) {
    __builtin_memcpy(v, p, 16);
  } else {
    uint32_t w[4];
    __builtin_memcpy(w, p, 16);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
}
template <class T, int E>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[E]) {
  if constexpr (E == 1) {
    if constexpr (sizeof(T) == 4) *p = v[0];
    else *p = to_bf16(v[0]);
  } else if constexpr (sizeof(T) == 4) {
    __builtin_memcpy(p, v, 16);
  } else {
    const uint32_t w[4] = {pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
    __builtin_memcpy(p, w, 16);
  }
}

// Sum over a team; TEAM > 64: over the workgroup, through LDS (scratch: a slot per wavefront, `turn` tells uses apart)
template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float* scratch) {
#pragma unroll
  for (int m = 1; m < (TEAM < 64 ? TEAM : 64); m <<= 1) v += __shfl_xor(v, m);
  if constexpr (TEAM > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TEAM / 64; ++w) v += scratch[w];
  }
  return v;
}

// Weights of a lane's columns (absent: `none`)
template <int E>
__device__ __forceinline__ void load_weights(float (&w)[E], const float* p, int at, float none) {
#pragma unroll
  for (int k = 0; k < E; ++k) w[k] = none;
  if (p != nullptr) __builtin_memcpy(w, p + at, 4 * E);
}

// Every workgroup takes every gridDim.x-th group of rows, so that weights are read once a workgroup and not once a row (from the L2 that was four
// times the rows' own bytes in bf16: 128 x 4096 rows of 512 took 0.92 ms).
template <class T, int E, int TEAM, int N>  // N vectors a lane
__global__ void __launch_bounds__(TEAM > kThreads ? TEAM : kThreads)
    layer_norm_kernel(int64_t rows, int width, const T* x, int64_t xs, const float* __restrict__ weight, const float* __restrict__ bias, float eps,
                      T* y, int64_t ys, float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  constexpr int kBlock = TEAM > kThreads ? TEAM : kThreads, kTeams = kBlock / TEAM;
  __shared__ float scratch[16];
  const int lane = threadIdx.x % TEAM;
  float w[N][E], b[N][E];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const Columns<E> c(u * TEAM + lane, width);
    load_weights<E>(w[u], weight, c.at, 1.f);
    load_weights<E>(b[u], bias, c.at, 0.f);
  }
  const float inv = 1.f / (float)width;
  for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < rows; row0 += (int64_t)gridDim.x * kTeams) {
    const int64_t row = row0 + threadIdx.x / TEAM;
    const bool on = row < rows;
    const T* xr = x + (on ? row : row0) * xs;
    float v[N][E];
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < N; ++u) load_vec<T, E>(v[u], xr + Columns<E>(u * TEAM + lane, width).at);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int skip = Columns<E>(u * TEAM + lane, width).skip;
#pragma unroll
      for (int k = 0; k < E; ++k) sum += k >= skip ? v[u][k] : 0.f;
    }
    const float mean = team_sum<TEAM>(sum, scratch) * inv;
    float sq = 0.f;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int skip = Columns<E>(u * TEAM + lane, width).skip;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        v[u][k] -= mean;
        sq += k >= skip ? v[u][k] * v[u][k] : 0.f;
      }
    }
    const float rstd = 1.f / sqrtf(team_sum<TEAM>(sq, scratch) * inv + eps);
    if (on) {
      T* yr = y + row * ys;
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const Columns<E> c(u * TEAM + lane, width);
        if (c.skip < E) {
#pragma unroll
          for (int k = 0; k < E; ++k) v[u][k] = v[u][k] * rstd * w[u][k] + b[u][k];
          store_vec<T, E>(yr + c.at, v[u]);
        }
      }
      if (lane == 0) {
        if (mean_out != nullptr) mean_out[row] = mean;
        if (rstd_out != nullptr) rstd_out[row] = rstd;
      }
    }
  }
}

// The gradient (rows of more than 4096 values with column sums spill 5 to 9 registers): a workgroup keeps its shares of the two column sums in registers over its rows: its teams' are added
// through LDS at the end and written out, [workgroup][2][width], for column_sum_kernel.
template <class T, int E, int TEAM, int N, bool WEIGHTS>
__global__ void __launch_bounds__(TEAM > kThreads ? TEAM : kThreads)
    layer_norm_backward_kernel(int64_t rows, int width, const T* dy, int64_t dys, const T* x, int64_t xs, const float* __restrict__ weight,
                               const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, int64_t dxs, float* __restrict__ part) {
  constexpr int kBlock = TEAM > kThreads ? TEAM : kThreads, kTeams = kBlock / TEAM, kWaves = kBlock / 64;
  __shared__ float scratch[16];
  const int lane = threadIdx.x % TEAM;
  const float inv = 1.f / (float)width;
  float w[N][E], dw[N][E], db[N][E];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    load_weights<E>(w[u], weight, Columns<E>(u * TEAM + lane, width).at, 1.f);
#pragma unroll
    for (int k = 0; k < E; ++k) dw[u][k] = db[u][k] = 0.f;
  }
  for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < rows; row0 += (int64_t)gridDim.x * kTeams) {
    const int64_t row = row0 + threadIdx.x / TEAM;
    const bool on = row < rows;
    const int64_t at = on ? row : rows - 1;
    const T *xr = x + at * xs, *gr = dy + at * dys;
    const float m = mean[at], r = rstd[at];
    float h[N][E], g[N][E];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int from = Columns<E>(u * TEAM + lane, width).at;
      load_vec<T, E>(h[u], xr + from);
      load_vec<T, E>(g[u], gr + from);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int skip = Columns<E>(u * TEAM + lane, width).skip;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        h[u][k] = (h[u][k] - m) * r;
        if constexpr (WEIGHTS) {
          dw[u][k] += on ? g[u][k] * h[u][k] : 0.f;
          db[u][k] += on ? g[u][k] : 0.f;
        }
        g[u][k] *= w[u][k];
        s1 += k >= skip ? g[u][k] : 0.f;
        s2 += k >= skip ? g[u][k] * h[u][k] : 0.f;
      }
    }
    s1 = team_sum<TEAM>(s1, scratch) * inv;
    s2 = team_sum<TEAM>(s2, scratch) * inv;
    if (on) {
      T* o = dx + row * dxs;
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const Columns<E> c(u * TEAM + lane, width);
        if (c.skip < E) {
#pragma unroll
          for (int k = 0; k < E; ++k) g[u][k] = r * (g[u][k] - s1 - h[u][k] * s2);
          store_vec<T, E>(o + c.at, g[u]);
        }
      }
    }
  }
  if constexpr (WEIGHTS) {
    float* p = part + (int64_t)blockIdx.x * 2 * width;
    if constexpr (TEAM >= kBlock) {
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const Columns<E> c(u * TEAM + lane, width);
          if (k >= c.skip) {
            p[c.at + k] = dw[u][k];
            p[width + c.at + k] = db[u][k];
          }
        }
    } else {
      __shared__ float shares[kWaves][2][TEAM * N * E];
      const int wave = threadIdx.x >> 6;
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int k = 0; k < E; ++k) {
#pragma unroll
          for (int m = TEAM; m < 64; m <<= 1) {
            dw[u][k] += __shfl_xor(dw[u][k], m);
            db[u][k] += __shfl_xor(db[u][k], m);
          }
          const Columns<E> c(u * TEAM + lane, width);
          if ((threadIdx.x & 63) < TEAM && k >= c.skip) {
            shares[wave][0][c.at + k] = dw[u][k];
            shares[wave][1][c.at + k] = db[u][k];
          }
        }
      __syncthreads();
      for (int at = threadIdx.x; at < 2 * width; at += kBlock) {
        const int which = at >= width, c = at - which * width;
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) s += shares[v][which][c];
        p[at] = s;
      }
    }
  }
}

// Sums of the workgroups' shares, in a fixed order: 32 groups of threads take every 32nd share of 32 columns, sixteen loads on their way together
__global__ void __launch_bounds__(1024) column_sum_kernel(const float* __restrict__ part, int n, int width, float* __restrict__ dweight,
                                                          float* __restrict__ dbias) {
  constexpr int kBatch = 16;
  __shared__ float shares[32][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, at = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (at < 2 * width) {
    for (int k0 = group; k0 < n; k0 += 32 * kBatch) {
      float v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) v[u] = part[(int64_t)min(k0 + 32 * u, n - 1) * 2 * width + at];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) s += k0 + 32 * u < n ? v[u] : 0.f;
    }
  }
  shares[group][lane] = s;
  __syncthreads();
  if (group == 0 && at < 2 * width) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) s += shares[w][lane];
    float* out = at < width ? dweight : dbias;
    if (out != nullptr) out[at < width ? at : at - width] = s;
  }
}

inline int team_of(int width) {  // lanes that a row takes
  int team = 8;
  while (team < 64 && team * kLane < width) team *= 2;
  return team * kLane >= width ? team : width <= 256 * kLane ? 256 : 1024;
}
inline int64_t shares_of(int64_t rows, int width) {  // workgroups of the gradient's kernel, each with its share of the column sums
  const int team = team_of(width), teams = team >= kThreads ? 1 : kThreads / team;
  const int64_t groups = (rows + teams - 1) / teams, most = team == 1024 ? 256 : 1024;
  return groups < most ? groups : most;
}

// The instance for a team.  (Rows shorter than sixteen bytes: the smallest.)
#define MARL_LN_TEAMS                          \
  constexpr int N = E == 1 ? 1 : kLane / E;    \
  if (E == 1 || team == 8) MARL_LN(8);         \
  else if (team == 16) MARL_LN(16);            \
  else if (team == 32) MARL_LN(32);            \
  else if (team == 64) MARL_LN(64);            \
  else if (team == 256) MARL_LN(256);          \
  else MARL_LN(1024)

template <class T, int E>
int32_t forward(int64_t rows, int width, const T* x, int64_t xs, const float* weight, const float* bias, float eps, T* y, int64_t ys, float* mean,
                float* rstd, hipStream_t s) {
  const int team = team_of(width);
  const int64_t teams = team >= kThreads ? 1 : kThreads / team, groups = (rows + teams - 1) / teams, most = team == 1024 ? 512 : 2048;
  const int64_t blocks = groups < most ? groups : most;  // as many as the chip holds at once
#define MARL_LN(TEAM)                                                                                                                        \
  hipLaunchKernelGGL((layer_norm_kernel<T, E, TEAM, N>), dim3((unsigned)blocks), dim3(TEAM > kThreads ? TEAM : kThreads), 0, s, rows, width, x, \
                     xs, weight, bias, eps, y, ys, mean, rstd)
  MARL_LN_TEAMS;
#undef MARL_LN
  return launch_status();
}

template <class T, int E, bool WEIGHTS>
int32_t backward(int64_t rows, int width, const T* dy, int64_t dys, const T* x, int64_t xs, const float* weight, const float* mean,
                 const float* rstd, T* dx, int64_t dxs, float* part, hipStream_t s) {
  const dim3 grid((unsigned)shares_of(rows, width));
  const int team = team_of(width);
#define MARL_LN(TEAM)                                                                                                                    \
  hipLaunchKernelGGL((layer_norm_backward_kernel<T, E, TEAM, N, WEIGHTS>), grid, dim3(TEAM > kThreads ? TEAM : kThreads), 0, s, rows, width, \
                     dy, dys, x, xs, weight, mean, rstd, dx, dxs, part)
  MARL_LN_TEAMS;
#undef MARL_LN
  return launch_status();
}

template <class T>
int32_t backward_of(bool wide, bool weights, int64_t rows, int width, const void* dy, int64_t dys, const void* x, int64_t xs, const float* weight,
                    const float* mean, const float* rstd, void* dx, int64_t dxs, float* part, hipStream_t s) {
  constexpr int E = 16 / sizeof(T);
  auto call = [&](auto f) { return f(rows, width, (const T*)dy, dys, (const T*)x, xs, weight, mean, rstd, (T*)dx, dxs, part, s); };
  if (wide) return weights ? call(backward<T, E, true>) : call(backward<T, E, false>);
  return weights ? call(backward<T, 1, true>) : call(backward<T, 1, false>);
}

int32_t check(int32_t precision, int64_t rows, int32_t width) {
  if (precision != 0 && precision != 1) return MARL_E_CONFIG;
  if (rows < 0 || rows > ((int64_t)1 << 40) || width < 1 || width > kMaxWidth) return MARL_E_SIZE;
  return MARL_OK;
}
int32_t check_rows(const void* p, int32_t precision) {
  if (p == nullptr) return MARL_E_NULL;
  return (reinterpret_cast<uintptr_t>(p) & (precision == 0 ? 3u : 1u)) != 0 ? MARL_E_ALIGN : MARL_OK;
}
bool overlapping(int64_t rows, int32_t width, int64_t stride) { return rows > 1 && (stride < 0 ? -stride : stride) < width; }  // rows of an output
// Rows written over the ones that are read, in other places
bool moved(int64_t rows, const void* out, int64_t out_stride, const void* in, int64_t in_stride) { return out == in && rows > 1 && out_stride != in_stride; }
int32_t check_floats(const float* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0 ? MARL_E_ALIGN : MARL_OK; }

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int32_t marl_layer_norm(int32_t precision, int64_t n_rows, int32_t width, const void* x, int64_t x_stride,
                        const float* weight, const float* bias, float eps, void* y, int64_t y_stride, float* mean,
                        float* rstd, void* stream) {
  int32_t rc = check(precision, n_rows, width);
  if (rc != MARL_OK || n_rows == 0) return rc;
  if (!(eps >= 0.f) || overlapping(n_rows, width, y_stride)) return MARL_E_CONFIG;
  if ((rc = check_rows(x, precision)) != MARL_OK || (rc = check_rows(y, precision)) != MARL_OK) return rc;
  if (moved(n_rows, y, y_stride, x, x_stride)) return MARL_E_CONFIG;
  for (const float* p : {weight, bias, (const float*)mean, (const float*)rstd})
    if ((rc = check_floats(p)) != MARL_OK) return rc;
  hipStream_t s = (hipStream_t)stream;
  const int elem = precision == 0 ? 4 : 2;
  const bool wide = width * elem >= 16;
  if (precision == 0)
    return (wide ? forward<float, 4> : forward<float, 1>)(n_rows, width, (const float*)x, x_stride, weight, bias, eps, (float*)y, y_stride, mean, rstd, s);
  return (wide ? forward<bf16_t, 8> : forward<bf16_t, 1>)(n_rows, width, (const bf16_t*)x, x_stride, weight, bias, eps, (bf16_t*)y, y_stride, mean,
                                                          rstd, s);
}

int32_t marl_layer_norm_workspace(int64_t n_rows, int32_t width, int64_t* bytes) {
  const int32_t rc = check(0, n_rows, width);
  if (rc != MARL_OK) return rc;
  if (bytes == nullptr) return MARL_E_NULL;
  *bytes = shares_of(n_rows, width) * 2 * width * 4;
  return MARL_OK;
}

int32_t marl_layer_norm_backward(int32_t precision, int64_t n_rows, int32_t width, const void* dy, int64_t dy_stride,
                                 const void* x, int64_t x_stride, const float* weight, const float* mean,
                                 const float* rstd, void* dx, int64_t dx_stride, float* dweight, float* dbias,
                                 void* workspace, void* stream) {
  int32_t rc = check(precision, n_rows, width);
  if (rc != MARL_OK) return rc;
  for (const float* p : {weight, (const float*)dweight, (const float*)dbias})
    if ((rc = check_floats(p)) != MARL_OK) return rc;
  const bool weights = dweight != nullptr || dbias != nullptr;
  if (n_rows > 0) {
    for (const void* p : {dy, x, (const void*)dx})
      if ((rc = check_rows(p, precision)) != MARL_OK) return rc;
    if (overlapping(n_rows, width, dx_stride) || moved(n_rows, dx, dx_stride, dy, dy_stride) || moved(n_rows, dx, dx_stride, x, x_stride)) return MARL_E_CONFIG;
    if (mean == nullptr || rstd == nullptr) return MARL_E_NULL;
    if ((rc = check_floats(mean)) != MARL_OK || (rc = check_floats(rstd)) != MARL_OK) return rc;
    if (weights) MARL_REQUIRE_PTR(workspace);
  }
  hipStream_t s = (hipStream_t)stream;
  int64_t shares = 0;
  if (n_rows > 0) {
    const int elem = precision == 0 ? 4 : 2;
    const bool wide = width * elem >= 16;
    shares = shares_of(n_rows, width);
    rc = (precision == 0 ? backward_of<float> : backward_of<bf16_t>)(wide, weights, n_rows, width, dy, dy_stride, x, x_stride, weight, mean, rstd, dx,
                                                                     dx_stride, (float*)workspace, s);
    if (rc != MARL_OK) return rc;
  }
  if (!weights) return MARL_OK;
  hipLaunchKernelGGL(column_sum_kernel, dim3((2 * width + 31) / 32), dim3(1024), 0, s, (const float*)workspace, (int)shares, width, dweight,
                     dbias);
  return launch_status();
}

}  // extern "C"
