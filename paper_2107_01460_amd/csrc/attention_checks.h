// Checks of the arguments that the attentions share, on the host and before any launch.
#pragma once
#include <initializer_list>

#include "common.h"

namespace marl {

constexpr int kMaxDim = 128;

inline int32_t check_dims(const marl_attention_dims* d) {
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
inline int32_t check_view(const marl_view& v, int precision, bool used) {
  if (!used) return MARL_OK;
  if (v.data == nullptr) return MARL_E_NULL;
  return (reinterpret_cast<uintptr_t>(v.data) & (precision == 0 ? 3u : 1u)) != 0 ? MARL_E_ALIGN : MARL_OK;
}
// An output's elements are places of their own: no stride of zero along a dimension that there is
inline int32_t check_output(const marl_view& v, const marl_attention_dims& d, int heads, bool used) {
  if (!used) return MARL_OK;
  const bool overlaps = (v.step == 0 && d.n_steps > 1) || (v.seq == 0 && d.n_seqs > 1) || (v.head == 0 && heads > 1);
  return overlaps ? MARL_E_CONFIG : MARL_OK;
}
// An output that begins where one of the others does
inline int32_t check_places(const marl_view& out, std::initializer_list<marl_view> others, bool used) {
  if (used)
    for (const marl_view& x : others)
      if (x.data == out.data) return MARL_E_CONFIG;
  return MARL_OK;
}
#define MARL_CHECK(x)                                        \
  do {                                                       \
    const int32_t rc_ = (x);                                 \
    if (rc_ != MARL_OK) return rc_;                          \
  } while (0)

}  // namespace marl
