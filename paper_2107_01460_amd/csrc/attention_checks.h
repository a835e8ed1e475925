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
// Contiguous memory of `bytes`; none: no array
struct Extent {
  uintptr_t from, bytes;
  bool meets(const Extent& o) const { return bytes > 0 && o.bytes > 0 && (from < o.from ? o.from - from < bytes : from - o.from < o.bytes); }
};
inline Extent extent(const void* p, int64_t bytes) { return {reinterpret_cast<uintptr_t>(p), p == nullptr ? 0 : (uintptr_t)bytes}; }
inline Extent places_of(const marl_attention_dims& d, const int32_t* positions) { return extent(positions, (int64_t)(d.n_seqs / d.seqs_per_flag) * d.n_steps * 4); }
struct Stride {
  __int128 bytes;
  int64_t n;
};
// Rows of a block of memory of `span` bytes from `base` on, the widest stride first, that lie in [lo, hi)
inline bool reaches(__int128 base, __int128 span, const Stride* s, int dims, __int128 lo, __int128 hi) {
  if (base >= hi || base + span <= lo) return false;
  if (base >= lo || dims == 0) return true;
  const __int128 part = span - s->bytes * (s->n - 1);  // of one index
  const __int128 begins = (lo - base + s->bytes - 1) / s->bytes;  // the first index that begins at lo or behind it
  if (begins < s->n && base + begins * s->bytes < hi) return true;
  // those before it that end behind lo: one, unless indexes overlap (of many such ones the nearest are looked at)
  __int128 i = begins < s->n ? begins : s->n;
  for (int looked = 0; i-- > 0 && base + i * s->bytes + part > lo && looked < 64; ++looked)
    if (reaches(base + i * s->bytes, part, s + 1, dims - 1, lo, hi)) return true;
  return false;
}
// Whether any row of an array [n_steps][n_seqs][heads][dim] lies in e.  (Not the memory between its rows: an array may lie in the gaps of another.)
inline bool touches(const marl_view& v, const marl_attention_dims& d, int heads, int dim, const Extent& e) {
  if (e.bytes == 0) return false;
  const int elem = d.precision == 0 ? 4 : 2;
  Stride s[3];
  int dims = 0;
  __int128 base = reinterpret_cast<uintptr_t>(v.data), span = (int64_t)dim * elem;
  for (const Stride& x : {Stride{v.step, d.n_steps}, Stride{v.seq, d.n_seqs}, Stride{v.head, heads}}) {
    if (x.n < 2 || x.bytes == 0) continue;
    Stride here = {x.bytes * elem, x.n};
    if (here.bytes < 0) {
      base += here.bytes * (here.n - 1);
      here.bytes = -here.bytes;
    }
    span += here.bytes * (here.n - 1);
    int at = dims++;
    for (; at > 0 && s[at - 1].bytes < here.bytes; --at) s[at] = s[at - 1];
    s[at] = here;
  }
  const __int128 lo = e.from;
  return reaches(base, span, s, dims, lo, lo + e.bytes);
}
inline bool touches(const marl_view& v, const marl_attention_dims& d, int heads, int dim, std::initializer_list<Extent> all) {
  for (const Extent& e : all)
    if (touches(v, d, heads, dim, e)) return true;
  return false;
}
#define MARL_CHECK(x)                                        \
  do {                                                       \
    const int32_t rc_ = (x);                                 \
    if (rc_ != MARL_OK) return rc_;                          \
  } while (0)

}  // namespace marl
