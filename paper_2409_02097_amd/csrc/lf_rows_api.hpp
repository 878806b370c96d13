// Host side of the row-wise operators around the mixer: [B, N, C] views, what the kernels can address of them, which may meet.
#pragma once
#include "../../include/linfusion.h"
#include "lf_host_api.hpp"

namespace lfh {

struct RowView { const void* p; long long batch, token; size_t bytes; Places rows; };

// LINFUSION_OK when the kernels can address [B, N, C] rows at `p` with these element strides (null: dense) in accesses of
// `align` bytes
inline int row_view(const void* p, const long long* s, int B, long long N, int C, size_t esz, bool written, RowView* v, size_t align = 16) {
  v->p = p;
  v->batch = s ? s[0] : N * C;
  v->token = s ? s[1] : C;
  if (B == 1) v->batch = 0;   // (never used, whatever they say)
  if (N == 1) v->token = 0;
  v->bytes = 0;
  if (!p) return LINFUSION_OK;
  const long long vec = (long long)(align / esz);
  if (v->batch < 0 || v->token < 0) return LINFUSION_ERR_INVALID;
  if (((uintptr_t)p & (align - 1)) || v->batch % vec || v->token % vec) return LINFUSION_ERR_MISALIGNED;
  if (v->token >= 1LL << 27) return LINFUSION_ERR_INVALID;
  const long double span = (long double)(B - 1) * v->batch + (long double)(N - 1) * v->token + C;
  if (span >= (long double)(1LL << 45)) return LINFUSION_ERR_INVALID;
  if (written) {   // no two rows share memory, whichever of batch and token is the outer one
    const bool tokens_out = v->token > v->batch;
    const long long in = tokens_out ? v->batch : v->token, out = tokens_out ? v->token : v->batch;
    const long long n_in = tokens_out ? B : N, n_out = tokens_out ? N : B;
    if (n_in > 1 && in < C) return LINFUSION_ERR_OVERLAP;
    if (n_out > 1 && out < (n_in - 1) * in + C) return LINFUSION_ERR_OVERLAP;
  }
  v->bytes = (size_t)span * esz;
  const long long strides[3] = {v->batch, 0, v->token};
  v->rows = places(p, strides, B, 1, N, C, esz);
  return LINFUSION_OK;
}

inline bool same_rows(const RowView& a, const RowView& b) { return a.p == b.p && a.batch == b.batch && a.token == b.token; }
inline bool meet(const RowView& a, const RowView& b) { return a.p && b.p && overlaps(a.p, a.bytes, b.p, b.bytes) && !apart(a.rows, b.rows); }

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// A plain byte range beside the views.
struct Range { const void* p; size_t n; };
inline bool meet(const Range& a, const Range& b) { return a.p && b.p && a.n && b.n && overlaps(a.p, a.n, b.p, b.n); }
inline Range span(const RowView& v) { return Range{v.p, v.bytes}; }

}  // namespace lfh
