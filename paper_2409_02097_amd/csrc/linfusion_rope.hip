// Rotary positions with several axes (lf_rope.hpp): checks, launch shapes, entry point.
#include "../../include/linfusion.h"

#include <stdint.h>

#include <cmath>

#include "lf_host_api.hpp"
#include "lf_rope.hpp"

namespace {

using lfh::overlaps;

struct Side { const void* x; void* y; int H; long long sx[3], sy[3]; size_t nx, ny; };

int make_side(const void* x, void* y, int H, const long long* sx, const long long* sy, int B, long long N, int d,
              size_t esz, Side* s) {
  *s = Side{x, y, H, {H * N * d, N * d, d}, {H * N * d, N * d, d}, 0, 0};
  if (!x) return LINFUSION_OK;
  for (int i = 0; i < 3; ++i) {
    if (sx) s->sx[i] = sx[i];
    if (sy) s->sy[i] = sy[i];
  }
  const long long extent[3] = {B, H, N};
  for (int i = 0; i < 3; ++i)
    if (extent[i] == 1) s->sx[i] = s->sy[i] = 0;   // (never used, whatever they say)
  if (((uintptr_t)x | (uintptr_t)y) & 15) return LINFUSION_ERR_MISALIGNED;
  int rc = lfh::check_strides(s->sx, B, H, N, d, esz, false);
  if (rc != LINFUSION_OK) return rc;
  if ((rc = lfh::check_strides(s->sy, B, H, N, d, esz, true)) != LINFUSION_OK) return rc;
  s->nx = lfh::span_bytes(s->sx, B, H, N, d, esz);
  s->ny = lfh::span_bytes(s->sy, B, H, N, d, esz);
  return LINFUSION_OK;
}

bool in_place(const Side& s) {
  return s.x == s.y && s.sx[0] == s.sy[0] && s.sx[1] == s.sy[1] && s.sx[2] == s.sy[2];
}

// Whether the rows at `p` and `r` may share memory.  (q and k may be columns of one projection, each turned in place: their spans
// interleave, their rows do not.)
bool meet(const void* p, size_t np, const long long sp[3], int Hp, const void* r, size_t nr, const long long sr[3], int Hr, int B,
          long long N, int d, size_t esz) {
  return overlaps(p, np, r, nr) && !lfh::apart(lfh::places(p, sp, B, Hp, N, d, esz), lfh::places(r, sr, B, Hr, N, d, esz));
}

template <typename T, int MODE> int launch(const lf::RopeArgs& a, int B, unsigned wgs, hipStream_t st) {
  const int lds = (int)lf::rope_table_bytes(a.tokens, a.pairs) + (MODE != 0 ? 4 * 2 * 1024 : 0);
  auto kernel = lf::rope_rows<T, MODE>;
  if (!lfh::allow_lds(kernel, lds)) return LINFUSION_ERR_HIP;
  kernel<<<dim3(wgs, B), dim3(256), lds, st>>>(a);
  return LINFUSION_OK;
}

template <typename T> int run(const lf::RopeArgs& a, int B, unsigned wgs, int mode, hipStream_t st) {
  if (mode == 0) return launch<T, 0>(a, B, wgs, st);
  return mode == 1 ? launch<T, 1>(a, B, wgs, st) : launch<T, 2>(a, B, wgs, st);
}

}  // namespace

extern "C" int linfusion_rope(const void* q, const void* k, void* q_out, void* k_out, const int* positions, int axes,
                              const int* channels, const double* bases, const double* scales, int B, int H, int H_k,
                              long long N, int d, int dtype, unsigned flags, const int* lengths,
                              const long long q_strides[3], const long long k_strides[3],
                              const long long q_out_strides[3], const long long k_out_strides[3],
                              const long long position_strides[2], void* stream) {
  if (!q || !q_out || !positions || !channels || !bases || (!k) != (!k_out)) return LINFUSION_ERR_INVALID;
  if (B <= 0 || H <= 0 || N <= 0 || d <= 0 || B > 65535 || H > 65535 || (k && (H_k <= 0 || H_k > 65535)))
    return LINFUSION_ERR_INVALID;
  if (flags & ~(LINFUSION_FLAG_ROPE_NEIGHBOURS | LINFUSION_FLAG_ROPE_INVERSE)) return LINFUSION_ERR_INVALID;
  if (dtype != LINFUSION_DTYPE_F32 && dtype != LINFUSION_DTYPE_F16 && dtype != LINFUSION_DTYPE_BF16)
    return LINFUSION_ERR_UNSUPPORTED;
  if (d % 8 || d > 2 * lf::kRopePairs) return LINFUSION_ERR_UNSUPPORTED;
  if (axes < 1 || axes > lf::kRopeAxes) return LINFUSION_ERR_UNSUPPORTED;
  if (N >= 1LL << 28) return LINFUSION_ERR_INVALID;
  lf::RopeArgs a{};
  int at = 0;
  bool whole = true;
  for (int i = 0; i < axes; ++i) {
    const int c = channels[i];
    if (c <= 0 || c % 2 || c > d - at) return LINFUSION_ERR_INVALID;
    if (!(bases[i] > 0.0) || !std::isfinite(bases[i])) return LINFUSION_ERR_INVALID;
    const double scale = scales ? scales[i] : 1.0;
    if (!std::isfinite(scale)) return LINFUSION_ERR_INVALID;
    a.first[i] = at;
    const double step = std::pow(bases[i], -2.0 / c);
    double rate = scale / 6.283185307179586476925287;
    for (int p = 0; p < c / 2; ++p, rate *= step) a.rate[at / 2 + p] = rate;
    at += c;
    whole = whole && c % (dtype == LINFUSION_DTYPE_F32 ? 8 : 16) == 0;   // (then sections begin and halves end at whole 16 bytes)
  }
  for (int i = axes; i <= lf::kRopeAxes; ++i) a.first[i] = at;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2;
  Side s[2];
  int rc = make_side(q, q_out, H, q_strides, q_out_strides, B, N, d, esz, &s[0]);
  if (rc != LINFUSION_OK) return rc;
  if ((rc = make_side(k, k_out, H_k, k_strides, k_out_strides, B, N, d, esz, &s[1])) != LINFUSION_OK) return rc;
  if (((uintptr_t)positions | (uintptr_t)lengths) & 3) return LINFUSION_ERR_MISALIGNED;
  const long long pb = position_strides ? position_strides[0] : 0, pa = position_strides ? position_strides[1] : N;
  if (pb < 0 || pa < 0 || pb >= 1LL << 44 || pa >= 1LL << 44) return LINFUSION_ERR_INVALID;
  const size_t np = (size_t)((B - 1) * pb + (axes - 1) * pa + N) * 4;
  for (int i = 0; i < 2; ++i) {
    if (!s[i].x) continue;
    if (!in_place(s[i]) && meet(s[i].y, s[i].ny, s[i].sy, s[i].H, s[i].x, s[i].nx, s[i].sx, s[i].H, B, N, d, esz))
      return LINFUSION_ERR_OVERLAP;
    const Side& o = s[1 - i];
    if (o.x && meet(s[i].y, s[i].ny, s[i].sy, s[i].H, o.x, o.nx, o.sx, o.H, B, N, d, esz)) return LINFUSION_ERR_OVERLAP;
    if (overlaps(s[i].y, s[i].ny, positions, np)) return LINFUSION_ERR_OVERLAP;
    if (lengths && overlaps(s[i].y, s[i].ny, lengths, (size_t)B * 4)) return LINFUSION_ERR_OVERLAP;
  }
  if (k && meet(q_out, s[0].ny, s[0].sy, s[0].H, k_out, s[1].ny, s[1].sy, s[1].H, B, N, d, esz)) return LINFUSION_ERR_OVERLAP;
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  for (int i = 0; i < 2; ++i) {
    if (!s[i].x) continue;
    a.side[i] = lf::RopeSide{s[i].x, s[i].y, s[i].sx[0], s[i].sx[1], s[i].sx[2], s[i].sy[0], s[i].sy[1], s[i].sy[2], s[i].H,
                             s[i].sx[1] < s[i].sx[2]};
  }
  a.positions = positions;
  a.pos_batch = pb;
  a.pos_axis = pa;
  a.lengths = lengths;
  a.N = N;
  a.d = d;
  a.pairs = at / 2;
  a.axes = axes;
  a.inverse = (flags & LINFUSION_FLAG_ROPE_INVERSE) != 0;
  // Tokens per workgroup: 16 KB of rows, so that the angles are a small part of its work, while every CU has several workgroups
  // (us per call, 8 / 16 / 32 / 64 KB: bf16 81120 x 2 x 16 x 128 252 / 227 / 233 / 236, fp32 2 x 36503 x 2 x 8 x 40 60 / 57 / 60 / 66)
  const long long heads = H + (k ? H_k : 0), all = (long long)B * N;
  const auto many = [&](long long t) { return (N + t - 1) / t >= 1LL << 24; };   // (a grid has at most 2^32 threads a row)
  int tokens = 1;
  while (tokens < 64 && 2 * tokens * a.pairs * 8 <= 32768 &&
         (many(tokens) || (all / (2 * tokens) >= 4LL * lfh::num_cu() && tokens * heads * d * (long long)esz < 16384)))
    tokens *= 2;
  a.tokens = tokens;
  const long long wgs = (N + tokens - 1) / tokens;   // (32 tokens are always possible: below 2^24)
  const int mode = (flags & LINFUSION_FLAG_ROPE_NEIGHBOURS) ? 0 : (whole ? 1 : 2);
  const hipStream_t st = (hipStream_t)stream;
  rc = dtype == LINFUSION_DTYPE_F16   ? run<lf::F16>(a, B, (unsigned)wgs, mode, st)
       : dtype == LINFUSION_DTYPE_BF16 ? run<lf::BF16>(a, B, (unsigned)wgs, mode, st)
                                       : run<lf::F32>(a, B, (unsigned)wgs, mode, st);
  if (rc != LINFUSION_OK) return rc;
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}
