// The block boundary (lf_gate_norm.hpp): checks, launch shapes, entry points.
#include "../../include/linfusion.h"

#include <stdint.h>

#include <cmath>

#include "lf_gate_norm.hpp"
#include "lf_host_api.hpp"

namespace {

using lfh::overlaps;

constexpr int kMaxChannels = 8192;

struct View { const void* p; long long batch, token; size_t bytes; lfh::Places rows; };

// LINFUSION_OK when the kernels can address [B, N, C] rows at `p` with these element strides (null: dense)
int make_view(const void* p, const long long* s, int B, long long N, int C, size_t esz, bool written, View* v) {
  v->p = p;
  v->batch = s ? s[0] : N * C;
  v->token = s ? s[1] : C;
  if (B == 1) v->batch = 0;   // (never used, whatever they say)
  if (N == 1) v->token = 0;
  v->bytes = 0;
  if (!p) return LINFUSION_OK;
  const long long vec = (long long)(16 / esz);
  if (v->batch < 0 || v->token < 0) return LINFUSION_ERR_INVALID;
  if (((uintptr_t)p & 15) || v->batch % vec || v->token % vec) return LINFUSION_ERR_MISALIGNED;
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
  v->rows = lfh::places(p, strides, B, 1, N, C, esz);
  return LINFUSION_OK;
}

bool same_rows(const View& a, const View& b) { return a.p == b.p && a.batch == b.batch && a.token == b.token; }
bool meet(const View& a, const View& b) { return a.p && b.p && overlaps(a.p, a.bytes, b.p, b.bytes) && !lfh::apart(a.rows, b.rows); }

int check_sizes(int B, long long N, int C, int dtype) {
  if (B <= 0 || N <= 0 || C <= 0 || B > 65535) return LINFUSION_ERR_INVALID;
  if (dtype != LINFUSION_DTYPE_F32 && dtype != LINFUSION_DTYPE_F16 && dtype != LINFUSION_DTYPE_BF16)
    return LINFUSION_ERR_UNSUPPORTED;
  if (C % 8 || C > kMaxChannels) return LINFUSION_ERR_UNSUPPORTED;
  if (N > (1LL << 40) / C) return LINFUSION_ERR_INVALID;
  return LINFUSION_OK;
}

// vectors of fp32: [C], or modulation rows with `stride` elements between two batch rows
int check_vectors(int C, long long stride, std::initializer_list<const void*> mod,
                  std::initializer_list<const void*> channel) {
  if (stride < 0 || (stride != 0 && stride < C) || stride >= 1LL << 40) return LINFUSION_ERR_INVALID;
  if (stride % 4) return LINFUSION_ERR_MISALIGNED;
  for (const void* p : mod)
    if ((uintptr_t)p & 15) return LINFUSION_ERR_MISALIGNED;
  for (const void* p : channel)
    if ((uintptr_t)p & 15) return LINFUSION_ERR_MISALIGNED;
  return LINFUSION_OK;
}

size_t mod_bytes(int B, int C, long long stride) { return ((size_t)(B - 1) * (size_t)stride + (size_t)C) * 4; }

// Threads per token and tokens per workgroup.  A wave per token where two vectors of 8 channels a lane hold it and there is a token for
// every wave of the device; a workgroup per token for wide tokens and for few.  us forward / backward, wave : workgroup, fp16: 32768 x 640
// 31 / 51 : 32 / 109, 2048 x 1024 4.7 / 12.9 : 6.3 / 15.0, 512 x 640 3.7 / 9.1 : 3.5 / 9.0; three vectors a lane lose to the workgroup
// (32768 x 1280 55 : 51).
// Workgroups per CU: forward many short ones where a token takes a workgroup, whose start (the modulation of its channels) is small
// against four tokens or more, fewer where it takes a wave; backward, where each leaves partial sums, fewer still: but four of a
// workgroup per token, not two, where many tokens leave much of it idle (32768 x 1280 112 : 141 us; 32768 x 2048 185 : 161, 1024 x 1280
// 17 : 13), and one, not two, above 4096 channels, whose registers leave a CU room for no more (bf16 16384 x 5120 313 : 320, 20000 x 4104
// 321 : 329, 8192 x 8192 218 : 229, fp32 2048 x 8192 101 : 118, 512 x 5120 24 : 30; 16384 x 4096 224 : 176, 8192 x 2560 92 : 64).  Forward,
// 16, 64 and 256 of them take the same time for 2560 to 8192 channels.
struct Shape { int lanes, vpt, rows, wgs; };
Shape shape_of(int B, long long N, int C, bool backward) {
  Shape s;
  const int vecs = C / 8;
  const long long cus = lfh::num_cu(), tokens = (long long)B * N;
  s.lanes = vecs <= 128 && (tokens >= 4 * cus || vecs <= 64) ? 64 : 256;
  s.vpt = (vecs + s.lanes - 1) / s.lanes;
  const int per = 256 / s.lanes;
  int per_cu;
  if (backward) per_cu = s.lanes == 64 ? (C <= 512 ? 8 : 4) : (C <= 1536 && tokens >= 16 * cus ? 4 : (C <= 4096 ? 2 : 1));
  else per_cu = s.lanes == 64 ? 16 : 64;
  long long rows = (tokens + cus * per_cu - 1) / (cus * per_cu);
  if (!backward && rows < 4 && tokens > 4 * cus) rows = 4;
  rows = (rows + per - 1) / per * per;
  if (rows > N) rows = (N + per - 1) / per * per;
  if (rows > 1 << 20) rows = 1 << 20;
  s.rows = (int)rows;
  s.wgs = (int)((N + rows - 1) / rows);
  return s;
}

template <typename T, int LANES, int VPT, bool RMS, bool POST>
int launch_fwd(const lf::GateNormArgs& a, int B, const Shape& s, hipStream_t st) {
  lf::gate_norm_fwd<T, LANES, VPT, RMS, POST><<<dim3(s.wgs, B), dim3(256), 0, st>>>(a);
  return LINFUSION_OK;
}
template <typename T, int LANES, int VPT, bool RMS, bool POST>
int launch_bwd(const lf::GateNormBwdArgs& a, int B, const Shape& s, hipStream_t st) {
  const int lds = LANES < 256 ? 256 / LANES * 3 * a.C * 4 : 0;
  auto kernel = lf::gate_norm_bwd<T, LANES, VPT, RMS, POST>;
  if (!lfh::allow_lds(kernel, lds)) return LINFUSION_ERR_HIP;
  kernel<<<dim3(s.wgs, B), dim3(256), lds, st>>>(a);
  return LINFUSION_OK;
}

#define LF_NORM_KINDS(LAUNCH, T, L, V)                                                    \
  return rms ? (post ? LAUNCH<T, L, V, true, true>(a, B, s, st) : LAUNCH<T, L, V, true, false>(a, B, s, st)) \
             : (post ? LAUNCH<T, L, V, false, true>(a, B, s, st) : LAUNCH<T, L, V, false, false>(a, B, s, st))

template <typename T> int run_fwd(const lf::GateNormArgs& a, int B, const Shape& s, bool rms, bool post, hipStream_t st) {
  if (s.lanes == 64) {
    if (s.vpt == 1) { LF_NORM_KINDS(launch_fwd, T, 64, 1); }
    LF_NORM_KINDS(launch_fwd, T, 64, 2);
  }
  if (s.vpt == 1) { LF_NORM_KINDS(launch_fwd, T, 256, 1); }
  if (s.vpt == 2) { LF_NORM_KINDS(launch_fwd, T, 256, 2); }
  LF_NORM_KINDS(launch_fwd, T, 256, 4);
}
template <typename T> int run_bwd(const lf::GateNormBwdArgs& a, int B, const Shape& s, bool rms, bool post, hipStream_t st) {
  if (s.lanes == 64) {
    if (s.vpt == 1) { LF_NORM_KINDS(launch_bwd, T, 64, 1); }
    LF_NORM_KINDS(launch_bwd, T, 64, 2);
  }
  if (s.vpt == 1) { LF_NORM_KINDS(launch_bwd, T, 256, 1); }
  if (s.vpt == 2) { LF_NORM_KINDS(launch_bwd, T, 256, 2); }
  LF_NORM_KINDS(launch_bwd, T, 256, 4);
}

lf::NormView dev(const View& v) { return lf::NormView{v.batch, v.token}; }

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

// Workgroups of a backward call over the whole batch, at most.  shape_of's tokens per workgroup go in steps, so its number of them falls
// here and there for a token more; this one never does, and a workspace of the longest sequence and largest batch serves all.
size_t most_partials(int B, long long N, int C) {
  const size_t per = C <= 512 ? 4 : 1, per_cu = C <= 512 ? 8 : (C <= 1536 ? 4 : (C <= 4096 ? 2 : 1));
  const size_t by_tokens = B * (((size_t)N + per - 1) / per), by_cus = lfh::num_cu() * per_cu + B + B * ((size_t)N >> 20);
  return by_tokens < by_cus ? by_tokens : by_cus;
}

}  // namespace

extern "C" {

int linfusion_gate_norm_fwd(const void* x, const void* f, const float* gate, const float* scale, const float* shift,
                            const float* w_pre, const float* w_post, void* y, void* h, int B, long long N, int C,
                            int dtype, float residual_scale, float norm_eps, unsigned flags, const int* lengths,
                            const long long strides[4][2], long long mod_stride, void* stream) {
  if (!x || (!y && !h)) return LINFUSION_ERR_INVALID;
  int rc = check_sizes(B, N, C, dtype);
  if (rc != LINFUSION_OK) return rc;
  if (flags & ~(LINFUSION_FLAG_NORM_RMS | LINFUSION_FLAG_NORM_POST)) return LINFUSION_ERR_INVALID;
  const bool rms = (flags & LINFUSION_FLAG_NORM_RMS) != 0, post = (flags & LINFUSION_FLAG_NORM_POST) != 0;
  if ((post || gate) && !f) return LINFUSION_ERR_INVALID;
  if (w_post && !post) return LINFUSION_ERR_INVALID;
  if (!(norm_eps > 0.0f) || std::isinf(norm_eps) || !std::isfinite(residual_scale)) return LINFUSION_ERR_INVALID;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2;
  View vx, vf, vy, vh;
  if ((rc = make_view(x, strides ? strides[0] : nullptr, B, N, C, esz, false, &vx)) != LINFUSION_OK) return rc;
  if ((rc = make_view(f, strides ? strides[1] : nullptr, B, N, C, esz, false, &vf)) != LINFUSION_OK) return rc;
  if ((rc = make_view(y, strides ? strides[2] : nullptr, B, N, C, esz, true, &vy)) != LINFUSION_OK) return rc;
  if ((rc = make_view(h, strides ? strides[3] : nullptr, B, N, C, esz, true, &vh)) != LINFUSION_OK) return rc;
  if ((rc = check_vectors(C, mod_stride, {gate, scale, shift}, {w_pre, w_post})) != LINFUSION_OK) return rc;
  if ((uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  // y may be x itself: a token is read whole by the threads that write it
  if ((meet(vy, vx) && !same_rows(vy, vx)) || meet(vy, vf) || meet(vh, vx) || meet(vh, vf) || meet(vh, vy))
    return LINFUSION_ERR_OVERLAP;
  for (const View* o : {&vy, &vh}) {
    if (!o->p) continue;
    for (const float* m : {gate, scale, shift})
      if (m && overlaps(o->p, o->bytes, m, mod_bytes(B, C, mod_stride))) return LINFUSION_ERR_OVERLAP;
    for (const float* w : {w_pre, w_post})
      if (w && overlaps(o->p, o->bytes, w, (size_t)C * 4)) return LINFUSION_ERR_OVERLAP;
    if (lengths && overlaps(o->p, o->bytes, lengths, (size_t)B * 4)) return LINFUSION_ERR_OVERLAP;
  }
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const Shape s = shape_of(B, N, C, false);
  const lf::GateNormArgs a{x, f, y, h, dev(vx), dev(vf), dev(vy), dev(vh), gate, scale, shift, w_pre, w_post,
                           mod_stride, lengths, N, C, s.rows, residual_scale, norm_eps};
  const hipStream_t st = (hipStream_t)stream;
  rc = dtype == LINFUSION_DTYPE_F16   ? run_fwd<lf::F16>(a, B, s, rms, post, st)
       : dtype == LINFUSION_DTYPE_BF16 ? run_fwd<lf::BF16>(a, B, s, rms, post, st)
                                       : run_fwd<lf::F32>(a, B, s, rms, post, st);
  if (rc != LINFUSION_OK) return rc;
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

size_t linfusion_gate_norm_bwd_workspace_bytes(int B, long long N, int C) {
  if (check_sizes(B, N, C, LINFUSION_DTYPE_F32) != LINFUSION_OK) return 0;
  return up(most_partials(B, N, C) * 3 * C * 4) + up((size_t)B * 3 * C * 4);
}

int linfusion_gate_norm_bwd(const void* x, const void* f, const float* gate, const float* scale, const float* w_pre,
                            const float* w_post, const void* dy, const void* dh, void* dx, void* df, float* dgate,
                            float* dscale, float* dshift, float* dw_pre, float* dw_post, int B, long long N, int C,
                            int dtype, float residual_scale, float norm_eps, unsigned flags, const int* lengths,
                            const long long strides[6][2], long long mod_stride, long long dmod_stride,
                            void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || (!dy && !dh)) return LINFUSION_ERR_INVALID;
  if (!dx && !df && !dgate && !dscale && !dshift && !dw_pre && !dw_post) return LINFUSION_ERR_INVALID;
  int rc = check_sizes(B, N, C, dtype);
  if (rc != LINFUSION_OK) return rc;
  if (flags & ~(LINFUSION_FLAG_NORM_RMS | LINFUSION_FLAG_NORM_POST)) return LINFUSION_ERR_INVALID;
  const bool rms = (flags & LINFUSION_FLAG_NORM_RMS) != 0, post = (flags & LINFUSION_FLAG_NORM_POST) != 0;
  if ((post || gate || df || dgate) && !f) return LINFUSION_ERR_INVALID;
  if ((w_post || dw_post) && !post) return LINFUSION_ERR_INVALID;
  if (!(norm_eps > 0.0f) || std::isinf(norm_eps) || !std::isfinite(residual_scale)) return LINFUSION_ERR_INVALID;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2;
  View vx, vf, vdy, vdh, vdx, vdf;
  auto st2 = [&](int i) { return strides ? strides[i] : nullptr; };
  if ((rc = make_view(x, st2(0), B, N, C, esz, false, &vx)) != LINFUSION_OK) return rc;
  if ((rc = make_view(f, st2(1), B, N, C, esz, false, &vf)) != LINFUSION_OK) return rc;
  if ((rc = make_view(dy, st2(2), B, N, C, esz, false, &vdy)) != LINFUSION_OK) return rc;
  if ((rc = make_view(dh, st2(3), B, N, C, esz, false, &vdh)) != LINFUSION_OK) return rc;
  if ((rc = make_view(dx, st2(4), B, N, C, esz, true, &vdx)) != LINFUSION_OK) return rc;
  if ((rc = make_view(df, st2(5), B, N, C, esz, true, &vdf)) != LINFUSION_OK) return rc;
  if ((rc = check_vectors(C, mod_stride, {gate, scale}, {w_pre, w_post})) != LINFUSION_OK) return rc;
  if ((rc = check_vectors(C, dmod_stride, {dgate, dscale, dshift}, {dw_pre, dw_post})) != LINFUSION_OK) return rc;
  const bool shared = mod_stride == 0;
  if (!shared && B > 1 && dmod_stride < C && (dgate || dscale || dshift)) return LINFUSION_ERR_OVERLAP;
  if ((uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  if (meet(vdx, vx) || meet(vdx, vf) || meet(vdx, vdh) || (meet(vdx, vdy) && !same_rows(vdx, vdy)) || meet(vdf, vx) ||
      meet(vdf, vf) || meet(vdf, vdy) || meet(vdf, vdh) || meet(vdf, vdx))
    return LINFUSION_ERR_OVERLAP;
  // every written range against every other range: the tensors, the vectors, the workspace
  const size_t need = linfusion_gate_norm_bwd_workspace_bytes(B, N, C);
  const bool sums = dgate || dscale || dshift || dw_pre || dw_post;
  struct Range { const void* p; size_t n; };
  const size_t mb = mod_bytes(B, C, mod_stride), dmb = shared ? (size_t)C * 4 : mod_bytes(B, C, dmod_stride), cb = (size_t)C * 4;
  const Range reads[] = {{x, vx.bytes}, {f, vf.bytes}, {dy, vdy.bytes}, {dh, vdh.bytes}, {gate, mb}, {scale, mb},
                         {w_pre, cb}, {w_post, cb}, {lengths, (size_t)B * 4}};
  const Range vectors[] = {{dgate, dmb}, {dscale, dmb}, {dshift, dmb}, {dw_pre, cb}, {dw_post, cb}};
  const Range rows[] = {{dx, vdx.bytes}, {df, vdf.bytes}};
  for (int i = 0; i < 5; ++i) {
    if (!vectors[i].p) continue;
    // (interleaved modulation gradients, columns of one [B, 3 C] buffer, share a span but no element)
    const bool spread = i < 3 && !shared && dmod_stride > C;
    for (const Range& r : reads)
      if (r.p && overlaps(vectors[i].p, vectors[i].n, r.p, r.n)) return LINFUSION_ERR_OVERLAP;
    for (const Range& r : rows)
      if (r.p && overlaps(vectors[i].p, vectors[i].n, r.p, r.n)) return LINFUSION_ERR_OVERLAP;
    for (int j = i + 1; j < 5; ++j) {
      if (!vectors[j].p || !overlaps(vectors[i].p, vectors[i].n, vectors[j].p, vectors[j].n)) continue;
      if (!(spread && j < 3)) return LINFUSION_ERR_OVERLAP;
      const long long apart = ((const char*)vectors[j].p - (const char*)vectors[i].p) / 4;
      const long long m = ((apart % dmod_stride) + dmod_stride) % dmod_stride;
      if (m < C || dmod_stride - m < C) return LINFUSION_ERR_OVERLAP;
    }
  }
  for (const Range& r : rows) {
    if (!r.p) continue;
    for (int i = 4; i < 9; ++i)
      if (reads[i].p && overlaps(r.p, r.n, reads[i].p, reads[i].n)) return LINFUSION_ERR_OVERLAP;
  }
  if (sums) {
    if (!workspace || workspace_bytes < need) return LINFUSION_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return LINFUSION_ERR_MISALIGNED;
    for (const Range& r : reads)
      if (r.p && overlaps(workspace, need, r.p, r.n)) return LINFUSION_ERR_OVERLAP;
    for (const Range& r : vectors)
      if (r.p && overlaps(workspace, need, r.p, r.n)) return LINFUSION_ERR_OVERLAP;
    for (const Range& r : rows)
      if (r.p && overlaps(workspace, need, r.p, r.n)) return LINFUSION_ERR_OVERLAP;
  }
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const Shape s = shape_of(B, N, C, true);
  float* partials = sums ? (float*)workspace : nullptr;
  float* total = sums ? (float*)((char*)workspace + up((size_t)B * s.wgs * 3 * C * 4)) : nullptr;
  const lf::GateNormBwdArgs a{x, f, dy, dh, dx, df, dev(vx), dev(vf), dev(vdy), dev(vdh), dev(vdx), dev(vdf), gate, scale,
                              w_pre, w_post, mod_stride, lengths, partials, N, C, s.rows, residual_scale, norm_eps};
  const hipStream_t st = (hipStream_t)stream;
  rc = dtype == LINFUSION_DTYPE_F16   ? run_bwd<lf::F16>(a, B, s, rms, post, st)
       : dtype == LINFUSION_DTYPE_BF16 ? run_bwd<lf::BF16>(a, B, s, rms, post, st)
                                       : run_bwd<lf::F32>(a, B, s, rms, post, st);
  if (rc != LINFUSION_OK) return rc;
  if (sums) {
    const bool over_batch = shared || dw_pre || dw_post;
    const lf::GateNormVectors v{partials, over_batch ? total : nullptr, gate, scale, w_pre, w_post, dgate, dscale, dshift, dw_pre, dw_post,
                                mod_stride, dmod_stride, B, C, s.wgs, shared};
    lf::gate_norm_sums<<<dim3((C + 63) / 64, 3, B), dim3(1024), 0, st>>>(v);
    if (over_batch) lf::gate_norm_vectors<<<dim3((C + 63) / 64), dim3(64), 0, st>>>(v);
  }
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

}  // extern "C"
