// The gated delta rule (lf_delta.hpp, lf_delta_bwd.hpp, lf_delta_step.hpp): checks, workspace layout, launches.
#include "../../include/linfusion.h"

#include <stdint.h>

#include <cmath>

#include "lf_delta.hpp"
#include "lf_delta_bwd.hpp"
#include "lf_delta_step.hpp"
#include "lf_host_api.hpp"

namespace {

using lfh::overlaps;

constexpr int kMaxKey = 160, kMaxValue = 256;

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

struct Sizes {
  long long nc, heads;   // chunks of N tokens; B * H
  int dkb, dvb, dks, runs, run;
  size_t esz;
  size_t at_kt, at_u, at_s, at_decay, at_wt, at_tt, at_kn, at_ds;   // bytes into a record
  size_t record, record_saved, record_b;                            // bytes of one
  size_t parts, joined;
  size_t forward() const { return (size_t)heads * nc * record + parts + joined; }
  size_t saved() const { return (size_t)heads * nc * record_saved + parts + joined; }
  size_t backward() const { return (size_t)heads * (nc + 2) * record_b; }
};

int make_sizes(int B, int H, int H_k, long long N, int dk, int dv, int dtype, Sizes* z) {
  if (B <= 0 || H <= 0 || H_k <= 0 || N <= 0 || dk <= 0 || dv <= 0) return LINFUSION_ERR_INVALID;
  if ((long long)B * H > 65535 || H % H_k || N >= 1LL << 30) return LINFUSION_ERR_INVALID;
  if (dtype != LINFUSION_DTYPE_F32 && dtype != LINFUSION_DTYPE_F16 && dtype != LINFUSION_DTYPE_BF16)
    return LINFUSION_ERR_UNSUPPORTED;
  if (dk % 8 || dv % 8 || dk > kMaxKey || dv > kMaxValue) return LINFUSION_ERR_UNSUPPORTED;
  z->nc = (N + lf::kDeltaChunk - 1) / lf::kDeltaChunk;
  z->heads = (long long)B * H;
  z->dkb = (dk + 15) / 16;
  z->dvb = (dv + 15) / 16;
  z->esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2;
  z->dks = (dk + 31) / 32;
  const size_t terms = dtype == LINFUSION_DTYPE_F32 ? 3 : (dtype == LINFUSION_DTYPE_F16 ? 2 : 1), frag = lf::kFrag * 2;
  const size_t u = (size_t)z->dvb * 4096, state = (size_t)z->dvb * z->dkb * 1024;
  z->at_kt = 4 * z->dks * 3 * frag;
  z->at_u = z->at_kt + z->dkb * 2 * terms * frag;
  z->at_s = z->at_u + u;
  z->at_decay = z->at_s + state;
  z->record = up(z->at_decay + lf::kDecayBytes);
  z->at_wt = z->record;
  z->at_tt = z->at_wt + z->dkb * 2 * 3 * frag;
  z->record_saved = up(z->at_tt + 6 * lf::kFrag * 4);
  z->at_kn = u;
  z->at_ds = z->at_kn + 4 * z->dks * terms * frag;
  z->record_b = up(z->at_ds + state);
  // Runs: as many as give every CU a workgroup of the second pass, of 8 chunks at least; each costs delta_join a step, and the first
  // pass does (d_k + d_v) / d_v times the work of the second.  us of the scans in runs : in one, bf16, heads of 64: 64 x 4096 tokens in 2
  // 141 : 103, 40 x 4096 in 3 103 : 85, 32 x 8192 in 4 162 : 164, 24 x 8192 in 5 127 : 145, 20 x 8192 in 6 106 : 130; heads of 128: 16 x
  // 8192 in 4 306 : 264, 8 x 8192 in 8 182 : 210.  In 5 of 8 chunks, 4 x 2560 tokens, heads of 64: 26 : 36.
  const long long slices = (z->dvb + 1) / 2, few = z->nc / 8 < 32 ? z->nc / 8 : 32;
  long long runs = lfh::num_cu() / (z->heads * slices);
  if (runs > few) runs = few;
  if (runs < 5) runs = 1;
  z->run = (int)((z->nc + runs - 1) / runs);
  z->runs = (int)((z->nc + z->run - 1) / z->run);
  // Runs come and go with the rounding of `run` and with the heads; memory is for as many as any smaller call has.
  long long most = few < 5 ? 0 : z->heads * few;
  if (most > lfh::num_cu() / slices) most = lfh::num_cu() / slices;
  const size_t blocks = (size_t)most * z->dkb * 1024;
  z->parts = up(blocks * (z->dvb + z->dkb));
  z->joined = up(blocks * z->dvb);
  return LINFUSION_OK;
}

// What a call reads or writes; `same`: the one range it may coincide with; a view's `rows` may lie between another's.
struct Range { const void* p; size_t n; bool written; const void* same; lfh::Places rows; };
Range plain(const void* p, size_t n, bool written, const void* same = nullptr) { return Range{p, n, written, same, lfh::Places{}}; }

bool clash(const Range* r, int n) {
  for (int i = 0; i < n; ++i)
    for (int j = i + 1; j < n; ++j) {
      if (!r[i].p || !r[j].p || !(r[i].written || r[j].written)) continue;
      if (!overlaps(r[i].p, r[i].n, r[j].p, r[j].n)) continue;
      if (r[i].p == r[j].p && r[i].n == r[j].n && (r[i].same == r[j].p && r[i].same)) continue;
      if (r[i].rows.width && r[j].rows.width && lfh::apart(r[i].rows, r[j].rows)) continue;
      return true;
    }
  return false;
}

// rows of `d` channels of the tensors' type
int check_rows(const void* p, const long long* given, int B, int H, long long N, int d, size_t esz, bool written,
               lf::DeltaView* v, Range* range) {
  long long s[3] = {H * N * d, N * d, d};
  const long long extent[3] = {B, H, N};
  for (int i = 0; i < 3; ++i)
    if (extent[i] == 1) s[i] = 0;   // (never used, whatever it says)
    else if (given) s[i] = given[i];
  if ((uintptr_t)p & 15) return LINFUSION_ERR_MISALIGNED;
  const int rc = lfh::check_strides(s, B, H, N, d, esz, written);
  if (rc != LINFUSION_OK) return rc;
  *v = lf::DeltaView{s[0], s[1], s[2]};
  *range = Range{p, lfh::span_bytes(s, B, H, N, d, esz), written, nullptr, lfh::places(p, s, B, H, N, d, esz)};
  return LINFUSION_OK;
}

// two tensors of one fp32 value per token and head, at any strides: judged as rows of four at four times the strides
int check_scalars(const void* p0, const void* p1, const long long* given, int B, int H, long long N, bool written,
                  lf::DeltaView* v, Range* range0, Range* range1) {
  long long s[3] = {H * N, N, 1};
  const long long extent[3] = {B, H, N};
  for (int i = 0; i < 3; ++i)
    if (extent[i] == 1) s[i] = 0;
    else if (given) s[i] = given[i];
  if (((uintptr_t)p0 | (uintptr_t)p1) & 3) return LINFUSION_ERR_MISALIGNED;
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] >= 1LL << 44) return LINFUSION_ERR_INVALID;
  const long long wide[3] = {4 * s[0], 4 * s[1], 4 * s[2]};
  const int rc = lfh::check_strides(wide, B, H, N, 4, 4, written);
  if (rc != LINFUSION_OK) return rc;
  *v = lf::DeltaView{s[0], s[1], s[2]};
  const size_t bytes = (size_t)((B - 1) * s[0] + (H - 1) * s[1] + (N - 1) * s[2] + 1) * 4;
  *range0 = Range{p0, bytes, written, nullptr, lfh::places(p0, s, B, H, N, 1, 4)};
  *range1 = Range{p1, bytes, written, nullptr, lfh::places(p1, s, B, H, N, 1, 4)};
  return LINFUSION_OK;
}

void place_forward(lf::DeltaArgs* a, const Sizes& z, void* at, bool for_backward) {
  a->record = static_cast<unsigned char*>(at);
  a->size = (unsigned)(for_backward ? z.record_saved : z.record);
  a->for_backward = for_backward;
  a->at_kt = (unsigned)z.at_kt;
  a->at_u = (unsigned)z.at_u;
  a->at_s = (unsigned)z.at_s;
  a->at_decay = (unsigned)z.at_decay;
  a->at_wt = (unsigned)z.at_wt;
  a->at_tt = (unsigned)z.at_tt;
  a->parts = reinterpret_cast<float*>(a->record + (size_t)z.heads * z.nc * a->size);
  a->joined = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(a->parts) + z.parts);
}

void place_backward(lf::DeltaArgs* a, const Sizes& z, void* at) {
  a->record_b = static_cast<unsigned char*>(at);
  a->size_b = (unsigned)z.record_b;
  a->at_kn = (unsigned)z.at_kn;
  a->at_ds = (unsigned)z.at_ds;
}

#define LF_FOR_STEPS(X)                                                                           \
  switch (a.dks) {                                                                                \
    case 1: X(1) break;                                                                           \
    case 2: X(2) break;                                                                           \
    case 3: X(3) break;                                                                           \
    case 4: X(4) break;                                                                           \
    default: X(5) break;                                                                          \
  }

// 32 value channels a workgroup where that still gives three quarters of the CUs one: the slices' common reads from the L2 halve.  us a
// call with 16 / 32: 10 heads of 64, 65536 tokens 813 / 720, 96 heads of 40, 4096 tokens, forward and backward 843 / 821; with fewer
// workgroups it would leave CUs idle along a chain that is no shorter.
template <int NI, int KS, bool PARTIAL> void launch_scan(const lf::DeltaArgs& a, int slices, int runs, hipStream_t st) {
  const int pairs = (slices + 1) / 2;
  if (slices > 1 && 4LL * pairs * a.heads * runs >= 3LL * lfh::num_cu())
    lf::delta_scan<NI, KS, 2, PARTIAL><<<dim3(pairs * a.heads, runs), dim3(256), 0, st>>>(a);
  else
    lf::delta_scan<NI, KS, 1, PARTIAL><<<dim3(slices * a.heads, runs), dim3(256), 0, st>>>(a);
}

template <typename T, int KS> int launch_states(const lf::DeltaArgs& a, int BH, hipStream_t st) {
  constexpr int NI = lf::TermsOf<T>::kStored;
  const int lds = lf::delta_prepare_lds<T>(KS, (a.dvb + 1) / 2);
  auto prepare = lf::delta_prepare<T, KS>;
  if (!lfh::allow_lds(prepare, lds)) return LINFUSION_ERR_HIP;
  prepare<<<dim3(a.nc, BH), dim3(256), lds, st>>>(a);
  if (a.runs > 1) {
    launch_scan<NI, KS, true>(a, a.dvb + a.dkb, a.runs - 1, st);
    lf::delta_join<KS><<<dim3(a.dvb, BH), dim3(256), 0, st>>>(a);
  }
  launch_scan<NI, KS, false>(a, a.dvb, a.runs, st);
  return LINFUSION_OK;
}

// operands, U, the states and the decays of all chunks
template <typename T> int run_states(const lf::DeltaArgs& a, int BH, hipStream_t st) {
  int rc = LINFUSION_OK;
#define X(KS) rc = launch_states<T, KS>(a, BH, st);
  LF_FOR_STEPS(X)
#undef X
  return rc;
}

template <typename T, int KS> int launch_out(const lf::DeltaArgs& a, int BH, hipStream_t st) {
  const int lds = lf::delta_out_lds<T>(KS);
  auto kernel = lf::delta_out<T, KS>;
  if (!lfh::allow_lds(kernel, lds)) return LINFUSION_ERR_HIP;
  kernel<<<dim3(a.nc, BH), dim3(256), lds, st>>>(a);
  return LINFUSION_OK;
}

template <typename T> int run_fwd(const lf::DeltaArgs& a, int BH, hipStream_t st) {
  int rc = run_states<T>(a, BH, st);
  if (rc != LINFUSION_OK) return rc;
#define X(KS) rc = launch_out<T, KS>(a, BH, st);
  LF_FOR_STEPS(X)
#undef X
  return rc;
}

template <typename T, int KS, bool SHARED> int launch_gradients(const lf::DeltaArgs& a, int B, hipStream_t st) {
  const int lds = lf::delta_gradients_lds<T>(KS);
  auto kernel = lf::delta_gradients<T, KS, SHARED>;
  if (!lfh::allow_lds(kernel, lds)) return LINFUSION_ERR_HIP;
  kernel<<<dim3(a.nc, B * a.Hk), dim3(512), lds, st>>>(a);
  return LINFUSION_OK;
}

template <typename T, int KS> int launch_bwd(const lf::DeltaArgs& a, int B, hipStream_t st) {
  constexpr int NI = lf::TermsOf<T>::kStored;
  const int BH = B * a.H, lds = lf::delta_back_prepare_lds<T>(KS, (a.dvb + 1) / 2);
  auto prepare = lf::delta_back_prepare<T, KS>;
  if (!lfh::allow_lds(prepare, lds)) return LINFUSION_ERR_HIP;
  prepare<<<dim3(a.nc, BH), dim3(256), lds, st>>>(a);
  lf::delta_back_scan<NI, KS><<<dim3(a.dvb * BH), dim3(256), 0, st>>>(a);
  return a.H == a.Hk ? launch_gradients<T, KS, false>(a, B, st) : launch_gradients<T, KS, true>(a, B, st);
}

template <typename T> int run_bwd(const lf::DeltaArgs& a, int B, bool states, hipStream_t st) {
  int rc = LINFUSION_OK;
  if (states && (rc = run_states<T>(a, B * a.H, st)) != LINFUSION_OK) return rc;
#define X(KS) rc = launch_bwd<T, KS>(a, B, st);
  LF_FOR_STEPS(X)
#undef X
  return rc;
}

template <typename T, int ROWS> void launch_step(const lf::DeltaStepArgs& a, int BH, hipStream_t st) {
  lf::delta_step<T, ROWS><<<dim3((a.dv + lf::kStepCols - 1) / lf::kStepCols, BH), dim3(256), 0, st>>>(a);
}
template <typename T> void run_step(const lf::DeltaStepArgs& a, int BH, hipStream_t st) {
  if (a.dk <= 32) launch_step<T, 1>(a, BH, st);
  else if (a.dk <= 64) launch_step<T, 2>(a, BH, st);
  else if (a.dk <= 96) launch_step<T, 3>(a, BH, st);
  else if (a.dk <= 128) launch_step<T, 4>(a, BH, st);
  else launch_step<T, 5>(a, BH, st);
}

}  // namespace

extern "C" {

size_t linfusion_delta_workspace_bytes(int B, int H, int H_k, long long N, int d_k, int d_v, int dtype) {
  Sizes z;
  return make_sizes(B, H, H_k, N, d_k, d_v, dtype, &z) == LINFUSION_OK ? z.forward() : 0;
}

size_t linfusion_delta_saved_bytes(int B, int H, int H_k, long long N, int d_k, int d_v, int dtype) {
  Sizes z;
  return make_sizes(B, H, H_k, N, d_k, d_v, dtype, &z) == LINFUSION_OK ? z.saved() : 0;
}

size_t linfusion_delta_bwd_workspace_bytes(int B, int H, int H_k, long long N, int d_k, int d_v, int dtype) {
  Sizes z;
  return make_sizes(B, H, H_k, N, d_k, d_v, dtype, &z) == LINFUSION_OK ? z.saved() + z.backward() : 0;
}

int linfusion_delta_fwd(const void* q, const void* k, const void* v, const float* g, const float* beta,
                        const float* state_in, void* out, float* state_out, const int* lengths, void* saved,
                        size_t saved_bytes, int B, int H, int H_k, long long N, int d_k, int d_v, int dtype, float scale,
                        unsigned flags, const long long q_strides[3], const long long k_strides[3],
                        const long long v_strides[3], const long long out_strides[3], const long long gate_strides[3],
                        void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !g || !beta || !out) return LINFUSION_ERR_INVALID;
  if (flags || !std::isfinite(scale)) return LINFUSION_ERR_INVALID;
  Sizes z;
  int rc = make_sizes(B, H, H_k, N, d_k, d_v, dtype, &z);
  if (rc != LINFUSION_OK) return rc;
  lf::DeltaArgs a{};
  Range rq, rk, rv, ro, rg, rb;
  if ((rc = check_rows(q, q_strides, B, H_k, N, d_k, z.esz, false, &a.vq, &rq)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(k, k_strides, B, H_k, N, d_k, z.esz, false, &a.vk, &rk)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(v, v_strides, B, H, N, d_v, z.esz, false, &a.vv, &rv)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(out, out_strides, B, H, N, d_v, z.esz, true, &a.vo, &ro)) != LINFUSION_OK) return rc;
  if ((rc = check_scalars(g, beta, gate_strides, B, H, N, false, &a.vg, &rg, &rb)) != LINFUSION_OK) return rc;
  if (((uintptr_t)state_in | (uintptr_t)state_out | (uintptr_t)saved) & 15) return LINFUSION_ERR_MISALIGNED;
  if ((uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  if (saved && saved_bytes < z.saved()) return LINFUSION_ERR_WORKSPACE;
  if (!saved) {
    if (!workspace || workspace_bytes < z.forward()) return LINFUSION_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return LINFUSION_ERR_MISALIGNED;
  }
  const size_t ns = (size_t)z.heads * d_k * d_v * 4;
  const Range ranges[] = {rq, rk, rv, rg, rb, ro, plain(lengths, (size_t)B * 4, false), plain(state_in, ns, false, state_out),
                          plain(state_out, ns, true, state_in),
                          saved ? plain(saved, z.saved(), true) : plain(workspace, z.forward(), true)};
  if (clash(ranges, 10)) return LINFUSION_ERR_OVERLAP;
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta;
  a.state_in = state_in; a.out = out; a.state_out = state_out; a.lengths = lengths;
  a.N = N; a.H = H; a.Hk = H_k; a.heads = (int)z.heads; a.nc = (int)z.nc; a.runs = z.runs; a.run = z.run;
  a.dk = d_k; a.dv = d_v; a.dkb = z.dkb; a.dvb = z.dvb; a.dks = z.dks; a.scale = scale;
  place_forward(&a, z, saved ? saved : workspace, saved != nullptr);
  const hipStream_t st = (hipStream_t)stream;
  const int BH = (int)z.heads;
  rc = dtype == LINFUSION_DTYPE_F16   ? run_fwd<lf::F16>(a, BH, st)
       : dtype == LINFUSION_DTYPE_BF16 ? run_fwd<lf::BF16>(a, BH, st)
                                       : run_fwd<lf::F32>(a, BH, st);
  if (rc != LINFUSION_OK) return rc;
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

int linfusion_delta_bwd(const void* q, const void* k, const void* v, const float* g, const float* beta,
                        const float* state_in, const void* dout, const float* dstate_out, const void* saved,
                        size_t saved_bytes, void* dq, void* dk, void* dv, float* dg, float* dbeta, float* dstate_in,
                        const int* lengths, int B, int H, int H_k, long long N, int d_k, int d_v, int dtype, float scale,
                        unsigned flags, const long long q_strides[3], const long long k_strides[3],
                        const long long v_strides[3], const long long gate_strides[3], const long long dout_strides[3],
                        const long long dq_strides[3], const long long dk_strides[3], const long long dv_strides[3],
                        const long long dgate_strides[3], void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !g || !beta || !dout || !dq || !dk || !dv || !dg || !dbeta) return LINFUSION_ERR_INVALID;
  if (flags || !std::isfinite(scale)) return LINFUSION_ERR_INVALID;
  Sizes z;
  int rc = make_sizes(B, H, H_k, N, d_k, d_v, dtype, &z);
  if (rc != LINFUSION_OK) return rc;
  lf::DeltaArgs a{};
  Range rq, rk, rv, rg, rb, rdo, rdq, rdk, rdv, rdg, rdb;
  if ((rc = check_rows(q, q_strides, B, H_k, N, d_k, z.esz, false, &a.vq, &rq)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(k, k_strides, B, H_k, N, d_k, z.esz, false, &a.vk, &rk)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(v, v_strides, B, H, N, d_v, z.esz, false, &a.vv, &rv)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(dout, dout_strides, B, H, N, d_v, z.esz, false, &a.vdo, &rdo)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(dq, dq_strides, B, H_k, N, d_k, z.esz, true, &a.vdq, &rdq)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(dk, dk_strides, B, H_k, N, d_k, z.esz, true, &a.vdk, &rdk)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(dv, dv_strides, B, H, N, d_v, z.esz, true, &a.vdv, &rdv)) != LINFUSION_OK) return rc;
  if ((rc = check_scalars(g, beta, gate_strides, B, H, N, false, &a.vg, &rg, &rb)) != LINFUSION_OK) return rc;
  if ((rc = check_scalars(dg, dbeta, dgate_strides, B, H, N, true, &a.vdg, &rdg, &rdb)) != LINFUSION_OK) return rc;
  if (((uintptr_t)state_in | (uintptr_t)dstate_out | (uintptr_t)dstate_in | (uintptr_t)saved) & 15)
    return LINFUSION_ERR_MISALIGNED;
  if ((uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  if (saved && saved_bytes < z.saved()) return LINFUSION_ERR_WORKSPACE;
  const size_t need = z.backward() + (saved ? 0 : z.saved());
  if (!workspace || workspace_bytes < need) return LINFUSION_ERR_WORKSPACE;
  if ((uintptr_t)workspace & 15) return LINFUSION_ERR_MISALIGNED;
  const size_t ns = (size_t)z.heads * d_k * d_v * 4;
  const Range ranges[] = {rq, rk, rv, rg, rb, rdo, rdq, rdk, rdv, rdg, rdb, plain(lengths, (size_t)B * 4, false),
                          plain(state_in, ns, false), plain(saved, z.saved(), false), plain(dstate_out, ns, false, dstate_in),
                          plain(dstate_in, ns, true, dstate_out), plain(workspace, need, true)};
  if (clash(ranges, 17)) return LINFUSION_ERR_OVERLAP;
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta;
  a.state_in = state_in; a.lengths = lengths; a.dout = dout; a.dstate_out = dstate_out;
  a.dq = dq; a.dk_out = dk; a.dv_out = dv; a.dg = dg; a.dbeta = dbeta; a.dstate_in = dstate_in;
  a.N = N; a.H = H; a.Hk = H_k; a.heads = (int)z.heads; a.nc = (int)z.nc; a.runs = z.runs; a.run = z.run;
  a.dk = d_k; a.dv = d_v; a.dkb = z.dkb; a.dvb = z.dvb; a.dks = z.dks; a.scale = scale;
  place_backward(&a, z, workspace);
  place_forward(&a, z, saved ? const_cast<void*>(saved) : static_cast<unsigned char*>(workspace) + z.backward(), true);
  const hipStream_t st = (hipStream_t)stream;
  rc = dtype == LINFUSION_DTYPE_F16   ? run_bwd<lf::F16>(a, B, !saved, st)
       : dtype == LINFUSION_DTYPE_BF16 ? run_bwd<lf::BF16>(a, B, !saved, st)
                                       : run_bwd<lf::F32>(a, B, !saved, st);
  if (rc != LINFUSION_OK) return rc;
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

int linfusion_delta_step(const void* q, const void* k, const void* v, const float* g, const float* beta,
                         const float* state_in, float* state_out, void* out, int B, int H, int H_k, int d_k, int d_v,
                         int dtype, float scale, unsigned flags, const long long q_strides[2],
                         const long long k_strides[2], const long long v_strides[2], const long long out_strides[2],
                         const long long gate_strides[2], void* stream) {
  if (!q || !k || !v || !g || !beta || !state_out || !out) return LINFUSION_ERR_INVALID;
  if (flags || !std::isfinite(scale)) return LINFUSION_ERR_INVALID;
  Sizes z;
  int rc = make_sizes(B, H, H_k, 1, d_k, d_v, dtype, &z);
  if (rc != LINFUSION_OK) return rc;
  lf::DeltaView vq, vk, vv, vo, vg;
  Range rq, rk, rv, ro, rg, rb;
  struct Three { long long s[3]; };
  auto three = [](const long long* s, int heads, int d) {
    return s ? Three{{s[0], s[1], 0}} : Three{{(long long)heads * d, d, 0}};
  };
  if ((rc = check_rows(q, three(q_strides, H_k, d_k).s, B, H_k, 1, d_k, z.esz, false, &vq, &rq)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(k, three(k_strides, H_k, d_k).s, B, H_k, 1, d_k, z.esz, false, &vk, &rk)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(v, three(v_strides, H, d_v).s, B, H, 1, d_v, z.esz, false, &vv, &rv)) != LINFUSION_OK) return rc;
  if ((rc = check_rows(out, three(out_strides, H, d_v).s, B, H, 1, d_v, z.esz, true, &vo, &ro)) != LINFUSION_OK) return rc;
  if ((rc = check_scalars(g, beta, three(gate_strides, H, 1).s, B, H, 1, false, &vg, &rg, &rb)) != LINFUSION_OK) return rc;
  if (((uintptr_t)state_in | (uintptr_t)state_out) & 15) return LINFUSION_ERR_MISALIGNED;
  const size_t ns = (size_t)z.heads * d_k * d_v * 4;
  const Range ranges[] = {rq, rk, rv, rg, rb, ro, plain(state_in, ns, false, state_out), plain(state_out, ns, true, state_in)};
  if (clash(ranges, 8)) return LINFUSION_ERR_OVERLAP;
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const lf::DeltaStepArgs a{q, k, v, g, beta, state_in, out, state_out, vq.b, vq.h, vk.b, vk.h, vv.b, vv.h,
                            vg.b, vg.h, vo.b, vo.h, H, H_k, d_k, d_v, scale};
  const hipStream_t st = (hipStream_t)stream;
  const int BH = (int)z.heads;
  if (dtype == LINFUSION_DTYPE_F16) run_step<lf::F16>(a, BH, st);
  else if (dtype == LINFUSION_DTYPE_BF16) run_step<lf::BF16>(a, BH, st);
  else run_step<lf::F32>(a, BH, st);
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

}  // extern "C"
