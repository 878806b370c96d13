// The gated linear recurrence (lf_scan.hpp): checks, launches, entry points.
#include "lf_rows_api.hpp"
#include "lf_scan.hpp"

#include <initializer_list>

namespace {

using lfh::meet;
using lfh::Range;
using lfh::row_view;
using lfh::RowView;
using lfh::span;

constexpr int kMaxChannels = 8192;
constexpr unsigned kFlags = LINFUSION_FLAG_SCAN_REVERSE | LINFUSION_FLAG_SCAN_LEAKY | LINFUSION_FLAG_SCAN_SUM;
int check(int B, long long N, int C, int dtype, unsigned flags) {
  if (B <= 0 || N <= 0 || C <= 0 || B > 65535 || N >= 1LL << 30) return LINFUSION_ERR_INVALID;
  if (dtype != LINFUSION_DTYPE_F32 && dtype != LINFUSION_DTYPE_F16 && dtype != LINFUSION_DTYPE_BF16) return LINFUSION_ERR_UNSUPPORTED;
  if (C % 8 || C > kMaxChannels) return LINFUSION_ERR_UNSUPPORTED;
  if (flags & ~kFlags || (flags & LINFUSION_FLAG_SCAN_LEAKY && flags & LINFUSION_FLAG_SCAN_SUM)) return LINFUSION_ERR_INVALID;
  return LINFUSION_OK;
}

int mode_of(unsigned flags) {
  return flags & LINFUSION_FLAG_SCAN_LEAKY ? lf::kScanLeaky : (flags & LINFUSION_FLAG_SCAN_SUM ? lf::kScanSum : lf::kScanNorm);
}

bool misaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if ((uintptr_t)p & 15) return true;
  return false;
}

// every output against everything else (but the states, of which an output may be the input itself)
bool clash(std::initializer_list<RowView> in, std::initializer_list<RowView> out, std::initializer_list<Range> read,
           std::initializer_list<Range> written) {
  for (const RowView* o = out.begin(); o != out.end(); ++o) {
    for (const RowView& v : in)
      if (meet(*o, v)) return true;
    for (const RowView* p = o + 1; p != out.end(); ++p)
      if (meet(*o, *p)) return true;
    for (const Range& r : read)
      if (meet(span(*o), r)) return true;
    for (const Range& r : written)
      if (meet(span(*o), r)) return true;
  }
  for (const Range* w = written.begin(); w != written.end(); ++w) {
    for (const RowView& v : in)
      if (meet(*w, span(v))) return true;
    for (const Range& r : read)
      if (meet(*w, r)) return true;
    for (const Range* p = w + 1; p != written.end(); ++p)
      if (meet(*w, *p)) return true;
  }
  return false;
}

lf::ScanView dev(const RowView& v) { return lf::ScanView{v.batch, v.token}; }

long long chunks_of(long long N) { return (N + lf::kScanChunk - 1) / lf::kScanChunk; }
size_t states(int B, long long N, int C) { return lfh::up256((size_t)B * chunks_of(N) * C * 4); }   // one value per chunk and channel

constexpr size_t kTicketBytes = 256;

// Chunks of a group, groups of a stretch: few mean many values that wait for one another, many that a chunk reads many totals (65536 x 1280 bf16
// in groups of 4 235 us, 8 172, 16 162, 32 164; 2^20 x 64 in stretches of 4 547 us, 8 226, 16 174).
int group_size() {
  const int g = lfh::env_int("LINFUSION_SCAN_GROUP", lf::kScanGroup);
  return g < 4 ? 4 : (g > lf::kScanGroup ? lf::kScanGroup : g);
}
// Whether the chain from group to group (1.8 us each) takes longer than the chunks themselves (16 ns each where all CUs have some): stretches
// then (bf16, 65536 x 64: 22 us, 67 by groups; 2^20 x 64: 174, 922), groups else (65536 x 1280: 162, stretches 10 % more).
constexpr int kNarrow = 8;   // chunks side by side
bool narrow(long long chunks, int B, int C) {
  return chunks > group_size() && (long long)B * ((C + lf::kScanWidth - 1) / lf::kScanWidth) < kNarrow;
}

// Time lanes of a row of up to 32 tokens where several share a workgroup, else 0 (bf16 forward, 65535 x 2 x 64: 23 us, 503 with a workgroup
// for every row; 6240 x 13 x 2048 285 us, 1.33 GB).
int packed(int B, long long N) {
  if (B == 1 || N > 32) return 0;
  int seg = 1;
  while (seg * lf::kScanT < N) seg *= 2;
  return seg;
}

lf::ScanRecords records(void* workspace, int B, long long N, int C) {
  char* w = (char*)workspace;
  return lf::ScanRecords{(unsigned*)w, (unsigned long long*)(w + kTicketBytes), (unsigned*)(w + kTicketBytes + 2 * states(B, N, C))};
}

void clear(const lf::ScanRecords& r, int B, long long chunks, int C, hipStream_t st) {
  const long long count = (long long)B * chunks * C;
  lf::scan_clear<<<(unsigned)((count / 2 + 255) / 256), 256, 0, st>>>(r, count);
}

long long tiles_of(long long chunks, int B, int C) { return chunks * ((C + lf::kScanWidth - 1) / lf::kScanWidth) * B; }

template <typename T, int MODE, bool INPUT, int TT, int CHAIN>
int forward(const lf::ScanArgs& a0, hipStream_t st) {
  lf::ScanArgs a = a0;
  const long long chunks = (a.N + 32 * TT - 1) / (32 * TT);
  const long long tiles = tiles_of(chunks, CHAIN == lf::kPacked ? lf::packed_tiles(a.B, a.seg) : a.B, a.C);
  if (tiles > 0x7fffffffLL) return LINFUSION_ERR_INVALID;
  a.chunks = (int)chunks;
  if constexpr (CHAIN == lf::kGroups || CHAIN == lf::kStretches) clear(a.rec, a.B, chunks, a.C, st);
  lf::scan_fwd<T, MODE, INPUT, TT, CHAIN><<<(unsigned)tiles, 256, 0, st>>>(a);
  return LINFUSION_OK;
}
// One chunk holds up to 128 tokens, or 256 of 16-bit types with eight a thread.
template <typename T, int MODE, bool INPUT>
int forward(const lf::ScanArgs& a, hipStream_t st) {
  constexpr int kLong = lf::Stored<T>::kBytes == 4 ? lf::kScanT : 2 * lf::kScanT;
  if (a.seg) return forward<T, MODE, INPUT, lf::kScanT, lf::kPacked>(a, st);
  if (a.N <= lf::kScanChunk) return forward<T, MODE, INPUT, lf::kScanT, lf::kAlone>(a, st);
  if (kLong > lf::kScanT && a.N <= 32 * kLong) return forward<T, MODE, INPUT, kLong, lf::kAlone>(a, st);
  if (narrow(chunks_of(a.N), a.B, a.C)) return forward<T, MODE, INPUT, lf::kScanT, lf::kStretches>(a, st);
  return forward<T, MODE, INPUT, lf::kScanT, lf::kGroups>(a, st);
}

template <typename T, int MODE, bool INPUT>
int backward(const lf::ScanBackArgs& a, hipStream_t st) {
  const long long tiles = tiles_of(a.chunks, a.seg ? lf::packed_tiles(a.B, a.seg) : a.B, a.C);
  if (tiles > 0x7fffffffLL) return LINFUSION_ERR_INVALID;
  if (a.seg) {
    lf::scan_bwd<T, MODE, INPUT, lf::kPacked><<<(unsigned)tiles, 256, 0, st>>>(a);
    return LINFUSION_OK;
  }
  if (a.chunks == 1) {
    lf::scan_bwd<T, MODE, INPUT, lf::kAlone><<<(unsigned)tiles, 256, 0, st>>>(a);
    return LINFUSION_OK;
  }
  clear(a.rec, a.B, a.chunks, a.C, st);
  if (narrow(a.chunks, a.B, a.C)) lf::scan_bwd<T, MODE, INPUT, lf::kStretches><<<(unsigned)tiles, 256, 0, st>>>(a);
  else lf::scan_bwd<T, MODE, INPUT, lf::kGroups><<<(unsigned)tiles, 256, 0, st>>>(a);
  return LINFUSION_OK;
}

template <typename T, int MODE, bool INPUT>
int step(const lf::ScanStepArgs& a, hipStream_t st) {
  lf::scan_step<T, MODE, INPUT><<<dim3((a.C + 511) / 512, a.B), 64, 0, st>>>(a);
  return LINFUSION_OK;
}

// `f` with the type, the weight's kind and whether there is a gate on the inputs as types
template <typename F> int with(int dtype, int mode, bool input, F f) {
  auto by_input = [&](auto t, auto m) { return input ? f(t, m, std::true_type{}) : f(t, m, std::false_type{}); };
  auto by_mode = [&](auto t) {
    return mode == lf::kScanLeaky ? by_input(t, std::integral_constant<int, lf::kScanLeaky>{})
           : mode == lf::kScanSum ? by_input(t, std::integral_constant<int, lf::kScanSum>{})
                                  : by_input(t, std::integral_constant<int, lf::kScanNorm>{});
  };
  return dtype == LINFUSION_DTYPE_F16 ? by_mode(lf::F16{}) : dtype == LINFUSION_DTYPE_BF16 ? by_mode(lf::BF16{}) : by_mode(lf::F32{});
}

int launch_forward(const lf::ScanArgs& a, int dtype, int mode, hipStream_t st) {
  return with(dtype, mode, a.input != nullptr, [&](auto t, auto m, auto i) {
    return forward<decltype(t), decltype(m)::value, decltype(i)::value>(a, st);
  });
}

}  // namespace

extern "C" {

size_t linfusion_scan_workspace_bytes(int B, long long N, int C) {
  if (check(B, N, C, LINFUSION_DTYPE_F32, 0) != LINFUSION_OK) return 0;
  return N <= lf::kScanChunk ? 0 : kTicketBytes + 3 * states(B, N, C);
}

size_t linfusion_scan_saved_bytes(int B, long long N, int C) {
  if (check(B, N, C, LINFUSION_DTYPE_F32, 0) != LINFUSION_OK) return 0;
  return states(B, N, C);
}

size_t linfusion_scan_bwd_workspace_bytes(int B, long long N, int C) {
  if (check(B, N, C, LINFUSION_DTYPE_F32, 0) != LINFUSION_OK) return 0;
  return kTicketBytes + 5 * states(B, N, C);
}

int linfusion_scan_fwd(const void* x, const void* gate, const void* input, const float* rate, const float* state_in, void* out,
                       float* state_out, const int* lengths, void* saved, size_t saved_bytes, int B, long long N, int C, int dtype,
                       unsigned flags, const long long strides[4][2], void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !gate || !rate || !out) return LINFUSION_ERR_INVALID;
  int rc = check(B, N, C, dtype, flags);
  if (rc != LINFUSION_OK) return rc;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2, sb = (size_t)B * C * 4;
  auto at = [&](int i) { return strides ? strides[i] : nullptr; };
  RowView vx, vg, vi, vo;
  if ((rc = row_view(x, at(0), B, N, C, esz, false, &vx)) != LINFUSION_OK) return rc;
  if ((rc = row_view(gate, at(1), B, N, C, esz, false, &vg)) != LINFUSION_OK) return rc;
  if ((rc = row_view(input, at(2), B, N, C, esz, false, &vi)) != LINFUSION_OK) return rc;
  if ((rc = row_view(out, at(3), B, N, C, esz, true, &vo)) != LINFUSION_OK) return rc;
  if (misaligned({rate, state_in, state_out, saved, workspace}) || (uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  const size_t need = linfusion_scan_workspace_bytes(B, N, C), keep = linfusion_scan_saved_bytes(B, N, C);
  if ((need && (!workspace || workspace_bytes < need)) || (saved && saved_bytes < keep)) return LINFUSION_ERR_WORKSPACE;
  const Range s_in{state_in, sb}, s_out{state_out, sb}, ws{need ? workspace : nullptr, need}, kept{saved, keep};
  if (clash({vx, vg, vi}, {vo}, {Range{rate, (size_t)C * 4}, Range{lengths, (size_t)B * 4}}, {s_out, ws, kept})) return LINFUSION_ERR_OVERLAP;
  if (meet(span(vo), s_in) || meet(ws, s_in) || meet(kept, s_in) || (state_in != state_out && meet(s_in, s_out))) return LINFUSION_ERR_OVERLAP;
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const lf::ScanArgs a{x, gate, input, out, dev(vx), dev(vg), dev(vi), dev(vo), rate, state_in, state_out, (float*)saved,
                       records(workspace, B, N, C), lengths, N, B, C, 0, (int)chunks_of(N), group_size(), packed(B, N), (flags & LINFUSION_FLAG_SCAN_REVERSE) != 0};
  if ((rc = launch_forward(a, dtype, mode_of(flags), (hipStream_t)stream)) != LINFUSION_OK) return rc;
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

int linfusion_scan_bwd(const void* x, const void* gate, const void* input, const float* rate, const float* state_in, const void* dout,
                       const float* dstate_out, const void* saved, size_t saved_bytes, void* dx, void* dgate, void* dinput,
                       float* drate, float* dstate_in, const int* lengths, int B, long long N, int C, int dtype, unsigned flags,
                       const long long strides[7][2], void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !gate || !rate || !dout || !dx || !dgate || !drate || (input != nullptr) != (dinput != nullptr)) return LINFUSION_ERR_INVALID;
  int rc = check(B, N, C, dtype, flags);
  if (rc != LINFUSION_OK) return rc;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2, sb = (size_t)B * C * 4, one = states(B, N, C);
  auto at = [&](int i) { return strides ? strides[i] : nullptr; };
  RowView v[7];
  const void* const p[7] = {x, gate, input, dout, dx, dgate, dinput};
  for (int i = 0; i < 7; ++i)
    if ((rc = row_view(p[i], at(i), B, N, C, esz, i >= 4, &v[i])) != LINFUSION_OK) return rc;
  if (misaligned({rate, state_in, dstate_out, saved, drate, dstate_in, workspace}) || (uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  const size_t keep = linfusion_scan_saved_bytes(B, N, C), need = linfusion_scan_bwd_workspace_bytes(B, N, C) - (saved ? keep : 0);
  if (!workspace || workspace_bytes < need || (saved && saved_bytes < keep)) return LINFUSION_ERR_WORKSPACE;
  const Range ds_out{dstate_out, sb}, ds_in{dstate_in, sb}, ws{workspace, need};
  if (clash({v[0], v[1], v[2], v[3]}, {v[4], v[5], v[6]},
            {Range{rate, (size_t)C * 4}, Range{lengths, (size_t)B * 4}, Range{saved, keep}, Range{state_in, sb}},
            {ds_in, ws, Range{drate, (size_t)C * 4}}))
    return LINFUSION_ERR_OVERLAP;
  for (int i = 4; i < 7; ++i)
    if (meet(span(v[i]), ds_out)) return LINFUSION_ERR_OVERLAP;
  if (meet(ws, ds_out) || meet(Range{drate, (size_t)C * 4}, ds_out) || (dstate_in != dstate_out && meet(ds_in, ds_out))) return LINFUSION_ERR_OVERLAP;
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const hipStream_t st = (hipStream_t)stream;
  char* const w = (char*)workspace + kTicketBytes + 3 * one;   // behind the records
  const lf::ScanRecords rec = records(workspace, B, N, C);
  const bool reverse = (flags & LINFUSION_FLAG_SCAN_REVERSE) != 0;
  const float* starts = (const float*)saved;
  if (!saved) {   // the states between the chunks again
    const lf::ScanArgs f{x, gate, input, nullptr, dev(v[0]), dev(v[1]), dev(v[2]), lf::ScanView{0, 0}, rate, state_in, nullptr, (float*)(w + one),
                         rec, lengths, N, B, C, 0, (int)chunks_of(N), group_size(), packed(B, N), reverse};
    if ((rc = launch_forward(f, dtype, mode_of(flags), st)) != LINFUSION_OK) return rc;
    starts = f.saved;
  }
  const lf::ScanBackArgs a{x, gate, input, dout, dx, dgate, dinput, dev(v[0]), dev(v[1]), dev(v[2]), dev(v[3]), dev(v[4]), dev(v[5]), dev(v[6]),
                           rate, starts, dstate_out, dstate_in, (float*)w, rec, lengths, N, B, C, (int)chunks_of(N), group_size(), packed(B, N), reverse};
  rc = with(dtype, mode_of(flags), input != nullptr, [&](auto t, auto m, auto i) {
    return backward<decltype(t), decltype(m)::value, decltype(i)::value>(a, st);
  });
  if (rc != LINFUSION_OK) return rc;
  lf::scan_rate_sums<<<(C + 15) / 16, 1024, 0, st>>>(a.partials, drate, a.seg ? lf::packed_tiles(B, a.seg) : (long long)B * a.chunks, C);
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

int linfusion_scan_step(const void* x, const void* gate, const void* input, const float* rate, const float* state_in, float* state_out,
                        void* out, int B, int C, int dtype, unsigned flags, const long long strides[4], void* stream) {
  if (!x || !gate || !rate || !out) return LINFUSION_ERR_INVALID;
  int rc = check(B, 1, C, dtype, flags);
  if (rc != LINFUSION_OK) return rc;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2, sb = (size_t)B * C * 4;
  RowView v[4];
  const void* const p[4] = {x, gate, input, out};
  for (int i = 0; i < 4; ++i) {
    const long long s[2] = {strides ? strides[i] : C, 0};
    if ((rc = row_view(p[i], s, B, 1, C, esz, i == 3, &v[i])) != LINFUSION_OK) return rc;
  }
  if (misaligned({rate, state_in, state_out})) return LINFUSION_ERR_MISALIGNED;
  const Range s_in{state_in, sb}, s_out{state_out, sb};
  if (clash({v[0], v[1], v[2]}, {v[3]}, {Range{rate, (size_t)C * 4}}, {s_out})) return LINFUSION_ERR_OVERLAP;
  if (meet(span(v[3]), s_in) || (state_in != state_out && meet(s_in, s_out))) return LINFUSION_ERR_OVERLAP;
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const lf::ScanStepArgs a{x, gate, input, out, v[0].batch, v[1].batch, v[2].batch, v[3].batch, rate, state_in, state_out, B, C};
  rc = with(dtype, mode_of(flags), input != nullptr, [&](auto t, auto m, auto i) {
    return step<decltype(t), decltype(m)::value, decltype(i)::value>(a, (hipStream_t)stream);
  });
  if (rc != LINFUSION_OK) return rc;
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

}  // extern "C"
