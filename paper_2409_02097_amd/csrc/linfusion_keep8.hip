// Activations kept in 8 bits (lf_keep8.hpp): checks, launches, entry points.
#include "lf_keep8.hpp"
#include "lf_keep8_api.hpp"

namespace {

using lfh::meet;
using lfh::Range;
using lfh::RowView;
using lfh::span;

constexpr int kMaxChannels = 32768;

// tokens of a workgroup: enough workgroups for 16 a CU, whole rounds of its tokens
int rows_of(int B, long long N, int C, const lfh::Across& x) {
  const long long all = (long long)x.blocks * B, most = 16LL * lfh::num_cu(), round = 256 / x.lanes;
  long long rows = (N * all + most - 1) / most;
  rows = (rows + round - 1) / round * round;
  while ((N + rows - 1) / rows > 65535) rows *= 2;
  return (int)rows;
}

int views(const void* x, const void* codes, const void* exps, int B, long long N, int C, int dtype, const int* lengths,
          const long long strides[3][2], bool back, RowView v[3]) {
  if (!x || !codes || !exps || B <= 0 || N <= 0 || C <= 0 || B > 65535 || N >= 1LL << 31) return LINFUSION_ERR_INVALID;
  if (dtype != LINFUSION_DTYPE_F32 && dtype != LINFUSION_DTYPE_F16 && dtype != LINFUSION_DTYPE_BF16) return LINFUSION_ERR_UNSUPPORTED;
  if (C % 8 || C > kMaxChannels) return LINFUSION_ERR_UNSUPPORTED;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2;
  const int blocks = (C + lf::kKeepBlock - 1) / lf::kKeepBlock;
  int rc = lfh::row_view(x, strides ? strides[0] : nullptr, B, N, C, esz, back, &v[0]);
  if (rc == LINFUSION_OK) rc = lfh::row_view(codes, strides ? strides[1] : nullptr, B, N, C, 1, !back, &v[1], 8);
  if (rc == LINFUSION_OK) rc = lfh::row_view(exps, strides ? strides[2] : nullptr, B, N, blocks, 1, !back, &v[2], 1);
  if (rc != LINFUSION_OK) return rc;
  if ((uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  const Range l{lengths, (size_t)B * 4};
  if (meet(v[0], v[1]) || meet(v[0], v[2]) || (!back && meet(v[1], v[2]))) return LINFUSION_ERR_OVERLAP;
  if (back ? meet(span(v[0]), l) : meet(span(v[1]), l) || meet(span(v[2]), l)) return LINFUSION_ERR_OVERLAP;
  return LINFUSION_OK;
}

}  // namespace

namespace lfh {

void launch_unkeep8(const lf::KeepArgs& a0, int B, int dtype, hipStream_t st) {
  lf::KeepArgs a = a0;
  const Across x = across(a.C);
  a.rows = rows_of(B, a.N, a.C, x);
  a.lanes = x.lanes;
  const dim3 grid(x.blocks, (unsigned)((a.N + a.rows - 1) / a.rows), B);
  if (dtype == LINFUSION_DTYPE_F16) lf::unkeep8<lf::F16><<<grid, 256, 0, st>>>(a);
  else if (dtype == LINFUSION_DTYPE_BF16) lf::unkeep8<lf::BF16><<<grid, 256, 0, st>>>(a);
  else lf::unkeep8<lf::F32><<<grid, 256, 0, st>>>(a);
}

}  // namespace lfh

extern "C" {

int linfusion_keep8(const void* x, signed char* codes, unsigned char* exps, int B, long long N, int C, int dtype, unsigned flags,
                    const int* lengths, const long long strides[3][2], void* stream) {
  if (flags) return LINFUSION_ERR_INVALID;
  RowView v[3];
  int rc = views(x, codes, exps, B, N, C, dtype, lengths, strides, false, v);
  if (rc != LINFUSION_OK || (rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const lfh::Across x8 = lfh::across(C);
  const lf::KeepArgs a{x, codes, exps, v[0].batch, v[0].token, v[1].batch, v[1].token, v[2].batch, v[2].token, lengths, N, C, rows_of(B, N, C, x8), x8.lanes};
  const dim3 grid(x8.blocks, (unsigned)((N + a.rows - 1) / a.rows), B);
  const hipStream_t st = (hipStream_t)stream;
  if (dtype == LINFUSION_DTYPE_F16) lf::keep8<lf::F16><<<grid, 256, 0, st>>>(a);
  else if (dtype == LINFUSION_DTYPE_BF16) lf::keep8<lf::BF16><<<grid, 256, 0, st>>>(a);
  else lf::keep8<lf::F32><<<grid, 256, 0, st>>>(a);
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

int linfusion_unkeep8(const signed char* codes, const unsigned char* exps, void* x, int B, long long N, int C, int dtype, unsigned flags,
                      const int* lengths, const long long strides[3][2], void* stream) {
  if (flags) return LINFUSION_ERR_INVALID;
  RowView v[3];
  const long long turned[3][2] = {{strides ? strides[2][0] : 0, strides ? strides[2][1] : 0}, {strides ? strides[0][0] : 0, strides ? strides[0][1] : 0},
                                  {strides ? strides[1][0] : 0, strides ? strides[1][1] : 0}};
  int rc = views(x, codes, exps, B, N, C, dtype, lengths, strides ? turned : nullptr, true, v);
  if (rc != LINFUSION_OK || (rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const lf::KeepArgs a{codes, x, const_cast<unsigned char*>(exps), v[1].batch, v[1].token, v[0].batch, v[0].token, v[2].batch, v[2].token, lengths, N, C, 0, 0};
  lfh::launch_unkeep8(a, B, dtype, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

}  // extern "C"
