// Linear layers (lf_linear.hpp): checks, choice of tiles, entry points.
#include "lf_keep8_api.hpp"
#include "lf_linear.hpp"

#include <cmath>
#include <initializer_list>

namespace {

using lfh::meet;
using lfh::Range;
using lfh::row_view;
using lfh::RowView;
using lfh::span;

constexpr int kMaxChannels = 32768;

int check(int B, long long N, int K, int C, int dtype) {
  if (B <= 0 || N <= 0 || K <= 0 || C <= 0 || B > 65535 || N >= 1LL << 31 || (long long)B * N >= 1LL << 31) return LINFUSION_ERR_INVALID;
  if (dtype != LINFUSION_DTYPE_F32 && dtype != LINFUSION_DTYPE_F16 && dtype != LINFUSION_DTYPE_BF16) return LINFUSION_ERR_UNSUPPORTED;
  if (K % 8 || C % 8 || K > kMaxChannels || C > kMaxChannels) return LINFUSION_ERR_UNSUPPORTED;
  return LINFUSION_OK;
}

int check_act(int act, float slope, unsigned flags) {
  if (act < LINFUSION_ACT_NONE || act > LINFUSION_ACT_SILU) return LINFUSION_ERR_UNSUPPORTED;
  return flags || !std::isfinite(slope) ? LINFUSION_ERR_INVALID : LINFUSION_OK;
}

bool misaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if ((uintptr_t)p & 15) return true;
  return false;
}

lf::LinRows dev(const RowView& v) { return lf::LinRows{v.batch, v.token}; }

// ---- which tiles, how many splits of k -------------------------------------------------------------------------------

struct Plan { int kind, splits; long long k_split; };   // kind: index into the tile shapes below

// Tile shapes: rows, columns, waves along each, bytes of k of a step, workgroups that share a CU (LDS, registers).  The first for
// 16-bit types only.  Half steps leave room for more workgroups, whose starts and ends overlap more: for short k (49152 x 320 -> 1280 in bf16
// 60 us, whole steps 74), while long k loses (8192^3 1274, 1043).
#define LF_LINEAR_SHAPES(DO) \
  DO(0, 256, 256, 2, 4, 128, 1) DO(1, 128, 160, 2, 2, 128, 2) DO(2, 128, 128, 2, 2, 128, 2) DO(3, 128, 64, 2, 2, 128, 3) \
  DO(4, 64, 64, 2, 2, 128, 4) DO(5, 128, 128, 2, 2, 64, 4) DO(6, 128, 160, 2, 2, 64, 3) DO(7, 128, 64, 2, 2, 64, 5)
// (Where every lane finds its tokens, dW by 128 x 128 in half steps spills 14 to 16 registers.)
constexpr int kShapes = 8;
struct Shape { int m, n, step, per_cu; };
constexpr Shape kShape[kShapes] = {
#define LF_ROW(I, M, N, WR, WC, STEP, PER) {M, N, STEP, PER},
    LF_LINEAR_SHAPES(LF_ROW)
#undef LF_ROW
};

// What a product takes, in us: rounds of workgroups, each a start and end (`over`) and its steps (`step`, of a CU full of such
// tiles), the last round by how full it is; another launch where k is split, and the sums' way out and in.  Fitted to 449
// measured times of 16-bit products and 210 of fp32 ones (rows 154 to 81120, columns 64 to 5120, k 64 to 49152, all shapes, 1 to 32
// splits; off by 10 % and 3 % at the root mean square; of 47 products it chooses the best shape or one within 5 % for 44, and 1.25 times the
// best one's time at most).  The number of tiles alone chose 256 x 256 for 49152 x 1280 -> 320: 74 us where 128 x 160 takes 49.
struct Cost { double step[kShapes], over[kShapes], fill, join, join_mb; };
constexpr Cost kCost16{{1.55, 1.10, 0.91, 0.81, 0.68, 0.90, 0.88, 0.78}, {5.6, 6.1, 3.9, 2.9, 1.8, 4.2, 6.2, 3.0}, 0.58, 3.4, 0.79};
constexpr Cost kCost32{{0.0, 5.00, 3.87, 3.19, 2.22, 3.76, 3.80, 2.69}, {0.0, 4.9, 4.1, 0.2, 0.0, 3.0, 3.4, 0.0}, 0.87, 2.7, 1.01};

Plan plan(long long M, int N, long long K, int dtype) {
  const bool wide = dtype == LINFUSION_DTYPE_F32;
  const Cost& c = wide ? kCost32 : kCost16;
  const long long cus = lfh::num_cu();
  const int only = lfh::env_int("LINFUSION_LINEAR_TILES", 0) - 1, only_splits = lfh::env_int("LINFUSION_LINEAR_SPLITS", 0);
  Plan best{4, 1, K};
  double least = 1e300;
  for (int s = wide ? 1 : 0; s < kShapes; ++s) {
    if (only >= 0 && s != only) continue;
    const int k_step = kShape[s].step / (wide ? 4 : 2);
    const long long steps = (K + k_step - 1) / k_step;
    const long long tiles = ((M + kShape[s].m - 1) / kShape[s].m) * ((N + kShape[s].n - 1) / kShape[s].n), room = cus * kShape[s].per_cu;
    for (const int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (splits > steps || (splits > 1 && tiles * splits >= 2 * room)) break;   // (what most_partials counts on)
      if (only_splits && splits != only_splits) continue;
      const long long per = (steps + splits - 1) / splits, used = (steps + per - 1) / per;
      const double each = per * c.step[s] + c.over[s];
      const long long all = tiles * used, rest = all % room;
      double t = (double)(all / room) * each;
      if (rest) t += each * std::pow((double)((rest + cus - 1) / cus) / kShape[s].per_cu, c.fill);
      if (used > 1) t += c.join + c.join_mb * 1e-6 * (double)M * N * (used + 1);
      if (t < least) {
        least = t;
        best = Plan{s, (int)used, per * k_step};
      }
    }
  }
  return best;
}

// Bytes of the sums of splits, at most: never falls with M.
size_t most_partials(long long M, int N) {
  const size_t by_rows = (size_t)M * N * 64 * 4, by_tiles = (size_t)lfh::num_cu() * 2 * 65536 * 4;
  return lfh::up256(by_rows < by_tiles ? by_rows : by_tiles);
}

template <typename T, int BM, int BN, int WR, int WC, int STEP, bool AK, bool BK, int MAPPED>
int launch_tiles(const lf::LinArgs& g, hipStream_t st) {
  auto kernel = lf::linear_tiles<T, BM, BN, WR, WC, STEP, AK, BK, MAPPED>;
  constexpr int lds = 2 * (BM + BN) * STEP;
  if (!lfh::allow_lds(kernel, lds)) return LINFUSION_ERR_HIP;
  const long long all = (long long)g.tiles_m * g.tiles_n * g.splits;
  if (all > 0x7fffffffLL) return LINFUSION_ERR_INVALID;
  kernel<<<(unsigned)all, 64 * WR * WC, lds, st>>>(g);
  return LINFUSION_OK;
}

template <typename T, bool AK, bool BK, int MAPPED>
int product(lf::LinArgs g, Plan p, hipStream_t st) {
  if constexpr (!AK && MAPPED == lf::kRows) {   // whole steps for every batch row
    const long long k_step = kShape[p.kind].step / lf::Stored<T>::kBytes, steps = (g.per_row + k_step - 1) / k_step * (g.K / g.per_row);
    const long long per = (steps + p.splits - 1) / p.splits;
    g.K = steps * k_step;
    p = Plan{p.kind, (int)((steps + per - 1) / per), per * k_step};
  }
  g.tiles_m = (int)((g.M + kShape[p.kind].m - 1) / kShape[p.kind].m);
  g.tiles_n = (g.N + kShape[p.kind].n - 1) / kShape[p.kind].n;
  g.splits = p.splits;
  g.k_split = p.k_split;
  if (p.splits == 1) g.partials = nullptr;
  int rc = LINFUSION_ERR_UNSUPPORTED;
#define LF_CASE(I, TM, TN, WR, WC, STEP, PER)                                                    \
  if constexpr (lf::Stored<T>::kBytes == 2 || I > 0)                           \
    if (p.kind == I) rc = launch_tiles<T, TM, TN, WR, WC, STEP, AK, BK, MAPPED>(g, st);
  LF_LINEAR_SHAPES(LF_CASE)
#undef LF_CASE
  if (rc != LINFUSION_OK) return rc;
  if (p.splits > 1) {
    const long long threads = g.M * (g.N / 8);
    lf::linear_join<T, MAPPED != lf::kFlat && AK><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(g);
  }
  return LINFUSION_OK;
}

// Tokens of a batch row from which on a step of k takes those of one row alone.
constexpr unsigned kRowTokens = 32;

template <typename T, bool AK, bool BK>
int product(const lf::LinArgs& g, bool mapped, const Plan& p, hipStream_t st) {
  if (!mapped) return product<T, AK, BK, lf::kFlat>(g, p, st);
  if constexpr (!AK) {
    if (g.per_row < kRowTokens) return product<T, AK, BK, lf::kLanes>(g, p, st);
  }
  return product<T, AK, BK, lf::kRows>(g, p, st);
}

template <typename F> int by_type(int dtype, F f) {
  return dtype == LINFUSION_DTYPE_F16 ? f(lf::F16{}) : dtype == LINFUSION_DTYPE_BF16 ? f(lf::BF16{}) : f(lf::F32{});
}

// Whether one stride leads through all tokens of a view.
bool plain(const RowView& v, int B, long long N) { return !v.p || B == 1 || (N == 1 ? true : v.batch == N * v.token); }
// and that stride, as {0, stride}
lf::LinRows flat(const RowView& v, int B, long long N, bool mapped) {
  if (mapped) return dev(v);
  return lf::LinRows{0, N == 1 ? v.batch : v.token};
}

constexpr long long kFew = 64;   // tokens up to which the weights' way from memory is all there is

template <typename T, int MT> int launch_few(const lf::LinArgs& g, bool mapped, hipStream_t st) {
  const unsigned wgs = (unsigned)((g.N + 15) / 16);
  if (mapped) lf::linear_few<T, MT, true><<<wgs, 64 * lf::kFewWaves, 0, st>>>(g);
  else lf::linear_few<T, MT, false><<<wgs, 64 * lf::kFewWaves, 0, st>>>(g);
  return LINFUSION_OK;
}

// Workgroups along the tokens of linear_slope, and the tokens of a piece of a batch row.
struct Slices { int count, each; };
// (49152 x 1280 from kept values, GELU: six a CU with two tokens of a lane under way 68 us, four with four 75, two with four 93.)
long long most_workgroups(int C) {
  const long long most = 6LL * lfh::num_cu() / lfh::across(C).blocks;
  return most < 1 ? 1 : most;
}
Slices slices(int B, long long N, int C) {
  const long long most = most_workgroups(C);
  long long each = (B * N + most - 1) / most;
  const long long round = 2 * (256 / lfh::across(C).lanes);
  each = (each + round - 1) / round * round;
  if (each > N) each = (N + round - 1) / round * round;
  const long long pieces = (N + each - 1) / each * B;
  return Slices{(int)(pieces < most ? pieces : most), (int)each};
}
size_t most_slices(long long rows, int C) {   // never falls with the rows
  const long long most = most_workgroups(C);
  return lfh::up256((size_t)(most < rows ? most : rows) * C * 4);
}

}  // namespace

extern "C" {

size_t linfusion_linear_workspace_bytes(int B, long long N, int C_in, int C_out, int dtype) {
  if (check(B, N, C_in, C_out, dtype) != LINFUSION_OK) return 0;
  return most_partials(B * N, C_out);
}

int linfusion_linear_fwd(const void* x, const void* w, const void* bias, const void* residual, void* y, void* z, int B, long long N,
                         int C_in, int C_out, int dtype, int activation, float slope, unsigned flags, const int* lengths,
                         const long long strides[4][2], long long w_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !w || (!y && !z) || (residual && !y)) return LINFUSION_ERR_INVALID;
  int rc = check(B, N, C_in, C_out, dtype);
  if (rc != LINFUSION_OK || (rc = check_act(activation, slope, flags)) != LINFUSION_OK) return rc;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2;
  auto at = [&](int i) { return strides ? strides[i] : nullptr; };
  RowView vx, vr, vy, vz, vw;
  if ((rc = row_view(x, at(0), B, N, C_in, esz, false, &vx)) != LINFUSION_OK) return rc;
  if ((rc = row_view(residual, at(1), B, N, C_out, esz, false, &vr)) != LINFUSION_OK) return rc;
  if ((rc = row_view(y, at(2), B, N, C_out, esz, true, &vy)) != LINFUSION_OK) return rc;
  if ((rc = row_view(z, at(3), B, N, C_out, esz, true, &vz)) != LINFUSION_OK) return rc;
  const long long ws[2] = {0, w_stride ? w_stride : C_in};
  if (ws[1] < C_in && C_out > 1) return LINFUSION_ERR_INVALID;
  if ((rc = row_view(w, ws, 1, C_out, C_in, esz, false, &vw)) != LINFUSION_OK) return rc;
  if (misaligned({bias, workspace}) || (uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  const size_t need = linfusion_linear_workspace_bytes(B, N, C_in, C_out, dtype);
  if (!workspace || workspace_bytes < need) return LINFUSION_ERR_WORKSPACE;
  // y may be the residual itself: a lane reads what it writes
  const Range others[] = {span(vw), {bias, (size_t)C_out * esz}, {lengths, (size_t)B * 4}, {workspace, need}};
  for (const RowView* o : {&vy, &vz}) {
    if (meet(*o, vx) || (meet(*o, vr) && !(o == &vy && lfh::same_rows(vy, vr)))) return LINFUSION_ERR_OVERLAP;
    for (const Range& r : others)
      if (meet(span(*o), r)) return LINFUSION_ERR_OVERLAP;
  }
  if (meet(vy, vz)) return LINFUSION_ERR_OVERLAP;
  for (const Range& r : {span(vx), span(vr), others[0], others[1], others[2]})
    if (meet(others[3], r)) return LINFUSION_ERR_OVERLAP;
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const bool mapped = lengths || !plain(vx, B, N) || !plain(vr, B, N) || !plain(vy, B, N) || !plain(vz, B, N);
  auto rows = [&](const RowView& v) { return flat(v, B, N, mapped); };
  lf::LinArgs g{};
  g.A = x, g.B = w, g.va = rows(vx), g.vb = lf::LinRows{0, ws[1]};
  g.M = B * N, g.K = C_in, g.N = C_out, g.per_row = (unsigned)N, g.lengths = lengths, g.partials = (float*)workspace;
  g.out = lf::LinOut{y, z, residual, bias, rows(vy), rows(vz), rows(vr), activation, slope};
  const hipStream_t st = (hipStream_t)stream;
  rc = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (g.M <= 16) return launch_few<T, 1>(g, mapped, st);
    if (g.M <= 32) return launch_few<T, 2>(g, mapped, st);
    if (g.M <= kFew) return launch_few<T, 4>(g, mapped, st);
    return product<T, true, true>(g, mapped, plan(g.M, g.N, g.K, dtype), st);
  });
  if (rc != LINFUSION_OK) return rc;
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

size_t linfusion_linear_bwd_workspace_bytes(int B, long long N, int C_in, int C_out, int dtype) {
  if (check(B, N, C_in, C_out, dtype) != LINFUSION_OK) return 0;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2, rows = (size_t)(B * N);
  const size_t a = most_partials(B * N, C_in), b = most_partials(C_out, C_in);
  return lfh::up256(rows * C_out * esz) + lfh::up256(rows * C_in * esz) + most_slices(B * N, C_out) + (a > b ? a : b);
}

int linfusion_linear_bwd(const void* x, const unsigned char* x_exps, const void* w, const void* z, const unsigned char* z_exps,
                         const void* dy, void* dx, void* dw, void* dbias, int B, long long N, int C_in, int C_out, int dtype,
                         int activation, float slope, unsigned flags, const int* lengths, const long long strides[6][2],
                         long long w_stride, long long dw_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dy || (!dx && !dw && !dbias) || (dx && !w) || (dw && !x)) return LINFUSION_ERR_INVALID;
  int rc = check(B, N, C_in, C_out, dtype);
  if (rc != LINFUSION_OK || (rc = check_act(activation, slope, flags)) != LINFUSION_OK) return rc;
  if ((activation != LINFUSION_ACT_NONE && !z) || (x_exps && !x) || (z_exps && !z)) return LINFUSION_ERR_INVALID;
  const size_t esz = dtype == LINFUSION_DTYPE_F32 ? 4 : 2;
  auto at = [&](int i) { return strides ? strides[i] : nullptr; };
  RowView vx, vz, vdy, vdx, vxe, vze, vw, vdw;
  if ((rc = row_view(x, at(0), B, N, C_in, x_exps ? 1 : esz, false, &vx, x_exps ? 8 : 16)) != LINFUSION_OK) return rc;
  if ((rc = row_view(z, at(1), B, N, C_out, z_exps ? 1 : esz, false, &vz, z_exps ? 8 : 16)) != LINFUSION_OK) return rc;
  if ((rc = row_view(dy, at(2), B, N, C_out, esz, false, &vdy)) != LINFUSION_OK) return rc;
  if ((rc = row_view(dx, at(3), B, N, C_in, esz, true, &vdx)) != LINFUSION_OK) return rc;
  if ((rc = row_view(x_exps, at(4), B, N, (C_in + 31) / 32, 1, false, &vxe, 1)) != LINFUSION_OK) return rc;
  if ((rc = row_view(z_exps, at(5), B, N, (C_out + 31) / 32, 1, false, &vze, 1)) != LINFUSION_OK) return rc;
  const long long ws[2] = {0, w_stride ? w_stride : C_in}, dws[2] = {0, dw_stride ? dw_stride : C_in};
  if ((ws[1] < C_in || dws[1] < C_in) && C_out > 1) return LINFUSION_ERR_INVALID;
  if ((rc = row_view(w, ws, 1, C_out, C_in, esz, false, &vw)) != LINFUSION_OK) return rc;
  if ((rc = row_view(dw, dws, 1, C_out, C_in, esz, true, &vdw)) != LINFUSION_OK) return rc;
  if (misaligned({dbias, workspace}) || (uintptr_t)lengths & 3) return LINFUSION_ERR_MISALIGNED;
  const size_t need = linfusion_linear_bwd_workspace_bytes(B, N, C_in, C_out, dtype);
  if (!workspace || workspace_bytes < need) return LINFUSION_ERR_WORKSPACE;
  const Range reads[] = {span(vx), span(vxe), span(vw), span(vz), span(vze), span(vdy), {lengths, (size_t)B * 4}};
  const Range writes[] = {span(vdx), span(vdw), {dbias, (size_t)C_out * esz}, {workspace, need}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 7; ++j) {
      if (!meet(writes[i], reads[j])) continue;
      if (i == 0 && ((j == 0 && !meet(vdx, vx)) || (j == 3 && !meet(vdx, vz)) || (j == 5 && !meet(vdx, vdy)))) continue;   // columns of one buffer
      return LINFUSION_ERR_OVERLAP;
    }
    for (int j = i + 1; j < 4; ++j)
      if (meet(writes[i], writes[j])) return LINFUSION_ERR_OVERLAP;
  }
  if ((rc = lfh::check_device()) != LINFUSION_OK) return rc;
  const hipStream_t st = (hipStream_t)stream;
  const long long M = B * N;
  char* at_ws = (char*)workspace;
  void* const dz = at_ws;
  at_ws += lfh::up256((size_t)M * C_out * esz);
  void* const wide_x = at_ws;
  at_ws += lfh::up256((size_t)M * C_in * esz);
  float* const sums = (float*)at_ws;
  at_ws += most_slices(M, C_out);
  float* const partials = (float*)at_ws;
  const bool act = activation != LINFUSION_ACT_NONE;
  if (act || dbias) {
    const bool one = !lengths && plain(vdy, B, N) && plain(vz, B, N) && plain(vze, B, N);   // one stride leads through all tokens
    const int rows_b = one ? 1 : B;
    const long long rows_n = one ? M : N;
    auto rows = [&](const RowView& v) { return flat(v, B, N, !one); };
    const Slices s = slices(rows_b, rows_n, C_out);
    const lf::LinSlopeArgs a{dy, z, z_exps, rows(vdy), rows(vz), rows(vze), act ? dz : nullptr, dbias ? sums : nullptr, lengths, rows_n, rows_b,
                             C_out, s.each, lfh::across(C_out).lanes, activation, slope};
    const dim3 grid(lfh::across(C_out).blocks, s.count);
    rc = by_type(dtype, [&](auto t) {
      using T = decltype(t);
      if (z_exps) lf::linear_slope<T, true><<<grid, 256, 0, st>>>(a);
      else lf::linear_slope<T, false><<<grid, 256, 0, st>>>(a);
      if (dbias) lf::linear_bias<T><<<(C_out + 15) / 16, 1024, 0, st>>>(sums, dbias, s.count, C_out);
      return LINFUSION_OK;
    });
  }
  RowView vd = vdy;
  if (act) {
    vd.p = dz;
    vd.batch = B == 1 ? 0 : N * C_out;
    vd.token = N == 1 ? 0 : C_out;
  }
  lf::LinArgs g{};
  g.per_row = (unsigned)N, g.lengths = lengths, g.partials = partials;
  if (dx) {
    const bool mapped = lengths || !plain(vd, B, N) || !plain(vdx, B, N);
    g.A = vd.p, g.va = flat(vd, B, N, mapped), g.B = w, g.vb = lf::LinRows{0, ws[1]};
    g.M = M, g.K = C_out, g.N = C_in;
    g.out = lf::LinOut{dx, nullptr, nullptr, nullptr, flat(vdx, B, N, mapped), {}, {}, lf::kActNone, 0.0f};
    rc = by_type(dtype, [&](auto t) { return product<decltype(t), true, false>(g, mapped, plan(g.M, g.N, g.K, dtype), st); });
    if (rc != LINFUSION_OK) return rc;
  }
  if (dw) {
    if (x_exps) {
      const lf::KeepArgs k{x, wide_x, const_cast<unsigned char*>(x_exps), vx.batch, vx.token, N * C_in, C_in, vxe.batch, vxe.token, lengths, N, C_in, 0, 0};
      lfh::launch_unkeep8(k, B, dtype, st);
      vx.p = wide_x;
      vx.batch = B == 1 ? 0 : N * C_in;
      vx.token = N == 1 ? 0 : C_in;
    }
    const bool mapped = lengths || !plain(vd, B, N) || !plain(vx, B, N);
    g.A = vd.p, g.va = flat(vd, B, N, mapped), g.B = vx.p, g.vb = flat(vx, B, N, mapped);
    g.M = C_out, g.K = M, g.N = C_in;
    g.out = lf::LinOut{dw, nullptr, nullptr, nullptr, lf::LinRows{0, dws[1]}, {}, {}, lf::kActNone, 0.0f};
    rc = by_type(dtype, [&](auto t) { return product<decltype(t), false, false>(g, mapped, plan(g.M, g.N, g.K, dtype), st); });
    if (rc != LINFUSION_OK) return rc;
  }
  return hipGetLastError() == hipSuccess ? LINFUSION_OK : LINFUSION_ERR_HIP;
}

}  // extern "C"
