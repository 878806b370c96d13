// A gated linear recurrence, channel by channel.  Per (batch, channel), token after token:
//
//     s = sigmoid(gate_t);  i = sigmoid(input_t) (1 without);  g = -rate s;  a = e^g
//     m = sqrt(1 - a^2)  (kScanNorm),  1 - a  (kScanLeaky),  1  (kScanSum)
//     h = a h + m i x_t;  out_t = h
//
// Backward, with E behind the last token the gradient that arrives at its state:
//
//     D = dout_t + E;  dx = D m i;  dinput = D m x i (1 - i);  dg = D (a h' + (dm/dg) i x), h' the state before the token;
//     dgate = dg g (1 - s);  drate += -dg s;  E = a D
//
// where dm/dg = -a^2 / m, -a, 0.  Both directions are first-order linear recurrences, so a stretch of tokens turns the value
// it starts from into A h + R with A the product of its a.  A workgroup of 256 threads takes a chunk of 32 x T tokens of 64
// channels, a thread T tokens of 8 channels: a and m i x in registers, the stretches of a wave's eight time lanes and then of
// the four waves joined through LDS.  Long sequences are several chunks.  Everything is fp32, results are rounded once.
#pragma once
#include "lf_vec8.hpp"

namespace lf {

constexpr int kScanNorm = 0, kScanLeaky = 1, kScanSum = 2;
constexpr int kScanWidth = 64;   // channels of a workgroup

// tokens of a thread: eight of 16-bit types, four of fp32 and in the backward pass, which holds twice the values
template <typename T> struct ScanShape {
  static constexpr int kT = Stored<T>::kBytes == 4 ? 4 : 8, kChunk = 32 * kT;
  static constexpr int kBackT = 4, kBackChunk = 32 * kBackT;
};

struct ScanView { long long batch, token; };   // element strides; channels contiguous

struct ScanArgs {
  const void *x, *gate, *input;
  void* out;
  ScanView vx, vg, vi, vo;
  const float *rate, *state_in;
  float *state_out, *totals, *starts;   // totals: [B][chunks][2][C]; starts: [B][chunks][C], the state before each chunk
  float* saved;                         // null, or the states before the chunks of the backward pass, [B][back_chunks][C]
  const int* lengths;
  long long N;
  int C, chunks, back_chunks;
  bool reverse;
};

struct ScanBackArgs {
  const void *x, *gate, *input, *dout;
  void *dx, *dgate, *dinput;
  ScanView vx, vg, vi, vd, vdx, vdg, vdi;
  const float *rate, *starts, *dstate_out;
  float *dstate_in, *totals, *ends, *partials;   // ends: [B][chunks][C], E behind each chunk; partials: [B][chunks][C], of drate
  const int* lengths;
  long long N;
  int C, chunks;
  bool reverse;
};

// e^x on the hardware's exponential of 2; Precise adds back what rounding x log2(e) loses.  x is cut off where the result is 0 or
// near the largest value anyway; a NaN stays one.
template <bool Precise> LF_DEV float exp_of(float x) {
  constexpr float kLog2e = 1.44269504088896340736f;
  if constexpr (!Precise) return __builtin_amdgcn_exp2f(x * kLog2e);
  x = x < -120.0f ? -120.0f : x;
  x = x > 88.0f ? 88.0f : x;
  const float t = x * kLog2e, e = __builtin_amdgcn_exp2f(t);
  const float lost = __builtin_fmaf(x, kLog2e, -t) + x * 1.92596299112661746e-8f;
  return __builtin_fmaf(e, lost * 0.69314718055994530942f, e);
}

template <bool Precise> LF_DEV float sigmoid_of(float x) {
  const float s = __builtin_amdgcn_rcpf(1.0f + exp_of<Precise>(-x));
  return Precise && x < -88.0f ? 0.0f : s;
}

// 1 - e^-v for v >= 0, e = e^-v given: where they are near each other by the series, whose next term is below 2^-24 of the
// result (16-bit types: 2^-19).
template <bool Precise> LF_DEV float one_less(float v, float e) {
  float p;
  if constexpr (Precise) {
    p = __builtin_fmaf(v, -1.0f / 8, 1.0f);
    p = __builtin_fmaf(v * p, -1.0f / 7, 1.0f);
    p = __builtin_fmaf(v * p, -1.0f / 6, 1.0f);
    p = __builtin_fmaf(v * p, -1.0f / 5, 1.0f);
    p = __builtin_fmaf(v * p, -1.0f / 4, 1.0f);
    p = __builtin_fmaf(v * p, -1.0f / 3, 1.0f);
    p = __builtin_fmaf(v * p, -1.0f / 2, 1.0f);
    return v < 0.5f ? v * p : 1.0f - e;
  }
  p = __builtin_fmaf(v, -1.0f / 120, 1.0f / 24);
  p = __builtin_fmaf(v, -p, 1.0f / 6);
  p = __builtin_fmaf(v, -p, 0.5f);
  p = __builtin_fmaf(v, -p, 1.0f);
  return v < 0.25f ? v * p : 1.0f - e;
}

// What a token's gates say: a, and the weight m of the new value with r so that dm/dg = -a r (kScanNorm: r = a / m, 0 where m is 0).
struct ScanWeight { float a, m, r; };
template <bool Precise, int MODE> LF_DEV ScanWeight weight_of(float decay) {   // decay = -g
  ScanWeight w;
  w.a = exp_of<Precise>(-decay);
  if constexpr (MODE == kScanSum) {
    w.m = 1.0f;
    w.r = 0.0f;
  } else if constexpr (MODE == kScanLeaky) {
    w.m = one_less<Precise>(decay, w.a);
    w.r = 1.0f;
  } else {
    const float m2 = one_less<Precise>(2.0f * decay, w.a * w.a);
    const float q = m2 < 1.17549435e-38f ? 0.0f : __builtin_amdgcn_rsqf(m2);
    w.m = m2 * q;
    w.r = w.a * q;
  }
  return w;
}

// Where a row's tokens are in the order of the recurrence.
struct ScanRow {
  long long n, first, step;   // tokens that count; the first one; from one to the next
  LF_DEV ScanRow(const int* lengths, int b, long long N, bool reverse) {
    n = tokens_of(lengths, b, N);
    first = reverse ? n - 1 : 0;
    step = reverse ? -1 : 1;
  }
  LF_DEV long long token(long long t) const { return first + step * t; }
};

// The stretches of a chunk joined: from each thread's (A, R) of 8 channels the value its first token starts from, given the
// chunk's; and the chunk's own (A, R).  Time lane of a thread: threadIdx.x / 8 in the recurrence's order (BACK: 31 minus that).
struct ScanJoin {
  float stretch[32][2][kScanWidth];   // [time lane]
  float wave[4][2][kScanWidth];
};

// A wave's LDS operations complete in the order in which they are issued: between its lanes no barrier is needed, only the order.
LF_DEV void lds_in_order() { asm volatile("" ::: "memory"); }

// before the barrier: `A`, `R` are replaced by those of the wave's stretches in front of this thread's
template <bool BACK> LF_DEV void join_wave(ScanJoin& s, float (&A)[8], float (&R)[8]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = threadIdx.x >> 3, c = (lane & 7) * 8;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    *reinterpret_cast<f32x4*>(&s.stretch[at][0][c + 4 * q]) = f32x4{A[4 * q], A[4 * q + 1], A[4 * q + 2], A[4 * q + 3]};
    *reinterpret_cast<f32x4*>(&s.stretch[at][1][c + 4 * q]) = f32x4{R[4 * q], R[4 * q + 1], R[4 * q + 2], R[4 * q + 3]};
  }
  lds_in_order();
  float a[8], r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = wave * 8 + (BACK ? 7 - j : j);
    a[j] = s.stretch[t][0][lane];
    r[j] = s.stretch[t][1][lane];
  }
  float pa = 1.0f, pr = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = wave * 8 + (BACK ? 7 - j : j);
    s.stretch[t][0][lane] = pa;
    s.stretch[t][1][lane] = pr;
    pr = __builtin_fmaf(a[j], pr, r[j]);
    pa *= a[j];
  }
  s.wave[wave][0][lane] = pa;
  s.wave[wave][1][lane] = pr;
  lds_in_order();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x4 va = *reinterpret_cast<const f32x4*>(&s.stretch[at][0][c + 4 * q]), vr = *reinterpret_cast<const f32x4*>(&s.stretch[at][1][c + 4 * q]);
#pragma unroll
    for (int j = 0; j < 4; ++j) { A[4 * q + j] = va[j]; R[4 * q + j] = vr[j]; }
  }
}

// behind the barrier, lane c of every wave for channel c: the chunk's (A, R) in front of the wave (upto = the wave's place in the
// order) or whole (upto = 4)
template <bool BACK> LF_DEV void join_chunk(const ScanJoin& s, int upto, float& A, float& R) {
  const int lane = threadIdx.x & 63;
  A = 1.0f;
  R = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int of = BACK ? 3 - w : w;
    const float a = s.wave[of][0][lane], r = s.wave[of][1][lane];
    if (w < upto) {
      R = __builtin_fmaf(a, R, r);
      A *= a;
    }
  }
}

// A value per lane (channel) handed to the lanes that hold 8 channels each, inside a wave, through 64 floats of LDS.
LF_DEV void spread8(float* lds, float v, float (&x)[8]) {
  const int lane = threadIdx.x & 63, c = (lane & 7) * 8;
  lds[lane] = v;
  lds_in_order();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x4 t = *reinterpret_cast<const f32x4*>(lds + c + 4 * q);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * q + j] = t[j];
  }
}

constexpr int kScanWhole = 0, kScanTotals = 1, kScanApply = 2;

// PASS kScanTotals leaves every chunk's (A, R), scan_starts turns them into the states between the chunks, and kScanApply goes
// from those; a sequence of one chunk is kScanWhole alone.
template <typename T, int MODE, bool INPUT, int PASS>
__global__ __launch_bounds__(256) void scan_fwd(ScanArgs a) {
  constexpr int TT = ScanShape<T>::kT, L = ScanShape<T>::kChunk;
  constexpr bool kPrecise = Stored<T>::kBytes == 4;
  __shared__ ScanJoin lds;
  __shared__ float spread[4][kScanWidth];
  const int b = blockIdx.z, blocks = (a.C + kScanWidth - 1) / kScanWidth;
  const int chunk = blockIdx.x / blocks, c0 = (blockIdx.x - chunk * blocks) * kScanWidth;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = c0 + (lane & 7) * 8;
  const bool on = c < a.C;
  const ScanRow row(a.lengths, b, a.N, a.reverse);
  const long long t0 = (long long)chunk * L + (threadIdx.x >> 3) * TT;
  if (chunk && (long long)chunk * L >= row.n) return;   // (the whole workgroup)
  Raw8<T> rx[TT], rg[TT], ri[TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    rx[j] = rg[j] = ri[j] = none8<T>();
    if (!on || t0 + j >= row.n) continue;
    const long long n = row.token(t0 + j);
    rx[j] = load8_raw<T>(at<T>(a.x, b * a.vx.batch + n * a.vx.token + c));
    rg[j] = load8_raw<T>(at<T>(a.gate, b * a.vg.batch + n * a.vg.token + c));
    if constexpr (INPUT) ri[j] = load8_raw<T>(at<T>(a.input, b * a.vi.batch + n * a.vi.token + c));
  }
  float rate[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) rate[k] = 0.0f;
  if (on) load8_f32(a.rate + c, rate);
  float da[TT][8], u[TT][8], A[8], R[8];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    float x[8], g[8], in[8];
    widen8<T>(rx[j], x);
    widen8<T>(rg[j], g);
    widen8<T>(ri[j], in);
    const bool live = on && t0 + j < row.n;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const ScanWeight w = weight_of<kPrecise, MODE>(rate[k] * sigmoid_of<kPrecise>(g[k]));
      float v = w.m * x[k];
      if constexpr (INPUT) v *= sigmoid_of<kPrecise>(in[k]);
      da[j][k] = live ? w.a : 1.0f;
      u[j][k] = live ? v : 0.0f;
      R[k] = j ? __builtin_fmaf(da[j][k], R[k], u[j][k]) : u[j][k];
      A[k] = j ? A[k] * da[j][k] : da[j][k];
    }
  }
  join_wave<false>(lds, A, R);
  __syncthreads();
  const long long at0 = ((long long)b * a.chunks + chunk) * a.C;
  const int cl = c0 + lane;
  float ca, cr;
  if constexpr (PASS == kScanTotals) {
    join_chunk<false>(lds, 4, ca, cr);
    if (wave == 0 && cl < a.C) {
      a.totals[2 * at0 + cl] = ca;
      a.totals[2 * at0 + a.C + cl] = cr;
    }
    return;
  }
  float h0 = 0.0f;
  if (cl < a.C) {
    if constexpr (PASS == kScanApply) h0 = a.starts[at0 + cl];
    else h0 = a.state_in ? a.state_in[(long long)b * a.C + cl] : 0.0f;
  }
  join_chunk<false>(lds, wave, ca, cr);
  float h[8];
  const float mine = __builtin_fmaf(ca, h0, cr);   // the state before the wave's tokens
  constexpr int kEvery = ScanShape<T>::kBackChunk / (8 * TT);   // waves of a chunk of the backward pass
  if (a.saved && cl < a.C && wave % kEvery == 0) {
    const long long t = (long long)chunk * L + wave * 8 * TT;
    if (t == 0 || t < row.n) a.saved[((long long)b * a.back_chunks + t / ScanShape<T>::kBackChunk) * a.C + cl] = mine;
  }
  spread8(spread[wave], mine, h);
#pragma unroll
  for (int k = 0; k < 8; ++k) h[k] = __builtin_fmaf(A[k], h[k], R[k]);
#pragma unroll
  for (int j = 0; j < TT; ++j) {
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = __builtin_fmaf(da[j][k], h[k], u[j][k]);
    if (a.out && on && t0 + j < row.n) store8_stream<T>(at<T>(a.out, b * a.vo.batch + row.token(t0 + j) * a.vo.token + c), h);
  }
  if (wave == 3 && cl < a.C && a.state_out && (long long)(chunk + 1) * L >= row.n) {   // the chunk with the last token that counts
    join_chunk<false>(lds, 4, ca, cr);
    a.state_out[(long long)b * a.C + cl] = __builtin_fmaf(ca, h0, cr);
  }
}

// The values that the chunks of one (batch, channel) start from, one after the other (BACK: from the last one that counts).
template <bool BACK>
__global__ __launch_bounds__(64) void scan_starts(const float* totals, const float* first, float* starts, const int* lengths,
                                                  long long N, int C, int chunks, int L) {
  const int b = blockIdx.y, c = blockIdx.x * 64 + threadIdx.x;
  if (c >= C) return;
  long long used = (tokens_of(lengths, b, N) + L - 1) / L;
  if (used < 1) used = 1;
  float h = first ? first[(long long)b * C + c] : 0.0f;
  const long long row = (long long)b * chunks;
  constexpr int kAhead = 8;
  for (long long j0 = 0; j0 < used; j0 += kAhead) {
    float ta[kAhead], tr[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const long long j = BACK ? used - 1 - j0 - q : j0 + q;
      ta[q] = tr[q] = 0.0f;
      if (j0 + q >= used) continue;
      ta[q] = totals[2 * (row + j) * C + c];
      tr[q] = totals[2 * (row + j) * C + C + c];
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const long long j = BACK ? used - 1 - j0 - q : j0 + q;
      if (j0 + q >= used) break;
      starts[(row + j) * C + c] = h;
      h = __builtin_fmaf(ta[q], h, tr[q]);
    }
  }
}

// What backward's chunks do to E: E = a (dout + E) from a chunk's last token to its first.
template <typename T>
__global__ __launch_bounds__(256) void scan_back_totals(ScanBackArgs a) {
  constexpr int TT = ScanShape<T>::kBackT, L = ScanShape<T>::kBackChunk;
  constexpr bool kPrecise = Stored<T>::kBytes == 4;
  __shared__ ScanJoin lds;
  const int b = blockIdx.z, blocks = (a.C + kScanWidth - 1) / kScanWidth;
  const int chunk = blockIdx.x / blocks, c0 = (blockIdx.x - chunk * blocks) * kScanWidth;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = c0 + (lane & 7) * 8;
  const bool on = c < a.C;
  const ScanRow row(a.lengths, b, a.N, a.reverse);
  const long long t0 = (long long)chunk * L + (threadIdx.x >> 3) * TT;
  if (chunk && (long long)chunk * L >= row.n) return;
  Raw8<T> rg[TT], rd[TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    rg[j] = rd[j] = none8<T>();
    if (!on || t0 + j >= row.n) continue;
    const long long n = row.token(t0 + j);
    rg[j] = load8_raw<T>(at<T>(a.gate, b * a.vg.batch + n * a.vg.token + c));
    rd[j] = load8_raw<T>(at<T>(a.dout, b * a.vd.batch + n * a.vd.token + c));
  }
  float rate[8], A[8], R[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) { rate[k] = 0.0f; A[k] = 1.0f; R[k] = 0.0f; }
  if (on) load8_f32(a.rate + c, rate);
#pragma unroll
  for (int j = TT - 1; j >= 0; --j) {
    float g[8], d[8];
    widen8<T>(rg[j], g);
    widen8<T>(rd[j], d);
    const bool live = on && t0 + j < row.n;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float da = live ? exp_of<kPrecise>(-rate[k] * sigmoid_of<kPrecise>(g[k])) : 1.0f;
      R[k] = da * (R[k] + (live ? d[k] : 0.0f));
      A[k] *= da;
    }
  }
  join_wave<true>(lds, A, R);
  __syncthreads();
  const int cl = c0 + lane;
  if (wave == 0 && cl < a.C) {
    float ca, cr;
    join_chunk<true>(lds, 4, ca, cr);
    const long long at0 = 2 * ((long long)b * a.chunks + chunk) * a.C + cl;
    a.totals[at0] = ca;
    a.totals[at0 + a.C] = cr;
  }
}

// The gradients of a chunk, from the state in front of it and E behind it (ends; null: one chunk, dstate_out).
template <typename T, int MODE, bool INPUT>
__global__ __launch_bounds__(256) void scan_bwd(ScanBackArgs a) {
  constexpr int TT = ScanShape<T>::kBackT, L = ScanShape<T>::kBackChunk;
  constexpr bool kPrecise = Stored<T>::kBytes == 4;
  __shared__ ScanJoin there, back;
  __shared__ float spread[2][4][kScanWidth];
  const int b = blockIdx.z, blocks = (a.C + kScanWidth - 1) / kScanWidth;
  const int chunk = blockIdx.x / blocks, c0 = (blockIdx.x - chunk * blocks) * kScanWidth;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = c0 + (lane & 7) * 8;
  const bool on = c < a.C;
  const ScanRow row(a.lengths, b, a.N, a.reverse);
  const long long t0 = (long long)chunk * L + (threadIdx.x >> 3) * TT;
  const int cl = c0 + lane;
  const long long at0 = ((long long)b * a.chunks + chunk) * a.C;
  if (chunk && (long long)chunk * L >= row.n) {
    if (wave == 0 && cl < a.C) a.partials[at0 + cl] = 0.0f;
    return;
  }
  Raw8<T> rx[TT], rg[TT], ri[TT], rd[TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    rx[j] = rg[j] = ri[j] = rd[j] = none8<T>();
    if (!on || t0 + j >= row.n) continue;
    const long long n = row.token(t0 + j);
    rx[j] = load8_raw<T>(at<T>(a.x, b * a.vx.batch + n * a.vx.token + c));
    rg[j] = load8_raw<T>(at<T>(a.gate, b * a.vg.batch + n * a.vg.token + c));
    if constexpr (INPUT) ri[j] = load8_raw<T>(at<T>(a.input, b * a.vi.batch + n * a.vi.token + c));
    rd[j] = load8_raw<T>(at<T>(a.dout, b * a.vd.batch + n * a.vd.token + c));
  }
  float rate[8], h0 = 0.0f, e0 = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) rate[k] = 0.0f;
  if (on) load8_f32(a.rate + c, rate);
  if (cl < a.C) {
    h0 = a.starts[at0 + cl];
    e0 = a.ends ? a.ends[at0 + cl] : (a.dstate_out ? a.dstate_out[(long long)b * a.C + cl] : 0.0f);
  }
  float da[TT][8], u[TT][8], sg[TT][8], A[8], R[8], BA[8], BR[8];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    float x[8], g[8], in[8];
    widen8<T>(rx[j], x);
    widen8<T>(rg[j], g);
    widen8<T>(ri[j], in);
    const bool live = on && t0 + j < row.n;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      sg[j][k] = sigmoid_of<kPrecise>(g[k]);
      const ScanWeight w = weight_of<kPrecise, MODE>(rate[k] * sg[j][k]);
      float v = w.m * x[k];
      if constexpr (INPUT) v *= sigmoid_of<kPrecise>(in[k]);
      da[j][k] = live ? w.a : 1.0f;
      u[j][k] = live ? v : 0.0f;
      R[k] = j ? __builtin_fmaf(da[j][k], R[k], u[j][k]) : u[j][k];
      A[k] = j ? A[k] * da[j][k] : da[j][k];
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) { BA[k] = A[k]; BR[k] = 0.0f; }
#pragma unroll
  for (int j = TT - 1; j >= 0; --j) {
    float d[8];
    widen8<T>(rd[j], d);
#pragma unroll
    for (int k = 0; k < 8; ++k) BR[k] = da[j][k] * (BR[k] + d[k]);
  }
  join_wave<false>(there, A, R);
  join_wave<true>(back, BA, BR);
  __syncthreads();
  float ca, cr;
  float h[8], E[8];
  join_chunk<false>(there, wave, ca, cr);
  spread8(spread[0][wave], __builtin_fmaf(ca, h0, cr), h);
  join_chunk<true>(back, 3 - wave, ca, cr);
  spread8(spread[1][wave], __builtin_fmaf(ca, e0, cr), E);
  if (a.dstate_in && chunk == 0 && wave == 0 && cl < a.C) {
    join_chunk<true>(back, 4, ca, cr);
    a.dstate_in[(long long)b * a.C + cl] = __builtin_fmaf(ca, e0, cr);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    h[k] = __builtin_fmaf(A[k], h[k], R[k]);
    E[k] = __builtin_fmaf(BA[k], E[k], BR[k]);
  }
#pragma unroll
  for (int j = 0; j < TT; ++j)   // u: the state before the token
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float v = u[j][k];
      u[j][k] = h[k];
      h[k] = __builtin_fmaf(da[j][k], h[k], v);
    }
  float by_rate[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) by_rate[k] = 0.0f;
#pragma unroll
  for (int j = TT - 1; j >= 0; --j) {
    float x[8], in[8], d[8], dx[8], dg[8], di[8];
    widen8<T>(rx[j], x);
    widen8<T>(ri[j], in);
    widen8<T>(rd[j], d);
    const bool live = on && t0 + j < row.n;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float D = d[k] + E[k], s = sg[j][k], decay = rate[k] * s, ak = da[j][k];
      const ScanWeight w = weight_of<kPrecise, MODE>(decay);
      float i = 1.0f;
      if constexpr (INPUT) i = sigmoid_of<kPrecise>(in[k]);
      const float Di = D * i, Dmi = w.m * Di;
      dx[k] = Dmi;
      if constexpr (INPUT) di[k] = Dmi * x[k] * (1.0f - i);
      // dg = a (D h' - r D i x)
      const float by_log = ak * __builtin_fmaf(D, u[j][k], -w.r * Di * x[k]);
      dg[k] = -by_log * decay * (1.0f - s);
      by_rate[k] = live ? __builtin_fmaf(-by_log, s, by_rate[k]) : by_rate[k];
      E[k] = ak * D;
    }
    if (!live) continue;
    const long long n = row.token(t0 + j);
    store8_stream<T>(at<T>(a.dx, b * a.vdx.batch + n * a.vdx.token + c), dx);
    store8_stream<T>(at<T>(a.dgate, b * a.vdg.batch + n * a.vdg.token + c), dg);
    if constexpr (INPUT) store8_stream<T>(at<T>(a.dinput, b * a.vdi.batch + n * a.vdi.token + c), di);
  }
  __syncthreads();   // the stretches' LDS takes the sums
#pragma unroll
  for (int q = 0; q < 2; ++q)
    *reinterpret_cast<f32x4*>(&there.stretch[threadIdx.x >> 3][0][(lane & 7) * 8 + 4 * q]) =
        f32x4{by_rate[4 * q], by_rate[4 * q + 1], by_rate[4 * q + 2], by_rate[4 * q + 3]};
  __syncthreads();
  if (wave == 0 && cl < a.C) {
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j) sum += there.stretch[j][0][lane];
    a.partials[at0 + cl] = sum;
  }
}

// drate: the chunks' sums of every batch row, in a fixed order, in fp64 (a long sequence has thousands of them).
__global__ __launch_bounds__(1024) void scan_rate_sums(const float* partials, float* drate, long long parts, int C) {
  __shared__ double lds[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  double sum = 0.0;
  if (c < C)
    for (long long p = wave; p < parts; p += 16) sum += (double)partials[p * C + c];
  lds[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && c < C) {
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += lds[w][lane];
    drate[c] = (float)sum;
  }
}

struct ScanStepArgs {
  const void *x, *gate, *input;
  void* out;
  long long sx, sg, si, so;
  const float *rate, *state_in;
  float* state_out;
  int B, C;
};

// One token of every batch row: a thread takes 8 channels.
template <typename T, int MODE, bool INPUT>
__global__ __launch_bounds__(64) void scan_step(ScanStepArgs a) {
  constexpr bool kPrecise = Stored<T>::kBytes == 4;
  const int b = blockIdx.y, c = (blockIdx.x * 64 + threadIdx.x) * 8;
  if (c >= a.C) return;
  const Raw8<T> rx = load8_raw<T>(at<T>(a.x, b * a.sx + c)), rg = load8_raw<T>(at<T>(a.gate, b * a.sg + c));
  Raw8<T> ri = none8<T>();
  if constexpr (INPUT) ri = load8_raw<T>(at<T>(a.input, b * a.si + c));
  float x[8], g[8], in[8], rate[8], h[8];
  load8_f32(a.rate + c, rate);
  const long long at0 = (long long)b * a.C + c;
#pragma unroll
  for (int k = 0; k < 8; ++k) h[k] = 0.0f;
  if (a.state_in) load8_f32(a.state_in + at0, h);
  widen8<T>(rx, x);
  widen8<T>(rg, g);
  widen8<T>(ri, in);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const ScanWeight w = weight_of<kPrecise, MODE>(rate[k] * sigmoid_of<kPrecise>(g[k]));
    float v = w.m * x[k];
    if constexpr (INPUT) v *= sigmoid_of<kPrecise>(in[k]);
    h[k] = __builtin_fmaf(w.a, h[k], v);
  }
  if (a.state_out) store8<F32>(reinterpret_cast<unsigned char*>(a.state_out + at0), h);
  store8<T>(at<T>(a.out, b * a.so + c), h);
}

}  // namespace lf
