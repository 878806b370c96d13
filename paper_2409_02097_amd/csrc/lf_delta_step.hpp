// The gated delta rule for one new token: S' = e^g S, u = beta (v - S'^T k), S = S' + k u^T, o = scale S^T q.
// Bound: HBM, the state in and out once.  A workgroup holds 32 value channels of one head's state in registers (a thread 4 of
// them in every 32nd row), so that S0^T k and S0^T q come from one pass: o = scale (e^g S0^T q + (q.k) u).
// 64 rows of 16 heads of 128 x 128: 24.2 us for 135 MB (5.6 TB/s); one row of 8 heads of 64 x 64: 4.0 us, a launch's latency.
#pragma once
#include "lf_vec8.hpp"

namespace lf {

struct DeltaStepArgs {
  const void *q, *k, *v;
  const float *g, *beta, *state_in;
  void* out;
  float* state_out;
  long long qb, qh, kb, kh, vb, vh, gb, gh, ob, oh;   // element strides {batch, head}
  int H, Hk, dk, dv;
  float scale;
};

constexpr int kStepCols = 32;

template <typename T, int ROWS> __global__ __launch_bounds__(256) void delta_step(DeltaStepArgs a) {
  __shared__ float kq[2][32 * ROWS];
  __shared__ __align__(16) float part[4][2][kStepCols];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int b = (unsigned)blockIdx.y / (unsigned)a.H, h = blockIdx.y - b * a.H, hk = (unsigned)h / (unsigned)(a.H / a.Hk);
  const int c = blockIdx.x * kStepCols + (tid & 7) * 4, row0 = tid >> 3;
  const bool on = c < a.dv;
  const long long base = (long long)blockIdx.y * a.dk * a.dv + c;
  f32x4 s[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = row0 + 32 * i;
    s[i] = f32x4{0, 0, 0, 0};
    if (a.state_in && on && row < a.dk) s[i] = *reinterpret_cast<const f32x4*>(a.state_in + base + (long long)row * a.dv);
  }
  const float g = a.g[b * a.gb + h * a.gh], beta = a.beta[b * a.gb + h * a.gh], decay = expf(g);
  float v[4] = {0, 0, 0, 0};
  if (on) {
    const unsigned char* p = at<T>(a.v, b * a.vb + h * a.vh + c);
    if constexpr (Stored<T>::kBytes == 4) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(p);
      v[0] = w[0]; v[1] = w[1]; v[2] = w[2]; v[3] = w[3];
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2*>(p);
      unpack2<T>(w[0], v[0], v[1]);
      unpack2<T>(w[1], v[2], v[3]);
    }
  }
  for (int i = tid; i < 8 * ROWS; i += 256) {   // 8 channels a thread: first the key's, then the query's
    const int which = i / (4 * ROWS), ch = (i - which * 4 * ROWS) * 8;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (ch < a.dk) load8<T>(which ? at<T>(a.q, b * a.qb + hk * a.qh + ch) : at<T>(a.k, b * a.kb + hk * a.kh + ch), x);
#pragma unroll
    for (int j = 0; j < 8; ++j) kq[which][ch + j] = x[j];
  }
  __syncthreads();
  float qk = 0.0f;
#pragma unroll
  for (int i = 0; i < (ROWS + 1) / 2; ++i) {
    const int ch = lane + 64 * i;
    if (ch < 32 * ROWS) qk = __builtin_fmaf(kq[0][ch], kq[1][ch], qk);
  }
  qk = lanes_sum<64>(qk);
  f32x4 sk = {0, 0, 0, 0}, sq = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    sk += s[i] * kq[0][row0 + 32 * i];
    sq += s[i] * kq[1][row0 + 32 * i];
  }
#pragma unroll
  for (int m = 8; m < 64; m <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sk[j] += __shfl_xor(sk[j], m, 64);
      sq[j] += __shfl_xor(sq[j], m, 64);
    }
  if (lane < 8) {
    *reinterpret_cast<f32x4*>(&part[wave][0][lane * 4]) = sk;
    *reinterpret_cast<f32x4*>(&part[wave][1][lane * 4]) = sq;
  }
  __syncthreads();
  const int at4 = (tid & 7) * 4;
  f32x4 u, o;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float rk = (part[0][0][at4 + j] + part[1][0][at4 + j]) + (part[2][0][at4 + j] + part[3][0][at4 + j]);
    const float rq = (part[0][1][at4 + j] + part[1][1][at4 + j]) + (part[2][1][at4 + j] + part[3][1][at4 + j]);
    u[j] = beta * (v[j] - decay * rk);
    o[j] = a.scale * __builtin_fmaf(qk, u[j], decay * rq);
  }
  if (!on) return;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = row0 + 32 * i;
    if (row < a.dk)
      *reinterpret_cast<f32x4*>(a.state_out + base + (long long)row * a.dv) = s[i] * decay + u * kq[0][row];
  }
  if (row0 == 0) {
    unsigned char* p = at<T>(a.out, b * a.ob + h * a.oh + c);
    if constexpr (Stored<T>::kBytes == 4) *reinterpret_cast<f32x4*>(p) = o;
    else *reinterpret_cast<u32x2*>(p) = u32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
  }
}

}  // namespace lf
