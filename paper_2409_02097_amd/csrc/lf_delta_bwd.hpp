// Gradients of the gated delta rule (lf_delta.hpp), with dO those of the outputs times `scale` and dS1 that of the state a
// chunk ends with.  Back through a chunk's equations:
//
//     dU = P^T dO + (e^(gamma_63 - gamma) K) dS1,    P = Q K^T * D
//     dS0 = e^gamma_63 dS1 + (e^gamma Q)^T dO - W^T dU
//     dX = T^T dU,   dV = beta dX,   dbeta_i = dX_i.u_i / beta_i
//     dQ = e^gamma dO S0^T + (dO U^T * D) K                                   (lower part)
//     dK = -e^gamma dV S0^T + e^(gamma_63 - gamma) U dS1^T + (dO U^T * D)^T Q + M K + M^T K,   M = -(dV U^T * D)   (strictly lower)
//     dg_t = sum over the chunk's tokens i >= t of (q_i.dq_i - v_i.dv_i)  +  <dS1, S1>
//
// The last line holds because scaling the state by a factor from token t on is the same as scaling the queries there by it
// and the values by its inverse.  Only dU and dS0 depend on the chunk behind: P^T dO is formed for all chunks at once
// (delta_back_outputs), a scan runs from the last chunk to the first (delta_back_scan), and the rest follows for all chunks
// at once (delta_gradients), where the value heads that share a query and key head are summed in their order.
#pragma once
#include "lf_delta.hpp"

namespace lf {

// ---- P^T dO --------------------------------------------------------------------------------------------------------------------
inline int delta_back_outputs_lds(int dkb, int dvb) {
  const int wide = dkb > dvb ? dkb : dvb;
  return 64 * (16 * dkb + 4) * 4 + 64 * (16 * wide + 4) * 4 + 64 * kLdT * 4 + 64 * 8;
}

template <typename T> __global__ __launch_bounds__(256) void delta_back_outputs(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  const int wide = a.dkb > a.dvb ? a.dkb : a.dvb, ld = 16 * a.dkb + 4, ldo = 16 * a.dvb + 4;
  float* q = reinterpret_cast<float*>(smem);
  float* k = q + 64 * ld;
  float* mp = k + 64 * (16 * wide + 4);
  double* gamma = reinterpret_cast<double*>(mp + 64 * kLdT);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4;
  const long long c = (long long)blockIdx.y * a.nc + blockIdx.x;
  if (wave == 0) gamma[lane] = chunk_gamma(a, w);
  stage_rows<T>(q, ld, a.q, a.vq, w.b, w.hk, w.n0, w.valid, a.dk, a.dkb);
  stage_rows<T>(k, ld, a.k, a.vk, w.b, w.hk, w.n0, w.valid, a.dk, a.dkb);
  __syncthreads();
  chunk_scores<false>(a, q, k, ld, gamma, nullptr, mp);
  __syncthreads();
  float* o = k;
  stage_rows<T>(o, ldo, a.dout, a.vdo, w.b, w.h, w.n0, w.valid, a.dv, a.dvb);
  __syncthreads();
  for (int sl = 0; sl < a.dvb; ++sl) {
    f32x4 acc = {0, 0, 0, 0};
    for (int kb = wave; kb < 4; ++kb)
      acc = mfma_block(rows_near(mp + 16 * kb * kLdT + 16 * wave, kLdT), rows_near(o + 16 * kb * ldo + 16 * sl, ldo), acc);
    float* du = a.du + (c * a.dvb + sl) * 1024;
#pragma unroll
    for (int r = 0; r < 4; ++r) du[(16 * wave + row4 + r) * 16 + col] = acc[r] * a.scale;
  }
  (void)tid;
}

// ---- the scan backwards ----------------------------------------------------------------------------------------------------------
template <typename T, int BLOCKS> __global__ __launch_bounds__(256) void delta_back_scan(DeltaArgs a) {
  __shared__ __align__(16) float sl[16 * 4 * BLOCKS * kLdS];
  __shared__ __align__(16) float ul[64 * kLdS], ol[64 * kLdS];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4;
  const int slice = blockIdx.x, bh = blockIdx.y, ch = slice * 16 + col;
  const DeltaAt first(a, bh, 0);
  const long long tokens = tokens_of(a.lengths, first.b, a.N);
  f32x4 s[BLOCKS];
#pragma unroll
  for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * (wave + 4 * t) + row4 + r;
      s[t][r] = a.dstate_out && row < a.dk && ch < a.dv ? a.dstate_out[((long long)bh * a.dk + row) * a.dv + ch] : 0.0f;
    }
  for (int i = (int)((tokens + 63) / 64) - 1; i >= 0; --i) {
    const DeltaAt w(a, bh, i);
    const long long c = (long long)bh * a.nc + i;
    float* keep = a.ds + (c * a.dvb + slice) * a.dkb * 256;
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t) {
      if (wave + 4 * t >= a.dkb) continue;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (wave + 4 * t) + row4 + r;
        sl[row * kLdS + col] = s[t][r];
        keep[row * 16 + col] = s[t][r];
      }
    }
    __syncthreads();
    const float* decay = a.decay + c * kDecayRows;
    float* mu = a.du + (c * a.dvb + slice) * 1024;
    f32x4 acc = {0, 0, 0, 0};
    const int kn = 16 * wave + col;
    for (int kb = 0; kb < a.dkb; ++kb) {
      f32x4 key = {0, 0, 0, 0};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int kc = 16 * kb + row4 + r;
        if (kn < w.valid && kc < a.dk) key[r] = load1<T>(a.k, w.b * a.vk.b + w.hk * a.vk.h + (w.n0 + kn) * a.vk.n + kc);
      }
      acc = mfma_block(key, rows_near(sl + 16 * kb * kLdS, kLdS), acc);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * wave + row4 + r;
      const float u = __builtin_fmaf(acc[r], decay[kDecayLeft + row], mu[row * 16 + col]);
      mu[row * 16 + col] = u;
      ul[row * kLdS + col] = u;
      float o = 0.0f;
      if (row < w.valid && ch < a.dv) o = load1<T>(a.dout, w.b * a.vdo.b + w.h * a.vdo.h + (w.n0 + row) * a.vdo.n + ch);
      ol[row * kLdS + col] = o * a.scale * decay[kDecaySince + row];
    }
    __syncthreads();
    const float whole = decay[kDecaySince + 63];
    const float* mw = a.w + c * a.dkb * 1024;
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t) {
      if (wave + 4 * t >= a.dkb) continue;
      s[t] *= whole;
      const int kc = 16 * (wave + 4 * t) + col;
      for (int kb = 0; kb < 4; ++kb) {
        f32x4 qry = {0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int n = 16 * kb + row4 + r;
          if (n < w.valid && kc < a.dk) qry[r] = load1<T>(a.q, w.b * a.vq.b + w.hk * a.vq.h + (w.n0 + n) * a.vq.n + kc);
        }
        s[t] = mfma_block(qry, rows_near(ol + 16 * kb * kLdS, kLdS), s[t]);
        s[t] = mfma_block(-rows_near(mw + (wave + 4 * t) * 1024 + 256 * kb, 16), rows_near(ul + 16 * kb * kLdS, kLdS), s[t]);
      }
    }
    // (sl is written again by the next round: its readers are behind the barrier before the second product)
  }
  if (a.dstate_in) {
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (wave + 4 * t) + row4 + r;
        if (row < a.dk && ch < a.dv) a.dstate_in[((long long)bh * a.dk + row) * a.dv + ch] = s[t][r];
      }
  }
}

// ---- the gradients ------------------------------------------------------------------------------------------------------------
inline int delta_gradients_lds(int dkb) {
  return 2 * 64 * (16 * dkb + 4) * 4 + 2 * 64 * kLdT * 4 + 3 * 64 * kLdS * 4 + 64 * 8 + kDecayRows * 4 + 64 * 4 + 16;
}

template <typename T, int KB> __global__ __launch_bounds__(256) void delta_gradients(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int b = (unsigned)blockIdx.y / (unsigned)a.Hk, hk = blockIdx.y - b * a.Hk, group = a.H / a.Hk;
  const int ld = 16 * a.dkb + 4;
  float* q = reinterpret_cast<float*>(smem);
  float* k = q + 64 * ld;
  float* mt = k + 64 * ld;                  // T, then dO U^T * D
  float* mm = mt + 64 * kLdT;               // M
  float* tiles = mm + 64 * kLdT;            // dO, dV, U: 16 channels of a chunk each
  double* gamma = reinterpret_cast<double*>(tiles + 3 * 64 * kLdS);
  float* decay = reinterpret_cast<float*>(gamma + 64);
  float* dgamma = decay + kDecayRows;
  float* inner = dgamma + 64;
  float *to = tiles, *tv = tiles + 64 * kLdS, *tu = tiles + 2 * 64 * kLdS;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4;
  const DeltaAt any(a, b * a.H + hk * group, blockIdx.x);
  if (any.valid == 0) return;
  stage_rows<T>(q, ld, a.q, a.vq, b, hk, any.n0, any.valid, a.dk, a.dkb);
  stage_rows<T>(k, ld, a.k, a.vk, b, hk, any.n0, any.valid, a.dk, a.dkb);
  f32x4 sum_q[KB], sum_k[KB];
#pragma unroll
  for (int i = 0; i < KB; ++i) sum_q[i] = sum_k[i] = f32x4{0, 0, 0, 0};
  for (int member = 0; member < group; ++member) {
    const DeltaAt w(a, b * a.H + hk * group + member, blockIdx.x);
    const long long c = (long long)w.bh * a.nc + blockIdx.x;
    __syncthreads();
    if (wave == 0) gamma[lane] = chunk_gamma(a, w);
    decay[tid] = a.decay[c * kDecayRows + tid];
    for (int i = tid; i < 64 * 16; i += 256) {
      const int r = i >> 4, v = (i & 15) * 4;
      *reinterpret_cast<f32x4*>(mt + r * kLdT + v) = *reinterpret_cast<const f32x4*>(a.t + c * 4096 + r * 64 + v);
    }
    f32x4 dq[KB], dk[KB], mo[4], mv[4];
#pragma unroll
    for (int i = 0; i < KB; ++i) dq[i] = dk[i] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) mo[i] = mv[i] = f32x4{0, 0, 0, 0};
    float dbeta[4] = {0, 0, 0, 0}, vdv[4] = {0, 0, 0, 0}, ss = 0.0f;
    for (int sl = 0; sl < a.dvb; ++sl) {
      const float* du = a.du + (c * a.dvb + sl) * 1024;
      const float* mu = a.u + (c * a.dvb + sl) * 1024;
      const float* s0 = a.s + (((long long)w.bh * (a.nc + 1) + blockIdx.x) * a.dvb + sl) * a.dkb * 256;
      const float* s1 = s0 + (long long)a.dvb * a.dkb * 256;
      const float* ds = a.ds + (c * a.dvb + sl) * a.dkb * 256;
      const int ch = 16 * sl + col;
      __syncthreads();   // T is there; the tiles of the slice before are read
      f32x4 dx = {0, 0, 0, 0};
      for (int kb = wave; kb < 4; ++kb)
        dx = mfma_block(rows_near(mt + 16 * kb * kLdT + 16 * wave, kLdT), rows_near(du + 256 * kb, 16), dx);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = 16 * wave + row4 + r;
        const bool on = n < w.valid && ch < a.dv;
        const float beta = decay[kDecayBeta + n], u = mu[n * 16 + col];
        const float dv = beta == kDeltaTinyBeta ? 0.0f : beta * dx[r];
        float o = 0.0f;
        if (on) {
          o = load1<T>(a.dout, w.b * a.vdo.b + w.h * a.vdo.h + (w.n0 + n) * a.vdo.n + ch) * a.scale;
          vdv[r] = __builtin_fmaf(load1<T>(a.v, w.b * a.vv.b + w.h * a.vv.h + (w.n0 + n) * a.vv.n + ch), dv, vdv[r]);
          store1<T>(a.dv_out, w.b * a.vdv.b + w.h * a.vdv.h + (w.n0 + n) * a.vdv.n + ch, dv);
        }
        dbeta[r] = __builtin_fmaf(dx[r], u / beta, dbeta[r]);
        to[n * kLdS + col] = o;
        tv[n * kLdS + col] = dv;
        tu[n * kLdS + col] = u;
      }
      __syncthreads();
      const f32x4 fo = steps_near(to + 16 * wave * kLdS, kLdS), fv = steps_near(tv + 16 * wave * kLdS, kLdS);
      const f32x4 fu = steps_near(tu + 16 * wave * kLdS, kLdS);
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        if (nt > wave) continue;
        f32x4 un = steps_near(tu + 16 * nt * kLdS, kLdS);
        if (decay[kDecayBeta + 16 * nt + col] == kDeltaTinyBeta) un = f32x4{0, 0, 0, 0};
        mo[nt] = mfma_block(fo, un, mo[nt]);
        mv[nt] = mfma_block(-fv, un, mv[nt]);
      }
      const float since = decay[kDecaySince + 16 * wave + col], write = decay[kDecayWrite + 16 * wave + col];
#pragma unroll
      for (int nb = 0; nb < KB; ++nb) {
        if (nb >= a.dkb) continue;
        const f32x4 f0 = steps_near(s0 + 256 * nb, 16), f1 = steps_near(ds + 256 * nb, 16);
        dq[nb] = mfma_block(fo * since, f0, dq[nb]);
        dk[nb] = mfma_block(fv * -since, f0, dk[nb]);
        dk[nb] = mfma_block(fu * write, f1, dk[nb]);
      }
      for (int i = tid; i < a.dkb * 256; i += 256) ss = __builtin_fmaf(ds[i], s1[i], ss);
    }
    __syncthreads();
    for (int nt = 0; nt < 4; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * wave + row4 + r, j = 16 * nt + col;
        const float d = j <= i ? decay_between(gamma, i, j) : 0.0f;
        mt[i * kLdT + j] = j <= i ? mo[nt][r] * d : 0.0f;
        mm[i * kLdT + j] = j < i ? mv[nt][r] * d : 0.0f;
      }
    // the rows' sums over channels, and <dS1, S1>
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      dbeta[r] = lanes_sum<16>(dbeta[r]);
      vdv[r] = lanes_sum<16>(vdv[r]);
    }
    ss = lanes_sum<64>(ss);
    if (lane == 0) inner[wave] = ss;
    __syncthreads();
    float qdq[4] = {0, 0, 0, 0};
#pragma unroll
    for (int nb = 0; nb < KB; ++nb) {
      if (nb >= a.dkb) continue;
      for (int kb = 0; kb < 4; ++kb) {
        const f32x4 kk = rows_near(k + 16 * kb * ld + 16 * nb, ld);
        if (kb <= wave) {
          dq[nb] = mfma_block(steps_near(mt + 16 * wave * kLdT + 16 * kb, kLdT), kk, dq[nb]);
          dk[nb] = mfma_block(steps_near(mm + 16 * wave * kLdT + 16 * kb, kLdT), kk, dk[nb]);
        }
        if (kb >= wave) {
          dk[nb] = mfma_block(rows_near(mt + 16 * kb * kLdT + 16 * wave, kLdT), rows_near(q + 16 * kb * ld + 16 * nb, ld), dk[nb]);
          dk[nb] = mfma_block(rows_near(mm + 16 * kb * kLdT + 16 * wave, kLdT), kk, dk[nb]);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) qdq[r] = __builtin_fmaf(q[(16 * wave + row4 + r) * ld + 16 * nb + col], dq[nb][r], qdq[r]);
      sum_q[nb] += dq[nb];
      sum_k[nb] += dk[nb];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      qdq[r] = lanes_sum<16>(qdq[r]);
      const int n = 16 * wave + row4 + r;
      if (col == 0) {
        dgamma[n] = qdq[r] - vdv[r];
        if (n < w.valid) a.dbeta[w.b * a.vdg.b + w.h * a.vdg.h + (w.n0 + n) * a.vdg.n] = dbeta[r];
      }
    }
    __syncthreads();
    if (wave == 0) {
      float x = dgamma[lane];
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const float y = __shfl_down(x, m, 64);
        if (lane + m < 64) x += y;
      }
      x += (inner[0] + inner[1]) + (inner[2] + inner[3]);
      if (lane < w.valid) a.dg[w.b * a.vdg.b + w.h * a.vdg.h + (w.n0 + lane) * a.vdg.n] = x;
    }
  }
#pragma unroll
  for (int nb = 0; nb < KB; ++nb) {
    const int ch = 16 * nb + col;
    if (ch >= a.dk) continue;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = 16 * wave + row4 + r;
      if (n >= any.valid) continue;
      store1<T>(a.dq, b * a.vdq.b + hk * a.vdq.h + (any.n0 + n) * a.vdq.n + ch, sum_q[nb][r]);
      store1<T>(a.dk_out, b * a.vdk.b + hk * a.vdk.h + (any.n0 + n) * a.vdk.n + ch, sum_k[nb][r]);
    }
  }
}

}  // namespace lf
