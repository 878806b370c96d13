// The gated delta rule.  Per (batch, head), with keys and queries of d_k channels, values of d_v, log decays g and
// corrections beta, and an fp32 state S of d_k x d_v:
//
//     S' = e^g_t S;   u_t = beta_t (v_t - S'^T k_t);   S = S' + k_t u_t^T;   o_t = scale S^T q_t
//
// In chunks of 64 tokens, with gamma the running sum of g inside a chunk, D_ij = e^(gamma_i - gamma_j) for j <= i, and S0
// the state a chunk starts from:
//
//     A = strictly lower part of (beta_i k_i.k_j D_ij),   T = (I + A)^-1,   W = T (beta e^gamma K),   U0 = T (beta V)
//     U = U0 - W S0,   O = scale (e^gamma Q S0 + (Q K^T * D) U),   S1 = e^gamma_63 S0 + (e^(gamma_63 - gamma) K)^T U
//
// Only U and S1 depend on the chunk before: T, W, U0 are formed for all chunks at once (delta_prepare), a scan runs over the
// chunks with a slice of 16 value channels per workgroup (delta_scan), and the outputs follow for all chunks at once
// (delta_out).  gamma and its differences are fp64: behind a token that forgets nearly everything the differences of an
// fp32 sum have lost the small decays that follow it.  Everything that reaches the state or an fp32 result is fp32 accurate.
//
// Layout of what passes between the kernels, fp32: blocks of 16 channels, [channels / 16][rows][16], so that every matrix
// operand is a contiguous kilobyte.
#pragma once
#include "lf_vec8.hpp"

namespace lf {

constexpr int kDeltaChunk = 64;
constexpr float kDeltaTinyBeta = 1e-18f;

struct DeltaView { long long b, h, n; };   // element strides

struct DeltaArgs {
  const void *q, *k, *v;
  const float *g, *beta;
  const float* state_in;
  void* out;
  float* state_out;
  const int* lengths;
  DeltaView vq, vk, vv, vg, vo;
  float *t, *w, *u, *s, *decay;   // per chunk: [64][64], [dkb][64][16], [dvb][64][16], [dvb][16 dkb][16] (one more per head), [4][64]
  long long N;
  int H, Hk, nc;                  // chunks of N tokens
  int dk, dv, dkb, dvb;           // channels, and blocks of 16 of them
  float scale;
  // backward
  const void* dout;
  const float* dstate_out;
  void *dq, *dk_out, *dv_out;
  float *dg, *dbeta, *dstate_in;
  DeltaView vdo, vdq, vdk, vdv, vdg;
  float *du, *ds;                 // as u; as s (the gradient of a chunk's last state)
};

// rows of `decay`: e^gamma; e^(gamma_63 - gamma), 0 where beta is 0 (such a token leaves the state alone); beta, never 0 (u / beta
// is needed where beta is 0 too, for its gradient); e^(gamma_63 - gamma) everywhere
constexpr int kDecaySince = 0, kDecayWrite = 64, kDecayBeta = 128, kDecayLeft = 192, kDecayRows = 256;

struct DeltaAt {
  int b, h, hk, bh;
  long long n0;      // first token of the chunk
  int valid;         // tokens of it that count
  LF_DEV DeltaAt(const DeltaArgs& a, int bh_, int chunk) {
    bh = bh_;
    b = (unsigned)bh_ / (unsigned)a.H;
    h = bh_ - b * a.H;
    hk = (unsigned)h / (unsigned)(a.H / a.Hk);
    n0 = (long long)chunk * kDeltaChunk;
    const long long left = tokens_of(a.lengths, b, a.N) - n0;
    valid = left <= 0 ? 0 : (left < kDeltaChunk ? (int)left : kDeltaChunk);
  }
};

// ---- fp32 products of 16 x 16 blocks ----------------------------------------------------------------------------------
// Lane l: row (or column) l % 16 and, of a block of 16 contraction steps, steps 4 (l / 16) .. + 3: four instructions.
LF_DEV f32x4 mfma_block(f32x4 a, f32x4 b, f32x4 c) {
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[0], b[0], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[1], b[1], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[2], b[2], c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a[3], b[3], c, 0, 0, 0);
}
// operand of a matrix whose contraction steps are neighbours in memory, or whose rows (columns) are
LF_DEV f32x4 steps_near(const float* p, int ld) {
  const int l = threadIdx.x & 63;
  return *reinterpret_cast<const f32x4*>(p + (l & 15) * ld + 4 * (l >> 4));
}
LF_DEV f32x4 rows_near(const float* p, int ld) {
  const int l = threadIdx.x & 63;
  const float* r = p + 4 * (l >> 4) * ld + (l & 15);
  return f32x4{r[0], r[ld], r[2 * ld], r[3 * ld]};
}

template <typename T> LF_DEV float load1(const void* p, long long i) {
  if constexpr (Stored<T>::kBytes == 4) {
    return static_cast<const float*>(p)[i];
  } else {
    float x, y;
    unpack2<T>(static_cast<const uint16_t*>(p)[i], x, y);
    return x;
  }
}
template <typename T> LF_DEV void store1(void* p, long long i, float v) {
  if constexpr (Stored<T>::kBytes == 4) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = (uint16_t)pack2<T>(v, 0.0f);
}

// A chunk's rows of one head in LDS as fp32, `ld` apart, zeros behind the last token and channel.
template <typename T>
LF_DEV void stage_rows(float* to, int ld, const void* x, const DeltaView& v, int b, int h, long long n0, int valid, int d,
                       int blocks) {
  const int vecs = blocks * 2;
  for (int i = threadIdx.x; i < kDeltaChunk * vecs; i += blockDim.x) {
    const int t = (unsigned)i / (unsigned)vecs, c = (i - t * vecs) * 8;
    float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (t < valid && c < d) load8<T>(at<T>(x, b * v.b + h * v.h + (n0 + t) * v.n + c), y);
    float* p = to + t * ld + c;
    *reinterpret_cast<f32x4*>(p) = f32x4{y[0], y[1], y[2], y[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{y[4], y[5], y[6], y[7]};
  }
}

// gamma of the 64 tokens, by the first wave; a decay of -infinity counts as -10^4, which is none left
LF_DEV double chunk_gamma(const DeltaArgs& a, const DeltaAt& w) {
  const int t = threadIdx.x & 63;
  float g = 0.0f;
  if (t < w.valid) g = a.g[w.b * a.vg.b + w.h * a.vg.h + (w.n0 + t) * a.vg.n];
  double x = g < -1e4f ? -1e4 : (double)g;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const double y = __shfl_up(x, m, 64);
    if (t >= m) x += y;
  }
  return x;
}

LF_DEV float decay_between(const double* gamma, int i, int j) { return expf((float)(gamma[i] - gamma[j])); }

constexpr int kLdT = 68;   // leading dimension of a 64 x 64 matrix in LDS: both operand forms are free of bank conflicts

// ---- T, W, U0 of every chunk ----------------------------------------------------------------------------------------------
inline int delta_prepare_lds(int dkb, int dvb) {
  const int wide = dkb > dvb ? dkb : dvb;
  return 64 * (16 * wide + 4) * 4 + 2 * 64 * kLdT * 4 + 64 * 8 + kDecayRows * 4 + 64 * 4;
}

template <typename T> __global__ __launch_bounds__(256) void delta_prepare(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  const int wide = a.dkb > a.dvb ? a.dkb : a.dvb, ld = 16 * wide + 4;
  float* x = reinterpret_cast<float*>(smem);
  float* ma = x + 64 * ld;
  float* mt = ma + 64 * kLdT;
  double* gamma = reinterpret_cast<double*>(mt + 64 * kLdT);
  float* decay = reinterpret_cast<float*>(gamma + 64);
  float* both = decay + kDecayRows;   // beta e^gamma
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4;
  const long long c = (long long)blockIdx.y * a.nc + blockIdx.x;
  if (wave == 0) {
    const double y = chunk_gamma(a, w), last = __shfl(y, 63, 64);
    float beta = 0.0f;
    if (lane < w.valid) beta = a.beta[w.b * a.vg.b + w.h * a.vg.h + (w.n0 + lane) * a.vg.n];
    const bool none = fabsf(beta) < kDeltaTinyBeta;
    if (none) beta = kDeltaTinyBeta;
    const float since = expf((float)y), left = expf((float)(last - y));
    gamma[lane] = y;
    decay[kDecaySince + lane] = since;
    decay[kDecayWrite + lane] = none ? 0.0f : left;
    decay[kDecayBeta + lane] = beta;
    decay[kDecayLeft + lane] = left;
    both[lane] = beta * since;
  }
  stage_rows<T>(x, ld, a.k, a.vk, w.b, w.hk, w.n0, w.valid, a.dk, a.dkb);
  for (int i = tid; i < 64 * kLdT; i += 256) mt[i] = 0.0f;
  __syncthreads();
  if (tid < kDecayRows) a.decay[c * kDecayRows + tid] = decay[tid];
  // A, rows 16 wave .. + 15
  for (int nt = 0; nt <= wave; ++nt) {
    f32x4 acc = {0, 0, 0, 0};
    for (int kb = 0; kb < a.dkb; ++kb)
      acc = mfma_block(steps_near(x + 16 * wave * ld + 16 * kb, ld), steps_near(x + 16 * nt * ld + 16 * kb, ld), acc);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * wave + row4 + r, j = 16 * nt + col;
      ma[i * kLdT + j] = i > j ? decay[kDecayBeta + i] * acc[r] * decay_between(gamma, i, j) : 0.0f;
    }
  }
  __syncthreads();
  // the blocks on the diagonal, a column per lane, by substitution
  if (lane < 16) {
    const float* m = ma + 16 * wave * kLdT + 16 * wave;
    float t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = i == lane ? 1.0f : 0.0f;
#pragma unroll
      for (int l = 0; l < i; ++l) s = __builtin_fmaf(-m[i * kLdT + l], t[l], s);
      t[i] = s;
      mt[(16 * wave + i) * kLdT + 16 * wave + lane] = s;
    }
  }
  __syncthreads();
  // the blocks below it: T_ij = -T_ii sum_l A_il T_lj, by their distance from the diagonal
  for (int far = 1; far < 4; ++far) {
    const int i = wave + far, j = wave;
    float* tij = mt + 16 * i * kLdT + 16 * j;
    if (i < 4) {
      f32x4 acc = {0, 0, 0, 0};
      for (int l = j; l < i; ++l)
        acc = mfma_block(steps_near(ma + 16 * i * kLdT + 16 * l, kLdT), rows_near(mt + 16 * l * kLdT + 16 * j, kLdT), acc);
#pragma unroll
      for (int r = 0; r < 4; ++r) tij[(row4 + r) * kLdT + col] = acc[r];
    }
    __syncthreads();
    f32x4 acc = {0, 0, 0, 0};
    if (i < 4) acc = mfma_block(steps_near(mt + 16 * i * kLdT + 16 * i, kLdT), rows_near(tij, kLdT), acc);
    __syncthreads();
    if (i < 4) {
#pragma unroll
      for (int r = 0; r < 4; ++r) tij[(row4 + r) * kLdT + col] = -acc[r];
    }
    __syncthreads();
  }
  if (a.t) {
    for (int i = tid; i < 64 * 16; i += 256) {
      const int r = i >> 4, v = (i & 15) * 4;
      *reinterpret_cast<f32x4*>(a.t + c * 4096 + r * 64 + v) = *reinterpret_cast<const f32x4*>(mt + r * kLdT + v);
    }
  }
  // W, then U0 where the keys were
  auto times = [&](const float* scale, float* to, int blocks) {
    for (int nb = 0; nb < blocks; ++nb) {
      f32x4 acc = {0, 0, 0, 0};
      for (int kb = 0; kb <= wave; ++kb) {
        const f32x4 s = *reinterpret_cast<const f32x4*>(scale + 16 * kb + row4);
        acc = mfma_block(steps_near(mt + 16 * wave * kLdT + 16 * kb, kLdT) * s, rows_near(x + 16 * kb * ld + 16 * nb, ld), acc);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) to[((long long)nb * 64 + 16 * wave + row4 + r) * 16 + col] = acc[r];
    }
  };
  times(both, a.w + c * a.dkb * 1024, a.dkb);
  __syncthreads();
  stage_rows<T>(x, ld, a.v, a.vv, w.b, w.h, w.n0, w.valid, a.dv, a.dvb);
  __syncthreads();
  times(decay + kDecayBeta, a.u + c * a.dvb * 1024, a.dvb);
}

// ---- the scan ---------------------------------------------------------------------------------------------------------------
// A workgroup takes 16 value channels of one head through all chunks; its four waves hold the state's row blocks
// wave, wave + 4, ... as accumulators.
constexpr int kLdS = 20;

template <typename T, int BLOCKS> __global__ __launch_bounds__(256) void delta_scan(DeltaArgs a) {
  __shared__ __align__(16) float sl[16 * 4 * BLOCKS * kLdS];
  __shared__ __align__(16) float ul[64 * kLdS];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4;
  const int slice = blockIdx.x, bh = blockIdx.y, ch = slice * 16 + col;
  const DeltaAt first(a, bh, 0);
  const long long tokens = tokens_of(a.lengths, first.b, a.N);
  const int chunks = (int)((tokens + 63) / 64);
  f32x4 s[BLOCKS];
#pragma unroll
  for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * (wave + 4 * t) + row4 + r;
      s[t][r] = a.state_in && row < a.dk && ch < a.dv ? a.state_in[((long long)bh * a.dk + row) * a.dv + ch] : 0.0f;
    }
  for (int i = 0;; ++i) {
    float* keep = a.s + (((long long)bh * (a.nc + 1) + i) * a.dvb + slice) * a.dkb * 256;
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
    if (i == chunks) break;
    __syncthreads();
    const DeltaAt w(a, bh, i);
    const long long c = (long long)bh * a.nc + i;
    const float* decay = a.decay + c * kDecayRows;
    const float* mw = a.w + c * a.dkb * 1024 + 16 * wave * 16;
    float* mu = a.u + (c * a.dvb + slice) * 1024;
    f32x4 acc = {0, 0, 0, 0};
    for (int kb = 0; kb < a.dkb; ++kb)
      acc = mfma_block(steps_near(mw + kb * 1024, 16), rows_near(sl + 16 * kb * kLdS, kLdS), acc);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * wave + row4 + r;
      const float u = mu[row * 16 + col] - acc[r];
      mu[row * 16 + col] = u;
      ul[row * kLdS + col] = u * decay[kDecayWrite + row];
    }
    __syncthreads();
    const float whole = decay[kDecaySince + 63];
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t) {
      if (wave + 4 * t >= a.dkb) continue;
      s[t] *= whole;
      const int kc = 16 * (wave + 4 * t) + col;
      for (int kb = 0; kb < 4; ++kb) {
        f32x4 key = {0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int n = 16 * kb + row4 + r;
          if (n < w.valid && kc < a.dk) key[r] = load1<T>(a.k, w.b * a.vk.b + w.hk * a.vk.h + (w.n0 + n) * a.vk.n + kc);
        }
        s[t] = mfma_block(key, rows_near(ul + 16 * kb * kLdS, kLdS), s[t]);
      }
    }
  }
  if (a.state_out) {
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (wave + 4 * t) + row4 + r;
        if (row < a.dk && ch < a.dv) a.state_out[((long long)bh * a.dk + row) * a.dv + ch] = s[t][r];
      }
  }
}

// P_ij = q_i.k_j D_ij for j <= i, into `mp`; FORWARD: 0 where beta_j is 0 (the u_j that is kept is not)
template <bool FORWARD>
LF_DEV void chunk_scores(const DeltaArgs& a, const float* q, const float* k, int ld, const double* gamma,
                         const float* beta, float* mp) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, row4 = (lane >> 4) * 4;
  for (int nt = 0; nt < 4; ++nt) {
    f32x4 acc = {0, 0, 0, 0};
    if (nt <= wave)
      for (int kb = 0; kb < a.dkb; ++kb)
        acc = mfma_block(steps_near(q + 16 * wave * ld + 16 * kb, ld), steps_near(k + 16 * nt * ld + 16 * kb, ld), acc);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * wave + row4 + r, j = 16 * nt + col;
      const bool on = j <= i && !(FORWARD && beta[j] == kDeltaTinyBeta);
      mp[i * kLdT + j] = on ? acc[r] * decay_between(gamma, i, j) : 0.0f;
    }
  }
}

// ---- the outputs --------------------------------------------------------------------------------------------------------------
inline int delta_out_lds(int dkb) { return 2 * 64 * (16 * dkb + 4) * 4 + 64 * kLdT * 4 + 64 * 8 + kDecayRows * 4; }

template <typename T> __global__ __launch_bounds__(256) void delta_out(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  const int ld = 16 * a.dkb + 4;
  float* q = reinterpret_cast<float*>(smem);
  float* k = q + 64 * ld;
  float* mp = k + 64 * ld;
  double* gamma = reinterpret_cast<double*>(mp + 64 * kLdT);
  float* decay = reinterpret_cast<float*>(gamma + 64);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4;
  const long long c = (long long)blockIdx.y * a.nc + blockIdx.x;
  if (wave == 0) gamma[lane] = chunk_gamma(a, w);
  decay[tid] = a.decay[c * kDecayRows + tid];
  stage_rows<T>(q, ld, a.q, a.vq, w.b, w.hk, w.n0, w.valid, a.dk, a.dkb);
  stage_rows<T>(k, ld, a.k, a.vk, w.b, w.hk, w.n0, w.valid, a.dk, a.dkb);
  __syncthreads();
  chunk_scores<true>(a, q, k, ld, gamma, decay + kDecayBeta, mp);
  __syncthreads();
  for (int sl = 0; sl < a.dvb; ++sl) {
    const float* s0 = a.s + (((long long)blockIdx.y * (a.nc + 1) + blockIdx.x) * a.dvb + sl) * a.dkb * 256;
    const float* u = a.u + (c * a.dvb + sl) * 1024;
    f32x4 acc = {0, 0, 0, 0};
    for (int kb = 0; kb < a.dkb; ++kb)
      acc = mfma_block(steps_near(q + 16 * wave * ld + 16 * kb, ld), rows_near(s0 + 256 * kb, 16), acc);
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] *= decay[kDecaySince + 16 * wave + row4 + r];
    for (int kb = 0; kb <= wave; ++kb)
      acc = mfma_block(steps_near(mp + 16 * wave * kLdT + 16 * kb, kLdT), rows_near(u + 256 * kb, 16), acc);
    const int ch = 16 * sl + col;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = 16 * wave + row4 + r;
      if (n < w.valid && ch < a.dv) store1<T>(a.out, w.b * a.vo.b + w.h * a.vo.h + (w.n0 + n) * a.vo.n + ch, acc[r] * a.scale);
    }
  }
}

}  // namespace lf
