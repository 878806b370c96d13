// The boundary between two blocks of a transformer (block output f, residual stream x, modulation by row of the batch):
//
//     fhat = f,  or  norm(f) * w_post                                  (norm after the block)
//     y    = residual_scale * x + gate * fhat                          (the residual stream, rounded once)
//     h    = norm(y) * w_pre * (1 + scale) + shift                     (norm before the next block, of the unrounded y)
//
// norm(t) = (t - mean) / sqrt(mean((t - mean)^2) + eps) over a token's C channels, or t / sqrt(mean(t^2) + eps).
// Every token is read once and written once; sums and statistics are fp32, the variance from the deviations.  Bound: HBM.
// bf16, forward: 81120 tokens of 2048 channels 240 us for 1.33 GB (5.5 TB/s); 12 x 4096 of 320: 21 us for 126 MB (6.0 TB/s), backward
// 36 us for 189 MB (5.3 TB/s) and 4.8 us for the vectors' sums; fp16, 2 x 256 of 1280: 4.3 us.
#pragma once
#include "lf_vec8.hpp"

namespace lf {

struct NormView { long long batch, token; };   // element strides; channels contiguous

struct GateNormArgs {
  const void *x, *f;
  void *y, *h;
  NormView vx, vf, vy, vh;
  const float *gate, *scale, *shift, *w_pre, *w_post;
  long long mod_stride;   // elements between the modulation rows of two batch rows (0: shared)
  const int* lengths;
  long long N;
  int C, rows;            // channels; tokens per workgroup
  float residual_scale, eps;
};

struct GateNormBwdArgs {
  const void *x, *f, *dy, *dh;
  void *dx, *df;
  NormView vx, vf, vdy, vdh, vdx, vdf;
  const float *gate, *scale, *w_pre, *w_post;
  long long mod_stride;
  const int* lengths;
  float* partials;        // [B][workgroups][3][C]
  long long N;
  int C, rows;
  float residual_scale, eps;
};

// Sums `v` over the threads of a token: LANES lanes of a wave, or the whole workgroup of four waves (LANES = 256) through
// LDS.  `slot` alternates, so that a second sum needs no barrier behind the first one's reads.
template <int LANES> LF_DEV float token_sum(float v, float* lds, int slot) {
  v = lanes_sum<64>(v);
  if constexpr (LANES == 256) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[slot * 4 + wave] = v;
    __syncthreads();
    v = (lds[slot * 4] + lds[slot * 4 + 1]) + (lds[slot * 4 + 2] + lds[slot * 4 + 3]);
  }
  return v;
}

template <int LANES> LF_DEV void token_sum2(float& a, float& b, float* lds, int slot) {
  a = lanes_sum<64>(a);
  b = lanes_sum<64>(b);
  if constexpr (LANES == 256) {
    const int wave = threadIdx.x >> 6;
    float* p = lds + 8 + slot * 8;   // (behind the single sums' slots, which other waves may still be reading)
    if ((threadIdx.x & 63) == 0) { p[wave] = a; p[4 + wave] = b; }
    __syncthreads();
    a = (p[0] + p[1]) + (p[2] + p[3]);
    b = (p[4] + p[5]) + (p[6] + p[7]);
  }
}

// t -> (t - mean) * rate in place (RMS: t * rate); returns rate.  `on[i]`: whether the i-th vector of this thread exists.
template <int LANES, int VPT, bool RMS>
LF_DEV float normalise(float (&t)[VPT][8], const bool (&on)[VPT], float inv_c, float eps, float* lds, int& slot) {
  if constexpr (!RMS) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += on[i] ? t[i][j] : 0.0f;
    const float mean = token_sum<LANES>(s, lds, slot) * inv_c;
    slot ^= 1;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) t[i][j] -= mean;
  }
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s += on[i] ? t[i][j] * t[i][j] : 0.0f;
  const float var = token_sum<LANES>(s, lds, slot) * inv_c;
  slot ^= 1;
  const float rate = 1.0f / sqrtf(var + eps);
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) t[i][j] *= rate;
  return rate;
}

// One workgroup of 256 threads takes `rows` consecutive tokens of one batch row, LANES threads a token, with the modulation
// of its channels in registers (fp32: 12 bytes a channel beside 8 bytes of a 16-bit token, so they are read once per
// workgroup and not once per token).  LANES = 64: a wave per token, no barrier; 256: a workgroup per token, for wide tokens
// and for few of them.
template <typename T, int LANES, int VPT, bool RMS, bool POST>
__global__ __launch_bounds__(256) void gate_norm_fwd(GateNormArgs a) {
  __shared__ float lds[8];
  const int b = blockIdx.y, lane = threadIdx.x % LANES;
  const long long n_end = tokens_of(a.lengths, b, a.N);
  long long n = (long long)blockIdx.x * a.rows + threadIdx.x / LANES;
  const long long last = (long long)(blockIdx.x + 1) * a.rows;
  const long long stop = last < n_end ? last : n_end;
  if (n >= stop) return;   // (LANES = 256: the whole workgroup)
  bool on[VPT];
  int c[VPT];
  float gate[VPT][8], mul[VPT][8], add[VPT][8], post[POST ? VPT : 1][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    c[i] = (i * LANES + lane) * 8;
    on[i] = c[i] < a.C;
    const long long m = b * a.mod_stride + c[i];
#pragma unroll
    for (int j = 0; j < 8; ++j) { gate[i][j] = 1.0f; mul[i][j] = 1.0f; add[i][j] = 0.0f; }
    if constexpr (POST) {
#pragma unroll
      for (int j = 0; j < 8; ++j) post[i][j] = 1.0f;
      if (on[i] && a.w_post) load8_f32(a.w_post + c[i], post[i]);
    }
    if (!on[i]) continue;
    if (a.f && a.gate) load8_f32(a.gate + m, gate[i]);
    if (a.scale) {
      load8_f32(a.scale + m, mul[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) mul[i][j] += 1.0f;
    }
    if (a.w_pre) {
      float w[8];
      load8_f32(a.w_pre + c[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) mul[i][j] *= w[j];
    }
    if (a.shift) load8_f32(a.shift + m, add[i]);
  }
  const float inv_c = 1.0f / (float)a.C;
  int slot = 0;
  Raw8<T> next_x[VPT], next_f[VPT];   // the token after this one is on its way meanwhile
  auto request = [&](long long m) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      next_x[i] = none8<T>();
      next_f[i] = none8<T>();
      if (!on[i] || m >= stop) continue;
      next_x[i] = load8_raw<T>(at<T>(a.x, b * a.vx.batch + m * a.vx.token + c[i]));
      if (a.f) next_f[i] = load8_raw<T>(at<T>(a.f, b * a.vf.batch + m * a.vf.token + c[i]));
    }
  };
  request(n);
  for (; n < stop; n += 256 / LANES) {
    float y[VPT][8], f[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      widen8<T>(next_x[i], y[i]);
      widen8<T>(next_f[i], f[i]);
    }
    request(n + 256 / LANES);
    if constexpr (POST) {
      normalise<LANES, VPT, RMS>(f, on, inv_c, a.eps, lds, slot);
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) f[i][j] *= post[i][j];
    }
    if (a.f) {
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[i][j] = __builtin_fmaf(gate[i][j], f[i][j], a.residual_scale * y[i][j]);
    } else if (a.residual_scale != 1.0f) {
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[i][j] *= a.residual_scale;
    }
    if (a.y) {
#pragma unroll
      for (int i = 0; i < VPT; ++i)
        if (on[i]) store8_stream<T>(at<T>(a.y, b * a.vy.batch + n * a.vy.token + c[i]), y[i]);
    }
    if (a.h) {
      normalise<LANES, VPT, RMS>(y, on, inv_c, a.eps, lds, slot);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if (!on[i]) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) y[i][j] = __builtin_fmaf(y[i][j], mul[i][j], add[i][j]);
        store8_stream<T>(at<T>(a.h, b * a.vh.batch + n * a.vh.token + c[i]), y[i]);
      }
    }
  }
}

// The gradients, with unit = norm(y), m = w_pre (1 + scale), and dy, dh those that arrive at y and h:
//
//     dunit = dh m;   dY = dy + rate (dunit - mean(dunit) - unit mean(dunit unit))        (RMS: without mean(dunit))
//     dx = residual_scale dY;   dfhat = gate dY;   df = dfhat, or the same step back through norm(f) from dfhat w_post
//
// and three sums over the tokens of a batch row, from which the gradients of all vectors follow:
//
//     A = sum dh,   Bs = sum dh unit,   G = sum dY norm(f)      (POST: of the normalised f, else of f itself)
//
// y is formed again from x and f (as many bytes as reading it, and unrounded).  Each workgroup leaves its sums in
// `partials`, its waves' in a fixed order; gate_norm_sums adds them up in a fixed order too.
template <typename T, int LANES, int VPT, bool RMS, bool POST>
__global__ __launch_bounds__(256) void gate_norm_bwd(GateNormBwdArgs a) {
  extern __shared__ __align__(16) float sums[];   // LANES < 256: [256 / LANES][3][C]
  __shared__ float lds[24];
  const int b = blockIdx.y, lane = threadIdx.x % LANES;
  const long long n_end = tokens_of(a.lengths, b, a.N);
  const long long first = (long long)blockIdx.x * a.rows + threadIdx.x / LANES;
  const long long last = (long long)(blockIdx.x + 1) * a.rows;
  const long long stop = last < n_end ? last : n_end;
  bool on[VPT];
  int c[VPT];
  float gate[VPT][8], mul[VPT][8], post[POST ? VPT : 1][8];
  float sa[VPT][8], sb[VPT][8], sg[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    c[i] = (i * LANES + lane) * 8;
    on[i] = c[i] < a.C;
    const long long m = b * a.mod_stride + c[i];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      gate[i][j] = 1.0f; mul[i][j] = 1.0f;
      sa[i][j] = sb[i][j] = sg[i][j] = 0.0f;
    }
    if constexpr (POST) {
#pragma unroll
      for (int j = 0; j < 8; ++j) post[i][j] = 1.0f;
      if (on[i] && a.w_post) load8_f32(a.w_post + c[i], post[i]);
    }
    if (!on[i]) continue;
    if (a.f && a.gate) load8_f32(a.gate + m, gate[i]);
    if (a.scale) {
      load8_f32(a.scale + m, mul[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) mul[i][j] += 1.0f;
    }
    if (a.w_pre) {
      float w[8];
      load8_f32(a.w_pre + c[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) mul[i][j] *= w[j];
    }
  }
  const float inv_c = 1.0f / (float)a.C;
  int slot = 0, slot2 = 0;
  Raw8<T> next_x[VPT], next_f[VPT], next_h[VPT], next_y[VPT];
  auto request = [&](long long m) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      next_x[i] = next_f[i] = next_h[i] = next_y[i] = none8<T>();
      if (!on[i] || m >= stop) continue;
      next_x[i] = load8_raw<T>(at<T>(a.x, b * a.vx.batch + m * a.vx.token + c[i]));
      if (a.f) next_f[i] = load8_raw<T>(at<T>(a.f, b * a.vf.batch + m * a.vf.token + c[i]));
      if (a.dh) next_h[i] = load8_raw<T>(at<T>(a.dh, b * a.vdh.batch + m * a.vdh.token + c[i]));
      if (a.dy) next_y[i] = load8_raw<T>(at<T>(a.dy, b * a.vdy.batch + m * a.vdy.token + c[i]));
    }
  };
  request(first);
  for (long long n = first; n < stop; n += 256 / LANES) {
    float y[VPT][8], f[VPT][8], d[VPT][8], up[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      widen8<T>(next_x[i], y[i]);
      widen8<T>(next_f[i], f[i]);
      widen8<T>(next_h[i], d[i]);
      widen8<T>(next_y[i], up[i]);
    }
    request(n + 256 / LANES);
    float rate_f = 1.0f;
    if constexpr (POST) rate_f = normalise<LANES, VPT, RMS>(f, on, inv_c, a.eps, lds, slot);
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float fh = POST ? f[i][j] * post[POST ? i : 0][j] : f[i][j];
        y[i][j] = __builtin_fmaf(gate[i][j], fh, a.residual_scale * y[i][j]);
      }
    if (a.dh) {
      const float rate = normalise<LANES, VPT, RMS>(y, on, inv_c, a.eps, lds, slot);
      float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if (!on[i]) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sa[i][j] += d[i][j];
          sb[i][j] = __builtin_fmaf(d[i][j], y[i][j], sb[i][j]);
          d[i][j] *= mul[i][j];
          s1 += d[i][j];
          s2 = __builtin_fmaf(d[i][j], y[i][j], s2);
        }
      }
      token_sum2<LANES>(s1, s2, lds, slot2);
      slot2 ^= 1;
      s1 = RMS ? 0.0f : s1 * inv_c;
      s2 *= inv_c;
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) d[i][j] = (d[i][j] - s1 - y[i][j] * s2) * rate;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) d[i][j] += up[i][j];
    // d is dY now; y is free
    if (a.dx) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if (!on[i]) continue;
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = a.residual_scale * d[i][j];
        store8_stream<T>(at<T>(a.dx, b * a.vdx.batch + n * a.vdx.token + c[i]), g);
      }
    }
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (!on[i]) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sg[i][j] = __builtin_fmaf(d[i][j], f[i][j], sg[i][j]);
        d[i][j] *= gate[i][j];
        if constexpr (POST) {
          d[i][j] *= post[POST ? i : 0][j];
          s1 += d[i][j];
          s2 = __builtin_fmaf(d[i][j], f[i][j], s2);
        }
      }
    }
    if (a.df) {
      if constexpr (POST) {
        token_sum2<LANES>(s1, s2, lds, slot2);
        slot2 ^= 1;
        s1 = RMS ? 0.0f : s1 * inv_c;
        s2 *= inv_c;
      }
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if (!on[i]) continue;
        if constexpr (POST) {
#pragma unroll
          for (int j = 0; j < 8; ++j) d[i][j] = (d[i][j] - s1 - f[i][j] * s2) * rate_f;
        }
        store8_stream<T>(at<T>(a.df, b * a.vdf.batch + n * a.vdf.token + c[i]), d[i]);
      }
    }
  }
  if (!a.partials) return;
  float* mine = a.partials + ((long long)b * gridDim.x + blockIdx.x) * 3 * a.C;
  if constexpr (LANES == 256) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (!on[i]) continue;
      store8<F32>(reinterpret_cast<unsigned char*>(mine + c[i]), sa[i]);
      store8<F32>(reinterpret_cast<unsigned char*>(mine + a.C + c[i]), sb[i]);
      store8<F32>(reinterpret_cast<unsigned char*>(mine + 2 * a.C + c[i]), sg[i]);
    }
  } else {
    constexpr int kPer = 256 / LANES;
    float* own = sums + (size_t)(threadIdx.x / LANES) * 3 * a.C;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (!on[i]) continue;
      store8<F32>(reinterpret_cast<unsigned char*>(own + c[i]), sa[i]);
      store8<F32>(reinterpret_cast<unsigned char*>(own + a.C + c[i]), sb[i]);
      store8<F32>(reinterpret_cast<unsigned char*>(own + 2 * a.C + c[i]), sg[i]);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 3 * a.C; e += 256) {
      float s = 0.0f;
      for (int k = 0; k < kPer; ++k) s += sums[(size_t)k * 3 * a.C + e];
      mine[e] = s;
    }
  }
}

struct GateNormVectors {
  const float* partials;   // [B][wgs][3][C]
  float* sums;             // [B][3][C]: A, Bs, G
  const float *gate, *scale, *w_pre, *w_post;
  float *dgate, *dscale, *dshift, *dw_pre, *dw_post;
  long long mod_stride, dmod_stride;
  int B, C, wgs;
  bool shared;             // one modulation row for the whole batch: its gradient is the sum over the batch
};

// The vectors' gradients: dshift = A, dscale = Bs w_pre, dgate = G w_post per modulation row;
// dw_pre = sum_b Bs (1 + scale), dw_post = sum_b G gate.
// First the workgroups' partial sums: 64 elements per workgroup, each of its sixteen waves a sixteenth of the partials in their
// order, the sixteenths in theirs (with four waves a sum over 2048 partials of one batch row took 30 us).  Where every
// modulation row has its own gradient that ends here; for the sums over the batch the totals are left for gate_norm_vectors.
__global__ __launch_bounds__(1024) void gate_norm_sums(GateNormVectors a) {
  constexpr int kWaves = 16;
  __shared__ float part[kWaves][64];
  const int lane = threadIdx.x & 63, share = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, which = blockIdx.y, b = blockIdx.z;
  const int per = (a.wgs + kWaves - 1) / kWaves, from = share * per, to = from + per < a.wgs ? from + per : a.wgs;
  const long long step = 3LL * a.C;
  float s = 0.0f;
  if (c < a.C) {
    const float* p = a.partials + ((long long)b * a.wgs + from) * step + (long long)which * a.C + c;
    int w = from;
    for (; w + 8 <= to; w += 8, p += 8 * step) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = p[i * step];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; w < to; ++w, p += step) s += *p;
  }
  part[share][lane] = s;
  __syncthreads();
  if (share != 0 || c >= a.C) return;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) s += part[i][lane];
  if (a.sums) a.sums[((long long)b * 3 + which) * a.C + c] = s;
  if (a.shared) return;
  const long long o = b * a.dmod_stride + c;
  if (which == 0 && a.dshift) a.dshift[o] = s;
  if (which == 1 && a.dscale) a.dscale[o] = s * (a.w_pre ? a.w_pre[c] : 1.0f);
  if (which == 2 && a.dgate) a.dgate[o] = s * (a.w_post ? a.w_post[c] : 1.0f);
}

// The sums over the batch, one thread per channel, batch rows in their order.
__global__ __launch_bounds__(64) void gate_norm_vectors(GateNormVectors a) {
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (c >= a.C) return;
  float ta = 0.0f, tb = 0.0f, tg = 0.0f, pre = 0.0f, post = 0.0f;
#pragma unroll 4
  for (int b = 0; b < a.B; ++b) {
    const float* s = a.sums + (long long)b * 3 * a.C + c;
    const float va = s[0], vb = s[a.C], vg = s[2 * a.C];
    const long long m = b * a.mod_stride + c;
    pre = __builtin_fmaf(vb, a.scale ? 1.0f + a.scale[m] : 1.0f, pre);
    post = __builtin_fmaf(vg, a.gate ? a.gate[m] : 1.0f, post);
    ta += va;
    tb += vb;
    tg += vg;
  }
  if (a.shared) {
    if (a.dshift) a.dshift[c] = ta;
    if (a.dscale) a.dscale[c] = tb * (a.w_pre ? a.w_pre[c] : 1.0f);
    if (a.dgate) a.dgate[c] = tg * (a.w_post ? a.w_post[c] : 1.0f);
  }
  if (a.dw_pre) a.dw_pre[c] = pre;
  if (a.dw_post) a.dw_post[c] = post;
}

}  // namespace lf
