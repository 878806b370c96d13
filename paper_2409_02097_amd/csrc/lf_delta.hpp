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
// Products run on the 16-bit matrix instruction with operands as sums of bf16 terms (lf_terms.hpp): three where a state or
// an fp32 result depends on them, two where a 16-bit output does.  What passes between the kernels is stored as its reader
// takes it, a contiguous kilobyte for each operand or accumulator of a wave:
//     w    T (beta e^gamma K) as operand: [4 row blocks][d_k / 32][3 terms][64 lanes][8 steps]
//     kt   K^T as operand: [d_k / 16][2][terms][64][8], once per query and key head
//     u    U0, then U, and s the state before each chunk and behind the last, as fp32 accumulators: [d_v / 16][row blocks][64][4]
#pragma once
#include "lf_terms.hpp"

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
  uint16_t *w, *kt, *wt, *tt;     // operands; wt = W^T, tt = (T beta)^T: for the backward pass, else null
  float *u, *s, *decay;           // accumulators; per chunk [4][64]
  long long N;
  int H, Hk, nc;                  // chunks of N tokens
  int dk, dv, dkb, dvb, dks;      // channels, blocks of 16 of them, and of 32
  float scale;
  // backward
  const void* dout;
  const float* dstate_out;
  void *dq, *dk_out, *dv_out;
  float *dg, *dbeta, *dstate_in;
  DeltaView vdo, vdq, vdk, vdv, vdg;
  uint16_t* kn;                   // K as operand
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

// Four neighbouring channels.
template <typename T> LF_DEV f32x4 load4(const unsigned char* p) {
  if constexpr (Stored<T>::kBytes == 4) {
    return *reinterpret_cast<const f32x4*>(p);
  } else {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    float a, b, c, d;
    unpack2<T>(w[0], a, b);
    unpack2<T>(w[1], c, d);
    return f32x4{a, b, c, d};
  }
}
template <typename T> LF_DEV void store4(unsigned char* p, const f32x4& v) {
  if constexpr (Stored<T>::kBytes == 4) *reinterpret_cast<f32x4*>(p) = v;
  else *reinterpret_cast<u32x2*>(p) = u32x2{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
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

constexpr int kLdT = 68;   // leading dimension of a 64 x 64 fp32 matrix in LDS: both operand forms are free of bank conflicts
constexpr int kLdP = 72;   // of a plane of one
constexpr int kLdU = 20;   // of planes of 16 value channels per token

LF_DEV int plane_ld(int steps) { return 32 * steps + 8; }
inline int plane_bytes(int rows, int steps) { return rows * (32 * steps + 8) * 2; }

constexpr int kFrag = 512;   // elements of one term of an operand

// An accumulator block as terms of an operand in global memory: its lane holds steps 4 g .. + 3 (g = lane / 16) of row (or
// column) lane % 16 of the 16 steps that are the `upper` half or not of the operand's 32.
template <int N> LF_DEV void store_operand(uint16_t* frag, bool upper, const f32x4& v) {
  const int l = threadIdx.x & 63, g = l >> 4;
  split4_lds<N>(frag + ((l & 15) + 16 * ((upper ? 2 : 0) + (g >> 1))) * 8 + (g & 1) * 4, kFrag, v);
}
template <int N> LF_DEV void store_frag(uint16_t* frag, const Terms<N>& t) {
#pragma unroll
  for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(frag + i * kFrag + (threadIdx.x & 63) * 8) = t.t[i];
}
template <int N> LF_DEV void load_frag(const uint16_t* frag, Terms<N>& t) {
#pragma unroll
  for (int i = 0; i < N; ++i) t.t[i] = *reinterpret_cast<const u32x4*>(frag + i * kFrag + (threadIdx.x & 63) * 8);
}

// ---- the operands and U0 of every chunk -----------------------------------------------------------------------------------
template <typename T> inline int delta_prepare_lds(int dks, int dvs) {
  const int wide = dks > dvs ? dks : dvs;
  return TermsOf<T>::kStored * plane_bytes(64, wide) + 64 * kLdT * 4 + 3 * 64 * kLdP * 2 + 64 * 8 + kDecayRows * 4 + 64 * 4;
}

template <typename T> __global__ __launch_bounds__(256) void delta_prepare(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NI = TermsOf<T>::kStored;
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  const int dvs = (a.dvb + 1) / 2, ld = plane_ld(a.dks), ldv = plane_ld(dvs), plane = 64 * ld;
  const int most = ld > ldv ? ld : ldv;
  float* mt = reinterpret_cast<float*>(smem);
  uint16_t* tp = reinterpret_cast<uint16_t*>(mt + 64 * kLdT);   // A, then T times a factor per column, as terms
  float* ma = reinterpret_cast<float*>(tp);
  uint16_t* x = tp + 3 * 64 * kLdP;                             // the keys, then the values
  double* gamma = reinterpret_cast<double*>(x + NI * 64 * most);
  float* decay = reinterpret_cast<float*>(gamma + 64);
  float* both = decay + kDecayRows;                             // beta e^gamma
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, g8 = (lane >> 4) * 8, row4 = (lane >> 4) * 4;
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
  stage_terms<T>(x, ld, a.k, w.b * a.vk.b + w.hk * a.vk.h + w.n0 * a.vk.n, a.vk.n, w.valid, a.dk, a.dks);
  for (int i = tid; i < 64 * kLdT; i += 256) mt[i] = 0.0f;
  __syncthreads();
  a.decay[c * kDecayRows + tid] = decay[tid];
  if (w.h % (a.H / a.Hk) == 0) {
    uint16_t* kt = a.kt + ((long long)(w.b * a.Hk + w.hk) * a.nc + blockIdx.x) * a.dkb * 2 * NI * kFrag;
    for (int i = wave; i < a.dkb * 2; i += 4) {
      Terms<NI> f;
      terms_across<NI>(x + 32 * (i & 1) * ld + 16 * (i >> 1), plane, ld, f);
      store_frag<NI>(kt + i * NI * kFrag, f);
    }
  }
  // A, rows 16 wave .. + 15
  for (int nt = 0; nt <= wave; ++nt) {
    f32x4 acc = {0, 0, 0, 0};
    for (int ks = 0; ks < a.dks; ++ks) {
      Terms<NI> fi, fj;
      terms_near<NI>(x + (16 * wave + col) * ld + 32 * ks + g8, plane, fi);
      terms_near<NI>(x + (16 * nt + col) * ld + 32 * ks + g8, plane, fj);
      acc = mul_terms<3>(fi, fj, acc);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * wave + row4 + r, j = 16 * nt + col;
      ma[i * kLdT + j] = i > j ? decay[kDecayBeta + i] * acc[r] * decay_between(gamma, i, j) : 0.0f;
    }
  }
  __syncthreads();
  // T: the blocks on the diagonal, a column per lane, by substitution
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
  // the blocks below it: T_ij = -T_ii sum_l A_il T_lj, by their distance from the diagonal; the inner sum waits in T_ij's place
  for (int far = 1; far < 4; ++far) {
    const int i = wave + far, j = wave;
    if (i < 4) {
      float* tij = mt + 16 * i * kLdT + 16 * j;
      f32x4 acc = {0, 0, 0, 0};
      for (int l = j; l < i; ++l)
        acc = mfma_block(steps_near(ma + 16 * i * kLdT + 16 * l, kLdT), rows_near(mt + 16 * l * kLdT + 16 * j, kLdT), acc);
#pragma unroll
      for (int r = 0; r < 4; ++r) tij[(row4 + r) * kLdT + col] = acc[r];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (only this wave uses the block until the barrier)
      acc = mfma_block(steps_near(mt + 16 * i * kLdT + 16 * i, kLdT), rows_near(tij, kLdT), f32x4{0, 0, 0, 0});
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int r = 0; r < 4; ++r) tij[(row4 + r) * kLdT + col] = -acc[r];
    }
    __syncthreads();
  }
  auto scaled = [&](const float* by) {   // T with a factor per column, as terms
    for (int i = tid; i < 64 * 8; i += 256) {
      const int r = i >> 3, v = (i & 7) * 8;
      float y[8];
      load8_f32(mt + r * kLdT + v, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= by[v + e];
      Terms<3> t;
      split8(y, t);
#pragma unroll
      for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4*>(tp + p * 64 * kLdP + r * kLdP + v) = t.t[p];
    }
  };
  scaled(both);
  __syncthreads();
  // T's rows 16 wave .. + 15 have nothing behind column 16 wave + 15
  const int steps = wave < 2 ? 1 : 2;
  Terms<3> ft[2];
  auto rows_of_t = [&]() {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      if (ks < steps) terms_near<3>(tp + (16 * wave + col) * kLdP + 32 * ks + g8, 64 * kLdP, ft[ks]);
  };
  rows_of_t();
  uint16_t* mw = a.w + (c * 4 + wave) * a.dks * 3 * kFrag;
  for (int cb = 0; cb < 2 * a.dks; ++cb) {
    f32x4 acc = {0, 0, 0, 0}, act = {0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if (ks >= steps) continue;
      Terms<NI> key;
      terms_across<NI>(x + 32 * ks * ld + 16 * cb, plane, ld, key);
      acc = mul_terms<3>(key, ft[ks], acc);
      if (a.wt) act = mul_terms<3>(ft[ks], key, act);
    }
    store_operand<3>(mw + (cb >> 1) * 3 * kFrag, cb & 1, acc);
    if (a.wt && cb < a.dkb) store_operand<3>(a.wt + ((c * a.dkb + cb) * 2 + (wave >> 1)) * 3 * kFrag, wave & 1, act);
  }
  __syncthreads();
  scaled(decay + kDecayBeta);
  stage_terms<T>(x, ldv, a.v, w.b * a.vv.b + w.h * a.vv.h + w.n0 * a.vv.n, a.vv.n, w.valid, a.dv, dvs);
  __syncthreads();
  rows_of_t();
  for (int vb = 0; vb < a.dvb; ++vb) {
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if (ks >= steps) continue;
      Terms<NI> val;
      terms_across<NI>(x + 32 * ks * ldv + 16 * vb, 64 * ldv, ldv, val);
      acc = mul_terms<3>(val, ft[ks], acc);
    }
    *reinterpret_cast<f32x4*>(a.u + (((c * a.dvb + vb) * 4 + wave) * 64 + lane) * 4) = acc;
  }
  if (a.tt) {
    for (int ks = 0; ks < 2; ++ks) {
      Terms<3> f;
      terms_across<3>(tp + 32 * ks * kLdP + 16 * wave, 64 * kLdP, kLdP, f);
      store_frag<3>(a.tt + ((c * 4 + wave) * 2 + ks) * 3 * kFrag, f);
    }
  }
}

// ---- the scan ---------------------------------------------------------------------------------------------------------------
// A workgroup takes 16 value channels of one head through all chunks; its four waves hold the state's row blocks
// wave, wave + 4, ... as accumulators and compute 16 tokens of U each.  Bound: the chain from one chunk's state to the next
// (two products, two passes through LDS); everything it reads from memory is requested a chunk ahead.
template <int NI, int KS> struct ScanIn {
  static constexpr int kBlocks = (2 * KS + 3) / 4;
  Terms<3> w[KS];
  Terms<NI> kt[kBlocks][2];
  f32x4 u0;
  float write, whole;
};

template <int NI, int KS> __global__ __launch_bounds__(256) void delta_scan(DeltaArgs a) {
  constexpr int kBlocks = ScanIn<NI, KS>::kBlocks, kLd = 32 * KS + 8, kPlane = 16 * kLd;
  __shared__ __align__(16) uint16_t sp[3 * kPlane];
  __shared__ __align__(16) uint16_t up[3 * 64 * kLdU];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  const int slice = blockIdx.x, bh = blockIdx.y, ch = slice * 16 + col;
  const DeltaAt first(a, bh, 0);
  const int chunks = (int)((tokens_of(a.lengths, first.b, a.N) + 63) / 64);
  f32x4 s[kBlocks];
#pragma unroll
  for (int t = 0; t < kBlocks; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * (wave + 4 * t) + row4 + r;
      s[t][r] = a.state_in && row < a.dk && ch < a.dv ? a.state_in[((long long)bh * a.dk + row) * a.dv + ch] : 0.0f;
    }
  for (int i = tid; i < 3 * kPlane / 8; i += 256) reinterpret_cast<u32x4*>(sp)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
  const long long c0 = (long long)bh * a.nc;
  const long long k0 = (long long)(first.b * a.Hk + first.hk) * a.nc;
  auto request = [&](ScanIn<NI, KS>& n, int i) {
    const uint16_t* mw = a.w + ((c0 + i) * 4 + wave) * a.dks * 3 * kFrag;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) load_frag<3>(mw + ks * 3 * kFrag, n.w[ks]);
    const uint16_t* kt = a.kt + (k0 + i) * a.dkb * 2 * NI * kFrag;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        if (wave + 4 * t < a.dkb) load_frag<NI>(kt + ((wave + 4 * t) * 2 + ks) * NI * kFrag, n.kt[t][ks]);
    n.u0 = *reinterpret_cast<const f32x4*>(a.u + ((((c0 + i) * a.dvb + slice) * 4 + wave) * 64 + lane) * 4);
    const float* decay = a.decay + (c0 + i) * kDecayRows;
    n.write = decay[kDecayWrite + 16 * wave + col];
    n.whole = decay[kDecaySince + 63];
  };
  auto keep = [&](int i) {
    float* to = a.s + (((long long)bh * (a.nc + 1) + i) * a.dvb + slice) * a.dkb * 256;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
      if (wave + 4 * t < a.dkb) *reinterpret_cast<f32x4*>(to + (wave + 4 * t) * 256 + lane * 4) = s[t];
  };
  auto chunk = [&](ScanIn<NI, KS>& in, ScanIn<NI, KS>& next, int i) {
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
      if (wave + 4 * t < a.dkb) split4_lds<3>(sp + col * kLd + 16 * (wave + 4 * t) + row4, kPlane, s[t]);
    if (i + 1 < chunks) request(next, i + 1);
    keep(i);
    lds_barrier();
    f32x4 acc = {0, 0, 0, 0}, acc2 = {0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      Terms<3> fs;
      terms_near<3>(sp + col * kLd + 32 * ks + g8, kPlane, fs);
      if (ks & 1) acc2 = mul_terms<3>(fs, in.w[ks], acc2);
      else acc = mul_terms<3>(fs, in.w[ks], acc);
    }
    const f32x4 u = in.u0 - (acc + acc2);
    *reinterpret_cast<f32x4*>(a.u + ((((c0 + i) * a.dvb + slice) * 4 + wave) * 64 + lane) * 4) = u;
    split4_lds<3>(up + (16 * wave + col) * kLdU + row4, 64 * kLdU, u * in.write);
    lds_barrier();
    Terms<3> fu[2];
    terms_across<3>(up, 64 * kLdU, kLdU, fu[0]);
    terms_across<3>(up + 32 * kLdU, 64 * kLdU, kLdU, fu[1]);
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      if (wave + 4 * t >= a.dkb) continue;
      s[t] *= in.whole;
      s[t] = mul_terms<3>(in.kt[t][0], fu[0], s[t]);
      s[t] = mul_terms<3>(in.kt[t][1], fu[1], s[t]);
    }
  };
  ScanIn<NI, KS> x, y;
  if (chunks > 0) request(x, 0);
  int i = 0;
  for (; i + 1 < chunks; i += 2) {
    chunk(x, y, i);
    chunk(y, x, i + 1);
  }
  if (i < chunks) chunk(x, y, i);
  keep(chunks);
  if (a.state_out) {
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (wave + 4 * t) + row4 + r;
        if (row < a.dk && ch < a.dv) a.state_out[((long long)bh * a.dk + row) * a.dv + ch] = s[t][r];
      }
  }
}

// ---- the outputs --------------------------------------------------------------------------------------------------------------
// Formed transposed, so that a lane has four neighbouring channels of a token: O^T = e^gamma S0^T Q^T + U^T P^T.
constexpr int kOutBlocks = 4;   // of 16 value channels at a time

template <typename T> inline int delta_out_lds(int dks) {
  constexpr int NI = TermsOf<T>::kStored, NO = TermsOf<T>::kOut;
  const int rows = 2 * NI * plane_bytes(64, dks);
  const int later = kOutBlocks * NO * (plane_bytes(16, dks) + 64 * kLdU * 2);
  return NO * 64 * kLdP * 2 + (rows > later ? rows : later) + 64 * 8 + kDecayRows * 4;
}

template <typename T, int KS> __global__ __launch_bounds__(256) void delta_out(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NI = TermsOf<T>::kStored, NO = TermsOf<T>::kOut, kLd = 32 * KS + 8, kSPlane = 16 * kLd, kUPlane = 64 * kLdU;
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  double* gamma = reinterpret_cast<double*>(smem);
  float* decay = reinterpret_cast<float*>(gamma + 64);
  uint16_t* pp = reinterpret_cast<uint16_t*>(decay + kDecayRows);
  uint16_t* q = pp + NO * 64 * kLdP;
  uint16_t* k = q + NI * 64 * kLd;
  uint16_t* sp = q;                                     // where q and k were
  uint16_t* up = sp + kOutBlocks * NO * kSPlane;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  const long long c = (long long)blockIdx.y * a.nc + blockIdx.x;
  if (wave == 0) gamma[lane] = chunk_gamma(a, w);
  decay[tid] = a.decay[c * kDecayRows + tid];
  stage_terms<T>(q, kLd, a.q, w.b * a.vq.b + w.hk * a.vq.h + w.n0 * a.vq.n, a.vq.n, w.valid, a.dk, KS);
  stage_terms<T>(k, kLd, a.k, w.b * a.vk.b + w.hk * a.vk.h + w.n0 * a.vk.n, a.vk.n, w.valid, a.dk, KS);
  __syncthreads();
  Terms<NI> fq[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) terms_near<NI>(q + (16 * wave + col) * kLd + 32 * ks + g8, 64 * kLd, fq[ks]);
  // P, four neighbouring columns j of row i at a time; 0 where beta_j is 0 (the u_j that is kept is not)
#pragma unroll
  for (int jt = 0; jt < 4; ++jt) {
    f32x4 acc = {0, 0, 0, 0};
    if (jt <= wave) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Terms<NI> fk;
        terms_near<NI>(k + (16 * jt + col) * kLd + 32 * ks + g8, 64 * kLd, fk);
        acc = mul_terms<NO>(fk, fq[ks], acc);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * wave + col, j = 16 * jt + row4 + r;
        const bool on = j <= i && decay[kDecayBeta + j] != kDeltaTinyBeta;
        acc[r] = on ? acc[r] * decay_between(gamma, i, j) : 0.0f;
      }
    }
    split4_lds<NO>(pp + (16 * wave + col) * kLdP + 16 * jt + row4, 64 * kLdP, acc);
  }
  __syncthreads();
  Terms<NO> fp[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) terms_near<NO>(pp + (16 * wave + col) * kLdP + 32 * ks + g8, 64 * kLdP, fp[ks]);
  const float since = decay[kDecaySince + 16 * wave + col];
  const int n = 16 * wave + col;
  // (the half block behind dkb of the last 32 channels: the queries there are 0, the state's planes are too)
  for (int i = tid; i < kOutBlocks * NO * kSPlane / 8; i += 256) reinterpret_cast<u32x4*>(sp)[i] = u32x4{0, 0, 0, 0};
  for (int vb0 = 0; vb0 < a.dvb; vb0 += kOutBlocks) {
    const int blocks = a.dvb - vb0 < kOutBlocks ? a.dvb - vb0 : kOutBlocks;
    __syncthreads();
    const float* s0 = a.s + (((long long)blockIdx.y * (a.nc + 1) + blockIdx.x) * a.dvb + vb0) * a.dkb * 256;
    for (int i = wave; i < blocks * a.dkb; i += 4) {
      const int vb = (unsigned)i / (unsigned)a.dkb, kb = i - vb * a.dkb;
      split4_lds<NO>(sp + vb * NO * kSPlane + col * kLd + 16 * kb + row4, kSPlane,
                     *reinterpret_cast<const f32x4*>(s0 + (long long)i * 256 + lane * 4));
    }
    const float* mu = a.u + (c * a.dvb + vb0) * 1024;
    for (int i = wave; i < blocks * 4; i += 4)
      split4_lds<NO>(up + (i >> 2) * NO * kUPlane + (16 * (i & 3) + col) * kLdU + row4, kUPlane,
                     *reinterpret_cast<const f32x4*>(mu + i * 256 + lane * 4));
    __syncthreads();
    for (int vb = 0; vb < blocks; ++vb) {
      f32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Terms<NO> fs;
        terms_near<NO>(sp + vb * NO * kSPlane + col * kLd + 32 * ks + g8, kSPlane, fs);
        acc = mul_terms<NO>(fs, fq[ks], acc);
      }
      acc *= since;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        if (2 * ks > wave) continue;
        Terms<NO> fu;
        terms_across<NO>(up + vb * NO * kUPlane + 32 * ks * kLdU, kUPlane, kLdU, fu);
        acc = mul_terms<NO>(fu, fp[ks], acc);
      }
      const int ch = 16 * (vb0 + vb) + row4;
      if (n < w.valid && ch < a.dv)
        store4<T>(at<T>(a.out, w.b * a.vo.b + w.h * a.vo.h + (w.n0 + n) * a.vo.n + ch), acc * a.scale);
    }
  }
}

}  // namespace lf
