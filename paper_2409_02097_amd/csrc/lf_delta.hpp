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
// chunks with 16 or 32 value channels per workgroup (delta_scan), and the outputs follow for all chunks at once
// (delta_out).  gamma and its differences are fp64: behind a token that forgets nearly everything the differences of an
// fp32 sum have lost the small decays that follow it.
//
// Products run on the 16-bit matrix instruction with operands as sums of bf16 terms (lf_terms.hpp), as many as hold all of a
// value: fp32 accurate for every type, because an output may be the small rest of a large state and its correction.  What
// passes between the kernels is stored as its reader takes it, a contiguous kilobyte for each operand or accumulator of a wave,
// all of a chunk and head in one record (a workgroup then touches a page or two of the workspace, not one per array):
//     w      T (beta e^gamma K) as operand: [4 row blocks][d_k / 32][3 terms][64 lanes][8 steps]
//     kt     K^T as operand: [d_k / 16][2][terms][64][8], in the record of the first value head that has the key head
//     u      U0, then U, and s the state before the chunk, as fp32 accumulators: [d_v / 16][row blocks][64][4]
//     decay  what follows from g and beta per token
//     wt     W^T as operand, [d_k / 16][2][3][64][8], and tt (T beta)^T, six operands of 64 x 8 fp32: for the backward pass
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
  unsigned char *record, *record_b;   // of the forward pass, of the backward pass
  unsigned size, size_b;              // bytes of one
  unsigned at_kt, at_u, at_s, at_decay, at_wt, at_tt, at_kn, at_ds;   // bytes into it; w, and du in the other, come first
  int for_backward;
  long long N;
  int H, Hk, heads, nc;           // B * H; chunks of N tokens
  int runs, run;                  // runs that the chunks are parted into, and how many make one
  float *parts, *joined;          // per run: what delta_scan<PARTIAL> leaves, and the state it starts from
  int dk, dv, dkb, dvb, dks;      // channels, blocks of 16 of them, and of 32
  float scale;
  // backward
  const void* dout;
  const float* dstate_out;
  void *dq, *dk_out, *dv_out;
  float *dg, *dbeta, *dstate_in;
  DeltaView vdo, vdq, vdk, vdv, vdg;

  LF_DEV unsigned char* rec(int bh, int chunk) const { return record + ((long long)bh * nc + chunk) * size; }
  LF_DEV unsigned char* rec_b(int bh, int chunk) const { return record_b + ((long long)bh * (nc + 2) + chunk) * size_b; }
};
template <typename P> LF_DEV P* part(unsigned char* record, unsigned at) { return reinterpret_cast<P*>(record + at); }

// rows of `decay`: e^gamma; e^(gamma_63 - gamma), 0 where beta is 0 (such a token leaves the state alone); beta, never 0 (u / beta
// is needed where beta is 0 too, for its gradient); e^(gamma_63 - gamma) everywhere
constexpr int kDecaySince = 0, kDecayWrite = 64, kDecayBeta = 128, kDecayLeft = 192, kDecayRows = 256;
constexpr int kDecayBytes = kDecayRows * 4 + 64 * 8;   // and gamma, as powers of two, in fp64

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

// Four neighbouring channels, as they are stored and widened.
template <typename T> struct Raw4Of { using type = u32x2; };
template <> struct Raw4Of<F32> { using type = f32x4; };
template <typename T> using Raw4 = typename Raw4Of<T>::type;
template <typename T> LF_DEV Raw4<T> load4_raw(const unsigned char* p) { return *reinterpret_cast<const Raw4<T>*>(p); }
template <typename T> LF_DEV f32x4 widen4(const Raw4<T>& w) {
  if constexpr (Stored<T>::kBytes == 4) {
    return w;
  } else {
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

// gamma of the 64 tokens, by one wave, as a power of two; a decay of -infinity counts as -10^4, which is none left
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
  return x * 1.4426950408889634074;
}

// 2^x of an fp64 power: the rounding of x to fp32 is off by 2^-24 of x, which matters the less the smaller the result
LF_DEV float power(double x) { return __builtin_amdgcn_exp2f((float)x); }
LF_DEV float decay_between(const double* gamma, int i, int j) { return power(gamma[i] - gamma[j]); }

constexpr int kLdP = 72;   // leading dimension in LDS of a 64 x 64 plane
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
// 10 heads of 64 channels, 65536 tokens, bf16: 139 to 176 us for 25 MB read and 500 MB of records written (3 to 3.6 TB/s); 96 heads of
// 40, 4096 tokens, with what the backward pass needs: 120 us, 450 MB (3.8 TB/s).
//
// A lower triangular matrix of 64 rows in LDS as its ten 16 x 16 blocks on and below the diagonal (fp32, 20 floats a row: both operand
// forms are free of bank conflicts): 13 KB, so that four workgroups of heads up to 64 fit a CU's LDS beside their keys.  What
// bounds the kernel is its chain of dependent small steps, so workgroups per CU are what counts.
constexpr int kLdB = 20, kBlock = 16 * kLdB;
LF_DEV int block_at(int i, int j) { return (i * (i + 1) / 2 + j) * kBlock; }

// Blocks of 32 value channels that pass through LDS at a time: all where a value is one term, two else (fp32 heads of 64 keys and 128
// values: 68 KB, two workgroups per CU, 18.8 us for 3 x 8 heads of 1000 tokens; all of them make it 95 KB, one, and 28.5 us).
template <typename T> LF_DEV_HOST int value_steps(int dvs) { return TermsOf<T>::kStored == 1 || dvs < 2 ? dvs : 2; }

template <typename T> inline int delta_prepare_lds(int dks, int dvs) {
  constexpr int N = TermsOf<T>::kStored;
  const int values = N * plane_bytes(64, value_steps<T>(dvs)), solve = 10 * kBlock * 4;
  return N * plane_bytes(64, dks) + solve + (values > solve ? values : solve) + 64 * 8 + kDecayRows * 4 + 64 * 4;
}

template <typename T, int KS> __global__ __launch_bounds__(256) void delta_prepare(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NI = TermsOf<T>::kStored, kLd = 32 * KS + 8, kPlane = 64 * kLd;
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  const int dvs = (a.dvb + 1) / 2, group = value_steps<T>(dvs), ldv = plane_ld(group);
  double* gamma = reinterpret_cast<double*>(smem);
  float* decay = reinterpret_cast<float*>(gamma + 64);
  float* both = decay + kDecayRows;                             // beta e^gamma
  float* mt = both + 64;                                        // T
  uint16_t* x = reinterpret_cast<uint16_t*>(mt + 10 * kBlock);  // the keys
  uint16_t* v = x + NI * kPlane;                                // A, then the values
  float* ma = reinterpret_cast<float*>(v);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15;
  const int g8 = (lane >> 4) * 8, row4 = (lane >> 4) * 4;
  unsigned char* rec = a.rec(w.bh, blockIdx.x);
  Rows<T, KS, 256> keys;
  keys.request(a.k, w.b * a.vk.b + w.hk * a.vk.h + w.n0 * a.vk.n, a.vk.n, w.valid, a.dk);
  if (wave == 0) {
    const double y = chunk_gamma(a, w), last = __shfl(y, 63, 64);
    float beta = 0.0f;
    if (lane < w.valid) beta = a.beta[w.b * a.vg.b + w.h * a.vg.h + (w.n0 + lane) * a.vg.n];
    const bool none = fabsf(beta) < kDeltaTinyBeta;
    if (none) beta = kDeltaTinyBeta;
    const float since = power(y), left = power(last - y);
    gamma[lane] = y;
    part<double>(rec, a.at_decay + kDecayRows * 4)[lane] = y;
    decay[kDecaySince + lane] = since;
    decay[kDecayWrite + lane] = none ? 0.0f : left;
    decay[kDecayBeta + lane] = beta;
    decay[kDecayLeft + lane] = left;
    both[lane] = beta * since;
  }
  keys.put(x, kLd);
  __syncthreads();
  part<float>(rec, a.at_decay)[tid] = decay[tid];
  if (w.h % (a.H / a.Hk) == 0) {
    uint16_t* kt = part<uint16_t>(rec, a.at_kt);
    for (int i = wave; i < a.dkb * 2; i += 4) {
      Terms<NI> f;
      terms_across<NI>(x + 32 * (i & 1) * kLd + 16 * (i >> 1), kPlane, kLd, f);
      store_frag<NI>(kt + i * NI * kFrag, f);
    }
  }
  // A, rows 16 wave .. + 15
  {
    Terms<NI> fi[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) terms_near<NI>(x + (16 * wave + col) * kLd + 32 * ks + g8, kPlane, fi[ks]);
    for (int nt = 0; nt <= wave; ++nt) {
      f32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Terms<NI> fj;
        terms_near<NI>(x + (16 * nt + col) * kLd + 32 * ks + g8, kPlane, fj);
        acc = mul_terms(fi[ks], fj, acc);
      }
      float* to = ma + block_at(wave, nt);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * wave + row4 + r, j = 16 * nt + col;
        to[(row4 + r) * kLdB + col] = i > j ? decay[kDecayBeta + i] * acc[r] * decay_between(gamma, i, j) : 0.0f;
      }
    }
  }
  // T: the blocks on the diagonal, a column per lane, by substitution (each wave its own: no barrier)
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  {
    const float* m = ma + block_at(wave, wave);
    float t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s0 = i == col ? 1.0f : 0.0f, s1 = 0.0f;
#pragma unroll
      for (int q = 0; q * 4 < i; ++q) {
        const f32x4 e = *reinterpret_cast<const f32x4*>(m + i * kLdB + 4 * q);
#pragma unroll
        for (int l = 0; l < 4; ++l) {
          if (4 * q + l >= i) continue;
          if (l & 1) s1 = __builtin_fmaf(-e[l], t[4 * q + l], s1);
          else s0 = __builtin_fmaf(-e[l], t[4 * q + l], s0);
        }
      }
      t[i] = s0 + s1;
    }
    if (lane < 16) {
      float* to = mt + block_at(wave, wave);
#pragma unroll
      for (int i = 0; i < 16; ++i) to[i * kLdB + lane] = t[i];
    }
  }
  __syncthreads();
  // the blocks below it: T_ij = -T_ii sum_l A_il T_lj, by their distance from the diagonal; the inner sum waits in T_ij's place
  for (int far = 1; far < 4; ++far) {
    const int i = wave + far, j = wave;
    if (i < 4) {
      float* tij = mt + block_at(i, j);
      f32x4 acc = {0, 0, 0, 0};
      for (int l = j; l < i; ++l)
        acc = mfma_block(steps_near(ma + block_at(i, l), kLdB), rows_near(mt + block_at(l, j), kLdB), acc);
#pragma unroll
      for (int r = 0; r < 4; ++r) tij[(row4 + r) * kLdB + col] = acc[r];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (only this wave uses the block until the barrier)
      acc = mfma_block(steps_near(mt + block_at(i, i), kLdB), rows_near(tij, kLdB), f32x4{0, 0, 0, 0});
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int r = 0; r < 4; ++r) tij[(row4 + r) * kLdB + col] = -acc[r];
    }
    __syncthreads();
  }
  auto put_values = [&](int step) {   // (A is read)
    stage_terms<T, 256>(v, ldv, a.v, w.b * a.vv.b + w.h * a.vv.h + w.n0 * a.vv.n + 32 * step, a.vv.n, w.valid, a.dv - 32 * step, group);
  };
  put_values(0);
  // T's rows 16 wave .. + 15 as an operand with a factor per column; nothing behind column 16 wave + 15
  const int steps = wave < 2 ? 1 : 2;
  auto rows_of_t = [&](const float* by, int ks, Terms<3>& f) {
    float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int j = 32 * ks + g8, jb = j >> 4;
    if (jb <= wave) {
      load8_f32(mt + block_at(wave, jb) + col * kLdB + (j & 15), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= by[j + e];
    }
    split8(y, f);
  };
  Terms<3> ft[2];
  rows_of_t(both, 0, ft[0]);
  if (steps > 1) rows_of_t(both, 1, ft[1]);
  uint16_t* mw = part<uint16_t>(rec, 0) + wave * KS * 3 * kFrag;
#pragma unroll
  for (int cb = 0; cb < 2 * KS; ++cb) {
    f32x4 acc = {0, 0, 0, 0}, act = {0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if (ks >= steps) continue;
      Terms<NI> key;
      terms_across<NI>(x + 32 * ks * kLd + 16 * cb, kPlane, kLd, key);
      acc = mul_terms(key, ft[ks], acc);
      if (a.for_backward) act = mul_terms(ft[ks], key, act);
    }
    store_operand<3>(mw + (cb >> 1) * 3 * kFrag, cb & 1, acc);
    if (a.for_backward && cb < a.dkb)
      store_operand<3>(part<uint16_t>(rec, a.at_wt) + (cb * 2 + (wave >> 1)) * 3 * kFrag, wave & 1, act);
  }
  rows_of_t(decay + kDecayBeta, 0, ft[0]);
  if (steps > 1) rows_of_t(decay + kDecayBeta, 1, ft[1]);
  __syncthreads();
  for (int vb = 0; vb < a.dvb; ++vb) {
    const int at_vb = vb % (2 * group);
    if (vb > 0 && at_vb == 0) {
      __syncthreads();
      put_values(vb / 2);
      __syncthreads();
    }
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if (ks >= steps) continue;
      Terms<NI> val;
      terms_across<NI>(v + 32 * ks * ldv + 16 * at_vb, 64 * ldv, ldv, val);
      acc = mul_terms(val, ft[ks], acc);
    }
    *reinterpret_cast<f32x4*>(part<float>(rec, a.at_u) + ((vb * 4 + wave) * 64 + lane) * 4) = acc;
  }
  if (a.for_backward) {   // (T beta)^T's rows j of this wave: nothing before column i = j, so six operands of the eight, in fp32
    const float by = decay[kDecayBeta + 16 * wave + col];
    for (int ks = wave >> 1; ks < 2; ++ks) {
      float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      const int i = 32 * ks + g8, ib = i >> 4;
      if (ib >= wave) {
        const float* p = mt + block_at(ib, wave) + (i & 15) * kLdB + col;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = p[e * kLdB] * by;
      }
      store8<F32>(rec + a.at_tt + ((wave < 2 ? 2 * wave + ks : 2 + wave) * 64 + lane) * 32, y);
    }
  }
}

// ---- the scan ---------------------------------------------------------------------------------------------------------------
// A workgroup takes 16 COLS value channels of one head through a run of chunks; its four waves hold the state's row blocks
// wave, wave + 4, ... as accumulators and compute 16 tokens of U each.  Bound: with few workgroups the chain from one chunk's
// state to the next (two products, two passes through LDS; what it reads is requested two chunks ahead where registers
// allow it), with many the operands' way from the L2, which every slice of a head reads anew: hence 32 channels where there
// are enough of them.  10 heads of 64 channels, 65536 tokens, bf16, in 12 runs: 184 us, 2.1 us a chunk (the first pass 196 us with two
// workgroups on most CUs); 96 heads of 40, 4096 tokens: 113 us, 1.8 us a chunk.  64 channels a workgroup were slower.
//
// With fewer workgroups than the device has room for, a head's chunks are parted into runs.  A run turns the state it starts
// from into M S + R with a d_k x d_k matrix M of its own: a first pass (PARTIAL) takes zeros and the columns of the identity
// through every run at once, delta_join takes the state through the runs, and the second pass starts each from its state.
template <int NI, int KS, int COLS> struct ScanIn {
  static constexpr int kBlocks = (2 * KS + 3) / 4;
  // chunks in flight and in work: three where the registers hold them (the first pass over 65536 tokens of 10 heads of 64, bf16: 185 us
  // against 193 with two; the others are the same)
  static constexpr int kDepth = 12 * KS + 8 * NI * kBlocks + 4 * COLS <= 114 ? 3 : 2;
  Terms<3> w[KS];
  Terms<NI> kt[kBlocks][2];
  f32x4 u0[COLS];
  float write, whole;
};

// The slices of a head on one XCD, whose L2 they share: workgroups are dealt to the eight XCDs in turn.
LF_DEV void slice_of_head(unsigned i, int slices, int heads, int& slice, int& bh) {
  const unsigned group = i / (8u * slices), r = i - group * 8u * slices;
  const unsigned here = heads - 8 * group < 8 ? heads - 8 * group : 8;
  slice = r / here;
  bh = 8 * group + (r - slice * here);
}

template <int NI, int KS, int COLS, bool PARTIAL> __global__ __launch_bounds__(256) void delta_scan(DeltaArgs a) {
  using In = ScanIn<NI, KS, COLS>;
  constexpr int kBlocks = In::kBlocks, kLd = 32 * KS + 8, kPlane = 16 * COLS * kLd, kLdU = 16 * COLS + 4, kUPlane = 64 * kLdU;
  __shared__ __align__(16) uint16_t sp[3 * kPlane];
  __shared__ __align__(16) uint16_t up[3 * kUPlane];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15;
  const int row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  const int slices = PARTIAL ? a.dvb + a.dkb : a.dvb, run = blockIdx.y;
  int group, bh;
  slice_of_head(blockIdx.x, (slices + COLS - 1) / COLS, a.heads, group, bh);
  const DeltaAt first(a, bh, 0);
  const int all = (int)((tokens_of(a.lengths, first.b, a.N) + 63) / 64);
  const int begin = run * a.run, end = begin + a.run < all ? begin + a.run : all;
  if (!PARTIAL && run > 0 && begin >= all) return;
  // A wave without a block of its own does the last one's work again, to the same bits, and so does a last odd slice: with
  // every load and store of a chunk unconditional, the compiler can wait for exactly those that it needs.
  int blk[kBlocks], slice[COLS];
  bool unit[COLS];   // columns of the identity, and no values
#pragma unroll
  for (int t = 0; t < kBlocks; ++t) blk[t] = wave + 4 * t < a.dkb ? wave + 4 * t : a.dkb - 1;
#pragma unroll
  for (int e = 0; e < COLS; ++e) {
    slice[e] = COLS * group + e < slices ? COLS * group + e : slices - 1;
    unit[e] = PARTIAL && slice[e] >= a.dvb;
  }
  f32x4 s[COLS][kBlocks];
#pragma unroll
  for (int e = 0; e < COLS; ++e)
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      float* joined = a.joined + ((((long long)bh * a.runs + run) * a.dvb + slice[e]) * a.dkb + blk[t]) * 256 + lane * 4;
      if (!PARTIAL && a.runs > 1) {
        s[e][t] = *reinterpret_cast<const f32x4*>(joined);
        continue;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * blk[t] + row4 + r, ch = slice[e] * 16 + col;
        if (unit[e]) s[e][t][r] = row == (slice[e] - a.dvb) * 16 + col ? 1.0f : 0.0f;
        else s[e][t][r] = a.state_in && run == 0 && row < a.dk && ch < a.dv ? a.state_in[((long long)bh * a.dk + row) * a.dv + ch] : 0.0f;
      }
      // (the second pass takes the first run's from here too: another run of it may have written over `state_in` by then)
      if (PARTIAL && run == 0 && !unit[e]) *reinterpret_cast<f32x4*>(joined) = s[e][t];
    }
  for (int i = tid; i < 3 * kPlane / 8; i += 256) reinterpret_cast<u32x4*>(sp)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
  const int key_head = bh - first.h + first.hk * (a.H / a.Hk);   // whose records have K^T
  int u_at[COLS];
#pragma unroll
  for (int e = 0; e < COLS; ++e) u_at[e] = ((unit[e] ? 0 : slice[e]) * 4 + wave) * 256 + lane * 4;
  // An address that differs by lane as far as the compiler can see: uniform loads would go through the scalar cache, whose
  // counter the barriers wait for, and its misses with it.
  int zero = 0;
  asm volatile("" : "+v"(zero));
  const unsigned char* ahead = a.rec(bh, begin);            // the record requested next
  const unsigned char* ahead_key = a.rec(key_head, begin);
  int requested = begin;
  auto request = [&](In& n) {
    const uint16_t* mw = reinterpret_cast<const uint16_t*>(ahead) + wave * KS * 3 * kFrag;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) load_frag<3>(mw + ks * 3 * kFrag, n.w[ks]);
    const uint16_t* kt = reinterpret_cast<const uint16_t*>(ahead_key + a.at_kt);
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) load_frag<NI>(kt + (blk[t] * 2 + ks) * NI * kFrag, n.kt[t][ks]);
#pragma unroll
    for (int e = 0; e < COLS; ++e) n.u0[e] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(ahead + a.at_u) + u_at[e]);
    const float* decay = reinterpret_cast<const float*>(ahead + a.at_decay);
    n.write = decay[kDecayWrite + 16 * wave + col];
    n.whole = decay[kDecaySince + 63 + zero];
    const unsigned step = ++requested < end ? a.size : 0;   // (the last one again behind the end)
    ahead += step;
    ahead_key += step;
  };
  unsigned char* here = a.rec(bh, begin);
  auto keep = [&](float* to) {   // `to`: the first slice
#pragma unroll
    for (int e = 0; e < COLS; ++e)
#pragma unroll
      for (int t = 0; t < kBlocks; ++t) *reinterpret_cast<f32x4*>(to + (slice[e] * a.dkb + blk[t]) * 256 + lane * 4) = s[e][t];
  };
  auto chunk = [&](In& in, In& next) {
#pragma unroll
    for (int e = 0; e < COLS; ++e)
#pragma unroll
      for (int t = 0; t < kBlocks; ++t) split4_lds<3>(sp + (16 * e + col) * kLd + 16 * blk[t] + row4, kPlane, s[e][t]);
    lds_barrier();
    f32x4 acc[COLS], acc2[COLS];
#pragma unroll
    for (int e = 0; e < COLS; ++e) acc[e] = acc2[e] = f32x4{0, 0, 0, 0};
    Terms<3> first_fs;
    terms_near<3>(sp + col * kLd + g8, kPlane, first_fs);
    __builtin_amdgcn_sched_barrier(0);
    request(next);                                           // while the planes are on their way
    if constexpr (!PARTIAL) keep(reinterpret_cast<float*>(here + a.at_s));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int e = 0; e < COLS; ++e) {
        Terms<3> fs;
        if (ks == 0 && e == 0) fs = first_fs;
        else terms_near<3>(sp + (16 * e + col) * kLd + 32 * ks + g8, kPlane, fs);
        if (COLS == 1 && (ks & 1)) acc2[e] = mul_terms(fs, in.w[ks], acc2[e]);
        else acc[e] = mul_terms(fs, in.w[ks], acc[e]);
      }
    f32x4 u[COLS];
#pragma unroll
    for (int e = 0; e < COLS; ++e) {
      f32x4 u0 = in.u0[e];
      if (unit[e]) u0 = f32x4{0, 0, 0, 0};
      u[e] = u0 - (acc[e] + acc2[e]);
      split4_lds<3>(up + (16 * wave + col) * kLdU + 16 * e + row4, kUPlane, u[e] * in.write);
    }
    lds_barrier();
#pragma unroll
    for (int e = 0; e < COLS; ++e) {
      Terms<3> fu[2];
      terms_across<3>(up + 16 * e, kUPlane, kLdU, fu[0]);
      terms_across<3>(up + 32 * kLdU + 16 * e, kUPlane, kLdU, fu[1]);
      if constexpr (!PARTIAL) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(here + a.at_u) + u_at[e]) = u[e];
#pragma unroll
      for (int t = 0; t < kBlocks; ++t) {
        f32x4 more = {0, 0, 0, 0};
        s[e][t] *= in.whole;
        s[e][t] = mul_terms(in.kt[t][0], fu[0], s[e][t]);
        more = mul_terms(in.kt[t][1], fu[1], more);
        s[e][t] += more;
      }
    }
    here += a.size;
  };
  if (begin < end) {
    In x, y;
    request(x);
    if constexpr (In::kDepth == 3) {
      In z;
      request(y);
      int i = begin;
      for (; i + 2 < end; i += 3) {
        chunk(x, z);
        chunk(y, x);
        chunk(z, y);
      }
      if (i < end) chunk(x, z);
      if (i + 1 < end) chunk(y, x);
    } else {
      int i = begin;
      for (; i + 1 < end; i += 2) {
        chunk(x, y);
        chunk(y, x);
      }
      if (i < end) chunk(x, y);
    }
  }
  if constexpr (PARTIAL) {
    keep(a.parts + ((long long)bh * a.runs + run) * (a.dvb + a.dkb) * a.dkb * 256);
  } else if (end == all && a.state_out) {
#pragma unroll
    for (int e = 0; e < COLS; ++e)
#pragma unroll
      for (int t = 0; t < kBlocks; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * blk[t] + row4 + r, ch = slice[e] * 16 + col;
          if (row < a.dk && ch < a.dv) a.state_out[((long long)bh * a.dk + row) * a.dv + ch] = s[e][t][r];
        }
  }
}

// The state that each run starts from, 16 value channels of one head: the first run's end, then M S + R run by run, in fp32 products.
// M's column k is a partial state's column k: the operand gathers its four steps from four lanes' accumulators.  A chain too, so what
// later runs need is requested ahead: 0.75 us a run for states of 64 x 64 (1.6 without), 3 for 128 x 128.
template <int KS> struct JoinIn {
  static constexpr int kBlocks = (2 * KS + 3) / 4, kDepth = KS <= 2 ? 4 : 2;
  f32x4 r[kBlocks], m[kBlocks][2 * KS];
};

template <int KS> __global__ __launch_bounds__(256) void delta_join(DeltaArgs a) {
  using In = JoinIn<KS>;
  constexpr int kBlocks = In::kBlocks;
  __shared__ __align__(16) float sl[32 * KS * kLdB];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15;
  const int row4 = (lane >> 4) * 4, slice = blockIdx.x, bh = blockIdx.y, slices = a.dvb + a.dkb, last = a.runs - 2;
  int blk[kBlocks];   // (as in delta_scan)
#pragma unroll
  for (int t = 0; t < kBlocks; ++t) blk[t] = wave + 4 * t < a.dkb ? wave + 4 * t : a.dkb - 1;
  const int step = slices * a.dkb * 256;
  const float* ahead = a.parts + (long long)bh * a.runs * step;
  int requested = 0;
  auto request = [&](In& n) {
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      n.r[t] = *reinterpret_cast<const f32x4*>(ahead + (slice * a.dkb + blk[t]) * 256 + lane * 4);
#pragma unroll
      for (int kb = 0; kb < 2 * KS; ++kb) {
        const int k = kb < a.dkb ? kb : a.dkb - 1;
        const float* m = ahead + ((a.dvb + k) * a.dkb + blk[t]) * 256 + (row4 + 16 * (col >> 2)) * 4 + (col & 3);
        n.m[t][kb] = f32x4{m[0], m[4], m[8], m[12]};
      }
    }
    ahead += requested++ < last ? step : 0;   // (the last one again behind the end)
  };
  float* to = a.joined + (((long long)bh * a.runs + 1) * a.dvb + slice) * a.dkb * 256 + lane * 4;
  auto join = [&](int run, const In& in, In& next) {
    request(next);
    f32x4 s[kBlocks];
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      s[t] = in.r[t];
      if (run == 0) continue;
#pragma unroll
      for (int kb = 0; kb < 2 * KS; ++kb)
        if (kb < a.dkb) s[t] = mfma_block(in.m[t][kb], rows_near(sl + 16 * kb * kLdB, kLdB), s[t]);
    }
    lds_barrier();
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
#pragma unroll
      for (int r = 0; r < 4; ++r) sl[(16 * blk[t] + row4 + r) * kLdB + col] = s[t][r];
      *reinterpret_cast<f32x4*>(to + blk[t] * 256) = s[t];
    }
    to += a.dvb * a.dkb * 256;
    lds_barrier();
  };
  In x, y;
  request(x);
  if constexpr (In::kDepth == 4) {
    In z, w;
    request(y);
    request(z);
    int run = 0;
    for (; run + 3 <= last; run += 4) {
      join(run, x, w);
      join(run + 1, y, x);
      join(run + 2, z, y);
      join(run + 3, w, z);
    }
    if (run <= last) join(run, x, w);
    if (run + 1 <= last) join(run + 1, y, x);
    if (run + 2 <= last) join(run + 2, z, y);
  } else {
    int run = 0;
    for (; run + 1 <= last; run += 2) {
      join(run, x, y);
      join(run + 1, y, x);
    }
    if (run <= last) join(run, x, y);
  }
}

// ---- the outputs --------------------------------------------------------------------------------------------------------------
// Formed transposed, so that a lane has four neighbouring channels of a token: O^T = e^gamma S0^T Q^T + U^T P^T.
// Bound: what it reads, U and the state in fp32.  10 heads of 64 channels, 65536 tokens, bf16: 143 us for 470 MB (3.3 TB/s).
//
// Value channels pass through LDS 32 at a time (three terms each; 64 of them leave room for fewer workgroups).  us a forward call, 32 : 64:
// bf16 10 heads of 64, 65536 tokens 658 : 674; 8 heads of 128, 8192 tokens 215 : 231; 64 heads of 32, 4096 tokens 123 : 128; fp16 32 heads of
// 128, 2048 tokens 141 : 154; fp32 16 heads of 64, 4096 tokens 105 : 107; fp16 8 heads of 64, 197 tokens 29.7 : 28.6.
constexpr int kOutBlocks = 2;   // of 16 value channels

template <typename T> inline int delta_out_lds(int dks) {
  constexpr int NI = TermsOf<T>::kStored;
  const int keys = NI * plane_bytes(64, dks), scores = 3 * 64 * kLdP * 2, rows = keys + (keys > scores ? keys : scores);
  const int later = kOutBlocks * 3 * (plane_bytes(16, dks) + 64 * kLdU * 2);
  return (rows > later ? rows : later) + 64 * 8 + 2 * 64 * 4;
}

template <typename T, int KS> __global__ __launch_bounds__(256) void delta_out(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NI = TermsOf<T>::kStored, KB = 2 * KS, kLd = 32 * KS + 8;
  constexpr int kSPlane = 16 * kLd, kUPlane = 64 * kLdU;
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  double* gamma = reinterpret_cast<double*>(smem);
  float* decay = reinterpret_cast<float*>(gamma + 64);   // e^gamma, beta
  uint16_t* q = reinterpret_cast<uint16_t*>(decay + 128);
  uint16_t* k = q + NI * 64 * kLd;
  uint16_t* pp = k;                                      // where the keys were
  uint16_t* sp = q;                                      // later, where all of these were
  uint16_t* up = sp + kOutBlocks * 3 * kSPlane;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15;
  const int row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  unsigned char* rec = a.rec(w.bh, blockIdx.x);
  Rows<T, KS, 256> queries, keys;
  queries.request(a.q, w.b * a.vq.b + w.hk * a.vq.h + w.n0 * a.vq.n, a.vq.n, w.valid, a.dk);
  keys.request(a.k, w.b * a.vk.b + w.hk * a.vk.h + w.n0 * a.vk.n, a.vk.n, w.valid, a.dk);
  if (wave == 0) {
    gamma[lane] = part<double>(rec, a.at_decay + kDecayRows * 4)[lane];
    decay[lane] = part<float>(rec, a.at_decay)[kDecaySince + lane];
    decay[64 + lane] = part<float>(rec, a.at_decay)[kDecayBeta + lane];
  }
  // the first blocks of U and of the state, requested now, put down when there is room
  f32x4 s_in[KB], u_in[kOutBlocks];
  int vb0 = 0, blocks = a.dvb < kOutBlocks ? a.dvb : kOutBlocks;
  auto request = [&]() {   // wave w: block w of the state (all of its rows), 16 tokens of every block of U
    const float* s0 = part<float>(rec, a.at_s) + vb0 * a.dkb * 256;
    const float* mu = part<float>(rec, a.at_u) + vb0 * 1024;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      if (wave < blocks && kb < a.dkb) s_in[kb] = *reinterpret_cast<const f32x4*>(s0 + (wave * a.dkb + kb) * 256 + lane * 4);
#pragma unroll
    for (int i = 0; i < kOutBlocks; ++i)
      if (i < blocks) u_in[i] = *reinterpret_cast<const f32x4*>(mu + (i * 4 + wave) * 256 + lane * 4);
  };
  request();
  queries.put(q, kLd);
  keys.put(k, kLd);
  __syncthreads();
  Terms<NI> fq[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) terms_near<NI>(q + (16 * wave + col) * kLd + 32 * ks + g8, 64 * kLd, fq[ks]);
  // P's rows of this wave, four neighbouring columns j of row i at a time; 0 where beta_j is 0 (the u_j that is kept is not)
  f32x4 scores[4];
#pragma unroll
  for (int jt = 0; jt < 4; ++jt) {
    f32x4 acc = {0, 0, 0, 0};
    if (jt <= wave) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Terms<NI> fk;
        terms_near<NI>(k + (16 * jt + col) * kLd + 32 * ks + g8, 64 * kLd, fk);
        acc = mul_terms(fk, fq[ks], acc);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * wave + col, j = 16 * jt + row4 + r;
        const bool on = j <= i && decay[64 + j] != kDeltaTinyBeta;
        acc[r] = on ? acc[r] * decay_between(gamma, i, j) : 0.0f;
      }
    }
    scores[jt] = acc;
  }
  __syncthreads();   // the keys are read
#pragma unroll
  for (int jt = 0; jt < 4; ++jt) split4_lds<3>(pp + (16 * wave + col) * kLdP + 16 * jt + row4, 64 * kLdP, scores[jt]);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (rows that only this wave writes and reads)
  Terms<3> fp[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) terms_near<3>(pp + (16 * wave + col) * kLdP + 32 * ks + g8, 64 * kLdP, fp[ks]);
  const float since = decay[16 * wave + col];
  const int n = 16 * wave + col;
  for (;;) {
    __syncthreads();
    if (wave < blocks) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)   // (zeros in the half block behind d_k: the queries' zeros times what is there)
        split4_lds<3>(sp + wave * 3 * kSPlane + col * kLd + 16 * kb + row4, kSPlane, kb < a.dkb ? s_in[kb] : f32x4{0, 0, 0, 0});
    }
#pragma unroll
    for (int i = 0; i < kOutBlocks; ++i)
      if (i < blocks) split4_lds<3>(up + i * 3 * kUPlane + n * kLdU + row4, kUPlane, u_in[i]);
    const int here = blocks, at_block = vb0;
    vb0 += kOutBlocks;
    blocks = a.dvb - vb0 < kOutBlocks ? a.dvb - vb0 : kOutBlocks;
    if (vb0 < a.dvb) request();
    __syncthreads();
    for (int vb = 0; vb < here; ++vb) {
      f32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Terms<3> fs;
        terms_near<3>(sp + vb * 3 * kSPlane + col * kLd + 32 * ks + g8, kSPlane, fs);
        acc = mul_terms(fs, fq[ks], acc);
      }
      acc *= since;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        if (2 * ks > wave) continue;
        Terms<3> fu;
        terms_across<3>(up + vb * 3 * kUPlane + 32 * ks * kLdU, kUPlane, kLdU, fu);
        acc = mul_terms(fu, fp[ks], acc);
      }
      const int ch = 16 * (at_block + vb) + row4;
      if (n < w.valid && ch < a.dv)
        store4<T>(at<T>(a.out, w.b * a.vo.b + w.h * a.vo.h + (w.n0 + n) * a.vo.n + ch), acc * a.scale);
    }
    if (vb0 >= a.dvb) break;
  }
}

}  // namespace lf
