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
// and the values by its inverse.  Only dU and dS0 depend on the chunk behind: P^T dO and (e^gamma Q)^T dO are formed for all
// chunks at once (delta_back_prepare), a scan runs from the last chunk to the first (delta_back_scan), and the rest follows
// for all chunks at once (delta_gradients), where the value heads that share a query and key head are summed in their order.
//     kn   K as operand: [4 token blocks][d_k / 32][terms][64][8], once per query and key head
//     du   P^T dO, then dU, as u;   ds   as s, two places more per head: (e^gamma Q)^T dO of chunk c at c, dS1 two places on,
//          which every wave of the scan has behind it when dS1 is written
#pragma once
#include "lf_delta.hpp"

namespace lf {

// ---- what does not depend on the chunk behind ---------------------------------------------------------------------------------
template <typename T> inline int delta_back_prepare_lds(int dks, int dvs) {
  constexpr int NI = TermsOf<T>::kStored;
  const int keys = NI * plane_bytes(64, dks), out = NI * plane_bytes(64, dvs);
  return 64 * 8 + 64 * 4 + 3 * 64 * kLdP * 2 + (2 * keys > out ? 2 * keys : out);
}

template <typename T> __global__ __launch_bounds__(256) void delta_back_prepare(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NI = TermsOf<T>::kStored;
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  const int dvs = (a.dvb + 1) / 2, ld = plane_ld(a.dks), ldo = plane_ld(dvs), plane = 64 * ld;
  double* gamma = reinterpret_cast<double*>(smem);
  float* since = reinterpret_cast<float*>(gamma + 64);
  uint16_t* pp = reinterpret_cast<uint16_t*>(since + 64);
  uint16_t* q = pp + 3 * 64 * kLdP;
  uint16_t* k = q + NI * plane;
  uint16_t* o = q;                      // where q and k were
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  const long long c = (long long)blockIdx.y * a.nc + blockIdx.x;
  if (wave == 0) gamma[lane] = chunk_gamma(a, w);
  if (tid < 64) since[tid] = a.decay[c * kDecayRows + kDecaySince + tid];
  stage_terms<T>(q, ld, a.q, w.b * a.vq.b + w.hk * a.vq.h + w.n0 * a.vq.n, a.vq.n, w.valid, a.dk, a.dks);
  stage_terms<T>(k, ld, a.k, w.b * a.vk.b + w.hk * a.vk.h + w.n0 * a.vk.n, a.vk.n, w.valid, a.dk, a.dks);
  __syncthreads();
  if (w.h % (a.H / a.Hk) == 0) {
    uint16_t* kn = a.kn + (((long long)(w.b * a.Hk + w.hk) * a.nc + blockIdx.x) * 4 + wave) * a.dks * NI * kFrag;
    for (int ks = 0; ks < a.dks; ++ks) {
      Terms<NI> f;
      terms_near<NI>(k + (16 * wave + col) * ld + 32 * ks + g8, plane, f);
      store_frag<NI>(kn + ks * NI * kFrag, f);
    }
  }
  // P transposed, [j][i]: four neighbouring rows i of column j at a time; rows i of tile `it`, columns of this wave's
  for (int it = 0; it < 4; ++it) {
    f32x4 acc = {0, 0, 0, 0};
    if (it >= wave) {
      for (int ks = 0; ks < a.dks; ++ks) {
        Terms<NI> fq, fk;
        terms_near<NI>(q + (16 * it + col) * ld + 32 * ks + g8, plane, fq);
        terms_near<NI>(k + (16 * wave + col) * ld + 32 * ks + g8, plane, fk);
        acc = mul_terms<3>(fq, fk, acc);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * it + row4 + r, j = 16 * wave + col;
        acc[r] = j <= i ? acc[r] * decay_between(gamma, i, j) : 0.0f;
      }
    }
    split4_lds<3>(pp + (16 * wave + col) * kLdP + 16 * it + row4, 64 * kLdP, acc);
  }
  // (e^gamma Q)^T as operands of this wave's channel blocks, before the queries make room: scaled, then split again
  __syncthreads();
  Terms<3> fq[3][2];   // channel blocks wave, wave + 4, wave + 8
#pragma unroll
  for (int t = 0; t < 3; ++t)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if (wave + 4 * t >= a.dkb) continue;
      Terms<NI> f;
      terms_across<NI>(q + 32 * ks * ld + 16 * (wave + 4 * t), plane, ld, f);
      float y[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float lo = 0.0f, hi = 0.0f;
#pragma unroll
        for (int p = NI - 1; p >= 0; --p) {
          float l1, h1;
          unpack2<BF16>(f.t[p][e], l1, h1);
          lo += l1;
          hi += h1;
        }
        const float* by = since + 32 * ks + g8 + 2 * e;
        y[2 * e] = lo * by[0] * a.scale;
        y[2 * e + 1] = hi * by[1] * a.scale;
      }
      split8(y, fq[t][ks]);
    }
  __syncthreads();
  stage_terms<T>(o, ldo, a.dout, w.b * a.vdo.b + w.h * a.vdo.h + w.n0 * a.vdo.n, a.vdo.n, w.valid, a.dv, dvs);
  Terms<3> fp[2];      // P^T's rows j of this wave
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) terms_near<3>(pp + (16 * wave + col) * kLdP + 32 * ks + g8, 64 * kLdP, fp[ks]);
  __syncthreads();
  for (int vb = 0; vb < a.dvb; ++vb) {
    Terms<NI> fo[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) terms_across<NI>(o + 32 * ks * ldo + 16 * vb, 64 * ldo, ldo, fo[ks]);
    f32x4 acc = {0, 0, 0, 0};   // rows: value channels, columns: tokens j
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) acc = mul_terms<3>(fo[ks], fp[ks], acc);
    *reinterpret_cast<f32x4*>(a.du + (((c * a.dvb + vb) * 4 + wave) * 64 + lane) * 4) = acc * a.scale;
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      if (wave + 4 * t >= a.dkb) continue;
      f32x4 z = {0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) z = mul_terms<3>(fq[t][ks], fo[ks], z);
      *reinterpret_cast<f32x4*>(a.ds + (((c + 2 * w.bh) * a.dvb + vb) * a.dkb + wave + 4 * t) * 256 + lane * 4) = z;
    }
  }
}

// ---- the scan backwards ----------------------------------------------------------------------------------------------------------
template <int NI, int KS> struct BackScanIn {
  static constexpr int kBlocks = (2 * KS + 3) / 4;
  Terms<NI> kn[KS];
  Terms<3> wt[kBlocks][2];
  f32x4 du, z[kBlocks];
  float left, whole;
};

template <int NI, int KS> __global__ __launch_bounds__(256) void delta_back_scan(DeltaArgs a) {
  constexpr int kBlocks = BackScanIn<NI, KS>::kBlocks, kLd = 32 * KS + 8, kPlane = 16 * kLd;
  __shared__ __align__(16) uint16_t sp[3 * kPlane];
  __shared__ __align__(16) uint16_t up[3 * 64 * kLdU];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15;
  const int row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  const int slice = blockIdx.x, bh = blockIdx.y, ch = slice * 16 + col;
  const DeltaAt first(a, bh, 0);
  const int chunks = (int)((tokens_of(a.lengths, first.b, a.N) + 63) / 64);
  int blk[kBlocks];   // (as in delta_scan)
#pragma unroll
  for (int t = 0; t < kBlocks; ++t) blk[t] = wave + 4 * t < a.dkb ? wave + 4 * t : a.dkb - 1;
  f32x4 s[kBlocks];
#pragma unroll
  for (int t = 0; t < kBlocks; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * blk[t] + row4 + r;
      s[t][r] = a.dstate_out && row < a.dk && ch < a.dv ? a.dstate_out[((long long)bh * a.dk + row) * a.dv + ch] : 0.0f;
    }
  for (int i = tid; i < 3 * kPlane / 8; i += 256) reinterpret_cast<u32x4*>(sp)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
  const long long c0 = (long long)bh * a.nc;
  const long long k0 = (long long)(first.b * a.Hk + first.hk) * a.nc;
  auto request = [&](BackScanIn<NI, KS>& n, int i) {
    const uint16_t* kn = a.kn + ((k0 + i) * 4 + wave) * a.dks * NI * kFrag;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) load_frag<NI>(kn + ks * NI * kFrag, n.kn[ks]);
    const uint16_t* wt = a.wt + (c0 + i) * a.dkb * 2 * 3 * kFrag;
    const float* z = a.ds + ((c0 + 2 * bh + i) * a.dvb + slice) * a.dkb * 256;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      n.z[t] = *reinterpret_cast<const f32x4*>(z + blk[t] * 256 + lane * 4);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) load_frag<3>(wt + (blk[t] * 2 + ks) * 3 * kFrag, n.wt[t][ks]);
    }
    n.du = *reinterpret_cast<const f32x4*>(a.du + ((((c0 + i) * a.dvb + slice) * 4 + wave) * 64 + lane) * 4);
    const float* decay = a.decay + (c0 + i) * kDecayRows;
    n.left = decay[kDecayLeft + 16 * wave + col];
    n.whole = decay[kDecaySince + 63];
  };
  auto chunk = [&](BackScanIn<NI, KS>& in, BackScanIn<NI, KS>& next, int i) {
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
      split4_lds<3>(sp + col * kLd + 16 * blk[t] + row4, kPlane, s[t]);
    request(next, i > 0 ? i - 1 : 0);
    float* to = a.ds + ((c0 + 2 * bh + i + 2) * a.dvb + slice) * a.dkb * 256;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
      *reinterpret_cast<f32x4*>(to + blk[t] * 256 + lane * 4) = s[t];
    lds_barrier();
    f32x4 acc = {0, 0, 0, 0}, acc2 = {0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      Terms<3> fs;
      terms_near<3>(sp + col * kLd + 32 * ks + g8, kPlane, fs);
      if (ks & 1) acc2 = mul_terms<3>(fs, in.kn[ks], acc2);
      else acc = mul_terms<3>(fs, in.kn[ks], acc);
    }
    const f32x4 u = in.du + (acc + acc2) * in.left;
    *reinterpret_cast<f32x4*>(a.du + ((((c0 + i) * a.dvb + slice) * 4 + wave) * 64 + lane) * 4) = u;
    split4_lds<3>(up + (16 * wave + col) * kLdU + row4, 64 * kLdU, -u);
    lds_barrier();
    Terms<3> fu[2];
    terms_across<3>(up, 64 * kLdU, kLdU, fu[0]);
    terms_across<3>(up + 32 * kLdU, 64 * kLdU, kLdU, fu[1]);
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      s[t] = s[t] * in.whole + in.z[t];
      s[t] = mul_terms<3>(in.wt[t][0], fu[0], s[t]);
      s[t] = mul_terms<3>(in.wt[t][1], fu[1], s[t]);
    }
  };
  BackScanIn<NI, KS> x, y;
  int i = chunks - 1;
  if (chunks > 0) request(x, i);
  for (; i > 0; i -= 2) {
    chunk(x, y, i);
    chunk(y, x, i - 1);
  }
  if (i == 0) chunk(x, y, 0);
  if (a.dstate_in) {
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * blk[t] + row4 + r;
        if (row < a.dk && ch < a.dv) a.dstate_in[((long long)bh * a.dk + row) * a.dv + ch] = s[t][r];
      }
  }
}

// ---- the gradients ------------------------------------------------------------------------------------------------------------
// Formed transposed (rows: channels, columns: tokens), a wave per 16 tokens.  32 value channels at a time pass through LDS:
// dU (then dV in its place), dO, U as [token][channel], S0 and dS1 as [channel][key channel].
constexpr int kLdV = 40;

template <typename T> inline int delta_gradients_lds(int dks) {
  constexpr int NI = TermsOf<T>::kStored;
  const int first = 3 * 3 * 64 * kLdV * 2 + 2 * 3 * plane_bytes(32, dks);
  const int second = 2 * 3 * 64 * kLdP * 2 + NI * plane_bytes(64, dks);
  return (first > second ? first : second) + 64 * 8 + kDecayRows * 4 + 16;
}

// sum over the four lanes of a wave that share l % 16
LF_DEV float groups_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

template <typename T, int KS, bool SHARED> __global__ __launch_bounds__(256) void delta_gradients(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NI = TermsOf<T>::kStored, KB = 2 * KS, kLd = 32 * KS + 8, kVPlane = 64 * kLdV, kSPlane = 32 * kLd;
  const int b = (unsigned)blockIdx.y / (unsigned)a.Hk, hk = blockIdx.y - b * a.Hk, group = SHARED ? a.H / a.Hk : 1;
  double* gamma = reinterpret_cast<double*>(smem);
  float* decay = reinterpret_cast<float*>(gamma + 64);
  float* inner = decay + kDecayRows;
  uint16_t* pv = reinterpret_cast<uint16_t*>(inner + 4);   // dU, then dV
  uint16_t* po = pv + 3 * kVPlane;
  uint16_t* pu = po + 3 * kVPlane;
  uint16_t* ps = pu + 3 * kVPlane;
  uint16_t* pd = ps + 3 * kSPlane;
  uint16_t* pm = pv;                                       // later: dO U^T * D, M, and the keys, then the queries
  uint16_t* pn = pm + 3 * 64 * kLdP;
  uint16_t* x = pn + 3 * 64 * kLdP;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  const int n = 16 * wave + col;                           // this lane's token
  const DeltaAt any(a, b * a.H + hk * group, blockIdx.x);
  if (any.valid == 0) return;
  const bool on = n < any.valid;
  f32x4 sum_q[SHARED ? KB : 1], sum_k[SHARED ? KB : 1];
  if constexpr (SHARED) {
#pragma unroll
    for (int i = 0; i < KB; ++i) sum_q[i] = sum_k[i] = f32x4{0, 0, 0, 0};
  }
  for (int member = 0; member < group; ++member) {
    const DeltaAt w(a, b * a.H + hk * group + member, blockIdx.x);
    const long long c = (long long)w.bh * a.nc + blockIdx.x;
    __syncthreads();
    if (wave == 0) gamma[lane] = chunk_gamma(a, w);
    decay[tid] = a.decay[c * kDecayRows + tid];
    f32x4 dq[KB], dk[KB], dw[KB], mo[4], mv[4];
#pragma unroll
    for (int i = 0; i < KB; ++i) dq[i] = dk[i] = dw[i] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) mo[i] = mv[i] = f32x4{0, 0, 0, 0};
    Terms<3> ft[2];   // (T beta)^T's rows of this wave: nothing before them
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      if (2 * ks + 1 >= wave) load_frag<3>(a.tt + ((c * 4 + wave) * 2 + ks) * 3 * kFrag, ft[ks]);
    float dbeta = 0.0f, ss = 0.0f;
    double vdv = 0.0;
    for (int i = tid; i < 2 * 3 * kSPlane / 8; i += 256) reinterpret_cast<u32x4*>(ps)[i] = u32x4{0, 0, 0, 0};
    for (int vb = 0; vb < a.dvb; vb += 2) {
      __syncthreads();   // the planes of the channels before are read; the zeros are there
      f32x4 u[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int ch = 16 * (vb + e) + row4;
        f32x4 du = {0, 0, 0, 0}, o = {0, 0, 0, 0};
        u[e] = f32x4{0, 0, 0, 0};
        if (vb + e < a.dvb) {
          const long long at4 = (((c * a.dvb + vb + e) * 4 + wave) * 64 + lane) * 4;
          du = *reinterpret_cast<const f32x4*>(a.du + at4);
          u[e] = *reinterpret_cast<const f32x4*>(a.u + at4);
          if (on && ch < a.dv) o = load4<T>(at<T>(a.dout, w.b * a.vdo.b + w.h * a.vdo.h + (w.n0 + n) * a.vdo.n + ch)) * a.scale;
        }
        const bool none = decay[kDecayBeta + n] == kDeltaTinyBeta;
        split4_lds<3>(pv + n * kLdV + 16 * e + row4, kVPlane, du);
        split4_lds<3>(po + n * kLdV + 16 * e + row4, kVPlane, o);
        split4_lds<3>(pu + n * kLdV + 16 * e + row4, kVPlane, none ? f32x4{0, 0, 0, 0} : u[e]);
        if (vb + e < a.dvb) {
          const float* s0 = a.s + (((long long)w.bh * (a.nc + 1) + blockIdx.x) * a.dvb + vb + e) * a.dkb * 256 + lane * 4;
          const float* s1 = s0 + (long long)a.dvb * a.dkb * 256;
          const float* ds = a.ds + ((c + 2 * w.bh + 2) * a.dvb + vb + e) * a.dkb * 256 + lane * 4;
          for (int kb = wave; kb < a.dkb; kb += 4) {
            const f32x4 d1 = *reinterpret_cast<const f32x4*>(ds + kb * 256), t1 = *reinterpret_cast<const f32x4*>(s1 + kb * 256);
            split4_lds<3>(ps + (16 * e + col) * kLd + 16 * kb + row4, kSPlane, *reinterpret_cast<const f32x4*>(s0 + kb * 256));
            split4_lds<3>(pd + (16 * e + col) * kLd + 16 * kb + row4, kSPlane, d1);
            ss += (d1[0] * t1[0] + d1[1] * t1[1]) + (d1[2] * t1[2] + d1[3] * t1[3]);
          }
        } else {   // an odd last block: zeros where the one before it was
          for (int kb = wave; kb < a.dkb; kb += 4) {
            split4_lds<3>(ps + (16 * e + col) * kLd + 16 * kb + row4, kSPlane, f32x4{0, 0, 0, 0});
            split4_lds<3>(pd + (16 * e + col) * kLd + 16 * kb + row4, kSPlane, f32x4{0, 0, 0, 0});
          }
        }
      }
      __syncthreads();
      f32x4 dv[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          if (2 * ks + 1 < wave) continue;
          Terms<3> f;
          terms_across<3>(pv + 32 * ks * kLdV + 16 * e, kVPlane, kLdV, f);
          acc = mul_terms<3>(f, ft[ks], acc);
        }
        const int ch = 16 * (vb + e) + row4;
        const float beta = decay[kDecayBeta + n];
        const f32x4 per = acc * (1.0f / beta) * (u[e] * (1.0f / beta));
        dbeta += (per[0] + per[1]) + (per[2] + per[3]);
        dv[e] = beta == kDeltaTinyBeta ? f32x4{0, 0, 0, 0} : acc;
        if (on && ch < a.dv) {
          const f32x4 v = load4<T>(at<T>(a.v, w.b * a.vv.b + w.h * a.vv.h + (w.n0 + n) * a.vv.n + ch));
          vdv += (double)(v[0] * dv[e][0] + v[1] * dv[e][1]) + (double)(v[2] * dv[e][2] + v[3] * dv[e][3]);
          store4<T>(at<T>(a.dv_out, w.b * a.vdv.b + w.h * a.vdv.h + (w.n0 + n) * a.vdv.n + ch), dv[e]);
        }
      }
      __syncthreads();   // dU is read
#pragma unroll
      for (int e = 0; e < 2; ++e) split4_lds<3>(pv + n * kLdV + 16 * e + row4, kVPlane, dv[e]);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (its own rows are all a wave reads of dV)
      Terms<3> fo, fv, fu;
      terms_near<3>(po + n * kLdV + g8, kVPlane, fo);
      terms_near<3>(pv + n * kLdV + g8, kVPlane, fv);
      terms_near<3>(pu + n * kLdV + g8, kVPlane, fu);
#pragma unroll
      for (int jt = 0; jt < 4; ++jt) {
        if (jt > wave) continue;
        Terms<3> fj;
        terms_near<3>(pu + (16 * jt + col) * kLdV + g8, kVPlane, fj);
        mo[jt] = mul_terms<3>(fj, fo, mo[jt]);
        mv[jt] = mul_terms<3>(fj, fv, mv[jt]);
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if (kb >= a.dkb) continue;
        Terms<3> f0, f1;
        terms_across<3>(ps + 16 * kb, kSPlane, kLd, f0);
        terms_across<3>(pd + 16 * kb, kSPlane, kLd, f1);
        dq[kb] = mul_terms<3>(f0, fo, dq[kb]);
        dk[kb] = mul_terms<3>(f0, fv, dk[kb]);
        dw[kb] = mul_terms<3>(f1, fu, dw[kb]);
      }
    }
    __syncthreads();
    const float since = decay[kDecaySince + n], write = decay[kDecayWrite + n];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      dq[kb] *= since;
      dk[kb] = dw[kb] * write - dk[kb] * since;
    }
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      f32x4 e = mo[jt], m = mv[jt];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 16 * jt + row4 + r;
        const float d = j <= n ? decay_between(gamma, n, j) : 0.0f;
        e[r] = j <= n ? e[r] * d : 0.0f;
        m[r] = j < n ? -m[r] * d : 0.0f;
      }
      split4_lds<3>(pm + n * kLdP + 16 * jt + row4, 64 * kLdP, e);
      split4_lds<3>(pn + n * kLdP + 16 * jt + row4, 64 * kLdP, m);
    }
    stage_terms<T>(x, kLd, a.k, b * a.vk.b + hk * a.vk.h + any.n0 * a.vk.n, a.vk.n, any.valid, a.dk, KS);
    ss = lanes_sum<64>(ss);
    if (lane == 0) inner[wave] = ss;
    dbeta = groups_sum(dbeta);
    __syncthreads();
    Terms<3> fe[2], fm[2], em[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      terms_near<3>(pm + n * kLdP + 32 * ks + g8, 64 * kLdP, fe[ks]);
      terms_near<3>(pn + n * kLdP + 32 * ks + g8, 64 * kLdP, fm[ks]);
      terms_across<3>(pn + 32 * ks * kLdP + 16 * wave, 64 * kLdP, kLdP, em[ks]);
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if (kb >= a.dkb) continue;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        Terms<NI> f;
        terms_across<NI>(x + 32 * ks * kLd + 16 * kb, 64 * kLd, kLd, f);
        if (2 * ks <= wave) {
          dq[kb] = mul_terms<3>(f, fe[ks], dq[kb]);
          dk[kb] = mul_terms<3>(f, fm[ks], dk[kb]);
        }
        if (2 * ks + 1 >= wave) dk[kb] = mul_terms<3>(f, em[ks], dk[kb]);
      }
    }
    __syncthreads();
    stage_terms<T>(x, kLd, a.q, b * a.vq.b + hk * a.vq.h + any.n0 * a.vq.n, a.vq.n, any.valid, a.dk, KS);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) terms_across<3>(pm + 32 * ks * kLdP + 16 * wave, 64 * kLdP, kLdP, fe[ks]);
    __syncthreads();
    double qdq = 0.0;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if (kb >= a.dkb) continue;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        if (2 * ks + 1 < wave) continue;
        Terms<NI> f;
        terms_across<NI>(x + 32 * ks * kLd + 16 * kb, 64 * kLd, kLd, f);
        dk[kb] = mul_terms<3>(f, fe[ks], dk[kb]);
      }
      const int ch = 16 * kb + row4;
      if (on && ch < a.dk) {
        const f32x4 q = load4<T>(at<T>(a.q, b * a.vq.b + hk * a.vq.h + (any.n0 + n) * a.vq.n + ch));
        qdq += (double)(q[0] * dq[kb][0] + q[1] * dq[kb][1]) + (double)(q[2] * dq[kb][2] + q[3] * dq[kb][3]);
      }
      if constexpr (SHARED) {
        sum_q[kb] += dq[kb];
        sum_k[kb] += dk[kb];
      }
    }
    double both = qdq - vdv;
    both += __shfl_xor(both, 16, 64);
    both += __shfl_xor(both, 32, 64);
    double* dg64 = reinterpret_cast<double*>(pm);   // (the planes there are read)
    __syncthreads();
    if (lane < 16) {
      dg64[n] = both;
      if (on) a.dbeta[w.b * a.vdg.b + w.h * a.vdg.h + (w.n0 + n) * a.vdg.n] = dbeta;
    }
    __syncthreads();
    if (wave == 0) {
      double y = dg64[lane];
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const double z = __shfl_down(y, m, 64);
        if (lane + m < 64) y += z;
      }
      y += ((double)inner[0] + inner[1]) + ((double)inner[2] + inner[3]);
      if (lane < w.valid) a.dg[w.b * a.vdg.b + w.h * a.vdg.h + (w.n0 + lane) * a.vdg.n] = (float)y;
    }
    if constexpr (!SHARED) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const int ch = 16 * kb + row4;
        if (!on || ch >= a.dk) continue;
        store4<T>(at<T>(a.dq, b * a.vdq.b + hk * a.vdq.h + (any.n0 + n) * a.vdq.n + ch), dq[kb]);
        store4<T>(at<T>(a.dk_out, b * a.vdk.b + hk * a.vdk.h + (any.n0 + n) * a.vdk.n + ch), dk[kb]);
      }
    }
  }
  if constexpr (SHARED) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int ch = 16 * kb + row4;
      if (!on || ch >= a.dk) continue;
      store4<T>(at<T>(a.dq, b * a.vdq.b + hk * a.vdq.h + (any.n0 + n) * a.vdq.n + ch), sum_q[kb]);
      store4<T>(at<T>(a.dk_out, b * a.vdk.b + hk * a.vdk.h + (any.n0 + n) * a.vdk.n + ch), sum_k[kb]);
    }
  }
}

}  // namespace lf
