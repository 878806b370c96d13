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
// and the values by its inverse.  Its sums cancel: dg is off by 1e-6 of its largest value where a recurrence in fp32 is off by 4e-7,
// whatever its products are formed in.
//
// Only dU and dS0 depend on the chunk behind: P^T dO and (e^gamma Q)^T dO are formed for all
// chunks at once (delta_back_prepare), a scan runs from the last chunk to the first (delta_back_scan), and the rest follows
// for all chunks at once (delta_gradients), where the value heads that share a query and key head are summed in their order.
// The backward pass has records of its own, two more than chunks per head:
//     du   P^T dO, then dU, as u
//     kn   K as operand: [4 token blocks][d_k / 32][terms][64][8], in the record of the first value head that has the key head
//     ds   as s: (e^gamma Q)^T dO of chunk c in record c, dS1 two records on, which every wave of the scan has behind it by then
#pragma once
#include "lf_delta.hpp"

namespace lf {

// ---- what does not depend on the chunk behind ---------------------------------------------------------------------------------
// 96 heads of 40 channels, 4096 tokens, bf16: 65 us for 230 MB (3.5 TB/s).
template <typename T> inline int delta_back_prepare_lds(int dks, int dvs) {
  constexpr int NI = TermsOf<T>::kStored;
  const int keys = NI * plane_bytes(64, dks), out = NI * plane_bytes(64, value_steps<T>(dvs)), scores = 3 * 64 * kLdP * 2;
  return 64 * 8 + 64 * 4 + (keys > out ? keys : out) + (keys > scores ? keys : scores);
}

template <typename T, int KS> __global__ __launch_bounds__(256) void delta_back_prepare(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NI = TermsOf<T>::kStored, ld = 32 * KS + 8, plane = 64 * ld, kOwn = (2 * KS + 3) / 4;
  const DeltaAt w(a, blockIdx.y, blockIdx.x);
  if (w.valid == 0) return;
  const int dvs = (a.dvb + 1) / 2, group = value_steps<T>(dvs), ldo = plane_ld(group);
  double* gamma = reinterpret_cast<double*>(smem);
  float* since = reinterpret_cast<float*>(gamma + 64);
  uint16_t* q = reinterpret_cast<uint16_t*>(since + 64);
  uint16_t* o = q;                      // where the queries were
  uint16_t* k = q + NI * (ld > ldo ? plane : 64 * ldo);
  uint16_t* pp = k;                     // where the keys were
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15;
  const int row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  unsigned char *rec = a.rec(w.bh, blockIdx.x), *rec_b = a.rec_b(w.bh, blockIdx.x);
  Rows<T, KS, 256> queries, keys;
  queries.request(a.q, w.b * a.vq.b + w.hk * a.vq.h + w.n0 * a.vq.n, a.vq.n, w.valid, a.dk);
  keys.request(a.k, w.b * a.vk.b + w.hk * a.vk.h + w.n0 * a.vk.n, a.vk.n, w.valid, a.dk);
  if (wave == 0) {
    gamma[lane] = part<double>(rec, a.at_decay + kDecayRows * 4)[lane];
    since[lane] = part<float>(rec, a.at_decay)[kDecaySince + lane];
  }
  queries.put(q, ld);
  keys.put(k, ld);
  __syncthreads();
  if (w.h % (a.H / a.Hk) == 0) {
    uint16_t* kn = part<uint16_t>(rec_b, a.at_kn) + wave * KS * NI * kFrag;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      Terms<NI> f;
      terms_near<NI>(k + (16 * wave + col) * ld + 32 * ks + g8, plane, f);
      store_frag<NI>(kn + ks * NI * kFrag, f);
    }
  }
  // P transposed, [j][i]: four neighbouring rows i of column j at a time; rows i of tile `it`, columns of this wave's
  f32x4 scores[4];
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    f32x4 acc = {0, 0, 0, 0};
    if (it >= wave) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Terms<NI> fq, fk;
        terms_near<NI>(q + (16 * it + col) * ld + 32 * ks + g8, plane, fq);
        terms_near<NI>(k + (16 * wave + col) * ld + 32 * ks + g8, plane, fk);
        acc = mul_terms(fq, fk, acc);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * it + row4 + r, j = 16 * wave + col;
        acc[r] = j <= i ? acc[r] * decay_between(gamma, i, j) : 0.0f;
      }
    }
    scores[it] = acc;
  }
  // (e^gamma Q)^T as operands of this wave's channel blocks, before the queries make room: scaled, then split again
  Terms<3> fq[kOwn][2];   // channel blocks wave, wave + 4, ...
#pragma unroll
  for (int t = 0; t < kOwn; ++t)
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
  __syncthreads();   // queries and keys are read
#pragma unroll
  for (int it = 0; it < 4; ++it) split4_lds<3>(pp + (16 * wave + col) * kLdP + 16 * it + row4, 64 * kLdP, scores[it]);
  auto put_gradients = [&](int step) {
    stage_terms<T, 256>(o, ldo, a.dout, w.b * a.vdo.b + w.h * a.vdo.h + w.n0 * a.vdo.n + 32 * step, a.vdo.n, w.valid, a.dv - 32 * step, group);
  };
  put_gradients(0);
  __syncthreads();
  Terms<3> fp[2];      // P^T's rows j of this wave
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) terms_near<3>(pp + (16 * wave + col) * kLdP + 32 * ks + g8, 64 * kLdP, fp[ks]);
  for (int vb = 0; vb < a.dvb; ++vb) {
    const int at_vb = vb % (2 * group);
    if (vb > 0 && at_vb == 0) {
      __syncthreads();
      put_gradients(vb / 2);
      __syncthreads();
    }
    Terms<NI> fo[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) terms_across<NI>(o + 32 * ks * ldo + 16 * at_vb, 64 * ldo, ldo, fo[ks]);
    f32x4 acc = {0, 0, 0, 0};   // rows: value channels, columns: tokens j
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) acc = mul_terms(fo[ks], fp[ks], acc);
    *reinterpret_cast<f32x4*>(part<float>(rec_b, 0) + ((vb * 4 + wave) * 64 + lane) * 4) = acc * a.scale;
#pragma unroll
    for (int t = 0; t < kOwn; ++t) {
      if (wave + 4 * t >= a.dkb) continue;
      f32x4 z = {0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) z = mul_terms(fq[t][ks], fo[ks], z);
      *reinterpret_cast<f32x4*>(part<float>(rec_b, a.at_ds) + (vb * a.dkb + wave + 4 * t) * 256 + lane * 4) = z;
    }
  }
}

// ---- the scan backwards ----------------------------------------------------------------------------------------------------------
// A slice of 16 value channels per workgroup, a chunk's chain as in delta_scan.  96 heads of 40 channels, 4096 tokens, bf16: 128 us for
// 440 MB (3.4 TB/s), 2 us a chunk.
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
  int slice, bh;
  slice_of_head(blockIdx.x, a.dvb, a.heads, slice, bh);
  const int ch = slice * 16 + col;
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
  const int key_head = bh - first.h + first.hk * (a.H / a.Hk);
  const int u_at = (slice * 4 + wave) * 256 + lane * 4;
  int zero = 0;   // (as in delta_scan)
  asm volatile("" : "+v"(zero));
  const int last = chunks > 0 ? chunks - 1 : 0;
  const unsigned char *ahead = a.rec(bh, last), *ahead_b = a.rec_b(bh, last), *ahead_key = a.rec_b(key_head, last);
  int requested = last;
  auto request = [&](BackScanIn<NI, KS>& n) {
    const uint16_t* kn = reinterpret_cast<const uint16_t*>(ahead_key + a.at_kn) + wave * KS * NI * kFrag;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) load_frag<NI>(kn + ks * NI * kFrag, n.kn[ks]);
    const uint16_t* wt = reinterpret_cast<const uint16_t*>(ahead + a.at_wt);
    const float* z = reinterpret_cast<const float*>(ahead_b + a.at_ds) + slice * a.dkb * 256;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      n.z[t] = *reinterpret_cast<const f32x4*>(z + blk[t] * 256 + lane * 4);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) load_frag<3>(wt + (blk[t] * 2 + ks) * 3 * kFrag, n.wt[t][ks]);
    }
    n.du = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(ahead_b) + u_at);
    const float* decay = reinterpret_cast<const float*>(ahead + a.at_decay);
    n.left = decay[kDecayLeft + 16 * wave + col];
    n.whole = decay[kDecaySince + 63 + zero];
    if (requested-- > 0) {   // (the first one again before the beginning)
      ahead -= a.size;
      ahead_b -= a.size_b;
      ahead_key -= a.size_b;
    }
  };
  unsigned char* here = a.rec_b(bh, last);
  auto chunk = [&](BackScanIn<NI, KS>& in, BackScanIn<NI, KS>& next) {
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) split4_lds<3>(sp + col * kLd + 16 * blk[t] + row4, kPlane, s[t]);
    lds_barrier();
    f32x4 acc = {0, 0, 0, 0}, acc2 = {0, 0, 0, 0};
    Terms<3> first_fs;
    terms_near<3>(sp + col * kLd + g8, kPlane, first_fs);
    __builtin_amdgcn_sched_barrier(0);
    request(next);
    float* to = reinterpret_cast<float*>(here + 2 * (size_t)a.size_b + a.at_ds) + slice * a.dkb * 256;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) *reinterpret_cast<f32x4*>(to + blk[t] * 256 + lane * 4) = s[t];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      Terms<3> fs;
      if (ks == 0) fs = first_fs;
      else terms_near<3>(sp + col * kLd + 32 * ks + g8, kPlane, fs);
      if (ks & 1) acc2 = mul_terms(fs, in.kn[ks], acc2);
      else acc = mul_terms(fs, in.kn[ks], acc);
    }
    const f32x4 u = in.du + (acc + acc2) * in.left;
    split4_lds<3>(up + (16 * wave + col) * kLdU + row4, 64 * kLdU, -u);
    lds_barrier();
    Terms<3> fu[2];
    terms_across<3>(up, 64 * kLdU, kLdU, fu[0]);
    terms_across<3>(up + 32 * kLdU, 64 * kLdU, kLdU, fu[1]);
    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(here) + u_at) = u;
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) {
      f32x4 more = in.z[t];
      s[t] *= in.whole;
      s[t] = mul_terms(in.wt[t][0], fu[0], s[t]);
      more = mul_terms(in.wt[t][1], fu[1], more);
      s[t] += more;
    }
    here -= a.size_b;
  };
  if (chunks > 0) {
    BackScanIn<NI, KS> x, y;
    int i = chunks - 1;
    request(x);
    for (; i > 0; i -= 2) {
      chunk(x, y);
      chunk(y, x);
    }
    if (i == 0) chunk(x, y);
  }
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
// Formed transposed (rows: channels, columns: tokens).  Eight waves: wave w takes tokens 16 (w % 4) .. + 15 and one half of the
// channels.  32 value channels at a time pass through LDS: dU (then dV in its place), dO, U as [token][channel], S0 and dS1 as
// [channel][key channel].  Bound: the chain of small products between its barriers, vector and LDS units a third busy each; 282 us for
// 96 heads of 40 channels, 4096 tokens, bf16.  What comes next is requested a round ahead, keys and queries behind the last one.
constexpr int kLdV = 40;

template <typename T> inline int delta_gradients_lds(int dks) {
  constexpr int NI = TermsOf<T>::kStored;
  const int first = (3 + NI + 3) * 64 * kLdV * 2 + 2 * 3 * plane_bytes(32, dks);
  const int second = 2 * 3 * 64 * kLdP * 2 + NI * plane_bytes(64, dks);
  return (first > second ? first : second) + 64 * 8 + kDecayRows * 4 + 8 * 4 + 2 * 64 * 8 + 2 * 64 * 4;
}

// sum over the four lanes of a wave that share l % 16
LF_DEV float groups_sum(float v) { return swap_add<32>(swap_add<16>(v)); }

// The same value, as far as the compiler can see another: what follows from it is computed where it is used and not kept in
// registers through a loop.
template <typename X> LF_DEV X again(X x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Two workgroups per CU, which leaves 128 registers a lane, where the planes are small enough and what is held fits: a workgroup is a
// chain of barriers.  4096 tokens, us with two : one: 12 x 8 heads of 40 channels, bf16 281 : 344; 4 x 16 heads of 64, fp16 265 : 274, of
// 32, fp32 120 : 180, of 32 with 4 key heads, bf16 111 : 140.  Not with the sums over value heads beside keys of more than 32 (2 x 16
// heads of 64, 4 key heads, bf16 148 : 122) or beside fp32 rows (4 x 16 heads of 32, 4 key heads, the whole call 265 : 260), nor for more
// than 64 (4 x 16 heads of 96, bf16 416 : 362; fp32 of 64, the whole call 591 : 482): the rest is in scratch memory.
template <typename T, int KS, bool SHARED> constexpr int gradients_waves() {   // per SIMD
  constexpr bool wide = TermsOf<T>::kStored == 3;
  return (KS == 1 && !(SHARED && wide)) || (KS == 2 && !SHARED && !wide) ? 4 : 2;
}

template <typename T, int KS, bool SHARED> __global__ __launch_bounds__(512, (gradients_waves<T, KS, SHARED>())) void delta_gradients(DeltaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NI = TermsOf<T>::kStored, kLd = 32 * KS + 8, kVPlane = 64 * kLdV, kSPlane = 32 * kLd, kPPlane = 64 * kLdP;
  constexpr int kOwn = (2 * KS + 3) / 4;
  const int b = (unsigned)blockIdx.y / (unsigned)a.Hk, hk = blockIdx.y - b * a.Hk, group = SHARED ? a.H / a.Hk : 1;
  double* gamma = reinterpret_cast<double*>(smem);
  double* dg64 = gamma + 64;                               // [2][64]
  float* decay = reinterpret_cast<float*>(dg64 + 128);
  float* db32 = decay + kDecayRows;                        // [2][64]
  float* inner = db32 + 128;                               // [8]
  uint16_t* pv = reinterpret_cast<uint16_t*>(inner + 8);   // dU, then dV
  uint16_t* pu = pv + 3 * kVPlane;
  uint16_t* po = pu + 3 * kVPlane;
  uint16_t* ps = po + NI * kVPlane;
  uint16_t* pd = ps + 3 * kSPlane;
  uint16_t* pm = pv;                                       // later: dO U^T * D, M, and the keys, then the queries
  uint16_t* pn = pm + 3 * kPPlane;
  uint16_t* x = pn + 3 * kPPlane;
  const int tid = threadIdx.x, wave8 = __builtin_amdgcn_readfirstlane(tid >> 6), wave = wave8 & 3, half = wave8 >> 2;
  const int lane = tid & 63, col = lane & 15, row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8;
  const int n = 16 * wave + col;                           // this lane's token
  const DeltaAt any(a, b * a.H + hk * group, blockIdx.x);
  if (any.valid == 0) return;
  const bool on = n < any.valid;
  Rows<T, KS, 512> keys, queries;
  auto channels_of = [&](const uint16_t* rows, int ch) {   // four channels of this lane's token, from their terms
    f32x4 y = {0, 0, 0, 0};
#pragma unroll
    for (int k = NI - 1; k >= 0; --k) {
      const u32x2 e = *reinterpret_cast<const u32x2*>(rows + k * 64 * kLd + n * kLd + ch);
      float e0, e1, e2, e3;
      unpack2<BF16>(e[0], e0, e1);
      unpack2<BF16>(e[1], e2, e3);
      y += f32x4{e0, e1, e2, e3};
    }
    return y;
  };
  f32x4 sum_q[SHARED ? KS : 1], sum_k[SHARED ? KS : 1];
  if constexpr (SHARED) {
#pragma unroll
    for (int i = 0; i < KS; ++i) sum_q[i] = sum_k[i] = f32x4{0, 0, 0, 0};
  }
  for (int member = 0; member < group; ++member) {
    const DeltaAt w(a, b * a.H + hk * group + member, blockIdx.x);
    unsigned char *rec = a.rec(w.bh, blockIdx.x), *rec_b = a.rec_b(w.bh, blockIdx.x);
    const float* ds = part<float>(a.rec_b(w.bh, blockIdx.x + 2), a.at_ds);
    // requested in the order in which they are waited for: the decays, ...
    double gamma_in = 0.0;
    float decay_in = 0.0f;
    if (tid < kDecayRows) decay_in = part<float>(rec, a.at_decay)[tid];
    else if (wave8 == 4) gamma_in = part<double>(rec, a.at_decay + kDecayRows * 4)[lane];
    // ... 16 value channels of this wave's tokens, and row blocks wave, wave + 4, ... of S0 and dS1: block vb + half
    f32x4 du, u, s0[kOwn], d1[kOwn];
    Raw4<T> o, v;
    auto request = [&](int vb) {
      const f32x4 none = {0, 0, 0, 0};
      const int lane = again(tid & 63), row4 = (lane >> 4) * 4, n = 16 * wave + (lane & 15);
      const int ch = 16 * vb + row4;
      du = u = none;
      o = v = Raw4<T>{};
#pragma unroll
      for (int t = 0; t < kOwn; ++t) s0[t] = d1[t] = none;
      if (vb >= a.dvb) return;
      const int at4 = ((vb * 4 + wave) * 64 + lane) * 4;
      du = *reinterpret_cast<const f32x4*>(part<float>(rec_b, 0) + at4);
      u = *reinterpret_cast<const f32x4*>(part<float>(rec, a.at_u) + at4);
      if (on && ch < a.dv) {
        o = load4_raw<T>(at<T>(a.dout, w.b * a.vdo.b + w.h * a.vdo.h + (w.n0 + n) * a.vdo.n + ch));
        v = load4_raw<T>(at<T>(a.v, w.b * a.vv.b + w.h * a.vv.h + (w.n0 + n) * a.vv.n + ch));
      }
#pragma unroll
      for (int t = 0; t < kOwn; ++t) {
        const int kb = wave + 4 * t;
        if (kb >= a.dkb) continue;
        s0[t] = *reinterpret_cast<const f32x4*>(part<float>(rec, a.at_s) + (vb * a.dkb + kb) * 256 + lane * 4);
        d1[t] = *reinterpret_cast<const f32x4*>(ds + (vb * a.dkb + kb) * 256 + lane * 4);
      }
    };
    request(half);
    __syncthreads();   // (the member before has been read)
    if (tid < kDecayRows) decay[tid] = decay_in;
    else if (wave8 == 4) gamma[lane] = gamma_in;
    f32x4 dq[KS], dk[KS], dw[KS], mx[4];
#pragma unroll
    for (int i = 0; i < KS; ++i) dq[i] = dk[i] = dw[i] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) mx[i] = f32x4{0, 0, 0, 0};
    float dbeta = 0.0f, ss = 0.0f;
    double vdv = 0.0;
    __syncthreads();
    const float beta = decay[kDecayBeta + n], per_beta = 1.0f / beta;
    const bool none = beta == kDeltaTinyBeta;
    for (int vb = 0; vb < a.dvb; vb += 2) {
      const int lane = again(tid & 63), col = lane & 15, row4 = (lane >> 4) * 4, g8 = (lane >> 4) * 8, n = 16 * wave + col;
      const bool on = n < any.valid;
      const int ch = 16 * (vb + half) + row4;
      split4_lds<3>(pv + n * kLdV + 16 * half + row4, kVPlane, du);
      split4_lds<3>(pu + n * kLdV + 16 * half + row4, kVPlane, none ? f32x4{0, 0, 0, 0} : u);
      split4_lds<NI>(po + n * kLdV + 16 * half + row4, kVPlane, widen4<T>(o));
#pragma unroll
      for (int t = 0; t < kOwn; ++t) {
        const int kb = wave + 4 * t;
        if (kb >= 2 * KS) continue;   // (zeros behind d_k too)
        split4_lds<3>(ps + (16 * half + col) * kLd + 16 * kb + row4, kSPlane, s0[t]);
        split4_lds<3>(pd + (16 * half + col) * kLd + 16 * kb + row4, kSPlane, d1[t]);
        ss += (d1[t][0] * s0[t][0] + d1[t][1] * s0[t][1]) + (d1[t][2] * s0[t][2] + d1[t][3] * s0[t][3]);
      }
      // (T beta)^T's rows of this wave, nothing before them
      auto tt_at = [&](int ks) { return load8_raw<F32>(rec + a.at_tt + ((wave < 2 ? 2 * wave + ks : 2 + wave) * 64 + lane) * 32); };
      Raw8<F32> tt[2];
      tt[0] = tt_at(0);   // (waves without one: the other again)
      tt[1] = tt_at(1);
      const f32x4 u_now = u;
      const Raw4<T> v_raw = v;
      lds_barrier();
      f32x4 dv = {0, 0, 0, 0};
#pragma unroll
      for (int ks = 1; ks >= 0; --ks) {
        if (ks == 0 && wave > 1) continue;
        Terms<3> f, ft;
        float y[8];
        widen8<F32>(tt[ks], y);
        split8(y, ft);
        terms_across<3>(pv + 32 * ks * kLdV + 16 * half, kVPlane, kLdV, f);
        dv = mul_terms(f, ft, dv);
        __builtin_amdgcn_sched_barrier(0);
      }
      const float by = again(per_beta);
      const f32x4 per = (dv * by) * (u_now * by);
      dbeta += (per[0] + per[1]) + (per[2] + per[3]);
      if (none) dv = f32x4{0, 0, 0, 0};
      if (on && ch < a.dv) {
        const f32x4 v_now = widen4<T>(v_raw);
        vdv += (double)(v_now[0] * dv[0] + v_now[1] * dv[1]) + (double)(v_now[2] * dv[2] + v_now[3] * dv[3]);
        store4<T>(at<T>(a.dv_out, w.b * a.vdv.b + w.h * a.vdv.h + (w.n0 + n) * a.vdv.n + ch), dv);
      }
      lds_barrier();   // dU is read
      split4_lds<3>(pv + n * kLdV + 16 * half + row4, kVPlane, dv);
      if (vb + 2 < a.dvb) request(vb + 2 + half);
      lds_barrier();
      Terms<3> fv, fu;
      Terms<NI> fo;
      terms_near<3>(pv + n * kLdV + g8, kVPlane, fv);
      terms_near<3>(pu + n * kLdV + g8, kVPlane, fu);
      terms_near<NI>(po + n * kLdV + g8, kVPlane, fo);
#pragma unroll
      for (int jt = 0; jt < 4; ++jt) {
        if (jt > wave) continue;
        __builtin_amdgcn_sched_barrier(0);   // (one operand at a time: two workgroups per CU have 128 registers a lane)
        Terms<3> fj;
        terms_near<3>(pu + (16 * jt + col) * kLdV + g8, kVPlane, fj);
        if (half == 0) mx[jt] = mul_terms(fj, fo, mx[jt]);
        else mx[jt] = mul_terms(fj, fv, mx[jt]);
      }
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const int kb = 2 * i + half;
        __builtin_amdgcn_sched_barrier(0);
        Terms<3> f;
        terms_across<3>(ps + 16 * kb, kSPlane, kLd, f);
        dq[i] = mul_terms(f, fo, dq[i]);
        dk[i] = mul_terms(f, fv, dk[i]);
        terms_across<3>(pd + 16 * kb, kSPlane, kLd, f);
        dw[i] = mul_terms(f, fu, dw[i]);
      }
      lds_barrier();   // the planes are read
    }
    keys.request(a.k, b * a.vk.b + hk * a.vk.h + any.n0 * a.vk.n, a.vk.n, any.valid, a.dk);
    queries.request(a.q, b * a.vq.b + hk * a.vq.h + any.n0 * a.vq.n, a.vq.n, any.valid, a.dk);
    const float since = decay[kDecaySince + n], write = decay[kDecayWrite + n];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      dq[i] *= since * a.scale;
      dw[i] *= write;
      dk[i] = dw[i] - dk[i] * since;
    }
    // half 0: scale dO U^T * D;  half 1: M
    uint16_t* mine = half ? pn : pm;
    const float factor = half ? -1.0f : a.scale;
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      __builtin_amdgcn_sched_barrier(0);
      f32x4 e = mx[jt];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 16 * jt + row4 + r;
        e[r] = j + half <= n ? e[r] * factor * decay_between(gamma, n, j) : 0.0f;
      }
      split4_lds<3>(mine + n * kLdP + 16 * jt + row4, kPPlane, e);
    }
    keys.put(x, kLd);
    dbeta = groups_sum(dbeta);
    if (lane < 16) db32[half * 64 + n] = dbeta;
    lds_barrier();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      __builtin_amdgcn_sched_barrier(0);
      Terms<3> fe, fm, em;
      terms_near<3>(pm + n * kLdP + 32 * ks + g8, kPPlane, fe);
      terms_near<3>(pn + n * kLdP + 32 * ks + g8, kPPlane, fm);
      terms_across<3>(pn + 32 * ks * kLdP + 16 * wave, kPPlane, kLdP, em);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        Terms<NI> f;
        terms_across<NI>(x + 32 * ks * kLd + 16 * (2 * i + half), 64 * kLd, kLd, f);
        if (2 * ks <= wave) {
          dq[i] = mul_terms(f, fe, dq[i]);
          dk[i] = mul_terms(f, fm, dk[i]);
        }
        if (2 * ks + 1 >= wave) dk[i] = mul_terms(f, em, dk[i]);
      }
    }
    // <dS1, S1> = e^gamma_63 <dS1, S0> + sum of k.(e^(gamma_63 - gamma) dS1 u) over the tokens
    ss *= decay[kDecaySince + 63];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const f32x4 k = channels_of(x, 16 * (2 * i + half) + row4);
      ss += (k[0] * dw[i][0] + k[1] * dw[i][1]) + (k[2] * dw[i][2] + k[3] * dw[i][3]);
    }
    ss = lanes_sum<64>(ss);
    if (lane == 0) inner[wave8] = ss;
    lds_barrier();
    queries.put(x, kLd);
    lds_barrier();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if (2 * ks + 1 < wave) continue;
      __builtin_amdgcn_sched_barrier(0);
      Terms<3> fe;
      terms_across<3>(pm + 32 * ks * kLdP + 16 * wave, kPPlane, kLdP, fe);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        Terms<NI> f;
        terms_across<NI>(x + 32 * ks * kLd + 16 * (2 * i + half), 64 * kLd, kLd, f);
        dk[i] = mul_terms(f, fe, dk[i]);
      }
    }
    double both = -vdv;   // q.dq - v.dv, the queries from their planes
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int ch = 16 * (2 * i + half) + row4;
      const f32x4 q = channels_of(x, ch);
      both += (double)(q[0] * dq[i][0] + q[1] * dq[i][1]) + (double)(q[2] * dq[i][2] + q[3] * dq[i][3]);
      if constexpr (SHARED) {
        sum_q[i] += dq[i];
        sum_k[i] += dk[i];
      } else if (on && ch < a.dk) {
        store4<T>(at<T>(a.dq, b * a.vdq.b + hk * a.vdq.h + (any.n0 + n) * a.vdq.n + ch), dq[i]);
        store4<T>(at<T>(a.dk_out, b * a.vdk.b + hk * a.vdk.h + (any.n0 + n) * a.vdk.n + ch), dk[i]);
      }
    }
    both += __shfl_xor(both, 16, 64);
    both += __shfl_xor(both, 32, 64);
    if (lane < 16) dg64[half * 64 + n] = both;
    __syncthreads();
    if (wave8 == 0) {
      double y = dg64[lane] + dg64[64 + lane];
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const double z = __shfl_down(y, m, 64);
        if (lane + m < 64) y += z;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) y += (double)inner[i];
      if (lane < w.valid) {
        const long long to = w.b * a.vdg.b + w.h * a.vdg.h + (w.n0 + lane) * a.vdg.n;
        a.dg[to] = (float)y;
        a.dbeta[to] = db32[lane] + db32[64 + lane];
      }
    }
  }
  if constexpr (SHARED) {
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int ch = 16 * (2 * i + half) + row4;
      if (!on || ch >= a.dk) continue;
      store4<T>(at<T>(a.dq, b * a.vdq.b + hk * a.vdq.h + (any.n0 + n) * a.vdq.n + ch), sum_q[i]);
      store4<T>(at<T>(a.dk_out, b * a.vdk.b + hk * a.vdk.h + (any.n0 + n) * a.vdk.n + ch), sum_k[i]);
    }
  }
}

}  // namespace lf
