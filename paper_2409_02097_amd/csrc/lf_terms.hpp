// fp32 values as sums of bf16 terms, for products on the 16-bit matrix instruction.
//
// A value is the sum of its nearest bf16, the nearest bf16 of what is left, and so on: N terms carry 8 N bits (24: all of
// fp32; a stored bf16 is one term, a stored fp16 two, exactly).  A product of two such sums keeps the pairs of terms i, j
// with i + j < 3, every pair dropped being near 2^-24 of the product: fp32 accurate.  Each pair is one instruction at 16 times
// the rate of the fp32 one (six of them, or three where one side is a stored bf16).
#pragma once
#include "lf_vec8.hpp"

namespace lf {

template <typename T> struct TermsOf { static constexpr int kStored = 1; };
template <> struct TermsOf<F16> { static constexpr int kStored = 2; };
template <> struct TermsOf<F32> { static constexpr int kStored = 3; };

template <int N> struct Terms { u32x4 t[N]; };   // an operand of 16 x 16 x 32: 8 contraction steps of one row (or column)

// the terms of a pair of values, packed
template <int N> LF_DEV void split_pair(float a, float b, uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    w[i] = pack2<BF16>(a, b);
    if (i + 1 < N) {
      asm("" : "+v"(w[i]));
      float x, y;
      unpack2<BF16>(w[i], x, y);
      a -= x;
      b -= y;
    }
  }
}

// Four values into N planes of 16-bit words at `p` (8 bytes each, `plane` elements apart).
template <int N> LF_DEV void split4_lds(uint16_t* p, int plane, const f32x4& v) {
  uint32_t a[N], b[N];
  split_pair<N>(v[0], v[1], a);
  split_pair<N>(v[2], v[3], b);
#pragma unroll
  for (int i = 0; i < N; ++i) *reinterpret_cast<u32x2*>(p + i * plane) = u32x2{a[i], b[i]};
}

template <int N> LF_DEV void split8(const float (&x)[8], Terms<N>& out) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[N];
    split_pair<N>(x[2 * j], x[2 * j + 1], w);
#pragma unroll
    for (int i = 0; i < N; ++i) out.t[i][j] = w[i];
  }
}

// Eight stored channels as terms.
template <typename T> LF_DEV void terms_of(const Raw8<T>& r, Terms<TermsOf<T>::kStored>& out) {
  if constexpr (TermsOf<T>::kStored == 1) {
    out.t[0] = r.w;
  } else {
    float x[8];
    widen8<T>(r, x);
    split8(x, out);
  }
}

// Operands from planes in LDS: 8 contraction steps that are neighbours in memory (`p` at the lane's row and first step), ...
template <int N> LF_DEV void terms_near(const uint16_t* p, int plane, Terms<N>& out) {
#pragma unroll
  for (int i = 0; i < N; ++i) out.t[i] = *reinterpret_cast<const u32x4*>(p + i * plane);
}
// ... or rows of them: `p` at the first step and column of a block of 32 steps by 16 columns, `ld` elements a step.
template <int N> LF_DEV void terms_across(const uint16_t* p, int plane, int ld, Terms<N>& out) {
  const int l = threadIdx.x & 63, g = l >> 4, i = l & 15;
  const uint16_t* at = p + (8 * g + (i >> 2)) * ld + 4 * (i & 3);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const u32x2 a = lds_read_tr16(at + k * plane), b = lds_read_tr16(at + k * plane + 4 * ld);
    out.t[k] = u32x4{a[0], a[1], b[0], b[1]};
  }
}

template <int NA, int NB> LF_DEV f32x4 mul_terms(const Terms<NA>& a, const Terms<NB>& b, f32x4 c) {
#pragma unroll
  for (int s = 2; s >= 0; --s)      // the small products first
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int j = s - i;
      if (j >= 0 && j < NB) c = mfma_16x16x32<BF16>(a.t[i], b.t[j], c);
    }
  return c;
}

// A chunk's rows of one head, 8 channels a vector: requested first, put down as term planes in LDS later ([64][ld] each, zeros
// behind the last token and channel; `steps` blocks of 32 channels).  Requests of several tensors are in flight together.
template <typename T, int STEPS, int THREADS> struct Rows {
  static constexpr int kVecs = (64 * 4 * STEPS + THREADS - 1) / THREADS;
  Raw8<T> raw[kVecs];
  LF_DEV void request(const void* x, long long base, long long row, int valid, int d) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int e = threadIdx.x + THREADS * i, t = e / (4 * STEPS), c = (e - t * 4 * STEPS) * 8;
      raw[i].w = u32x4{0, 0, 0, 0};
      if constexpr (Stored<T>::kBytes == 4) raw[i].w2 = u32x4{0, 0, 0, 0};
      if (t < valid && c < d) raw[i] = load8_raw<T>(at<T>(x, base + t * row + c));
    }
  }
  LF_DEV void put(uint16_t* to, int ld) const {
    constexpr int N = TermsOf<T>::kStored;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int e = threadIdx.x + THREADS * i, t = e / (4 * STEPS), c = (e - t * 4 * STEPS) * 8;
      Terms<N> y;
      terms_of<T>(raw[i], y);
      if (e < 64 * 4 * STEPS) {
#pragma unroll
        for (int k = 0; k < N; ++k) *reinterpret_cast<u32x4*>(to + k * 64 * ld + t * ld + c) = y.t[k];
      }
    }
  }
};
// The same in one go for a number of steps known at run time, four vectors in flight.
template <typename T, int THREADS>
LF_DEV void stage_terms(uint16_t* to, int ld, const void* x, long long base, long long row, int valid, int d, int steps) {
  constexpr int N = TermsOf<T>::kStored;
  const int vecs = steps * 4;
  for (int i0 = threadIdx.x; i0 < 64 * vecs; i0 += 4 * THREADS) {
    Raw8<T> raw[4];
    int t[4], c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = i0 + THREADS * i;
      t[i] = (unsigned)e / (unsigned)vecs;
      c[i] = (e - t[i] * vecs) * 8;
      raw[i].w = u32x4{0, 0, 0, 0};
      if constexpr (Stored<T>::kBytes == 4) raw[i].w2 = u32x4{0, 0, 0, 0};
      if (t[i] < valid && c[i] < d) raw[i] = load8_raw<T>(at<T>(x, base + t[i] * row + c[i]));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (t[i] >= 64) continue;
      Terms<N> y;
      terms_of<T>(raw[i], y);
#pragma unroll
      for (int k = 0; k < N; ++k) *reinterpret_cast<u32x4*>(to + k * 64 * ld + t[i] * ld + c[i]) = y.t[k];
    }
  }
}

}  // namespace lf
