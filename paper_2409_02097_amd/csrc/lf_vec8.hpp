// Eight neighbouring channels of a token as fp32 values, whatever they are stored as: one 16-byte access of the 16-bit
// types, two of fp32.  Shared by the row-wise operators around the mixer (block boundary, rotary positions, delta rule).
#pragma once
#include "lf_common.hpp"

namespace lf {

#define LF_DEV_HOST __host__ __device__ __forceinline__

struct F32 {};   // tag: IEEE binary32 storage

template <typename T> struct Stored { static constexpr int kBytes = 2; };
template <> struct Stored<F32> { static constexpr int kBytes = 4; };

// element `i` of a tensor of T
template <typename T> LF_DEV const unsigned char* at(const void* p, long long i) {
  return static_cast<const unsigned char*>(p) + i * Stored<T>::kBytes;
}
template <typename T> LF_DEV unsigned char* at(void* p, long long i) {
  return static_cast<unsigned char*>(p) + i * Stored<T>::kBytes;
}

template <typename T> struct Raw8 { u32x4 w; };
template <> struct Raw8<F32> { u32x4 w, w2; };

template <typename T> LF_DEV Raw8<T> load8_raw(const unsigned char* p) {
  Raw8<T> r;
  r.w = *reinterpret_cast<const u32x4*>(p);
  if constexpr (Stored<T>::kBytes == 4) r.w2 = *reinterpret_cast<const u32x4*>(p + 16);
  return r;
}

template <typename T> LF_DEV Raw8<T> none8() {
  Raw8<T> r;
  r.w = u32x4{0, 0, 0, 0};
  if constexpr (Stored<T>::kBytes == 4) r.w2 = u32x4{0, 0, 0, 0};
  return r;
}

template <typename T> LF_DEV void widen8(const Raw8<T>& r, float (&x)[8]) {
  if constexpr (Stored<T>::kBytes == 4) {
    const f32x4 a = __builtin_bit_cast(f32x4, r.w), b = __builtin_bit_cast(f32x4, r.w2);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(r.w[i], x[2 * i], x[2 * i + 1]);
  }
}

template <typename T> LF_DEV void load8(const unsigned char* p, float (&x)[8]) { widen8<T>(load8_raw<T>(p), x); }

// rounded once, to nearest even
template <typename T> LF_DEV Raw8<T> narrow8(const float (&x)[8]) {
  Raw8<T> r;
  if constexpr (Stored<T>::kBytes == 4) {
    r.w = __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]});
    r.w2 = __builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]});
  } else {
    r.w = u32x4{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])};
  }
  return r;
}

template <typename T> LF_DEV void store8(unsigned char* p, const float (&x)[8]) {
  const Raw8<T> r = narrow8<T>(x);
  *reinterpret_cast<u32x4*>(p) = r.w;
  if constexpr (Stored<T>::kBytes == 4) *reinterpret_cast<u32x4*>(p + 16) = r.w2;
}

template <typename T> LF_DEV void store8_stream(unsigned char* p, const float (&x)[8]) {
  const Raw8<T> r = narrow8<T>(x);
  st_stream(reinterpret_cast<u32x4*>(p), r.w);
  if constexpr (Stored<T>::kBytes == 4) st_stream(reinterpret_cast<u32x4*>(p + 16), r.w2);
}

LF_DEV void load8_f32(const float* p, float (&x)[8]) { load8<F32>(reinterpret_cast<const unsigned char*>(p), x); }

// Sum over the LANES neighbouring lanes (16 or 64); every one of them gets it.  Without LDS: exchanges inside a row of 16 lanes
// as modifiers of the additions, rows and halves by the swapping moves (a step through the LDS crossbar takes 60 cycles or more, and
// the row-wise operators wait for four to eight of these sums per token).
template <int CTRL> LF_DEV float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// v plus the other row's (LANES = 16: rows 0 and 1, 2 and 3) or the other half's.  (The two copies are kept apart: with one value
// as both operands this compiler takes both results for the first.)
template <int LANES> LF_DEV float swap_add(float v) {
  unsigned a = __builtin_bit_cast(unsigned, v), b = a;
  asm("" : "+v"(b));
  const auto r = LANES == 16 ? __builtin_amdgcn_permlane16_swap(a, b, false, false) : __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
template <int LANES> LF_DEV float lanes_sum(float v) {
  static_assert(LANES == 16 || LANES == 64, "a row or a wave");
  v = dpp_add<0xB1>(v);    // lanes 1 apart
  v = dpp_add<0x4E>(v);    // 2 apart
  v = dpp_add<0x141>(v);   // the other half of 8
  v = dpp_add<0x140>(v);   // of 16
  if constexpr (LANES == 64) {
    v = swap_add<16>(v);
    v = swap_add<32>(v);
  }
  return v;
}

// Sum over the rows of partials [parts][C] in column c, for the first 16 threads of a workgroup of 1024, whose thread t has column t % 16:
// 64 rows at a time, in a fixed order, in fp64 (a long batch has thousands of rows).
LF_DEV double column_sum(double (&lds)[64][17], const float* partials, long long parts, int C, int c) {
  const int lane = threadIdx.x & 15, row = threadIdx.x >> 4;
  double sum = 0.0;
  for (long long p0 = row; p0 < parts; p0 += 64 * 8) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const long long p = p0 + 64 * j;
      v[j] = p < parts && c < C ? partials[p * C + c] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += (double)v[j];
  }
  lds[row][lane] = sum;
  __syncthreads();
  if (row == 0) {
#pragma unroll 8
    for (int r = 1; r < 64; ++r) sum += lds[r][lane];
  }
  return sum;
}

// tokens of row b that count: `lengths` (null: all N) clamped to [0, N]
LF_DEV long long tokens_of(const int* lengths, int b, long long N) {
  if (!lengths) return N;
  const long long n = lengths[b];
  return n < 0 ? 0 : (n > N ? N : n);
}

}  // namespace lf
