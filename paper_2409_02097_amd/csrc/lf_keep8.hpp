// Activations kept in 8 bits: every block of 32 channels of a token has an exponent, the least e with 127 * 2^e not below the
// block's largest magnitude, and every value is the integer nearest to x / 2^e (ties to even), -127 .. 127.  The exponent's byte is
// e + 127, e at least -126; 255 marks a block that holds an infinity or a NaN, which comes back as NaN throughout.  The scale being
// a power of two, both ways are exact but for that one rounding: off by at most 2^e / 2, i.e. by at most 1 / 127 of the block's largest
// magnitude, or 2^-127 where that is more.  Bound: HBM (81120 x 2048 bf16, 504 MB each: keep8 92 us, unkeep8 89 us, 5.5 and 5.7 TB/s).
#pragma once
#include "lf_vec8.hpp"

namespace lf {

constexpr int kKeepBlock = 32;

struct KeepArgs {
  const void* x;              // values (keep), or codes (back)
  void* codes;                // codes (keep), or values (back)
  unsigned char* exps;
  long long xb, xt, cb, ct, eb, et;   // strides {batch, token} of x, codes, exps
  const int* lengths;
  long long N;
  int C, rows, lanes;         // tokens of a workgroup; lanes of a token, a multiple of four
};

// e + 127 of a block whose largest magnitude is `most` (its bits as an integer keep the order of magnitudes, infinities and NaN last)
LF_DEV int keep_exponent(uint32_t most) {
  if (most >= 0x7f800000u) return 255;
  const int power = (int)(most >> 23), fraction = (int)(most & 0x7fffffu);   // most = (1 + fraction / 2^23) 2^(power - 127)
  const int e = power - 6 + (fraction > 0x7e0000 ? 1 : 0);                   // 127 = (1 + 0x7e0000 / 2^23) 2^6
  return e < 1 ? 1 : e;
}

template <typename T> struct Largest { static constexpr float value = 3.40282347e38f; };
template <> struct Largest<F16> { static constexpr float value = 65504.0f; };
template <> struct Largest<BF16> { static constexpr float value = 3.38953139e38f; };

// Eight codes as values of T, exact (the one multiple of 2^e that may lie above T's largest value, 64 * 2^e, is that value).  A code is
// read as the unsigned byte code + 128: (byte - 128) 2^e in one exact multiply-add.
template <typename T> LF_DEV void keep_values(u32x2 codes, int e, float (&x)[8]) {
  constexpr float most = Largest<T>::value;
  constexpr int kTop = (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 5;   // the exponent byte of 2^e where 64 * 2^e is above `most`
  constexpr int kFar = kTop < 247 ? kTop : 247;                               // (or 128 * 2^e above fp32's)
  const float scale = e == 255 ? __builtin_nanf("") : __builtin_bit_cast(float, (uint32_t)e << 23), off = -128.0f * scale;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t w = codes[j >> 2] ^ 0x80808080u;
    x[j] = __builtin_fmaf((float)(w >> (8 * (j & 3)) & 255u), scale, off);
  }
  if (e >= kFar) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = (float)(int8_t)(codes[j >> 2] >> (8 * (j & 3))) * scale;
      x[j] = v > most ? most : (v < -most ? -most : v);   // (a NaN stays one)
    }
  }
}

// The largest of four neighbouring lanes' values.
LF_DEV uint32_t quad_max(uint32_t v) {
  uint32_t w = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);
  v = v > w ? v : w;
  w = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);
  return v > w ? v : w;
}

// `lanes` lanes of 8 channels a token, as many tokens at a time as that leaves, four times as many under way; four lanes share a block.
constexpr int kKeepAhead = 4;

template <typename T> __global__ __launch_bounds__(256) void keep8(KeepArgs a) {
  const int row = threadIdx.x / a.lanes, lane = threadIdx.x - row * a.lanes, together = 256 / a.lanes;
  const int b = blockIdx.z, c = (blockIdx.x * a.lanes + lane) * 8;
  const long long end = tokens_of(a.lengths, b, a.N), first = (long long)blockIdx.y * a.rows;
  const long long stop = first + a.rows < end ? first + a.rows : end;
  if (row >= together) return;
  const bool on = c < a.C;
  for (long long n0 = first + row; n0 < stop; n0 += together * kKeepAhead) {   // (four neighbouring lanes together)
    Raw8<T> raw[kKeepAhead];
#pragma unroll
    for (int q = 0; q < kKeepAhead; ++q) {
      raw[q] = none8<T>();
      if (on && n0 + together * q < stop) raw[q] = load8_raw<T>(at<T>(a.x, b * a.xb + (n0 + together * q) * a.xt + c));
    }
#pragma unroll
    for (int q = 0; q < kKeepAhead; ++q) {
      const long long n = n0 + together * q;
      float x[8];
      widen8<T>(raw[q], x);
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t m = __builtin_bit_cast(uint32_t, x[j]) & 0x7fffffffu;
        most = most > m ? most : m;
      }
      const int e = keep_exponent(quad_max(most));
      if (!on || n >= stop) continue;
      u32x2 codes = {0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int v = e == 255 ? 0 : (int)__builtin_rintf(__builtin_amdgcn_ldexpf(x[j], 127 - e));
        codes[j >> 2] |= (uint32_t)(v & 255) << (8 * (j & 3));
      }
      *reinterpret_cast<u32x2*>(static_cast<unsigned char*>(a.codes) + b * a.cb + n * a.ct + c) = codes;
      if ((lane & 3) == 0) a.exps[b * a.eb + n * a.et + c / kKeepBlock] = (unsigned char)e;
    }
  }
}

template <typename T> __global__ __launch_bounds__(256) void unkeep8(KeepArgs a) {
  const int row = threadIdx.x / a.lanes, lane = threadIdx.x - row * a.lanes, together = 256 / a.lanes;
  const int b = blockIdx.z, c = (blockIdx.x * a.lanes + lane) * 8;
  const long long end = tokens_of(a.lengths, b, a.N), first = (long long)blockIdx.y * a.rows;
  const long long stop = first + a.rows < end ? first + a.rows : end;
  if (c >= a.C || row >= together) return;
  for (long long n0 = first + row; n0 < stop; n0 += together * kKeepAhead) {
    u32x2 codes[kKeepAhead];
    int e[kKeepAhead];
#pragma unroll
    for (int q = 0; q < kKeepAhead; ++q) {
      const long long n = n0 + together * q;
      if (n >= stop) continue;
      codes[q] = *reinterpret_cast<const u32x2*>(static_cast<const unsigned char*>(a.x) + b * a.xb + n * a.xt + c);
      e[q] = a.exps[b * a.eb + n * a.et + c / kKeepBlock];
    }
#pragma unroll
    for (int q = 0; q < kKeepAhead; ++q) {
      const long long n = n0 + together * q;
      if (n >= stop) continue;
      float x[8];
      keep_values<T>(codes[q], e[q], x);
      store8_stream<T>(at<T>(a.codes, b * a.cb + n * a.ct + c), x);
    }
  }
}

}  // namespace lf
