// Rotary positions with several axes: an axis owns a section of a head's channels, in pairs, and turns pair i of its c
// channels by  theta = pos * scale * base^(-2 i / c):
//
//     (x1, x2) -> (x1 cos theta - x2 sin theta, x2 cos theta + x1 sin theta)
//
// Turning by -theta is the inverse and the gradient.  Bound: HBM, each value read once and written once.  The angles depend
// on the token and the pair, not on the head: a workgroup takes a few tokens of one batch row through all heads of q and k
// and computes each sine and cosine once.  theta is formed in turns, in fp64: a position of 10^5 leaves an fp32 product
// no more than 3 correct digits of the angle, and the fraction of the fp64 product is exact to 2^-36.
// bf16, 81120 tokens of 2 x 16 heads of 128: 214 to 234 us for 1.33 GB (6.2 to 5.7 TB/s; as one section of halves 222, as sections
// of 44 + 42 + 42, halves, 263); fp32, 2 x 36503 tokens of 2 x 8 heads of 40: 57 us for 374 MB
// (6.6 TB/s); fp16, 2 x 256 tokens of 2 x 8 heads of 160: 5.8 us.
#pragma once
#include "lf_vec8.hpp"

namespace lf {

constexpr int kRopeAxes = 4;
constexpr int kRopePairs = 128;   // d <= 256

struct RopeSide {
  const void* x;
  void* y;
  long long xb, xh, xn, yb, yh, yn;   // element strides {batch, head, token}
  int H;
  int by_token;                       // heads of a token are the nearer neighbours in memory
};

struct RopeArgs {
  RopeSide side[2];
  const int* positions;
  long long pos_batch, pos_axis;
  const int* lengths;
  long long N;
  int d, pairs, axes, tokens;         // tokens: per workgroup
  int first[kRopeAxes + 1];           // first channel of each section; behind the last one channels have no position
  unsigned inverse;
  double rate[kRopePairs];            // turns per unit of position
};

// cos and sin of `turns` of a full turn.  The hardware's own (argument in turns; absolute error near 2^-20) for the 16-bit
// types, whose results are rounded to 2^-9 or 2^-12; the library's for fp32.
template <typename T> LF_DEV f32x2 turn_of(double turns) {
  const float r = (float)(turns - __builtin_rint(turns));
  if constexpr (Stored<T>::kBytes == 4) {
    float s, c;
    sincospif(2.0f * r, &s, &c);
    return f32x2{c, s};
  } else {
    return f32x2{__builtin_amdgcn_cosf(r), __builtin_amdgcn_sinf(r)};
  }
}

inline __host__ __device__ size_t rope_table_bytes(int tokens, int pairs) { return ((size_t)tokens * pairs * 8 + 15) & ~(size_t)15; }

// MODE 0: neighbouring channels are paired (pair = channel / 2).  1: a section's first half with its second half, all
// halves whole 16-byte pieces; 2: the same, halves of any size.
// A wave takes whole rows, a lane 16 bytes of one, kRows of them in flight; the halves change places through LDS that only the
// wave itself uses, after its loads and before its stores, so a call may work in place.
template <typename T, int MODE>
__global__ __launch_bounds__(256) void rope_rows(RopeArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int E = 16 / Stored<T>::kBytes, kRows = 2;   // channels a lane; groups of rows in flight
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int b = blockIdx.y;
  const long long n_end = tokens_of(a.lengths, b, a.N);
  const long long n0 = (long long)blockIdx.x * a.tokens;
  if (n0 >= n_end) return;
  const int tokens = n_end - n0 < a.tokens ? (int)(n_end - n0) : a.tokens;
  f32x2* table = reinterpret_cast<f32x2*>(smem);                       // [tokens][pairs]
  unsigned char* stage = smem + rope_table_bytes(a.tokens, a.pairs) + (size_t)wave * kRows * 1024;
  for (int i = tid; i < tokens * a.pairs; i += 256) {
    const int t = (unsigned)i / (unsigned)a.pairs, p = i - t * a.pairs;
    int axis = 0;
#pragma unroll
    for (int s = 1; s < kRopeAxes; ++s)
      if (s < a.axes && 2 * p >= a.first[s]) axis = s;
    const int pos = a.positions[b * a.pos_batch + axis * a.pos_axis + n0 + t];
    f32x2 cs = turn_of<T>((double)pos * a.rate[p]);
    if (a.inverse) cs[1] = -cs[1];
    table[i] = cs;
  }
  __syncthreads();
  const int chunks = a.d / E, per = 64 / chunks;       // pieces per row, rows per wave and step
  const int own = lane / chunks, c0 = (lane - own * chunks) * E;
  // where this lane's channels stand: the pair of the first, the partner's channel, and the sign of its part
  int pair = c0 >> 1, partner = 0;
  float sign = 1.0f;
  const bool turned = c0 < a.first[a.axes];
  if constexpr (MODE == 1) {
    int s0 = 0, s1 = a.first[1];
#pragma unroll
    for (int s = 1; s < kRopeAxes; ++s)
      if (s < a.axes && c0 >= a.first[s]) { s0 = a.first[s]; s1 = a.first[s + 1]; }
    const int half = (s1 - s0) >> 1, o = c0 - s0;
    const bool upper = o >= half;
    pair = (s0 >> 1) + (upper ? o - half : o);
    partner = upper ? c0 - half : c0 + half;
    sign = upper ? 1.0f : -1.0f;
  }
  auto widen = [](const u32x4& w, float (&x)[E]) {
    if constexpr (E == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = __builtin_bit_cast(f32x4, w)[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) unpack2<T>(w[j], x[2 * j], x[2 * j + 1]);
    }
  };
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    const RopeSide& side = a.side[which];
    if (!side.x) continue;
    const int rows = tokens * side.H, step = 4 * per;
    for (int r0 = wave * per; r0 < rows; r0 += kRows * step) {
      u32x4 raw[kRows];
      int t[kRows], h[kRows];
      bool on[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int r = r0 + k * step + own;
        on[k] = own < per && r < rows;
        if (side.by_token) { t[k] = (int)((unsigned)r / (unsigned)side.H); h[k] = r - t[k] * side.H; }
        else { h[k] = (int)((unsigned)r / (unsigned)tokens); t[k] = r - h[k] * tokens; }
        if (on[k]) raw[k] = *reinterpret_cast<const u32x4*>(at<T>(side.x, b * side.xb + h[k] * side.xh + (n0 + t[k]) * side.xn + c0));
      }
      if constexpr (MODE != 0) {
#pragma unroll
        for (int k = 0; k < kRows; ++k)
          if (on[k]) *reinterpret_cast<u32x4*>(stage + (k * 64 + lane) * 16) = raw[k];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (LDS that only this wave uses)
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        if (!on[k]) continue;
        const f32x2* cs = table + t[k] * a.pairs;
        float x[E], y[E];
        widen(raw[k], x);
        if constexpr (MODE == 0) {
          if (turned) {
#pragma unroll
            for (int j = 0; j < E / 2; ++j) {
              if (pair + j < a.pairs) {
                const f32x2 e = cs[pair + j];
                y[2 * j] = x[2 * j] * e[0] - x[2 * j + 1] * e[1];
                y[2 * j + 1] = x[2 * j + 1] * e[0] + x[2 * j] * e[1];
              } else {
                y[2 * j] = x[2 * j];
                y[2 * j + 1] = x[2 * j + 1];
              }
            }
          }
        } else if constexpr (MODE == 1) {
          if (turned) {
            float z[E];
            widen(*reinterpret_cast<const u32x4*>(stage + (k * 64 + lane + (partner - c0) / E) * 16), z);
#pragma unroll
            for (int j = 0; j < E; ++j) {
              const f32x2 e = cs[pair + j];
              y[j] = x[j] * e[0] + sign * (z[j] * e[1]);
            }
          }
        } else if (turned) {
          const unsigned char* row = stage + (k * 64 + own * chunks) * 16;
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const int c = c0 + j;
            y[j] = x[j];
            if (c >= a.first[a.axes]) continue;
            int s0 = 0, s1 = a.first[1];
#pragma unroll
            for (int s = 1; s < kRopeAxes; ++s)
              if (s < a.axes && c >= a.first[s]) { s0 = a.first[s]; s1 = a.first[s + 1]; }
            const int half = (s1 - s0) >> 1, o = c - s0;
            const bool upper = o >= half;
            const f32x2 e = cs[(s0 >> 1) + (upper ? o - half : o)];
            const int other = upper ? c - half : c + half;
            float z;
            if constexpr (E == 4) {
              z = *reinterpret_cast<const float*>(row + other * 4);
            } else {
              float dummy;
              unpack2<T>(*reinterpret_cast<const uint16_t*>(row + other * 2), z, dummy);
            }
            y[j] = x[j] * e[0] + (upper ? z * e[1] : -(z * e[1]));
          }
        }
        u32x4 out = raw[k];   // channels without a position keep their bits
        if (turned) {
          if constexpr (E == 4) out = __builtin_bit_cast(u32x4, f32x4{y[0], y[1], y[2], y[3]});
          else out = u32x4{pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3]), pack2<T>(y[4], y[5]), pack2<T>(y[6], y[7])};
        }
        st_stream(reinterpret_cast<u32x4*>(at<T>(side.y, b * side.yb + h[k] * side.yh + (n0 + t[k]) * side.yn + c0)), out);
      }
      if constexpr (MODE != 0) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  }
}

}  // namespace lf
