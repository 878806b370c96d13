// Linear layers: z = x W^T + b, y = residual + act(z), and their gradients dx = dz W, dW = dz^T x with dz = dy act'(z).
//
// One tiled matrix product serves all three: out[m][n] = sum_k A(m, k) B(n, k), fp32 sums on the matrix instructions (16-bit types:
// 16 x 16 x 32; fp32: 16 x 16 x 4, whose operands are exact).  Either operand may lie with k contiguous (x, W, dz in rows) or with
// its own index contiguous (W for dx; dz and x for dW): the second kind is staged as rows of k and read from LDS by transposing
// reads (fp32: word by word), so that no tensor is transposed in memory.  Tiles of 128 or 64 bytes of k go from memory to LDS without
// passing registers, one step ahead of the products; 16-byte pieces are dealt over a row so that operand reads meet every bank
// evenly.  Where something is not there (channels behind the last, tokens behind a row's length, the end of k) a lane copies from 16
// bytes of zeros instead.  The result is formed transposed, so that a lane holds four neighbouring channels of a token.
#pragma once
#include "lf_keep8.hpp"

namespace lf {

constexpr int kActNone = 0, kActLeaky = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4;

__device__ static const u32x4 kZeros16[1] = {};   // what absent pieces are copied from

struct LinRows { long long batch, token; };   // element strides of [B, N, C] rows; a matrix of plain rows: {0, row stride}

// What is done with z, and where it goes.
struct LinOut {
  void *y, *z;
  const void *residual, *bias;
  LinRows vy, vz, vr;
  int act;
  float slope;
};

struct LinArgs {
  const void *A, *B;
  LinRows va, vb;
  long long M, K;      // rows of the result, products per element
  int N;               // columns of the result
  unsigned per_row;    // tokens of a batch row (which index tokens are depends on the product)
  const int* lengths;
  float* partials;     // [splits][M][N] where k is split, else null
  long long k_split;   // k of a split (a multiple of the tile's)
  int tiles_m, tiles_n, splits;
  LinOut out;
};

// ---- activations -----------------------------------------------------------------------------------------------------

// e^x as 2^(x log2 e) on the hardware's unit: for results of 16 bits.
LF_DEV float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// The normal distribution's tail beyond |z|, Q = exp(-z^2 / 2) P(t) with t = 1 / (1 + 0.3 |z|), and e = exp(-z^2 / 2) for its density.  P
// is a polynomial of degree 6 without a constant, fitted to Q exp(z^2 / 2) for the least of the larger of two errors: Q is off by 2.4e-7 at most and by 1.7e-5
// of itself as far as e is a normal number (|z| to 13.2); arithmetic in fp32 makes that 3.7e-7 and 2.3e-5, an eightieth of bf16's half step.  For
// results of 16 bits (81120 x 8192 of them, with erfc: 1000 of a call's 3200 us).
LF_DEV float normal_tail(float z, float& e) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, __builtin_fabsf(z), 1.0f));
  e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170368f);
  float p = __builtin_fmaf(t, -0.07902849465608597f, 0.22102923691272736f);
  p = __builtin_fmaf(t, p, -0.02159360982477665f);
  p = __builtin_fmaf(t, p, 0.14607316255569458f);
  p = __builtin_fmaf(t, p, 0.1134302094578743f);
  p = __builtin_fmaf(t, p, 0.12008927762508392f);
  return e * t * p;
}

// Precise: for fp32 results; else for 16-bit ones.
template <bool Precise> LF_DEV float logistic(float x) {
  if constexpr (Precise) return 1.0f / (1.0f + expf(-x));
  return __builtin_amdgcn_rcpf(1.0f + exp_fast(-x));
}

template <bool Precise> LF_DEV float act_of(float z, int act, float slope) {
  switch (act) {
    case kActLeaky: return z > 0.0f ? z : slope * z;
    case kActGelu: {
      if constexpr (Precise) return 0.5f * z * erfcf(z * -0.70710678118654752440f);
      float e;
      return fmaxf(z, 0.0f) - fminf(__builtin_fabsf(z), 64.0f) * normal_tail(z, e);   // z (1 - Q) above 0, z Q below (Q is 0 long before 64)
    }
    case kActGeluTanh: return z * logistic<Precise>(1.59576912160573071176f * z * __builtin_fmaf(0.044715f * z, z, 1.0f));
    case kActSilu: return z * logistic<Precise>(z);
    default: return z;
  }
}

template <bool Precise> LF_DEV float act_slope(float z, int act, float slope) {
  switch (act) {
    case kActLeaky: return z > 0.0f ? 1.0f : slope;
    case kActGelu: {
      constexpr float kDensity = 0.39894228040143267794f;
      if constexpr (Precise) return __builtin_fmaf(z, kDensity * expf(-0.5f * z * z), 0.5f * erfcf(z * -0.70710678118654752440f));
      float e;
      const float q = normal_tail(z, e);
      return __builtin_fmaf(z, kDensity * e, z > 0.0f ? 1.0f - q : q);
    }
    case kActGeluTanh: {
      z = z > 30.0f ? 30.0f : (z < -30.0f ? -30.0f : z);   // 1 or 0 from there on, and no infinity times 0
      const float z2 = z * z, p = logistic<Precise>(1.59576912160573071176f * z * __builtin_fmaf(0.044715f, z2, 1.0f));
      return __builtin_fmaf(z * p * (1.0f - p), 1.59576912160573071176f * __builtin_fmaf(0.134145f, z2, 1.0f), p);
    }
    case kActSilu: {
      const float p = logistic<Precise>(z);
      return p * __builtin_fmaf(z, 1.0f - p, 1.0f);
    }
    default: return 1.0f;
  }
}

// ---- tokens and results ----------------------------------------------------------------------------------------------

// Where a token is, and whether it counts.
struct LinToken { unsigned b, n; bool on; };
template <bool MAPPED> LF_DEV LinToken token_at(long long m, long long count, unsigned per_row, const int* lengths) {
  LinToken t{0, (unsigned)m, m < count};
  if constexpr (MAPPED) {
    if (t.on) {
      t.b = (unsigned)m / per_row;
      t.n = (unsigned)m - t.b * per_row;
      if (lengths) t.on = (long long)t.n < (long long)lengths[t.b];
    }
  }
  return t;
}
LF_DEV long long place(const LinRows& v, const LinToken& t) { return t.b * v.batch + t.n * v.token; }

// z of eight channels (n ..) of a token to what the call asks for, bias and residual (where there is one) at hand
template <typename T> LF_DEV void finish8(const LinOut& o, const LinToken& t, int n, float (&z)[8], const float (&bias)[8], const Raw8<T>& residual) {
#pragma unroll
  for (int j = 0; j < 8; ++j) z[j] += bias[j];
  if (o.z) store8_stream<T>(at<T>(o.z, place(o.vz, t) + n), z);
  if (!o.y) return;
  if (o.act != kActNone) {
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = act_of<Stored<T>::kBytes == 4>(z[j], o.act, o.slope);
  }
  if (o.residual) {
    float v[8];
    widen8<T>(residual, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] += v[j];
  }
  store8_stream<T>(at<T>(o.y, place(o.vy, t) + n), z);
}
template <typename T> LF_DEV void bias8(const LinOut& o, int n, float (&bias)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) bias[j] = 0.0f;
  if (o.bias) load8<T>(at<T>(o.bias, n), bias);
}
template <typename T> LF_DEV Raw8<T> residual8(const LinOut& o, const LinToken& t, int n) {
  return o.residual ? load8_raw<T>(at<T>(o.residual, place(o.vr, t) + n)) : none8<T>();
}
template <typename T> LF_DEV void finish8(const LinOut& o, const LinToken& t, int n, float (&z)[8]) {
  const Raw8<T> residual = residual8<T>(o, t, n);
  float bias[8];
  bias8<T>(o, n, bias);
  finish8<T>(o, t, n, z, bias, residual);
}

// ---- the tiled product -----------------------------------------------------------------------------------------------

template <int N> LF_DEV void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Copies 64 x 16 bytes, lane l's from `p`, to the LDS address `lds` + 16 l.  Written out: before a transposing read the compiler waits for
// every copy of its own that is under way, though it goes to the other buffer (8192^3 with B's own index contiguous, bf16: 1093 us so, 905
// without).  (m0, which nothing else here uses, has to be written an instruction before it is read.)  No register receives anything, and wait_copies stands before the barrier behind which the copy is read.
LF_DEV void copy_kb(const unsigned char* p, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory");
}
LF_DEV unsigned lds_address(unsigned char* p) { return (unsigned)(uintptr_t)(LF_LDS unsigned char*)p; }

// An operand's tile of X rows (or columns) and STEP bytes of k, 128 or 64.  KC: k contiguous, X rows of STEP bytes, 16-byte piece c of row r
// at c ^ turn_row(r).  Else rows of k of X values, with groups of 16 values (16-bit: 32 bytes; fp32: 64) of row k at g ^ turn(k), for as
// many groups as make a power of two.
template <typename T, int X, bool KC, int STEP> struct LinTile {
  static constexpr int kSize = Stored<T>::kBytes, kVec = 16 / kSize, kK = STEP / kSize;
  static constexpr int kBytes = X * STEP;
  static constexpr int kRow = KC ? STEP : X * kSize, kPieces = kRow / 16;
  static LF_DEV int turn_row(int r) { return STEP == 128 ? r & 7 : (r >> 2) & 3; }
  static constexpr int kGroups = X / 16, kGroupPieces = kSize;   // (transposed) groups of a row; pieces of a group: 2 or 4
  static constexpr int kMask = (kGroups & -kGroups) - 1;
  static_assert(kBytes % 1024 == 0, "whole copies");
  // rows that one transposing read (16-bit: k = 8 g + r; fp32: k = 4 g + j) brings together get different turns
  static LF_DEV int turn(int k) { return (kSize == 2 ? ((k & 3) | ((k >> 3) & 3) << 2) : ((k >> 2) & 3)) & kMask; }
};

// How tokens are found.  kFlat: one stride leads through all of them.  kRows: batch row and token; where tokens are k, a step's are all of one
// batch row, whose length a wave reads once (a division and a length for every copy: 101 us for 3 x 1000 x 640 to 1280 in fp32, 62 so).
// kLanes (tokens are k, batch rows of a few tokens, of which a step takes several): every lane for itself.
constexpr int kFlat = 0, kRows = 1, kLanes = 2;

// The steps of a tile's k.
struct LinStep { long long k0, end; int b, len; };   // k from k0 to end; kRows: tokens of batch row b, from token k0 on, that count below len
template <int K, bool ROWS> struct LinSteps {
  long long at, stop, by;   // steps
  long long k_end;
  unsigned per, n;          // ROWS: steps of a batch row, its tokens
  const int* lengths;
  // ROWS: the splits take steps in turn, so that rows of any lengths are shared evenly; else each a stretch
  LF_DEV LinSteps(int split, int splits, long long k_split, long long k_all, unsigned per_row, const int* len) {
    k_end = (split + 1) * k_split < k_all ? (split + 1) * k_split : k_all;
    at = ROWS ? split : split * (k_split / K);
    stop = ROWS ? k_all / K : (k_end + K - 1) / K;
    by = ROWS ? splits : 1;
    n = per_row;
    per = (per_row + K - 1) / K;
    lengths = len;
  }
  // the next step with something in it; false: none left
  LF_DEV bool next(LinStep& s) {
    if constexpr (!ROWS) {
      if (at >= stop) return false;
      s = LinStep{at * K, k_end, 0, 0};
      ++at;
      return true;
    }
    for (; at < stop; at += by) {
      const unsigned b = (unsigned)at / per, first = ((unsigned)at - b * per) * K;
      int len = (int)n;
      if (lengths) {   // (a scalar load: it must not wait for the copies under way)
        len = *(const __attribute__((address_space(4))) int*)(lengths + b);
        len = len < 0 ? 0 : (len > (int)n ? (int)n : len);
      }
      if ((int)first >= len) continue;
      s = LinStep{first, 0, (int)b, len};
      at += by;
      return true;
    }
    return false;
  }
};

// The copies of a tile that a thread takes part in: `COUNT` of them.
template <typename T, int X, bool KC, int STEP, int WAVES, int MAPPED> struct LinCopy {
  using Tile = LinTile<T, X, KC, STEP>;
  static constexpr int kCopies = Tile::kBytes / 1024, kCount = (kCopies + WAVES - 1) / WAVES;
  const unsigned char* p[kCount];
  int k[kCount];   // KC: the piece's first k; else the row of k
  bool on[kCount];

  // x0: the tile's first row or column; `limit`: how many there are
  LF_DEV void start(const void* base, const LinRows& v, long long x0, long long limit, unsigned per_row, const int* lengths, int wave) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < kCount; ++j) {
      const int f = (wave + WAVES * j) * 64 + lane, row = f / Tile::kPieces, pos = f % Tile::kPieces;
      if constexpr (KC) {
        const int piece = pos ^ Tile::turn_row(row);
        const LinToken t = token_at<MAPPED != kFlat>(x0 + row, limit, per_row, lengths);
        on[j] = t.on;
        k[j] = piece * Tile::kVec;
        p[j] = t.on ? at<T>(base, (MAPPED != kFlat ? place(v, t) : (x0 + row) * v.token) + k[j]) : nullptr;
      } else {
        const int group = (pos / Tile::kGroupPieces) ^ Tile::turn(row), piece = group * Tile::kGroupPieces + pos % Tile::kGroupPieces;
        const long long x = x0 + piece * Tile::kVec;
        on[j] = x < limit;
        k[j] = row;
        p[j] = at<T>(base, on[j] ? x : 0);
      }
    }
  }
  LF_DEV void step(unsigned lds, const LinRows& v, const LinStep& s, unsigned per_row, const int* lengths, int wave) const {
#pragma unroll
    for (int j = 0; j < kCount; ++j) {
      if (kCopies % WAVES && wave + WAVES * j >= kCopies) break;   // (a whole wave)
      const unsigned char* from;
      bool there;
      if constexpr (KC) {
        there = on[j] && s.k0 + k[j] < s.end;
        from = p[j] + s.k0 * Tile::kSize;
      } else if constexpr (MAPPED == kLanes) {
        const LinToken t = token_at<true>(s.k0 + k[j], s.end, per_row, lengths);
        there = on[j] && t.on;
        from = p[j] + place(v, t) * Tile::kSize;
      } else if constexpr (MAPPED == kRows) {
        there = on[j] && (int)s.k0 + k[j] < s.len;
        from = p[j] + (s.b * v.batch + s.k0 * v.token) * Tile::kSize + k[j] * v.token * Tile::kSize;
      } else {
        there = on[j] && s.k0 + k[j] < s.end;
        from = p[j] + s.k0 * v.token * Tile::kSize + k[j] * v.token * Tile::kSize;
      }
      copy_kb(there ? from : reinterpret_cast<const unsigned char*>(kZeros16), lds + (wave + WAVES * j) * 1024);
    }
  }
};

// Operands of 16 rows (columns) from a tile: 16-bit, 32 k of lane l's row l % 16, eight of them from 8 (l / 16) on; fp32, 16 k, four of them
// from 4 (l / 16) on: the j-th instruction takes every lane's j-th.
template <typename T, int X, bool KC, int STEP> struct LinRead {
  using Tile = LinTile<T, X, KC, STEP>;
  static constexpr int kSteps = STEP / 64;   // per tile
  int base, turn[KC ? kSteps : 1];
  LF_DEV void start(int x) {   // x: the wave's first row or column, a multiple of 16
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    if constexpr (KC) {
      base = (x + i) * STEP;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) turn[s] = ((4 * s + g) ^ Tile::turn_row(i)) * 16;
    } else if constexpr (Tile::kSize == 2) {
      base = (8 * g + (i >> 2)) * Tile::kRow + (i & 3) * 8;
      turn[0] = Tile::turn(8 * g + (i >> 2));
    } else {
      base = 4 * g * Tile::kRow + i * 4;
      turn[0] = 0;   // (goes by the row)
    }
  }
  // tile t of 16 from x on (`x` again: transposed places depend on it), step s
  LF_DEV u32x4 get(const unsigned char* lds, int x, int t, int s) const {
    if constexpr (KC) {
      return *reinterpret_cast<const u32x4*>(lds + base + turn[s] + t * 16 * STEP);
    } else if constexpr (Tile::kSize == 2) {
      const unsigned char* q = lds + base + s * 32 * Tile::kRow + ((x / 16 + t) ^ turn[0]) * 32;
      const u32x2 a = lds_read_tr16(reinterpret_cast<const uint16_t*>(q)), b = lds_read_tr16(reinterpret_cast<const uint16_t*>(q + 4 * Tile::kRow));
      return u32x4{a[0], a[1], b[0], b[1]};
    } else {
      const int g = (threadIdx.x & 63) >> 4;
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j)   // (turn(16 s + 4 g + j) is g)
        v[j] = *reinterpret_cast<const uint32_t*>(lds + base + (s * 16 + j) * Tile::kRow + ((x / 16 + t) ^ (g & Tile::kMask)) * 64);
      return v;
    }
  }
};

template <typename T> LF_DEV f32x4 lin_product(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (Stored<T>::kBytes == 2) {
    return mfma_16x16x32<T>(a, b, c);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  }
}

// Which tile of the result, and which split of k, a workgroup takes.  Workgroups are dealt to the eight XCDs in turn: each XCD gets a
// stretch of the list, which goes through bands of eight rows of tiles column by column, so that those on an XCD at a time share
// operands in its L2.  `ragged` (rows that may not count): the list as it is, so that no XCD's stretch is empty.
struct LinPlace {
  int m, n, split;
  LF_DEV LinPlace(int tiles_m, int tiles_n, bool ragged) {
    const unsigned all = gridDim.x, id = blockIdx.x, xcd = id % 8, at = id / 8;
    const unsigned each = all / 8, more = all % 8;
    unsigned t = ragged ? id : xcd * each + (xcd < more ? xcd : more) + at;
    const unsigned tiles = (unsigned)tiles_m * (unsigned)tiles_n;
    split = t / tiles;
    t -= split * tiles;
    const unsigned band = 8 * (unsigned)tiles_n, first = t / band * 8, in = t % band;
    const unsigned high = (unsigned)tiles_m - first < 8 ? (unsigned)tiles_m - first : 8;
    m = first + in % high;
    n = in / high;
  }
};

// WR x WC waves, each with BM / WR rows and BN / WC columns of the tile.  AK, BK: whether A, B have k contiguous.  Tokens are the rows
// of the result where A has k contiguous, else k.
template <typename T, int BM, int BN, int WR, int WC, int STEP, bool AK, bool BK, int MAPPED>
__global__ __launch_bounds__(64 * WR * WC, STEP == 64 && BM * BN <= 128 * 128 ? 4 : 1) void linear_tiles(LinArgs g) {
  constexpr int kWaves = WR * WC, WM = BM / WR, WN = BN / WC, MT = WM / 16, NT = WN / 16;
  using TA = LinTile<T, BM, AK, STEP>;
  using TB = LinTile<T, BN, BK, STEP>;
  constexpr int kBuffer = TA::kBytes + TB::kBytes;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const LinPlace tile(g.tiles_m, g.tiles_n, AK && g.lengths != nullptr);
  const long long m0 = (long long)tile.m * BM;
  const int n0 = tile.n * BN;
  if constexpr (AK && MAPPED != kFlat) {   // nothing to do where no row of the tile counts
    if (g.lengths) {
      bool some = false;
      for (int r = threadIdx.x; r < BM; r += 64 * kWaves) some |= token_at<true>(m0 + r, g.M, g.per_row, g.lengths).on;
      if (!__syncthreads_or(some)) return;
    }
  }
  constexpr bool kByRows = !AK && MAPPED == kRows;
  LinSteps<TA::kK, kByRows> steps(tile.split, g.splits, g.k_split, g.K, g.per_row, g.lengths);
  LinCopy<T, BM, AK, STEP, kWaves, MAPPED> ca;
  LinCopy<T, BN, BK, STEP, kWaves, AK ? kFlat : MAPPED> cb;
  ca.start(g.A, g.va, m0, g.M, g.per_row, g.lengths, wave);
  cb.start(g.B, g.vb, n0, g.N, g.per_row, g.lengths, wave);
  const int wm = wave / WC * WM, wn = wave % WC * WN;
  LinRead<T, BM, AK, STEP> ra;
  LinRead<T, BN, BK, STEP> rb;
  ra.start(wm);
  rb.start(wn);
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  int side = 0;
  const unsigned base = lds_address(smem);
  auto request = [&](const LinStep& s) {
    const unsigned to = base + side * kBuffer;
    ca.step(to, g.va, s, g.per_row, g.lengths, wave);
    cb.step(to + TA::kBytes, g.vb, s, g.per_row, g.lengths, wave);
  };
  LinStep s;
  bool more = steps.next(s);
  if (more) request(s);
  while (more) {
    wait_copies<0>();
    __syncthreads();   // this step's tiles are there, and nobody reads the other buffer any more
    const unsigned char* la = smem + side * kBuffer;
    side ^= 1;
    more = steps.next(s);
    if (more) request(s);
    const unsigned char* lb = la + TA::kBytes;
#pragma unroll
    for (int q = 0; q < STEP / 64; ++q) {
      u32x4 a[MT], b[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) b[j] = rb.get(lb, wn, j, q);
#pragma unroll
      for (int i = 0; i < MT; ++i) a[i] = ra.get(la, wm, i, q);
      __builtin_amdgcn_s_setprio(1);   // one wave of a SIMD multiplies while the other one reads (8192^3 in bf16: 869 us without, 835 with)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = lin_product<T>(b[j], a[i], acc[i][j]);
      __builtin_amdgcn_s_setprio(0);
    }
  }
  // Lane l has columns 4 (l / 16) .. + 3 of a tile of 16 and row l % 16: through LDS, a wave's rows for itself, into rows of eight
  // channels a lane, so that stores are whole lines and the activation's code is there once.
  constexpr int kUnits = WN / 4, kTurn = (kUnits & -kUnits) - 1;   // 16 bytes each; row r's unit u is at u ^ (r & kTurn)
  constexpr int kRegion = 2 * kBuffer / kWaves, kFit = kRegion / (16 * WN * 4);
  constexpr int kPass = kFit >= MT ? MT : (kFit >= (MT + 1) / 2 && MT % 2 == 0 ? MT / 2 : (kFit >= 2 && MT % 2 == 0 ? 2 : 1));
  static_assert(kFit >= kPass && MT % kPass == 0, "whole passes");
  constexpr int kRowLanes = WN / 8, kTogether = 64 / kRowLanes;   // lanes of a row; rows at a time
  constexpr int kAtOnce = 4;   // rows of a lane whose residuals are requested together
  __syncthreads();
  unsigned char* mine = smem + wave * kRegion;
  const int row = lane / kRowLanes, u = lane % kRowLanes * 2, n = n0 + wn + 4 * u;
  const bool on = lane < kTogether * kRowLanes && n < g.N;
  float bias[8];
  if (on && !g.partials) bias8<T>(g.out, n, bias);
#pragma unroll
  for (int p = 0; p < MT; p += kPass) {
#pragma unroll
    for (int i = 0; i < kPass; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int r = 16 * i + (lane & 15), v = 4 * j + (lane >> 4);
        *reinterpret_cast<f32x4*>(mine + r * (WN * 4) + (v ^ (r & kTurn)) * 16) = acc[p + i][j];
      }
    asm volatile("" ::: "memory");   // (a wave's LDS operations complete in order)
#pragma unroll 1
    for (int r0 = 0; r0 < 16 * kPass; r0 += kTogether * kAtOnce) {
      LinToken t[kAtOnce];
      Raw8<T> residual[kAtOnce];
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        const int r = r0 + q * kTogether + row;
        t[q] = token_at<MAPPED != kFlat && AK>(m0 + wm + 16 * p + r, g.M, g.per_row, g.lengths);
        t[q].on = t[q].on && on && r < 16 * kPass;
        residual[q] = none8<T>();
        if (t[q].on && !g.partials) residual[q] = residual8<T>(g.out, t[q], n);
      }
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        if (!t[q].on) continue;
        const int r = r0 + q * kTogether + row;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(mine + r * (WN * 4) + (u ^ (r & kTurn)) * 16);
        const f32x4 hi = *reinterpret_cast<const f32x4*>(mine + r * (WN * 4) + ((u + 1) ^ (r & kTurn)) * 16);
        if (g.partials) {
          float* to = g.partials + (tile.split * g.M + m0 + wm + 16 * p + r) * g.N + n;
          *reinterpret_cast<f32x4*>(to) = lo;
          *reinterpret_cast<f32x4*>(to + 4) = hi;
        } else {
          float z[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          finish8<T>(g.out, t[q], n, z, bias, residual[q]);
        }
      }
    }
    asm volatile("" ::: "memory");
  }
}

// The splits' sums, eight columns a thread, in their order.
template <typename T, bool MAPPED> __global__ __launch_bounds__(256) void linear_join(LinArgs g) {
  const long long across = g.N / 8, id = (long long)blockIdx.x * 256 + threadIdx.x;
  if (id >= g.M * across) return;
  const long long m = id / across;
  const int n = (int)(id - m * across) * 8;
  const LinToken t = token_at<MAPPED>(m, g.M, g.per_row, g.lengths);
  if (!t.on) return;
  float z[8], v[8];
  load8_f32(g.partials + m * g.N + n, z);
  for (int s = 1; s < g.splits; ++s) {
    load8_f32(g.partials + (s * g.M + m) * g.N + n, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] += v[j];
  }
  finish8<T>(g.out, t, n, z);
}

// ---- few tokens ------------------------------------------------------------------------------------------------------

// Up to 16 MT tokens: every weight is read once, straight into operand registers, 16 channels a workgroup, whose eight waves share k.
// Bound: the weights' way from memory, for few of them its latency.
constexpr int kFewWaves = 8;
template <typename T, int MT, bool MAPPED> __global__ __launch_bounds__(64 * kFewWaves) void linear_few(LinArgs g) {
  constexpr int kVec = 16 / Stored<T>::kBytes, kK = 4 * kVec, kAhead = MT == 4 ? 4 : 6;   // k of a product; products requested together
  __shared__ __attribute__((aligned(16))) float lds[kFewWaves][16 * MT][20];   // (rows spread over the banks)
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
  const int n0 = blockIdx.x * 16;
  f32x4 acc[MT];
  const unsigned char* px[MT];
  bool on[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const LinToken m = token_at<MAPPED>(16 * t + i, g.M, g.per_row, g.lengths);
    on[t] = m.on;
    px[t] = at<T>(g.A, on[t] ? place(g.va, m) : 0);
  }
  const bool row = n0 + i < g.N;
  const unsigned char* pw = at<T>(g.B, row ? (n0 + i) * g.vb.token : 0);
  for (long long k0 = (long long)wave * kAhead * kK; k0 < g.K; k0 += kFewWaves * kAhead * kK) {
    u32x4 w[kAhead], x[MT][kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const long long k = k0 + j * kK + q * kVec;
      const bool there = k < g.K;
      w[j] = u32x4{0, 0, 0, 0};
      if (row && there) w[j] = ld_stream(reinterpret_cast<const u32x4*>(at<T>(pw, k)));
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        x[t][j] = u32x4{0, 0, 0, 0};
        if (on[t] && there) x[t][j] = *reinterpret_cast<const u32x4*>(at<T>(px[t], k));
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[t] = lin_product<T>(w[j], x[t][j], acc[t]);
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) *reinterpret_cast<f32x4*>(&lds[wave][16 * t + i][4 * q]) = acc[t];
  __syncthreads();
  // eight channels a thread
  const int m = threadIdx.x >> 1, half = threadIdx.x & 1, n = n0 + 8 * half;
  if (m >= 16 * MT || n >= g.N) return;
  const LinToken t = token_at<MAPPED>(m, g.M, g.per_row, g.lengths);
  if (!t.on) return;
  float z[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    z[j] = lds[0][m][8 * half + j];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) z[j] += lds[w][m][8 * half + j];
  }
  finish8<T>(g.out, t, n, z);
}

// ---- dz, and the bias's gradient ---------------------------------------------------------------------------------------

struct LinSlopeArgs {
  const void *dy, *z;               // z: values, or codes of eight bits with `z_exps`
  const unsigned char* z_exps;
  LinRows vdy, vz, ve;              // ve: of the exponents' rows
  void* dz;                         // [B * N][C] rows, or null (no activation)
  float* partials;                  // [workgroups along the tokens][C], or null
  const int* lengths;
  long long N;
  int B, C, each, lanes, act;       // each: tokens of a piece of a batch row; a workgroup takes pieces in turn; lanes: of a token
  float slope;
};

// dz = dy act'(z), rounded once to the type (it is an operand of two products), and the sums of the unrounded values over a
// workgroup's tokens.  That rounding is beside the results' own in dx and dw of 16-bit types: bf16 2.4e-3 of their norm off, 1.7e-3 with dz as two terms of the
// type.  Those double the products' work: dx and dw of 49152 x 1280 to 320 take 101 and 101 us for 71 and 57, of 320 to 1280 115 and 108 for 48 and 57, of 16384 x
// 1280 to 5120 405 and 381 for 204 and 221, and the way out of dz of 1280 channels 24 us more.  One term is also what a layer hands back whose activation is a call
// of its own.  `lanes` lanes of 8 channels a token, as many tokens at a time as that leaves, twice as many under way (absent ones from 16 bytes of zeros, without
// branches).  Bound: HBM (49152 x 1280 bf16 from kept z: 315 MB), with GELU the vector instructions too.
template <typename T, bool KEPT> __global__ __launch_bounds__(256) void linear_slope(LinSlopeArgs a) {
  __shared__ float lds[256][8];
  constexpr int kAhead = 2;
  const int row = threadIdx.x / a.lanes, lane = threadIdx.x - row * a.lanes, rows = 256 / a.lanes, c = (blockIdx.x * a.lanes + lane) * 8;
  const bool on = c < a.C && row < rows;
  const unsigned char* const none = reinterpret_cast<const unsigned char*>(kZeros16);
  const long long per = (a.N + a.each - 1) / a.each, pieces = per * a.B;
  float sum[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
  for (long long piece = blockIdx.y; piece < pieces; piece += gridDim.y) {
    const unsigned b = (unsigned)piece / (unsigned)per;
    const long long first = (long long)((unsigned)piece - b * (unsigned)per) * a.each, len = tokens_of(a.lengths, b, a.N);
    const long long end = first + a.each < len ? first + a.each : len;
    const unsigned char *pd = at<T>(a.dy, b * a.vdy.batch + c), *pe = a.z_exps + b * a.ve.batch + c / kKeepBlock;
    const unsigned char* pz = KEPT ? static_cast<const unsigned char*>(a.z) + b * a.vz.batch + c : at<T>(a.z, b * a.vz.batch + c);
    unsigned char* po = at<T>(a.dz, b * a.N * a.C + c);
    for (long long n0 = first; n0 < end; n0 += rows * kAhead) {
      Raw8<T> rd[kAhead], rz[KEPT ? 1 : kAhead];
      u32x2 codes[KEPT ? kAhead : 1];
      int exps[KEPT ? kAhead : 1];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        const long long n = n0 + row + rows * q;
        const bool there = on && n < end;
        if constexpr (Stored<T>::kBytes == 4) {
          rd[q] = none8<T>();
          if (there) rd[q] = load8_raw<T>(pd + n * a.vdy.token * 4);
        } else {
          rd[q].w = *reinterpret_cast<const u32x4*>(there ? pd + n * a.vdy.token * 2 : none);
        }
        if (!a.dz) continue;
        if constexpr (KEPT) {
          codes[q] = *reinterpret_cast<const u32x2*>(there ? pz + n * a.vz.token : none);
          exps[q] = *(there ? pe + n * a.ve.token : none);
        } else if constexpr (Stored<T>::kBytes == 4) {
          rz[q] = none8<T>();
          if (there) rz[q] = load8_raw<T>(pz + n * a.vz.token * 4);
        } else {
          rz[q].w = *reinterpret_cast<const u32x4*>(there ? pz + n * a.vz.token * 2 : none);
        }
      }
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        const long long n = n0 + row + rows * q;
        float d[8];
        widen8<T>(rd[q], d);
        if (a.dz) {
          float z[8];
          if constexpr (KEPT) keep_values<T>(codes[q], exps[q], z);
          else widen8<T>(rz[q], z);
#pragma unroll
          for (int j = 0; j < 8; ++j) d[j] *= act_slope<Stored<T>::kBytes == 4>(z[j], a.act, a.slope);
          if (on && n < end) store8<T>(po + n * a.C * Stored<T>::kBytes, d);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += d[j];
      }
    }
  }
  if (!a.partials) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) lds[threadIdx.x][j] = sum[j];
  __syncthreads();
  for (int t = threadIdx.x; t < 8 * a.lanes; t += 256) {
    const int cc = blockIdx.x * a.lanes * 8 + t;
    float all = 0.0f;
    for (int r = 0; r < rows; ++r) all += lds[r * a.lanes + (t >> 3)][t & 7];
    if (cc < a.C) a.partials[(long long)blockIdx.y * a.C + cc] = all;
  }
}

// The bias's gradient: the workgroups' sums.
template <typename T> __global__ __launch_bounds__(1024) void linear_bias(const float* partials, void* dbias, int parts, int C) {
  __shared__ double lds[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15);
  const double sum = column_sum(lds, partials, parts, C, c);
  if (threadIdx.x >= 16 || c >= C) return;
  if constexpr (Stored<T>::kBytes == 4) static_cast<float*>(dbias)[c] = (float)sum;
  else static_cast<uint16_t*>(dbias)[c] = (uint16_t)pack2<T>((float)sum, 0.0f);
}

}  // namespace lf
