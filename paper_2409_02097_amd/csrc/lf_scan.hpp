// A gated linear recurrence, channel by channel.  Per (batch, channel), token after token:
//
//     s = sigmoid(gate_t);  i = sigmoid(input_t) (1 without);  g = -rate s;  a = e^g
//     m = sqrt(1 - a^2)  (kScanNorm),  1 - a  (kScanLeaky),  1  (kScanSum)
//     h = a h + m i x_t;  out_t = h
//
// Backward, with E behind the last token the gradient that arrives at its state:
//
//     D = dout_t + E;  dx = D m i;  dinput = D m x i (1 - i);  dg = D (a h' + (dm/dg) i x), h' the state before the token;
//     dgate = dg g (1 - s);  drate += -dg s;  E = a D
//
// where dm/dg = -a^2 / m, -a, 0.  Both directions are first-order linear recurrences, so a stretch of tokens turns the value
// it starts from into A h + R with A the product of its a.  A workgroup of 256 threads takes a chunk of 128 tokens of 64
// channels, a thread four tokens of 8 channels: a and m i x in registers, the stretches of a wave's eight time lanes and then of
// the four waves joined through LDS.  The chunks of a long sequence tell each other theirs inside the launch (ScanRecords), so that
// every tensor is read once and written once.  Everything is fp32, results are rounded once.
// One MI355X: 65536 x 1280 bf16 with a gate on the inputs 162 us with the records' clearing, 671 MB at 4.2 TB/s, where a copy of
// 1 GiB makes 5.2; 12 x 4096 x 320 bf16, 46 us forward (126 MB) and 63 back (220 MB at 3.5 TB/s).
#pragma once
#include "lf_vec8.hpp"

namespace lf {

constexpr int kScanNorm = 0, kScanLeaky = 1, kScanSum = 2;
constexpr int kScanWidth = 64;   // channels of a workgroup

// (eight tokens a thread where a sequence is several chunks: half the workgroups on a CU, and no faster)
constexpr int kScanT = 4, kScanChunk = 32 * kScanT;   // tokens of a thread; of a chunk

struct ScanView { long long batch, token; };   // element strides; channels contiguous

// What the chunks of a sequence tell each other: every chunk's (A, R), and what stands for groups of them, as soon as they are known.  All ones:
// not yet (scan_clear).  The workgroups take chunks by `ticket`, nearer the sequence's start (backward: its end) first, so that a workgroup
// only ever waits for ones that have started and wait for earlier ones alone: every wait ends.
struct ScanRecords {
  unsigned* ticket;
  unsigned long long* totals;   // [B][chunks][C]
  unsigned* values;             // [B][chunks][C]
};

struct ScanArgs {
  const void *x, *gate, *input;
  void* out;                    // null: only `saved`
  ScanView vx, vg, vi, vo;
  const float *rate, *state_in;
  float *state_out, *saved;     // saved: null, or [B][chunks of kScanChunk][C], the state before each chunk
  ScanRecords rec;
  const int* lengths;
  long long N;
  int B, C, chunks, saved_chunks, group, seg;
  bool reverse;
};

struct ScanBackArgs {
  const void *x, *gate, *input, *dout;
  void *dx, *dgate, *dinput;
  ScanView vx, vg, vi, vd, vdx, vdg, vdi;
  const float *rate, *starts, *dstate_out;
  float *dstate_in, *partials;  // partials: [B][chunks][C], of drate
  ScanRecords rec;
  const int* lengths;
  long long N;
  int B, C, chunks, group, seg;
  bool reverse;
};

// v < limit ? a : b, both formed in any case: left to itself the compiler makes branches of such choices, one per element (65536 x 1280 in
// bf16: 142 us for what takes 60 without).
LF_DEV float below(float v, float limit, float a, float b) {
  asm volatile("" : "+v"(a));
  return v < limit ? a : b;
}
// c ? 0 : x, x formed in any case
LF_DEV float unless(bool c, float x) {
  asm volatile("" : "+v"(x));
  return c ? 0.0f : x;
}

// 1 / (1 + e^-x), the exponential by the hardware's of 2; Precise adds back what rounding x log2(e) loses.
// `e`: e^-x.
template <bool Precise> LF_DEV float sigmoid_of(float x, float& e) {
  constexpr float kLog2e = 1.44269504088896340736f;
  const float t = x * -kLog2e;
  e = __builtin_amdgcn_exp2f(t);
  if constexpr (!Precise) return __builtin_amdgcn_rcpf(1.0f + e);
  const float lost = __builtin_fmaf(x, -1.92596299112661746e-8f, __builtin_fmaf(x, -kLog2e, -t));
  e = unless(x > 104.0f, __builtin_fmaf(e, lost * 0.69314718055994530942f, e));   // (no 0 times infinity)
  const float s = __builtin_amdgcn_rcpf(1.0f + e);
  return unless(x < -88.0f, s);
}
template <bool Precise> LF_DEV float sigmoid_of(float x) {
  float e;
  return sigmoid_of<Precise>(x, e);
}

// A sigmoid and one less it in one number, the smaller of the two, as next to 1 a sigmoid no longer holds what is left: s below x = 0, else s - 1, whose sign
// says which (a zero's too).  s (1 - s) is |v| (1 - |v|) either way.
template <bool Precise> LF_DEV float smaller_sigmoid(float x, float& s) {
  float e;
  s = sigmoid_of<Precise>(x, e);
  float v = -(e * s);
  asm("" : "+v"(v));   // (no branch)
  v = x < 0.0f ? s : v;
  asm volatile("" : "+v"(v));   // (or what it is chosen from is kept until it is needed)
  return v;
}

// 1 - 2^-d for d >= 0, e = 2^-d given, or with TWICE 1 - 4^-d, e = 4^-d: where e is near 1 by the series, whose next term is below 2^-24
// of the result (16-bit types: below 2^-18.9 twice, 2^-24 once).
template <bool Precise, bool TWICE> LF_DEV float one_less(float d, float e) {
  constexpr float k1[10] = {0.693147181f, 0.240226507f, 0.0555041087f, 0.00961812911f, 0.00133335581f, 0.000154035304f, 1.52527338e-05f, 1.32154868e-06f, 1.0178086e-07f, 7.05491162e-09f};
  constexpr float k2[8] = {1.38629436f, 0.960906028f, 0.444032869f, 0.153890066f, 0.0426673861f, 0.00985825945f, 0.00195234993f, 0.000338316462f};   // (ln 2)^n / n!, (2 ln 2)^n / n!
  constexpr int kTerms = Precise ? 8 : (TWICE ? 4 : 6);
  constexpr float kLimit = Precise ? (TWICE ? 0.36f : 0.72f) : (TWICE ? 0.09f : 0.36f);   // the exponent below 1/2; 1/8, 1/4
  float p = TWICE ? k2[kTerms - 1] : k1[kTerms - 1];
#pragma unroll
  for (int i = kTerms - 2; i >= 0; --i) p = __builtin_fmaf(d, -p, TWICE ? k2[i] : k1[i]);
  return below(d, kLimit, d * p, 1.0f - e);
}

// The weight m of the new value for a = 2^-d.
template <bool Precise, int MODE> LF_DEV float weight_of(float d, float a) {
  if constexpr (MODE == kScanSum) return 1.0f;
  if constexpr (MODE == kScanLeaky) return one_less<Precise, false>(d, a);
  return __builtin_amdgcn_sqrtf(one_less<Precise, true>(d, a * a));
}

// What absent gates read as: minus infinity, whose sigmoid is 0, so that a = 1 and the state stays as it is.
template <typename T> struct ShutBits;
template <> struct ShutBits<F16> { static constexpr uint32_t value = 0xfc00fc00u; };
template <> struct ShutBits<BF16> { static constexpr uint32_t value = 0xff80ff80u; };
template <> struct ShutBits<F32> { static constexpr uint32_t value = 0xff800000u; };
template <typename T> LF_DEV Raw8<T> shut8() {
  constexpr uint32_t w = ShutBits<T>::value;
  Raw8<T> r;
  r.w = u32x4{w, w, w, w};
  if constexpr (Stored<T>::kBytes == 4) r.w2 = u32x4{w, w, w, w};
  return r;
}

// Has a value from memory arrive before anything behind this leaves: a state that is given may be overwritten in place as soon as another
// wave, or the chunk behind, has heard from this one.
LF_DEV void arrive(float& v) { asm volatile("" : "+v"(v)::"memory"); }

// Makes the compiler take a row for a new one, so that what was formed from it is formed again and not kept in registers meanwhile.
template <typename T> LF_DEV void forget(Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w = r.w[i];
    asm("" : "+v"(w));
    r.w[i] = w;
    if constexpr (Stored<T>::kBytes == 4) {
      w = r.w2[i];
      asm("" : "+v"(w));
      r.w2[i] = w;
    }
  }
}

// Where a row's tokens are in the order of the recurrence.
struct ScanRow {
  long long n;       // tokens that count
  bool reverse;
  LF_DEV ScanRow(const int* lengths, int b, long long N, bool rev) : n(tokens_of(lengths, b, N)), reverse(rev) {}
  LF_DEV long long token(long long t) const { return reverse ? n - 1 - t : t; }
  // the bytes from a token's row to the next one's in this order
  template <typename T> LF_DEV long long step(const ScanView& v) const { return (reverse ? -v.token : v.token) * Stored<T>::kBytes; }
};

LF_DEV void load_rate(const float* p, bool on, float (&rate)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) rate[k] = 0.0f;
  if (on) load8_f32(p, rate);
}

// The rows of a thread's tokens of up to four tensors, token after token, so that work on the first can begin while the others are on
// their way; `absent` where there are none.
template <typename T> struct ScanLoad {
  const unsigned char* p;   // the first token's
  long long step;           // bytes to the next one's
  Raw8<T> absent;
};
template <typename T> LF_DEV void load_token(bool there, int j, ScanLoad<T>& l, Raw8<T>* r) {
  r[j] = l.absent;
  if (there) r[j] = load8_raw<T>(l.p);
  l.p += l.step;
}
template <typename T, int TT, typename... More> LF_DEV void load_rows(int live, bool full, More&&... more) {
  auto all = [&](bool there, int j) { (load_token<T>(there, j, more.first, more.second), ...); };
  if (full) {   // (a whole workgroup's)
#pragma unroll
    for (int j = 0; j < TT; ++j) all(true, j);
  } else {
#pragma unroll
    for (int j = 0; j < TT; ++j) all(j < live, j);
  }
}
template <typename T> struct ScanPair { ScanLoad<T> first; Raw8<T>* second; };
template <typename T> LF_DEV ScanPair<T> rows_of(const void* base, const ScanView& v, const ScanRow& row, int b, long long n, int c, const Raw8<T>& absent, Raw8<T>* r) {
  return ScanPair<T>{ScanLoad<T>{at<T>(base, b * v.batch + n * v.token + c), row.step<T>(v), absent}, r};
}

// The stretches of a chunk joined: from each thread's (A, R) of 8 channels the value its first token starts from, given the
// chunk's; and the chunk's own (A, R).  Time lane of a thread: threadIdx.x / 8 in the recurrence's order (BACK: 31 minus that).
struct ScanJoin {
  float stretch[32][2][kScanWidth];   // [time lane]
  float wave[4][2][kScanWidth];
};

// A wave's LDS operations complete in the order in which they are issued: between its lanes no barrier is needed, only the order.
LF_DEV void lds_in_order() { asm volatile("" ::: "memory"); }

// before the barrier: `A`, `R` are replaced by those of the wave's stretches in front of this thread's (of the `seg` among which it is)
template <bool BACK> LF_DEV void join_wave(ScanJoin& s, float (&A)[8], float (&R)[8], int seg = 8) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = threadIdx.x >> 3, c = (lane & 7) * 8;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    *reinterpret_cast<f32x4*>(&s.stretch[at][0][c + 4 * q]) = f32x4{A[4 * q], A[4 * q + 1], A[4 * q + 2], A[4 * q + 3]};
    *reinterpret_cast<f32x4*>(&s.stretch[at][1][c + 4 * q]) = f32x4{R[4 * q], R[4 * q + 1], R[4 * q + 2], R[4 * q + 3]};
  }
  lds_in_order();
  float a[8], r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = wave * 8 + (BACK ? 7 - j : j);
    a[j] = s.stretch[t][0][lane];
    r[j] = s.stretch[t][1][lane];
  }
  float pa = 1.0f, pr = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = wave * 8 + (BACK ? 7 - j : j);
    if ((j & (seg - 1)) == 0) {
      pa = 1.0f;
      pr = 0.0f;
    }
    s.stretch[t][0][lane] = pa;
    s.stretch[t][1][lane] = pr;
    pr = __builtin_fmaf(a[j], pr, r[j]);
    pa *= a[j];
  }
  s.wave[wave][0][lane] = pa;
  s.wave[wave][1][lane] = pr;
  lds_in_order();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x4 va = *reinterpret_cast<const f32x4*>(&s.stretch[at][0][c + 4 * q]), vr = *reinterpret_cast<const f32x4*>(&s.stretch[at][1][c + 4 * q]);
#pragma unroll
    for (int j = 0; j < 4; ++j) { A[4 * q + j] = va[j]; R[4 * q + j] = vr[j]; }
  }
}

// behind the barrier, lane c of every wave for channel c: the chunk's (A, R) in front of the wave (upto = the wave's place in the
// order) or whole (upto = 4)
template <bool BACK> LF_DEV void join_chunk(const ScanJoin& s, int upto, float& A, float& R) {
  const int lane = threadIdx.x & 63;
  A = 1.0f;
  R = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int of = BACK ? 3 - w : w;
    const float a = s.wave[of][0][lane], r = s.wave[of][1][lane];
    if (w < upto) {
      R = __builtin_fmaf(a, R, r);
      A *= a;
    }
  }
}

// A value per lane (channel) handed to the lanes that hold 8 channels each, inside a wave, through 64 floats of LDS.
LF_DEV void spread8(float* lds, float v, float (&x)[8]) {
  const int lane = threadIdx.x & 63, c = (lane & 7) * 8;
  lds[lane] = v;
  lds_in_order();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x4 t = *reinterpret_cast<const f32x4*>(lds + c + 4 * q);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * q + j] = t[j];
  }
}

struct ScanPlace { int chunk, b, c0; };
inline __host__ __device__ int packed_tiles(int B, int seg) { return (int)(((long long)B * seg + 31) / 32); }

// A thread's batch row and its first token; packed: of the rows of a workgroup its own (`on`: whether there is one).
template <bool PACKED> struct ScanThread {
  int b, t0;
  bool on;
  LF_DEV ScanThread(const ScanPlace& p, int c, int B, int C, int seg, int tokens, int chunk) : b(p.b), on(c < C) {
    const int at = threadIdx.x >> 3;
    if constexpr (PACKED) {
      b = p.b * (32 / seg) + at / seg;
      on = on && b < B;
      b = b < B ? b : B - 1;
      t0 = (at & (seg - 1)) * tokens;
    } else {
      t0 = p.chunk * chunk + at * tokens;
    }
  }
};


// ---- between chunks ----------------------------------------------------------------------------------------------------

constexpr unsigned kNotYet = 0xffffffffu;
LF_DEV unsigned told(float v) { return v != v ? 0x7fc00000u : __builtin_bit_cast(unsigned, v); }   // (never kNotYet)

LF_DEV void tell_totals(unsigned long long* p, float A, float R) {
  __hip_atomic_store(p, (unsigned long long)told(R) << 32 | told(A), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
LF_DEV void tell_value(unsigned* p, float h) { __hip_atomic_store(p, told(h), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

template <typename W> LF_DEV W heard(const W* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// `w` as it was read from `p`, read again until it is there (lanes that read nothing have 0)
template <typename W> LF_DEV void await(W& w, const W* p) {
  while (__any((unsigned)w == kNotYet)) {
    __builtin_amdgcn_s_sleep(1);
    if ((unsigned)w == kNotYet) w = heard(p);
  }
}

// How a row's chunks hear of one another.  kAlone: there is one.  kGroups: in groups; a group's last chunk tells the value behind it, so a row is a
// chain of groups.  kStretches: the groups in stretches of as many; a group's last chunk tells the group's totals, a stretch's last one the value behind
// it, so a row is a chain of stretches, for rows with too few channels beside one another to hide the longer chain.  kPacked: rows of 32 tokens or
// fewer, several in a workgroup: `seg` time lanes (1, 2, 4 or 8) each, nothing to be told and no barrier.
constexpr int kAlone = 0, kGroups = 1, kStretches = 2, kPacked = 3;

constexpr int kScanGroup = 16;   // chunks of a group, groups of a stretch, at most
struct ScanFound { float value[kScanWidth]; };

// The value that a chunk starts from, lane c's for its channel: from the value behind the group of chunks before its own (its row's first
// one, `start`, in the first group) through the totals of its group's chunks before it, one after the other.  Only a group's last chunk
// tells its value, so that results do not depend on who was first, and a chunk reads 16 totals or fewer, not a row's.  `order`: the chunk's
// place in its row's order (backward: from the row's end); `i0`: its record for this channel, `next`: from a chunk's record to the one's
// after it in the order.  `totals`: LDS for `group` of them.
LF_DEV float look_back(const ScanRecords& r, ScanFound& lds, float (&totals)[32][2][kScanWidth], int group, int order, long long i0, long long next,
                       float start, bool on) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int before = order % group;   // chunks of the group before this one
  if (wave == 0) {
    float v = start;
    if (order >= group) {
      const unsigned* p = r.values + i0 - next * (before + 1);
      unsigned w = 0;
      if (on) w = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      while (__any(w == kNotYet)) {
        __builtin_amdgcn_s_sleep(1);
        if (w == kNotYet) w = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      v = __builtin_bit_cast(float, w);
    }
    lds.value[lane] = v;
  }
  // The waves take the chunks in turn, from the furthest on; those of a wave are requested together, four at a time.  (Written out: with await
  // bf16 takes two registers more, so that three workgroups share a CU and not four: 65536 x 1280 194 us for 179.)
  for (int e0 = wave; e0 < before; e0 += 16) {
    unsigned long long t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      t[k] = 0;
      if (on && e0 + 4 * k < before)
        t[k] = __hip_atomic_load(r.totals + i0 - next * (before - e0 - 4 * k), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      while (__any((unsigned)t[k] == kNotYet)) {
        __builtin_amdgcn_s_sleep(1);
        if ((unsigned)t[k] == kNotYet)
          t[k] = __hip_atomic_load(r.totals + i0 - next * (before - e0 - 4 * k), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      if (e0 + 4 * k < before) {
        totals[e0 + 4 * k][0][lane] = __builtin_bit_cast(float, (unsigned)t[k]);
        totals[e0 + 4 * k][1][lane] = __builtin_bit_cast(float, (unsigned)(t[k] >> 32));
      }
    }
  }
  __syncthreads();
  float h = lds.value[lane];
  for (int e = 0; e < before; ++e) h = __builtin_fmaf(totals[e][0][lane], h, totals[e][1][lane]);
  return h;
}

// A group's totals: eight bytes a channel in the rows of `values` of its last chunk, whose record for channel c is i, and of the one before.
LF_DEV unsigned long long* group_totals(const ScanRecords& r, long long i, long long next, int c) {
  return reinterpret_cast<unsigned long long*>(r.values + (i - c - (next > 0 ? next : 0))) + c;
}

// The same with stretches: from the value behind the stretch before (`start` in the first) through the totals of this stretch's groups before and of
// this group's chunks before.  c: the channel; A, R: the chunk's totals, of which a group's last chunk makes the group's.  The value behind
// a stretch is told in the row before those of its last group's totals.  `totals`: 16 KB of LDS.
LF_DEV float look_far(const ScanRecords& r, ScanFound& lds, float (&totals)[32][2][kScanWidth], int group, int order, long long i0, long long next,
                      int c, float start, float A, float R, bool on) {
  constexpr int kEach = kScanGroup / 4;   // of a wave
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int before = order % group, groups = order / group % group;   // chunks, groups before this one
  const long long last = i0 - next * (before + 1);                    // the last chunk of the group before
  // the waves take the chunks and the groups in turn, from the furthest on; all of a wave's are requested together
  unsigned long long t[kEach], g[kEach];
  unsigned w = 0;
  const bool far = wave == 0 && order >= group * group;
  const unsigned* const from = r.values + last - next * ((long long)groups * group + 2);
  if (far && on) w = heard(from);
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int e = wave + 4 * k;
    t[k] = g[k] = 0;
    if (on && e < before) t[k] = heard(r.totals + i0 - next * (before - e));
    if (on && e < groups) g[k] = heard(group_totals(r, last - next * ((long long)(groups - 1 - e) * group), next, c));
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int e = wave + 4 * k;
    await(t[k], r.totals + i0 - next * (before - e));
    if (e < before) {
      totals[kScanGroup + e][0][lane] = __builtin_bit_cast(float, (unsigned)t[k]);
      totals[kScanGroup + e][1][lane] = __builtin_bit_cast(float, (unsigned)(t[k] >> 32));
    }
  }
  if (before == group - 1) {
    __syncthreads();
    if (wave == 0) {
      float ga = 1.0f, gr = 0.0f;
      for (int e = 0; e < before; ++e) {
        const float a = totals[kScanGroup + e][0][lane];
        gr = __builtin_fmaf(a, gr, totals[kScanGroup + e][1][lane]);
        ga *= a;
      }
      if (on) tell_totals(group_totals(r, i0, next, c), ga * A, __builtin_fmaf(A, gr, R));
    }
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int e = wave + 4 * k;
    await(g[k], group_totals(r, last - next * ((long long)(groups - 1 - e) * group), next, c));
    if (e < groups) {
      totals[e][0][lane] = __builtin_bit_cast(float, (unsigned)g[k]);
      totals[e][1][lane] = __builtin_bit_cast(float, (unsigned)(g[k] >> 32));
    }
  }
  if (far) {
    await(w, from);
    start = __builtin_bit_cast(float, w);
  }
  if (wave == 0) lds.value[lane] = start;
  __syncthreads();
  float h = lds.value[lane];
  for (int e = 0; e < groups; ++e) h = __builtin_fmaf(totals[e][0][lane], h, totals[e][1][lane]);
  for (int e = 0; e < before; ++e) h = __builtin_fmaf(totals[kScanGroup + e][0][lane], h, totals[kScanGroup + e][1][lane]);
  return h;
}

// Records to "not yet", the ticket to 0.
__global__ __launch_bounds__(256) void scan_clear(ScanRecords r, long long count) {
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 2;
  if (i == 0) *r.ticket = 0;
  if (i >= count) return;   // (count is even)
  *reinterpret_cast<u32x4*>(r.totals + i) = u32x4{kNotYet, kNotYet, kNotYet, kNotYet};
  *reinterpret_cast<u32x2*>(r.values + i) = u32x2{kNotYet, kNotYet};
}

// A workgroup's tile: a chunk of a batch row and 64 channels, by ticket (ONE: by its index): a chunk of all rows and channels, then the
// next one.  Waiting for the ticket costs 17 of 160 us (65536 x 1280 bf16); workgroups that stay and draw their next ticket early hold it while
// others wait for its tile (218 us, 176 when drawn as late as the results' way out), and several tiles a ticket leave fewer chunks under way
// (two 190, four 214).
template <bool ONE, bool BACK> LF_DEV ScanPlace take_tile(const ScanRecords& r, int B, int C, int chunks, unsigned& lds) {
  unsigned id = blockIdx.x;
  if constexpr (!ONE) {
    if (threadIdx.x == 0) lds = __hip_atomic_fetch_add(r.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    id = (unsigned)__builtin_amdgcn_readfirstlane((int)lds);
  }
  const unsigned blocks = (unsigned)(C + kScanWidth - 1) / kScanWidth, per = blocks * (unsigned)B;
  const unsigned at = id / per, rest = id - at * per, b = rest / blocks;
  return ScanPlace{BACK ? chunks - 1 - (int)at : (int)at, (int)b, (int)(rest - b * blocks) * kScanWidth};
}

// ---- forward -----------------------------------------------------------------------------------------------------------

struct ScanForwardLds {
  ScanJoin join;
  ScanFound found;
  float spread[4][kScanWidth];
  unsigned id;
};
// TT tokens a thread.
// Bound: HBM and vector instructions, nearly level (46 issue slots a value with the norm's weight, six of them transcendental: the vector
// units are busy 62 % of the time), then the wait for a ticket (take_tile).
template <typename T, int MODE, bool INPUT, int TT, int CHAIN>
__global__ __launch_bounds__(256) void scan_fwd(ScanArgs a) {
  constexpr int L = 32 * TT;
  constexpr bool ONE = CHAIN == kAlone || CHAIN == kPacked;
  constexpr bool kPrecise = Stored<T>::kBytes == 4;
  __shared__ ScanForwardLds shared;
  ScanJoin& lds = shared.join;
  const ScanPlace p = take_tile<ONE, false>(a.rec, CHAIN == kPacked ? packed_tiles(a.B, a.seg) : a.B, a.C, a.chunks, shared.id);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = p.c0 + (lane & 7) * 8, cl = p.c0 + lane;
  const ScanThread<CHAIN == kPacked> me(p, c, a.B, a.C, a.seg, TT, L);
  const bool on = me.on;
  const ScanRow row(a.lengths, me.b, a.N, a.reverse);
  const int t0 = me.t0;
  if (p.chunk && (long long)p.chunk * L >= row.n) return;   // (the whole workgroup)
  const int live = on ? (row.n - t0 < TT ? (int)(row.n - t0) : TT) : 0;   // this thread's tokens that count (below 0: none)
  Raw8<T> rx[TT], rg[TT], ri[INPUT ? TT : 1];
  const bool full = CHAIN != kPacked && (long long)(p.chunk + 1) * L <= row.n && p.c0 + kScanWidth <= a.C;
  float rate[8], h0 = 0.0f;   // (rate requested first: loads are waited for in their order)
  load_rate(a.rate + c, on, rate);
  {
    const long long n = row.token(t0);
    ScanPair<T> g = rows_of<T>(a.gate, a.vg, row, me.b, n, c, shut8<T>(), rg), x = rows_of<T>(a.x, a.vx, row, me.b, n, c, none8<T>(), rx);
    if constexpr (INPUT) load_rows<T, TT>(live, full, g, x, rows_of<T>(a.input, a.vi, row, me.b, n, c, none8<T>(), ri));
    else load_rows<T, TT>(live, full, g, x);
  }
  if (CHAIN != kPacked && cl < a.C && a.state_in && (ONE || p.chunk < (CHAIN == kStretches ? a.group * a.group : a.group))) h0 = a.state_in[(long long)p.b * a.C + cl];
  float da[TT][8], u[TT][8], A[8], R[8];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    float x[8], g[8], in[8];
    widen8<T>(rx[j], x);
    widen8<T>(rg[j], g);
    if constexpr (INPUT) widen8<T>(ri[j], in);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float d = rate[k] * 1.44269504088896340736f * sigmoid_of<kPrecise>(g[k]);
      da[j][k] = __builtin_amdgcn_exp2f(-d);
      u[j][k] = weight_of<kPrecise, MODE>(d, da[j][k]) * x[k];
      if constexpr (INPUT) u[j][k] *= sigmoid_of<kPrecise>(in[k]);
      R[k] = j ? __builtin_fmaf(da[j][k], R[k], u[j][k]) : u[j][k];
      A[k] = j ? A[k] * da[j][k] : da[j][k];
    }
  }
  float h[8];
  if constexpr (CHAIN == kPacked) {
    join_wave<false>(lds, A, R, a.seg);
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = 0.0f;
    if (on && a.state_in) load8_f32(a.state_in + (long long)me.b * a.C + c, h);
    if (on && a.saved && t0 == 0) store8<F32>(reinterpret_cast<unsigned char*>(a.saved + (long long)me.b * a.C + c), h);
  } else {
    join_wave<false>(lds, A, R);
    arrive(h0);
    __syncthreads();
    float ca, cr;
    const long long row0 = (long long)p.b * a.chunks * a.C + cl;
    const bool whole = wave == 0 && cl < a.C;   // the threads that speak for the chunk
    const long long i0 = row0 + (long long)p.chunk * a.C;
    if constexpr (!ONE) {
      join_chunk<false>(lds, 4, ca, cr);
      if (whole) tell_totals(a.rec.totals + i0, ca, cr);
      if constexpr (CHAIN == kGroups) h0 = look_back(a.rec, shared.found, lds.stretch, a.group, p.chunk, i0, a.C, h0, cl < a.C);
      else h0 = look_far(a.rec, shared.found, lds.stretch, a.group, p.chunk, i0, a.C, cl, h0, ca, cr, cl < a.C);
    }
    if (whole) {
      join_chunk<false>(lds, 4, ca, cr);
      const float end = __builtin_fmaf(ca, h0, cr);
      if (CHAIN == kGroups && p.chunk % a.group == a.group - 1) tell_value(a.rec.values + i0, end);
      if (CHAIN == kStretches && p.chunk % (a.group * a.group) == a.group * a.group - 1) tell_value(a.rec.values + i0 - 2 * a.C, end);
      if (a.state_out && (long long)(p.chunk + 1) * L >= row.n) a.state_out[(long long)p.b * a.C + cl] = end;   // the last token is here
    }
    join_chunk<false>(lds, wave, ca, cr);
    const float mine = __builtin_fmaf(ca, h0, cr);   // the state before the wave's tokens
    if (a.saved && cl < a.C && wave * 8 * TT % kScanChunk == 0) {
      const long long t = (long long)p.chunk * L + wave * 8 * TT;
      if (t == 0 || t < row.n) a.saved[((long long)p.b * a.saved_chunks + t / kScanChunk) * a.C + cl] = mine;
    }
    spread8(shared.spread[wave], mine, h);
  }
  if (!a.out) return;
  unsigned char* po = at<T>(a.out, me.b * a.vo.batch + row.token(t0) * a.vo.token + c);
  const long long so = row.step<T>(a.vo);
#pragma unroll
  for (int k = 0; k < 8; ++k) h[k] = __builtin_fmaf(A[k], h[k], R[k]);
#pragma unroll
  for (int j = 0; j < TT; ++j) {
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = __builtin_fmaf(da[j][k], h[k], u[j][k]);
    if (j < live) store8_stream<T>(po, h);
    po += so;
  }
  if constexpr (CHAIN == kPacked) {   // whose tokens reach the last that counts (without any: the first)
    const bool ends = row.n > t0 ? row.n <= t0 + TT : (row.n == 0 && t0 == 0);
    if (on && a.state_out && ends) store8<F32>(reinterpret_cast<unsigned char*>(a.state_out + (long long)me.b * a.C + c), h);
  }
}

// ---- backward ----------------------------------------------------------------------------------------------------------

// The gradients of a chunk, from the state in front of it and E behind it, which comes from the chunks behind as the state does from
// those before.  Bound: registers, which leave two workgroups a CU (three spill: 100 us where two take 60, 12 x 4096 x 320 bf16), and for fp32 with a gate on
// the inputs not even those: 3 to 9 values a lane go through scratch, 23 to 27 in a chain of stretches.
struct ScanBackLds {
  ScanJoin there, back;
  ScanFound found;
  float spread[2][4][kScanWidth];
  f32x4 weights[kScanT][2][256];
  unsigned id;
};
template <typename T, int MODE, bool INPUT, int CHAIN>
__global__ __launch_bounds__(256, 2) void scan_bwd(ScanBackArgs a) {
  constexpr int TT = kScanT, L = kScanChunk;
  constexpr bool ONE = CHAIN == kAlone || CHAIN == kPacked;
  constexpr bool kPrecise = Stored<T>::kBytes == 4;
  __shared__ ScanBackLds shared;
  ScanJoin &there = shared.there, &back = shared.back;
  const ScanPlace p = take_tile<ONE, true>(a.rec, CHAIN == kPacked ? packed_tiles(a.B, a.seg) : a.B, a.C, a.chunks, shared.id);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = p.c0 + (lane & 7) * 8, cl = p.c0 + lane;
  const ScanThread<CHAIN == kPacked> me(p, c, a.B, a.C, a.seg, TT, L);
  const bool on = me.on;
  const ScanRow row(a.lengths, me.b, a.N, a.reverse);
  const long long row0 = (long long)p.b * a.chunks * a.C + cl, at0 = row0 + (long long)p.chunk * a.C;
  const int last = row.n ? (int)((row.n - 1) / L) : 0;   // (packed: 0)
  if (p.chunk > last) {   // (the whole workgroup)
    if (wave == 0 && cl < a.C) a.partials[at0] = 0.0f;
    return;
  }
  const int t0 = me.t0;
  const int live = on ? (row.n - t0 < TT ? (int)(row.n - t0) : TT) : 0;
  const long long n0 = row.token(t0);
  Raw8<T> rx[TT], rg[TT], ri[INPUT ? TT : 1], rd[TT];
  const bool full = CHAIN != kPacked && (long long)(p.chunk + 1) * L <= row.n && p.c0 + kScanWidth <= a.C;
  float rate[8], h0 = 0.0f, e0 = 0.0f;
  load_rate(a.rate + c, on, rate);
  if (CHAIN != kPacked && cl < a.C) h0 = a.starts[at0];
  if (CHAIN != kPacked && cl < a.C && a.dstate_out && (ONE || last - p.chunk < (CHAIN == kStretches ? a.group * a.group : a.group))) e0 = a.dstate_out[(long long)p.b * a.C + cl];
  {
    ScanPair<T> g = rows_of<T>(a.gate, a.vg, row, me.b, n0, c, shut8<T>(), rg), x = rows_of<T>(a.x, a.vx, row, me.b, n0, c, none8<T>(), rx);
    ScanPair<T> d = rows_of<T>(a.dout, a.vd, row, me.b, n0, c, none8<T>(), rd);
    if constexpr (INPUT) load_rows<T, TT>(live, full, g, x, rows_of<T>(a.input, a.vi, row, me.b, n0, c, none8<T>(), ri), d);
    else load_rows<T, TT>(live, full, g, x, d);
  }
  // (m i waits in LDS: with it and what follows from it in registers 75 of them spill)
  float da[TT][8], u[TT][8], sg[TT][8], A[8], R[8], BA[8], BR[8];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    float x[8], g[8], in[8], mi[8];
    widen8<T>(rx[j], x);
    widen8<T>(rg[j], g);
    if constexpr (INPUT) widen8<T>(ri[j], in);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float s;
      sg[j][k] = smaller_sigmoid<kPrecise>(g[k], s);
      const float d = rate[k] * 1.44269504088896340736f * s, ak = __builtin_amdgcn_exp2f(-d);
      da[j][k] = ak;
      mi[k] = weight_of<kPrecise, MODE>(d, ak);
      if constexpr (INPUT) mi[k] *= sigmoid_of<kPrecise>(in[k]);
      u[j][k] = mi[k] * x[k];
      R[k] = j ? __builtin_fmaf(ak, R[k], u[j][k]) : u[j][k];
      A[k] = j ? A[k] * ak : ak;
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) shared.weights[j][q][threadIdx.x] = f32x4{mi[4 * q], mi[4 * q + 1], mi[4 * q + 2], mi[4 * q + 3]};
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) { BA[k] = A[k]; BR[k] = 0.0f; }
#pragma unroll
  for (int j = TT - 1; j >= 0; --j) {
    float d[8];
    widen8<T>(rd[j], d);
#pragma unroll
    for (int k = 0; k < 8; ++k) BR[k] = da[j][k] * (BR[k] + d[k]);
  }
  float h[8], E[8];
  const bool whole = wave == 0 && cl < a.C;
  if constexpr (CHAIN == kPacked) {
    join_wave<false>(there, A, R, a.seg);
    join_wave<true>(back, BA, BR, a.seg);
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = E[k] = 0.0f;
    const long long of = (long long)me.b * a.C + c;
    if (on) load8_f32(a.starts + of, h);
    if (on && a.dstate_out) load8_f32(a.dstate_out + of, E);
  } else {
    join_wave<false>(there, A, R);
    join_wave<true>(back, BA, BR);
    arrive(e0);
    __syncthreads();
    float ca, cr;
    if constexpr (!ONE) {
      join_chunk<true>(back, 4, ca, cr);
      if (whole) tell_totals(a.rec.totals + at0, ca, cr);
      if constexpr (CHAIN == kGroups) e0 = look_back(a.rec, shared.found, back.stretch, a.group, last - p.chunk, at0, -(long long)a.C, e0, cl < a.C);
      else e0 = look_far(a.rec, shared.found, back.stretch, a.group, last - p.chunk, at0, -(long long)a.C, cl, e0, ca, cr, cl < a.C);
    }
    if (whole) {
      join_chunk<true>(back, 4, ca, cr);
      const float end = __builtin_fmaf(ca, e0, cr);
      if (CHAIN == kGroups && (last - p.chunk) % a.group == a.group - 1) tell_value(a.rec.values + at0, end);
      if (CHAIN == kStretches && (last - p.chunk) % (a.group * a.group) == a.group * a.group - 1) tell_value(a.rec.values + at0 + 2 * a.C, end);
      if (a.dstate_in && p.chunk == 0) a.dstate_in[(long long)p.b * a.C + cl] = end;
    }
    join_chunk<false>(there, wave, ca, cr);
    spread8(shared.spread[0][wave], __builtin_fmaf(ca, h0, cr), h);
    join_chunk<true>(back, 3 - wave, ca, cr);
    spread8(shared.spread[1][wave], __builtin_fmaf(ca, e0, cr), E);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    h[k] = __builtin_fmaf(A[k], h[k], R[k]);
    E[k] = __builtin_fmaf(BA[k], E[k], BR[k]);
  }
#pragma unroll
  for (int j = 0; j < TT; ++j)   // u: the state before the token
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float v = u[j][k];
      u[j][k] = h[k];
      h[k] = __builtin_fmaf(da[j][k], h[k], v);
    }
  float by_rate[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) by_rate[k] = 0.0f;
  const long long sdx = row.step<T>(a.vdx), sdg = row.step<T>(a.vdg), sdi = row.step<T>(a.vdi);
  unsigned char* pdx = at<T>(a.dx, me.b * a.vdx.batch + n0 * a.vdx.token + c) + (TT - 1) * sdx;
  unsigned char* pdg = at<T>(a.dgate, me.b * a.vdg.batch + n0 * a.vdg.token + c) + (TT - 1) * sdg;
  unsigned char* pdi = at<T>(a.dinput, me.b * a.vdi.batch + n0 * a.vdi.token + c) + (TT - 1) * sdi;
#pragma unroll
  for (int j = TT - 1; j >= 0; --j) {
    float x[8], in[8], d[8], dx[8], dg[8], di[8];
    forget(rx[j]);
    widen8<T>(rx[j], x);
    if constexpr (INPUT) {
      forget(ri[j]);
      widen8<T>(ri[j], in);
    }
    widen8<T>(rd[j], d);
    const f32x4 w0 = shared.weights[j][0][threadIdx.x], w1 = shared.weights[j][1][threadIdx.x];
#pragma unroll
    for (int k = 0; k < 8; ++k) {   // (a token that does not count: D = E, s = m = 0, a = 1)
      const float D = d[k] + E[k], mi = k < 4 ? w0[k & 3] : w1[k & 3];
      const float v = sg[j][k], other = 1.0f - __builtin_fabsf(v), s = __builtin_bit_cast(int, v) < 0 ? other : v;
      float i = 1.0f;
      dx[k] = D * mi;
      if constexpr (INPUT) {
        float e;
        i = sigmoid_of<kPrecise>(in[k], e);
        di[k] = dx[k] * x[k] * (__builtin_fminf(e, 0x1p126f) * i);   // 1 - i = e i (and no infinity times 0 where i, and so dx, is 0)
      }
      E[k] = da[j][k] * D;
      // -dg = a D (r i x - h') with dm/dg = -a r: r = a / m, 1, 0
      float rix = 0.0f;
      if constexpr (MODE == kScanLeaky) rix = i * x[k];
      if constexpr (MODE == kScanNorm) rix = below(mi, 1.17549435e-38f, 0.0f, da[j][k] * (i * __builtin_amdgcn_rcpf(mi))) * (i * x[k]);
      const float part = E[k] * (rix - u[j][k]);
      by_rate[k] = __builtin_fmaf(part, s, by_rate[k]);
      dg[k] = part * rate[k] * (__builtin_fabsf(v) * other);
    }
    if (j < live) {
      store8_stream<T>(pdx, dx);
      store8_stream<T>(pdg, dg);
      if constexpr (INPUT) store8_stream<T>(pdi, di);
    }
    pdx -= sdx;
    pdg -= sdg;
    pdi -= sdi;
  }
  if (CHAIN == kPacked && on && a.dstate_in && t0 == 0) store8<F32>(reinterpret_cast<unsigned char*>(a.dstate_in + (long long)me.b * a.C + c), E);
  __syncthreads();   // the stretches' LDS takes the sums
#pragma unroll
  for (int q = 0; q < 2; ++q)
    *reinterpret_cast<f32x4*>(&there.stretch[threadIdx.x >> 3][0][(lane & 7) * 8 + 4 * q]) =
        f32x4{by_rate[4 * q], by_rate[4 * q + 1], by_rate[4 * q + 2], by_rate[4 * q + 3]};
  __syncthreads();
  if (whole) {
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j) sum += there.stretch[j][0][lane];
    a.partials[at0] = sum;
  }
}

// drate: the chunks' sums of every batch row.
__global__ __launch_bounds__(1024) void scan_rate_sums(const float* partials, float* drate, long long parts, int C) {
  __shared__ double lds[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15);
  const double sum = column_sum(lds, partials, parts, C, c);
  if (threadIdx.x < 16 && c < C) drate[c] = (float)sum;
}

struct ScanStepArgs {
  const void *x, *gate, *input;
  void* out;
  long long sx, sg, si, so;
  const float *rate, *state_in;
  float* state_out;
  int B, C;
};

// One token of every batch row: a thread takes 8 channels.
template <typename T, int MODE, bool INPUT>
__global__ __launch_bounds__(64) void scan_step(ScanStepArgs a) {
  constexpr bool kPrecise = Stored<T>::kBytes == 4;
  const int b = blockIdx.y, c = (blockIdx.x * 64 + threadIdx.x) * 8;
  if (c >= a.C) return;
  const Raw8<T> rx = load8_raw<T>(at<T>(a.x, b * a.sx + c)), rg = load8_raw<T>(at<T>(a.gate, b * a.sg + c));
  Raw8<T> ri = none8<T>();
  if constexpr (INPUT) ri = load8_raw<T>(at<T>(a.input, b * a.si + c));
  float x[8], g[8], in[8], rate[8], h[8];
  load8_f32(a.rate + c, rate);
  const long long at0 = (long long)b * a.C + c;
#pragma unroll
  for (int k = 0; k < 8; ++k) h[k] = 0.0f;
  if (a.state_in) load8_f32(a.state_in + at0, h);
  widen8<T>(rx, x);
  widen8<T>(rg, g);
  widen8<T>(ri, in);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float d = rate[k] * 1.44269504088896340736f * sigmoid_of<kPrecise>(g[k]), da = __builtin_amdgcn_exp2f(-d);
    float v = weight_of<kPrecise, MODE>(d, da) * x[k];
    if constexpr (INPUT) v *= sigmoid_of<kPrecise>(in[k]);
    h[k] = __builtin_fmaf(da, h[k], v);
  }
  if (a.state_out) store8<F32>(reinterpret_cast<unsigned char*>(a.state_out + at0), h);
  store8<T>(at<T>(a.out, b * a.so + c), h);
}

}  // namespace lf
