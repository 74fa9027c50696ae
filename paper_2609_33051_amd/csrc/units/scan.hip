// The selective scan of packed prompts (Mamba-2 form), by chunks of 64 tokens on
// the matrix cores.  With g_t the sum of log decays from the chunk's start and
// S the state before it,
//     y_t = e^{g_t} S C_t + sum_{s <= t} e^{g_t - g_s} dt_s <B_s, C_t> x_s + D x_t,
//     S' = e^{g_L} S + sum_s (e^{g_L - g_s} dt_s x_s) B_s^T,
// every exponent <= 0.  A workgroup of four waves owns 128 value channels (one
// head, or two of a group: the scores <B_s, C_t> are theirs together) and a run of
// tokens, and goes through it chunk by chunk; the state stays in registers (32 value
// channels a wave) and each input is read once, a chunk ahead.
//
// Fragments.  Both operands of a product hold, per lane, 8 consecutive indices of
// a 32-deep reduction (lane group g = lane / 16: 8 g .. 8 g + 7) of the row or
// column lane % 16.  The state's accumulator tiles are assigned to channels so
// that two of them are such a fragment as they lie: tile kt, row m is channel
// 32 (kt / 2) + 8 (m / 4) + 4 (kt % 2) + m % 4.
//
// Long sequences: a sequence is split into segments of `seg` tokens, a fair
// share of the card.  A first launch runs the state part of every segment but a
// sequence's last, from zero (the first: from S_in), and keeps its end state and
// total decay; the second begins each segment from the states before it, joined.
#include <type_traits>

#include "../mixer.h"

namespace skssm {

constexpr int kChunk = 64;
constexpr int kValues = 128;        // value channels of a workgroup
constexpr int kGates = 4 * kChunk;  // tokens whose gates are computed together, a chunk per wave
// places in a chunk's record of gates (floats)
constexpr int kLeft = 0, kEnd = 64, kLocalRecord = 68, kLocal = 68, kStep = 196, kGate = 324, kPass = 388, kRecord = 484;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// 64 rows of COLS elements in LDS, for reads of 16 bytes of a row by the lanes of
// consecutive rows: the 16-byte chunks of a row are permuted by the row, so that the
// eight rows a read takes at once lie in different banks.
template <typename IO, int COLS> struct RowTile {
  static constexpr int kBytes = kChunk * COLS * (int)sizeof(IO), kChunks = COLS * (int)sizeof(IO) / 16;
  static constexpr int kPer = 16 / (int)sizeof(IO);  // elements of a chunk
  static __device__ __forceinline__ int at(int row, int col) {  // byte offset
    return row * (COLS * (int)sizeof(IO)) + (((col / kPer) ^ (row & 7)) << 4) + (col % kPer) * (int)sizeof(IO);
  }
};
// The same where columns are read too.  fp32: as above.  bf16: a transposed read takes
// 8-byte pieces of four rows, channels 32 q + 8 p + 4 h .. + 3 for p = 0..3: these are made
// neighbours (32 bytes: unit h COLS / 32 + q of the row), units are permuted by the row's
// low bits, so that the four rows cover 128 bytes, and pieces by the next two, so that
// 16 rows of one piece do.
template <typename IO, int COLS> struct ColTile : RowTile<IO, COLS> {};
template <int COLS> struct ColTile<bf16_t, COLS> : RowTile<bf16_t, COLS> {
  static __device__ __forceinline__ int at(int row, int col) {
    const int unit = ((col >> 2) & 1) * (COLS / 32) + (col >> 5), piece = (col >> 3) & 3;
    return row * (COLS * 2) + ((unit ^ (row & 3)) << 5) + ((piece ^ ((row >> 2) & 3)) << 3) + (col & 3) * 2;
  }
};

struct FragF32 { float e[8]; };

template <typename IO> struct Frags;
template <> struct Frags<bf16_t> {
  using F = bf16x8;
  // 8 consecutive columns of one row of a RowTile, and of a ColTile, from the places of the
  // first four and the last four
  static __device__ __forceinline__ F row(const char* t, const uint32_t* at, int off) {
    return __builtin_bit_cast(F, *reinterpret_cast<const uint4*>(t + at[0] + off));
  }
  static __device__ __forceinline__ F row_c(const char* t, const uint32_t* at, int off) {
    const uint2 a = *reinterpret_cast<const uint2*>(t + at[0] + off), b = *reinterpret_cast<const uint2*>(t + at[1] + off);
    return __builtin_bit_cast(F, make_uint4(a.x, a.y, b.x, b.y));
  }
  template <int COLS> static __device__ __forceinline__ void put_c(char* t, int row, int col, uint4 x) {
    *reinterpret_cast<uint2*>(t + ColTile<bf16_t, COLS>::at(row, col)) = make_uint2(x.x, x.y);
    *reinterpret_cast<uint2*>(t + ColTile<bf16_t, COLS>::at(row, col + 4)) = make_uint2(x.z, x.w);
  }
  // 8 consecutive rows of the column that the lane's place i = lane % 16 stands for, where
  // places 4 p .. 4 p + 3 are four consecutive columns: a transposed read takes, from
  // the 16 lanes of a group, four rows (i / 4) of four 8-byte pieces (i % 4)
  static constexpr int kCols = 2;  // places a lane holds: of row i / 4 and of row 4 + i / 4
  template <int COLS> static __device__ __forceinline__ void cols_at(uint32_t* at, int row0, int i, int col0, int step) {
#pragma unroll
    for (int q = 0; q < 2; ++q) at[q] = ColTile<bf16_t, COLS>::at(row0 + 4 * q + (i >> 2), col0 + step * (i & 3));
  }
  // (odd: the same places four columns on, COLS / 32 units)
  template <int COLS> static __device__ __forceinline__ F cols(const char* t, const uint32_t* at, int off, int odd) {
    typedef __attribute__((address_space(3))) shortx4* lds4;
    const uint32_t a = COLS == 128 ? at[0] + 128 * odd : at[0] ^ (COLS * odd), b = COLS == 128 ? at[1] + 128 * odd : at[1] ^ (COLS * odd);
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(t + a + off));
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(t + b + off));
    return __builtin_bit_cast(F, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  static __device__ __forceinline__ floatx4 mma(F a, F b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ F of(floatx4 lo, floatx4 hi) {
    return __builtin_bit_cast(F, make_uint4(bf16_pack2(lo[0], lo[1]), bf16_pack2(lo[2], lo[3]), bf16_pack2(hi[0], hi[1]), bf16_pack2(hi[2], hi[3])));
  }
  static __device__ __forceinline__ void store4(char* t, int at, float a, float b, float c, float d) {
    *reinterpret_cast<uint2*>(t + at) = make_uint2(bf16_pack2(a, b), bf16_pack2(c, d));
  }
};
template <> struct Frags<float> {
  using F = FragF32;
  static __device__ __forceinline__ F row(const char* t, const uint32_t* at, int off) {
    F f;
    const float4 a = *reinterpret_cast<const float4*>(t + at[0] + off), b = *reinterpret_cast<const float4*>(t + at[1] + off);
    f.e[0] = a.x; f.e[1] = a.y; f.e[2] = a.z; f.e[3] = a.w;
    f.e[4] = b.x; f.e[5] = b.y; f.e[6] = b.z; f.e[7] = b.w;
    return f;
  }
  static constexpr int kCols = 8;
  template <int COLS> static __device__ __forceinline__ void cols_at(uint32_t* at, int row0, int i, int col0, int step) {
#pragma unroll
    for (int q = 0; q < 8; ++q) at[q] = ColTile<float, COLS>::at(row0 + q, col0 + step * (i >> 2) + (i & 3));
  }
  static __device__ __forceinline__ F row_c(const char* t, const uint32_t* at, int off) { return row(t, at, off); }
  template <int COLS> static __device__ __forceinline__ void put_c(char* t, int row, int col, uint4 x) {
    *reinterpret_cast<uint4*>(t + ColTile<float, COLS>::at(row, col)) = x;
  }
  // (odd: the same places four columns on, the other chunk of a pair)
  template <int COLS> static __device__ __forceinline__ F cols(const char* t, const uint32_t* at, int off, int odd) {
    F f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.e[e] = *reinterpret_cast<const float*>(t + (at[e] ^ (16 * odd)) + off);
    return f;
  }
  static __device__ __forceinline__ floatx4 mma(const F& a, const F& b, floatx4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.e[e], b.e[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ F of(floatx4 lo, floatx4 hi) {
    F f;
#pragma unroll
    for (int e = 0; e < 4; ++e) { f.e[e] = lo[e]; f.e[e + 4] = hi[e]; }
    return f;
  }
  static __device__ __forceinline__ void store4(char* t, int at, float a, float b, float c, float d) {
    *reinterpret_cast<float4*>(t + at) = make_float4(a, b, c, d);
  }
};

// x weighted per token, as the state's update takes it: fp32, or three bf16 parts that
// hold the product's 24 bits (two leave the state 2e-6 off, six times what fp32
// sums do).
template <typename IO> struct Weighted;
template <> struct Weighted<float> {
  static constexpr int kParts = 1;
  FragF32 f;
  __device__ __forceinline__ void set(const FragF32& x, const float* w) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.e[e] = x.e[e] * w[e];
  }
  __device__ __forceinline__ const FragF32& part(int) const { return f; }
};
template <> struct Weighted<bf16_t> {
  static constexpr int kParts = 3;
  uint4 p[kParts];
  __device__ __forceinline__ void set(bf16x8 x, const float* w) {
    const uint4 u = __builtin_bit_cast(uint4, x);
    const uint32_t in[4] = {u.x, u.y, u.z, u.w};
    uint32_t h[kParts][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float a = bf16_lo(in[q]) * w[2 * q], b = bf16_hi(in[q]) * w[2 * q + 1];
#pragma unroll
      for (int k = 0; k < kParts; ++k) {
        h[k][q] = bf16_pack2(a, b);
        a -= bf16_lo(h[k][q]);
        b -= bf16_hi(h[k][q]);
      }
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) p[k] = make_uint4(h[k][0], h[k][1], h[k][2], h[k][3]);
  }
  __device__ __forceinline__ bf16x8 part(int k) const { return __builtin_bit_cast(bf16x8, p[k]); }
};

// A segment of a sequence.  Slots 0 .. batch-1 are the sequences' first segments;
// the window of packed rows [j seg, (j + 1) seg), j >= 1, holds at most one later
// segment's start (two starts of one sequence lie seg apart, and a later
// sequence's first one more than seg behind its own start).
struct Segment {
  int b, k, lo, hi, p0, p1;  // sequence, index in it, its rows, the segment's rows
  __device__ __forceinline__ bool later(const Sequences& q, int j, int seg) {
    const int64_t at = (int64_t)j * seg;
    if (at >= q.tokens) return false;
    b = q.of((int)at);
    lo = q.start(b);
    hi = q.start(b + 1);
    if (lo > at) return false;
    k = (int)((at - lo + seg - 1) / seg);
    const int64_t p = (int64_t)lo + (int64_t)k * seg;
    if (k < 1 || p >= hi || p >= at + seg) return false;
    p0 = (int)p;
    p1 = hi - p0 > seg ? p0 + seg : hi;
    return true;
  }
  __device__ __forceinline__ void first(const Sequences& q, int i, int seg) {
    b = i;
    k = 0;
    lo = q.start(b);
    hi = q.start(b + 1);
    if (hi < lo) hi = lo;
    p0 = lo;
    p1 = hi - lo > seg ? lo + seg : hi;
  }
};

// Inclusive sums over the wave's lanes, and one lane's value, in 64 bits.
template <int CTRL, int ROWS> __device__ __forceinline__ double dpp64(double x) {  // 0 where no lane is read
  const uint2 u = __builtin_bit_cast(uint2, x);
  const uint2 r = make_uint2(__builtin_amdgcn_update_dpp(0, (int)u.x, CTRL, ROWS, 0xF, false),
                             __builtin_amdgcn_update_dpp(0, (int)u.y, CTRL, ROWS, 0xF, false));
  return __builtin_bit_cast(double, r);
}
__device__ __forceinline__ double wave_scan(double x) {
  x += dpp64<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8
  x += dpp64<0x112, 0xF>(x);
  x += dpp64<0x114, 0xF>(x);
  x += dpp64<0x118, 0xF>(x);
  x += dpp64<0x142, 0xA>(x);  // lane 15 of rows 0 and 2 to rows 1 and 3
  x += dpp64<0x143, 0xC>(x);  // lane 31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ double lane_of(double x, int lane) {
  const uint2 u = __builtin_bit_cast(uint2, x);
  return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_readlane((int)u.x, lane), __builtin_amdgcn_readlane((int)u.y, lane)));
}

// LOCAL: the state part alone, over the segment before the slot's (first launch).
template <typename IO, int K, int V, bool LOCAL>
__global__ __launch_bounds__(256, sizeof(IO) == 2 ? 2 : 1) void scan_kernel(ScanArgs a, int seg, bool apart) {
  using FR = Frags<IO>;
  using F = typename FR::F;
  using TB = ColTile<IO, K>;
  using TX = ColTile<IO, kValues>;
  using TC = RowTile<IO, K>;
  using TM = RowTile<IO, kChunk>;
  constexpr int KT = K / 16, KF = K / 32, HEADS = kValues / V, PER = TB::kPer, ROW = (int)sizeof(IO) * 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  // workgroups go round the eight XCDs: each takes a run of heads, whose groups' B and C stay in its L2
  const int per_group = a.H / a.G, parts = a.G * ((per_group + HEADS - 1) / HEADS);
  const int slot = blockIdx.x / parts;
  int part = blockIdx.x % parts;
  if (parts % 8 == 0) part = (part % 8) * (parts / 8) + part / 8;
  const int grp = part / ((per_group + HEADS - 1) / HEADS), first = (part % ((per_group + HEADS - 1) / HEADS)) * HEADS;
  const int h0 = grp * per_group + first, heads = min(HEADS, per_group - first);
  const int hl = HEADS == 2 ? wave >> 1 : 0;             // the wave's head among the workgroup's
  const bool mine = hl < heads;                          // (an odd group's last workgroup has one head)
  const int h = h0 + (mine ? hl : 0), vbase = HEADS == 2 ? 32 * (wave & 1) : 32 * wave;

  Segment s;
  if (LOCAL) {
    if (!s.later(a.seq, slot + 1, seg)) return;
    s.p1 = s.p0;
    s.p0 -= seg;
    --s.k;
  } else if (slot < a.seq.batch) {
    s.first(a.seq, slot, seg);
  } else if (!s.later(a.seq, slot - a.seq.batch + 1, seg)) {
    return;
  }

  extern __shared__ __attribute__((aligned(16))) char lds[];
  char* const lb = lds;
  char* const lx = lb + TB::kBytes;
  char* const lc = lx + TX::kBytes;
  char* const lm = lc + TC::kBytes;
  float* const gates = reinterpret_cast<float*>(LOCAL ? lc : lm + HEADS * TM::kBytes);

  // channels: the lane's four state values (v of place i, k of group g) of tile (u, kt) in a tile-major state
  auto state_at = [&](int u, int kt) {
    const int v = vbase + 8 * (i >> 2) + 4 * u + (i & 3), k = 32 * (kt >> 1) + 8 * g + 4 * (kt & 1);
    return ((v >> 4) * (K / 16) + (k >> 4)) * 256 + 4 * ((v & 15) + 16 * ((k & 15) >> 2));
  };
  auto work_at = [&](int j) { return a.work + ((size_t)(j - 1) * a.H + h) * (V * K); };  // before segment start j
  float* const decays = a.work ? a.work + (size_t)(a.seq.tokens / seg) * a.H * (V * K) : nullptr;

  floatx4 S[2][KT];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) S[u][kt] = floatx4{0.f, 0.f, 0.f, 0.f};
  if (s.k == 0) {
    if (a.S_in) {
      const float* in = a.S_in + ((size_t)s.b * a.H + h) * (V * K);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[u][kt] = *reinterpret_cast<const floatx4*>(in + state_at(u, kt));
    }
  } else if (!LOCAL) {
    for (int k = 0; k < s.k; ++k) {  // the segments before this one, in order
      const int j = (int)(((int64_t)s.lo + (int64_t)(k + 1) * seg) / seg);
      const float* w = work_at(j);
      const float d = k ? __builtin_amdgcn_exp2f(decays[(size_t)(j - 1) * a.H + h]) : 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const floatx4 t = *reinterpret_cast<const floatx4*>(w + state_at(u, kt));
#pragma unroll
          for (int e = 0; e < 4; ++e) S[u][kt][e] = k ? fmaf(S[u][kt][e], d, t[e]) : t[e];
        }
    }
  }

  // A chunk's rows in registers on their way to LDS, 16-byte pieces, zero past the
  // segment: 256 threads take 256 / kChunks rows at a time.
  constexpr int RB = 256 / TB::kChunks, RX = 256 / TX::kChunks, NB = kChunk / RB, NX = kChunk / RX;
  const int rb = tid / TB::kChunks, cb = (tid % TB::kChunks) * PER, rx = tid / TX::kChunks, cx = (tid % TX::kChunks) * PER;
  const int xload = cx < heads * V ? cx : 0;  // (a missing head's columns: any values, its results are not stored)
  const uint32_t ob = (uint32_t)((rb * a.ldb + cb) * sizeof(IO)), oc = (uint32_t)((rb * a.ldc + cb) * sizeof(IO)),
                 ox = (uint32_t)((rx * a.ldx + xload) * sizeof(IO));
  const char* const b0 = static_cast<const char*>(a.b) + (size_t)grp * K * sizeof(IO);
  const char* const c0 = static_cast<const char*>(a.c) + (size_t)grp * K * sizeof(IO);
  const char* const x0 = static_cast<const char*>(a.x) + (size_t)h0 * V * sizeof(IO);
  const size_t nb = RB * a.ldb * sizeof(IO), nc = RB * a.ldc * sizeof(IO), nx = RX * a.ldx * sizeof(IO);
  const char* fb = b0 + (size_t)s.p0 * sizeof(IO) * a.ldb;
  const char* fc = c0 + (size_t)s.p0 * sizeof(IO) * a.ldc;
  const char* fx = x0 + (size_t)s.p0 * sizeof(IO) * a.ldx;
  uint4 pb[NB], pc[NB], px[NX];
  auto fetch = [&](int n) {  // the next chunk; n: rows to the segment's end
    auto rows = [&](auto all) {
      constexpr bool ALL = decltype(all)::value;
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        if (!ALL) pb[q] = pc[q] = make_uint4(0, 0, 0, 0);
        if (ALL || q * RB + rb < n) {
          pb[q] = *reinterpret_cast<const uint4*>(fb + ob);
          if (!LOCAL) pc[q] = *reinterpret_cast<const uint4*>(fc + oc);
        }
        fb += nb;
        fc += nc;
      }
#pragma unroll
      for (int q = 0; q < NX; ++q) {
        if (!ALL) px[q] = make_uint4(0, 0, 0, 0);
        if (ALL || q * RX + rx < n) px[q] = *reinterpret_cast<const uint4*>(fx + ox);
        fx += nx;
      }
    };
    if (n >= kChunk) rows(std::true_type{});
    else rows(std::false_type{});
  };
  auto put = [&]() {
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      FR::template put_c<K>(lb, q * RB + rb, cb, pb[q]);
      if (!LOCAL) *reinterpret_cast<uint4*>(lc + TC::at(q * RB + rb, cb)) = pc[q];
    }
#pragma unroll
    for (int q = 0; q < NX; ++q) FR::template put_c<kValues>(lx, q * RX + rx, cx, px[q]);
  };

  // Step sizes and decays of four chunks, a chunk per wave.  Sums of log decays run in
  // 64 bits: a token that forgets everything (held to 2^-150, which is 0 in fp32)
  // must not blur the differences of those after it.  A chunk's record, in LDS, with
  // the tile of 16 tokens t / 16 = w and G(w) the sum before it, base 2:
  //   kLocal  g_t - G(w) in two parts       kStep  g_s - G(w) - log2 dt_s in two parts
  //   kGate   2^{g_t}
  //   kPass   dt_s 2^{G(w) - g_s} of the tokens s before tile w = 1, 2, 3
  //   kLeft   dt_s 2^{g_L - g_s}            kEnd   g_L
  // LOCAL keeps kLeft and kEnd.
  auto record = [&](int head, int chunk) { return gates + (head * 4 + chunk) * (LOCAL ? kLocalRecord : kRecord); };
  float Dh[HEADS], A2[HEADS], bias[HEADS];
#pragma unroll
  for (int q = 0; q < HEADS; ++q) {
    const int hh = h0 + min(q, heads - 1);
    Dh[q] = !LOCAL && a.D ? a.D[hh] : 0.f;
    A2[q] = a.A[hh] * 1.44269504f;
    bias[q] = a.dt_bias ? a.dt_bias[hh] : 0.f;
  }
  float raw[HEADS];  // dt as stored, four chunks ahead
  auto steps = [&](int p) {
#pragma unroll
    for (int q = 0; q < HEADS; ++q)
      raw[q] = ld_elem(static_cast<const IO*>(a.dt) + (size_t)min(p + tid, s.p1 - 1) * a.lddt + h0 + min(q, heads - 1));
  };
  auto gate = [&](int p) {
    float dt[HEADS];
    double sum[HEADS];
#pragma unroll
    for (int q = 0; q < HEADS; ++q) {
      dt[q] = p + tid < s.p1 ? softplus(raw[q] + bias[q]) : 0.f;
      sum[q] = wave_scan((double)fmaxf(dt[q] * A2[q], -150.f));
    }
    if (p + kGates < s.p1) steps(p + kGates);
#pragma unroll
    for (int q = 0; q < HEADS; ++q) {
      const double end = lane_of(sum[q], 63);
      float* r = record(q, wave);
      r[kLeft + lane] = dt[q] * __builtin_amdgcn_exp2f((float)(end - sum[q]));
      if (lane == 0) r[kEnd] = (float)end;
      if (!LOCAL) {
        const double g1 = lane_of(sum[q], 15), g2 = lane_of(sum[q], 31), g3 = lane_of(sum[q], 47);
        const double loc = sum[q] - (lane < 16 ? 0.0 : lane < 32 ? g1 : lane < 48 ? g2 : g3);
        const float hi = (float)loc;
        r[kLocal + lane] = hi;
        r[kLocal + 64 + lane] = (float)(loc - (double)hi);
        // (no step: so far down that its power is 0 whatever t)
        const double low = dt[q] > 1e-37f ? loc - (double)__log2f(dt[q]) : 1e4;
        const float at = (float)low;
        r[kStep + lane] = at;
        r[kStep + 64 + lane] = (float)(low - (double)at);
        r[kGate + lane] = __builtin_amdgcn_exp2f((float)sum[q]);
        if (lane < 16) r[kPass + lane] = dt[q] * __builtin_amdgcn_exp2f((float)(g1 - sum[q]));
        if (lane < 32) r[kPass + 16 + lane] = dt[q] * __builtin_amdgcn_exp2f((float)(g2 - sum[q]));
        if (lane < 48) r[kPass + 48 + lane] = dt[q] * __builtin_amdgcn_exp2f((float)(g3 - sum[q]));
      }
    }
  };

  // the lane's places in the tiles: rows i (+ 16 per 16 ROW COLS bytes) of B, C and M, columns of B and x
  constexpr int NR = (int)sizeof(IO) / 2;  // 16-byte chunks of a fragment's row
  uint32_t brow[KF][2], crow[KF][NR], mrow[2][NR], bcol[KF][FR::kCols], xcol[FR::kCols];
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int kf = 0; kf < KF; ++kf) brow[kf][q] = TB::at(i, 32 * kf + 8 * g + 4 * q);
#pragma unroll
  for (int q = 0; q < NR; ++q) {
#pragma unroll
    for (int kf = 0; kf < KF; ++kf) crow[kf][q] = TC::at(i, 32 * kf + 8 * g + 4 * q);
#pragma unroll
    for (int sf = 0; sf < 2; ++sf) mrow[sf][q] = hl * TM::kBytes + TM::at(i, 32 * sf + 8 * g + 4 * q);
  }
#pragma unroll
  for (int kf = 0; kf < KF; ++kf) FR::template cols_at<K>(bcol[kf], 8 * g, i, 32 * kf, 8);
  FR::template cols_at<kValues>(xcol, 8 * g, i, 32 * wave, 8);
  const uint32_t oy = (uint32_t)((i * a.ldy + vbase + 8 * g) * sizeof(IO));
  const size_t ny = 16 * a.ldy * sizeof(IO);
  char* py = static_cast<char*>(a.y) + (size_t)h * V * sizeof(IO) + (size_t)s.p0 * sizeof(IO) * a.ldy;

  if (!LOCAL) {  // scores of tokens after t in the 32 that a fragment spans: zero throughout
    for (int q = tid; q < HEADS * TM::kBytes / 16; q += 256) reinterpret_cast<uint4*>(lm)[q] = make_uint4(0, 0, 0, 0);
  }
  float total = 0.f;
  if (s.p0 < s.p1) {
    steps(s.p0);
    fetch(s.p1 - s.p0);
  }
  int chunk = 0;
  for (int p = s.p0; p < s.p1; p += kChunk, chunk = (chunk + 1) & 3) {
    lds_barrier();
    put();
    if (chunk == 0) gate(p);
    lds_barrier();
    if (p + kChunk < s.p1) fetch(s.p1 - p - kChunk);
    const float* const rec = record(mine ? hl : 0, chunk);

    if constexpr (!LOCAL) {
      // scores of tiles (w, st): tokens t (place i) of tile w against s of tile st <= w, with
      // decay and step, as rows of M; D on the diagonal.  The ten tiles by wave:
      // its diagonal one, then 0: (1,0) (2,0)  1: (2,1) (3,0)  2: (3,1)  3: (3,2).  (What a missing
      // second head finds in its record is never stored.)
      auto score = [&](int tw, int ts, auto diagonal) {
        floatx4 m = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kf = 0; kf < KF; ++kf)
          m = FR::mma(FR::row_c(lb, brow[kf], ts * ROW * K), FR::row(lc, crow[kf], tw * ROW * K), m);
        const int to = TM::at(16 * tw + i, 16 * ts + 4 * g);
#pragma unroll
        for (int hh = 0; hh < HEADS; ++hh) {
          const float* r = record(hh, chunk);
          float f[4];
          if constexpr (decltype(diagonal)::value) {
            const float th = r[kLocal + 16 * tw + i], tl = r[kLocal + 64 + 16 * tw + i];
            const float4 sh = *reinterpret_cast<const float4*>(r + kStep + 16 * ts + 4 * g),
                         sl = *reinterpret_cast<const float4*>(r + kStep + 64 + 16 * ts + 4 * g);
            const float h4[4] = {sh.x, sh.y, sh.z, sh.w}, l4[4] = {sl.x, sl.y, sl.z, sl.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int o = 4 * g + e - i;  // s - t
              f[e] = m[e] * __builtin_amdgcn_exp2f((th - h4[e]) + (tl - l4[e]));
              f[e] = (o > 0 ? 0.f : f[e]) + (o == 0 ? Dh[hh] : 0.f);
            }
          } else {
            const float et = __builtin_amdgcn_exp2f(r[kLocal + 16 * tw + i]);
            const float4 w4 = *reinterpret_cast<const float4*>(r + kPass + (tw == 1 ? 0 : tw == 2 ? 16 : 48) + 16 * ts + 4 * g);
            f[0] = m[0] * et * w4.x; f[1] = m[1] * et * w4.y; f[2] = m[2] * et * w4.z; f[3] = m[3] * et * w4.w;
          }
          FR::store4(lm + hh * TM::kBytes, to, f[0], f[1], f[2], f[3]);
        }
      };
      score(wave, wave, std::true_type{});
      score(wave == 0 ? 1 : wave == 1 ? 2 : 3, wave == 0 ? 0 : wave == 3 ? 2 : 1, std::false_type{});
      if (wave < 2) score(wave + 2, 0, std::false_type{});
    }
    // Between products the vector units have work of their own: an instruction of the matrix
    // cores takes the time of four others (a product, then three of them, in the
    // orders asked for below).
    F xt[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int sf = 0; sf < 2; ++sf) xt[u][sf] = FR::template cols<kValues>(lx, xcol, sf * 2 * ROW * kValues, u);
    const float end = rec[kEnd], d = __builtin_amdgcn_exp2f(end);
    total += end;
    Weighted<IO> w[2][2];
    auto weigh = [&](int sf) {
      Vec<8> ws;
      ws.load(rec + kLeft + 32 * sf + 8 * g);
      w[0][sf].set(xt[0][sf], ws.e);
      w[1][sf].set(xt[1][sf], ws.e);
    };
    if constexpr (!LOCAL) {
      // y: the state's part first, so that its products run while the scores settle
      floatx4 y[4][2];
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int u = 0; u < 2; ++u) y[tt][u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kf = 0; kf < KF; ++kf) {
        const F s0 = FR::of(S[0][2 * kf], S[0][2 * kf + 1]), s1 = FR::of(S[1][2 * kf], S[1][2 * kf + 1]);
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
          const F ct = FR::row(lc, crow[kf], tt * ROW * K);
          y[tt][0] = FR::mma(s0, ct, y[tt][0]);
          y[tt][1] = FR::mma(s1, ct, y[tt][1]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) { S[u][2 * kf] *= d; S[u][2 * kf + 1] *= d; }
      }
      weigh(0);
      if constexpr (sizeof(IO) == 2) {
#pragma unroll
        for (int q = 0; q < 8 * KF; ++q) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x2, 5, 0);
        }
      }
#pragma unroll
      for (int tt = 0; tt < 4; ++tt) {
        const float et = rec[kGate + 16 * tt + i];
#pragma unroll
        for (int e = 0; e < 4; ++e) { y[tt][0][e] *= et; y[tt][1][e] *= et; }
      }
      lds_barrier();
      const int n = mine ? s.p1 - p : 0;
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int sf = 0; sf <= tt / 2; ++sf) {
          const F mt = FR::row(lm, mrow[sf], tt * ROW * kChunk);
          y[tt][0] = FR::mma(xt[0][sf], mt, y[tt][0]);
          y[tt][1] = FR::mma(xt[1][sf], mt, y[tt][1]);
        }
      auto rows = [&](auto all) {
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
          if (!decltype(all)::value && 16 * tt + i >= n) continue;
          Raw<IO, 8> o;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              if constexpr (sizeof(IO) == 2) o.w[2 * u + e / 2] = bf16_pack2(y[tt][u][e], y[tt][u][e + 1]);
              else { o.e[4 * u + e] = y[tt][u][e]; o.e[4 * u + e + 1] = y[tt][u][e + 1]; }
            }
          o.store(reinterpret_cast<IO*>(py + tt * ny + oy));
        }
      };
      if (n >= kChunk) rows(std::true_type{});
      else rows(std::false_type{});
      py += 4 * ny;
    } else {
      weigh(0);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[u][kt] *= d;
    }
    // the state: decayed already, now the chunk's tokens
#pragma unroll
    for (int sf = 0; sf < 2; ++sf) {
      if (sf == 0) weigh(1);
#pragma unroll
      for (int kt = 0; kt < KT; kt += 2) {
        const F b0t = FR::template cols<K>(lb, bcol[kt / 2], sf * 2 * ROW * K, 0), b1t = FR::template cols<K>(lb, bcol[kt / 2], sf * 2 * ROW * K, 1);
#pragma unroll
        for (int k = 0; k < Weighted<IO>::kParts; ++k) {
          S[0][kt] = FR::mma(b0t, w[0][sf].part(k), S[0][kt]);
          S[1][kt] = FR::mma(b0t, w[1][sf].part(k), S[1][kt]);
          S[0][kt + 1] = FR::mma(b1t, w[0][sf].part(k), S[0][kt + 1]);
          S[1][kt + 1] = FR::mma(b1t, w[1][sf].part(k), S[1][kt + 1]);
        }
      }
    }
    if constexpr (sizeof(IO) == 2) {
#pragma unroll
      for (int q = 0; q < 12 * KT / 2; ++q) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x2, 3, 1);
      }
    }
  }

  if (!mine) return;
  if (LOCAL) {
    float* w = work_at(slot + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) *reinterpret_cast<floatx4*>(w + state_at(u, kt)) = S[u][kt];
    if (vbase == 0 && lane == 0) decays[(size_t)slot * a.H + h] = total;
  } else if (s.p1 == s.hi) {
    // S_out in place of S_in: other segments' workgroups may still read it, so that a later
    // segment leaves its state where only this workgroup reads, for a copy after the launch
    float* out = apart && s.k > 0 ? work_at(slot - a.seq.batch + 1) : a.S_out + ((size_t)s.b * a.H + h) * (V * K);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) *reinterpret_cast<floatx4*>(out + state_at(u, kt)) = S[u][kt];
  }
}

// The end states that a launch in place left in the workspace, into S_out.
__global__ __launch_bounds__(256) void scan_states_kernel(ScanArgs a, int seg, int size) {
  const int h = blockIdx.x % a.H, j = blockIdx.x / a.H + 1;
  Segment s;
  if (!s.later(a.seq, j, seg) || s.p1 != s.hi) return;
  const float4* w = reinterpret_cast<const float4*>(a.work + ((size_t)(j - 1) * a.H + h) * size);
  float4* out = reinterpret_cast<float4*>(a.S_out + ((size_t)s.b * a.H + h) * size);
  for (int q = threadIdx.x; q < size / 4; q += 256) out[q] = w[q];
}

// Tokens of a segment: a fair share of all tokens for each of the two workgroups that a
// CU holds, in whole gates; sequences no longer than that are not split.
int scan_parts(int H, int G, int V) { return G * ((H / G + kValues / V - 1) / (kValues / V)); }
int scan_segment(const Sequences& q, int parts) {
  constexpr int64_t want = 512;
  int64_t seg = ((int64_t)q.tokens * parts + want - 1) / want;
  seg = (seg + kGates - 1) / kGates * kGates;
  const int longest = q.offsets ? q.tokens : q.each;
  return seg < kGates ? kGates : seg >= longest ? (longest > 0 ? longest : 1) : (int)seg;
}
int scan_windows(const Sequences& q, int seg) { return seg < (q.offsets ? q.tokens : q.each) ? q.tokens / seg : 0; }

size_t scan_workspace(int batch, int tokens, int H, int G, int K, int V) {
  Sequences q{};
  q.offsets = reinterpret_cast<const int32_t*>(4);  // lengths unknown: the most that any take
  q.batch = batch;
  q.tokens = tokens;
  const int seg = scan_segment(q, scan_parts(H, G, V));
  return (size_t)scan_windows(q, seg) * H * ((size_t)V * K + 1) * sizeof(float);
}

template <typename IO, int K, int V>
int launch_scan(const ScanArgs& a, hipStream_t s) {
  const int parts = scan_parts(a.H, a.G, V), seg = scan_segment(a.seq, parts), windows = scan_windows(a.seq, seg);
  const bool apart = windows && a.S_in && a.S_in == a.S_out;
  constexpr int heads = kValues / V;
  constexpr size_t local = RowTile<IO, K>::kBytes + RowTile<IO, kValues>::kBytes;
  constexpr size_t full = local + RowTile<IO, K>::kBytes + heads * RowTile<IO, kChunk>::kBytes;
  if (windows)
    hipLaunchKernelGGL((scan_kernel<IO, K, V, true>), dim3((unsigned)windows * (unsigned)parts), dim3(256),
                       local + heads * 4 * kLocalRecord * sizeof(float), s, a, seg, false);
  hipLaunchKernelGGL((scan_kernel<IO, K, V, false>), dim3((unsigned)(a.seq.batch + windows) * (unsigned)parts), dim3(256),
                     full + heads * 4 * kRecord * sizeof(float), s, a, seg, apart);
  if (apart) hipLaunchKernelGGL(scan_states_kernel, dim3((unsigned)windows * (unsigned)a.H), dim3(256), 0, s, a, seg, V * K);
  return 0;
}

template <typename IO>
int launch_scan(const ScanArgs& a, int K, int V, hipStream_t s) {
  if (K == 64 && V == 64) return launch_scan<IO, 64, 64>(a, s);
  if (K == 128 && V == 64) return launch_scan<IO, 128, 64>(a, s);
  if (K == 128 && V == 128) return launch_scan<IO, 128, 128>(a, s);
  return -2;
}

int run_scan(const ScanArgs& a, int K, int V, int io, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return io == 1 ? launch_scan<bf16_t>(a, K, V, s) : launch_scan<float>(a, K, V, s);
}

}  // namespace skssm
