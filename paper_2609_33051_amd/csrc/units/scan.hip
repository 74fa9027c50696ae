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
// Products.  The state's update and its reads run in tiles of 32 x 32, the scores
// in tiles of 16 x 16.  An instruction takes the vector units' issue slots for some
// 12 cycles whichever it is, 32x32x16 for 32 cycles of products and 16x16x32 for 16, and
// the vector work between them (weights, decays, roundings) is what bounds this kernel.
// Operands hold, per lane, 8 consecutive indices of the reduction (lane group h = lane /
// 32, or g = lane / 16) of the row or column lane % 32 (lane % 16).  The state's
// accumulator rows are assigned to channels so that eight of a lane's registers are
// such an operand as they lie: row 8 q + 4 h + e of a tile is channel 16 (q / 2) + 8 h + 4 (q % 2) + e.
//
// Long sequences: a sequence is split into segments of `seg` tokens, a fair
// share of the card.  A first launch runs the state part of every segment but a
// sequence's last, from zero (the first: from S_in), and keeps its end state and
// total decay; the second begins each segment from the states before it, joined.
//
// Measured, 128 heads of 128 x 64 in 8 groups, bf16: one prompt of 16384 tokens 330 us (states 110,
// outputs 220; its bytes take 96 at the best copy's rate, its products in this form 100 of
// the matrix units'), 37 prompts of 12000 tokens 211 us.  Matrix and vector units add up to
// 96 % of the first launch's time and 86 % of the second's: what is left is
// waiting at the barriers and for LDS, with the two waves a SIMD that registers and LDS allow.
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "../mixer.h"

namespace skssm {

constexpr int kChunk = 64;
constexpr int kValues = 128;        // value channels of a workgroup
constexpr int kGates = 4 * kChunk;  // tokens whose gates are computed together, a chunk per wave
// places in a chunk's record of gates (floats)
constexpr int kLeft = 0, kEnd = 64, kLocalRecord = 68, kLocal = 68, kStep = 196, kGate = 324, kPass = 388, kSkip = 452, kRecord = 456;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// 64 rows of COLS elements in LDS.  The 16-byte chunks of a row are permuted by the row, so
// that two reads keep their lanes in different banks: 16 bytes of consecutive
// rows, and the transposed read's four rows of 64 bytes (rows of 128 bytes differ by their
// place already where they follow one another).  The states' launch has no conflicts by its counters; the
// outputs' has them in 19 % of its LDS cycles, at what only it accesses: the operands and the tile of the scores.
template <typename IO, int COLS> struct Tile {
  static constexpr int kBytes = kChunk * COLS * (int)sizeof(IO), kChunks = COLS * (int)sizeof(IO) / 16;
  static constexpr int kPer = 16 / (int)sizeof(IO);  // elements of a chunk
  static __device__ __forceinline__ int at(int row, int col) {  // byte offset
    const int key = (kChunks >= 16 ? (row & 3) << 2 : (row & 2) << 1) | ((row >> 2) & 3);
    return row * (COLS * (int)sizeof(IO)) + (((col / kPer) ^ key) << 4) + (col % kPer) * (int)sizeof(IO);
  }
};

// The channel of row (column) m of a 32-wide tile of the state.
__device__ __forceinline__ int channel(int m) { return 16 * (m >> 4) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3); }

struct FragF32 { float e[8]; };

template <typename IO> struct Frags;
template <> struct Frags<bf16_t> {
  using F = bf16x8;
  static constexpr int kRow = 1, kCols = 2;  // places a lane holds of a row's and of a column's operand
  // 8 consecutive columns of one row
  template <int COLS> static __device__ __forceinline__ void row_at(uint32_t* at, int row, int col) { at[0] = Tile<bf16_t, COLS>::at(row, col); }
  static __device__ __forceinline__ F row(const char* t, const uint32_t* at, int off) {
    return __builtin_bit_cast(F, *reinterpret_cast<const uint4*>(t + at[0] + off));
  }
  // rows 8 h .. 8 h + 7 of column col0 + channel(lane % 32): a transposed read takes, from 16
  // lanes, four rows (i / 4) of four 8-byte pieces (i % 4) and leaves each lane a column
  template <int COLS> static __device__ __forceinline__ void cols_at(uint32_t* at, int lane, int col0) {
    const int i = lane & 15, p = i & 3;
#pragma unroll
    for (int q = 0; q < 2; ++q)
      at[q] = Tile<bf16_t, COLS>::at(8 * (lane >> 5) + 4 * q + (i >> 2), col0 + channel(16 * ((lane >> 4) & 1) + 4 * p));
  }
  static __device__ __forceinline__ F cols(const char* t, const uint32_t* at, int off) {
    typedef __attribute__((address_space(3))) shortx4* lds4;
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(t + at[0] + off));
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(t + at[1] + off));
    return __builtin_bit_cast(F, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  static __device__ __forceinline__ floatx4 mma(F a, F b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ floatx16 mma(F a, F b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ F of(const floatx16& s, int r) {  // registers r .. r + 7
    return __builtin_bit_cast(F, make_uint4(bf16_pack2(s[r], s[r + 1]), bf16_pack2(s[r + 2], s[r + 3]), bf16_pack2(s[r + 4], s[r + 5]),
                                            bf16_pack2(s[r + 6], s[r + 7])));
  }
  static __device__ __forceinline__ void store4(char* t, int at, float a, float b, float c, float d) {
    *reinterpret_cast<uint2*>(t + at) = make_uint2(bf16_pack2(a, b), bf16_pack2(c, d));
  }
};
template <> struct Frags<float> {
  using F = FragF32;
  static constexpr int kRow = 2, kCols = 8;
  template <int COLS> static __device__ __forceinline__ void row_at(uint32_t* at, int row, int col) {
    at[0] = Tile<float, COLS>::at(row, col);
    at[1] = Tile<float, COLS>::at(row, col + 4);
  }
  static __device__ __forceinline__ F row(const char* t, const uint32_t* at, int off) {
    F f;
    const float4 a = *reinterpret_cast<const float4*>(t + at[0] + off), b = *reinterpret_cast<const float4*>(t + at[1] + off);
    f.e[0] = a.x; f.e[1] = a.y; f.e[2] = a.z; f.e[3] = a.w;
    f.e[4] = b.x; f.e[5] = b.y; f.e[6] = b.z; f.e[7] = b.w;
    return f;
  }
  template <int COLS> static __device__ __forceinline__ void cols_at(uint32_t* at, int lane, int col0) {
#pragma unroll
    for (int q = 0; q < 8; ++q) at[q] = Tile<float, COLS>::at(8 * (lane >> 5) + q, col0 + channel(lane & 31));
  }
  static __device__ __forceinline__ F cols(const char* t, const uint32_t* at, int off) {
    F f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.e[e] = *reinterpret_cast<const float*>(t + at[e] + off);
    return f;
  }
  static __device__ __forceinline__ floatx4 mma(const F& a, const F& b, floatx4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.e[e], b.e[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ floatx16 mma(const F& a, const F& b, floatx16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.e[e], b.e[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ F of(const floatx16& s, int r) {
    F f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.e[e] = s[r + e];
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

// The sequence that is `rank`-th by length, longest first: workgroups start in this order, so
// that the card does not wait for a long sequence that began last.  Every wave counts for itself, a
// lane a sequence; for 64 sequences at the most, of three chunks on average: shorter ones
// leave nothing to wait for, and counting (over 256 sequences in 6 us a workgroup) is a large part of them.
// 128 heads of 128 x 64, uneven lengths, by packed order / by length (us): 37 sequences of 324 tokens on average
// 219 / 212, 16 of 200 85 / 82, 8 of 1000 160 / 163; with a count over all of up to 256: 100 of 400 613 / 609, of 200
// 352 / 363, of 80 199 / 220, 256 of 30 440 / 572, 37 of 100 91 / 94.
__device__ __forceinline__ int by_length(const Sequences& q, int rank, int lane) {
  if (!q.offsets || q.batch < 2 || q.batch > 64 || q.tokens < 3 * kChunk * q.batch) return rank;
  const int length = lane < q.batch ? q.start(lane + 1) - q.start(lane) : INT_MIN;
  int before = 0;
  for (int b = 0; b < q.batch; ++b) before += __builtin_amdgcn_readlane(length, b) + (b < lane) > length;
  return __builtin_ctzll(__ballot(lane < q.batch && before == rank));
}

// LOCAL: the state part alone, over the segment before the slot's (first launch).
template <typename IO, int K, int V, bool LOCAL>
__global__ __launch_bounds__(256, sizeof(IO) == 2 ? 2 : 1) void scan_kernel(ScanArgs a, int seg, bool apart) {
  using FR = Frags<IO>;
  using F = typename FR::F;
  using TB = Tile<IO, K>;
  using TX = Tile<IO, kValues>;
  using TM = Tile<IO, kChunk>;
  constexpr int KT = K / 32, HEADS = kValues / V, PER = TB::kPer, ROW = (int)sizeof(IO) * 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  const int c32 = lane & 31, h32 = lane >> 5;
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

  extern __shared__ __attribute__((aligned(16))) char lds[];
  Segment s;
  if (LOCAL) {
    if (!s.later(a.seq, slot + 1, seg)) return;
    s.p1 = s.p0;
    s.p0 -= seg;
    --s.k;
  } else if (slot < a.seq.batch) {
    s.first(a.seq, by_length(a.seq, slot, lane), seg);
  } else if (!s.later(a.seq, slot - a.seq.batch + 1, seg)) {
    return;
  }
  char* lb = lds;  // (LOCAL: of two buffers in turn)
  char* lx = lb + TB::kBytes;
  char* const lc = lx + TX::kBytes;
  char* const lm = lc + TB::kBytes;
  float* gates = reinterpret_cast<float*>(LOCAL ? lds + 2 * (TB::kBytes + TX::kBytes) : lm + HEADS * TM::kBytes);

  // the place of registers 4 q .. 4 q + 3 of tile kt (value channel of column c32, four key channels) in a tile-major state
  auto state_at = [&](int kt, int q) {
    const int v = vbase + channel(c32);
    return ((v >> 4) * (K / 16) + 2 * kt + (q >> 1)) * 256 + 4 * ((v & 15) + 16 * (2 * h32 + (q & 1)));
  };
  auto work_at = [&](int j) { return a.work + ((size_t)(j - 1) * a.H + h) * (V * K); };  // before segment start j
  float* const decays = a.work ? a.work + (size_t)(a.seq.tokens / seg) * a.H * (V * K) : nullptr;

  floatx16 S[KT];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[kt][r] = 0.f;
  // S = S d + a stored state
  auto add_state = [&](const float* from, float d) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const floatx4 t = *reinterpret_cast<const floatx4*>(from + state_at(kt, q));
#pragma unroll
        for (int e = 0; e < 4; ++e) S[kt][4 * q + e] = fmaf(S[kt][4 * q + e], d, t[e]);
      }
  };
  auto put_state = [&](float* to) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<floatx4*>(to + state_at(kt, q)) = floatx4{S[kt][4 * q], S[kt][4 * q + 1], S[kt][4 * q + 2], S[kt][4 * q + 3]};
  };
  if (s.k == 0) {
    if (a.S_in) add_state(a.S_in + ((size_t)s.b * a.H + h) * (V * K), 1.f);
  } else if (!LOCAL) {
    for (int k = 0; k < s.k; ++k) {  // the segments before this one, in order
      const int j = (int)(((int64_t)s.lo + (int64_t)(k + 1) * seg) / seg);
      add_state(work_at(j), k ? __builtin_amdgcn_exp2f(decays[(size_t)(j - 1) * a.H + h]) : 1.f);
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
    for (int q = 0; q < NB; ++q) *reinterpret_cast<uint4*>(lb + TB::at(q * RB + rb, cb)) = pb[q];
#pragma unroll
    for (int q = 0; q < NB; ++q)
      if (!LOCAL) *reinterpret_cast<uint4*>(lc + TB::at(q * RB + rb, cb)) = pc[q];
#pragma unroll
    for (int q = 0; q < NX; ++q) *reinterpret_cast<uint4*>(lx + TX::at(q * RX + rx, cx)) = px[q];
  };

  // Step sizes and decays of four chunks, a chunk per wave.  Sums of log decays run in
  // 64 bits: a token that forgets everything (held to 2^-150, which is 0 in fp32)
  // must not blur the differences of those after it.  A chunk's record, in LDS, with
  // the tile of 16 tokens t / 16 = w and G(w) the sum before it, base 2:
  //   kLocal  g_t - G(w) in two parts       kStep  g_s - G(w) - log2 dt_s in two parts
  //   kGate   2^{g_t}
  //   kPass   dt_s 2^{G(w + 1) - g_s}       kSkip  1 and 2^{G(w) - G(w' + 1)}, (w, w') = (2, 0), (3, 1), (3, 0)
  //   kLeft   dt_s 2^{g_L - g_s}            kEnd   g_L
  // LOCAL keeps kLeft and kEnd.
  auto record = [&](int head, int chunk) { return gates + (head * 4 + chunk) * (LOCAL ? kLocalRecord : kRecord); };
  const float D = !LOCAL && a.D ? a.D[h] : 0.f;
  float A2[HEADS], bias[HEADS];
#pragma unroll
  for (int q = 0; q < HEADS; ++q) {
    const int hh = h0 + min(q, heads - 1);
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
      const float log = dt[q] * A2[q];
      sum[q] = wave_scan((double)(log < -150.f ? -150.f : log));  // (NaN stays)
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
        r[kPass + lane] = dt[q] * __builtin_amdgcn_exp2f((float)((lane < 16 ? g1 : lane < 32 ? g2 : lane < 48 ? g3 : end) - sum[q]));
        const float skip = __builtin_amdgcn_exp2f((float)(lane == 1 ? g2 - g1 : lane == 2 ? g3 - g2 : lane == 3 ? g3 - g1 : 0.0));
        if (lane < 4) r[kSkip + lane] = skip;
      }
    }
  };

  // the lane's places in the tiles: rows i of B and C by 32 channels (scores), rows c32 of C by 16
  // channels, of M and of x, columns of B and x
  uint32_t row16[KT][FR::kRow], row32[2 * KT][FR::kRow], mrow[4][FR::kRow], xrow[2][FR::kRow], bcol[KT][FR::kCols], xcol[FR::kCols];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    FR::template row_at<K>(row16[kt], i, 32 * kt + 8 * g);
    FR::template row_at<K>(row32[2 * kt], c32, 32 * kt + 8 * h32);
    FR::template row_at<K>(row32[2 * kt + 1], c32, 32 * kt + 16 + 8 * h32);
    FR::template cols_at<K>(bcol[kt], lane, 32 * kt);
  }
#pragma unroll
  for (int st = 0; st < 4; ++st) FR::template row_at<kChunk>(mrow[st], c32, 16 * st + 8 * h32);
#pragma unroll
  for (int j = 0; j < 2; ++j) FR::template row_at<kValues>(xrow[j], c32, 32 * wave + 16 * j + 8 * h32);
  FR::template cols_at<kValues>(xcol, lane, 32 * wave);
  char* const lmh = lm + hl * TM::kBytes;
  const uint32_t oy = (uint32_t)((c32 * a.ldy + vbase + 8 * h32) * sizeof(IO));
  const size_t ny = 32 * a.ldy * sizeof(IO);
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
    if (LOCAL) {
      // waves still at the chunk before read the other buffer, and at most one is behind
      const bool odd = ((p - s.p0) / kChunk) & 1, high = ((p - s.p0) / kGates) & 1;
      lb = lds + (odd ? TB::kBytes + TX::kBytes : 0);
      lx = lb + TB::kBytes;
      gates = reinterpret_cast<float*>(lds + 2 * (TB::kBytes + TX::kBytes)) + (high ? HEADS * 4 * kLocalRecord : 0);
    } else {
      lds_barrier();
    }
    put();
    if (chunk == 0) gate(p);
    lds_barrier();
    if (p + kChunk < s.p1) fetch(s.p1 - p - kChunk);
    const float* const rec = record(mine ? hl : 0, chunk);

    if constexpr (!LOCAL) {
      // scores of tiles (w, st): tokens t (place i) of tile w against s of tile st <= w, with
      // decay and step, as rows of M.  The ten tiles by wave:
      // its diagonal one, then 0: (1,0), 1: (2,1), 2: (3,1), 3: (3,2), then (2,0) and (3,0), each
      // head by a wave of its own where there are two.  (What a missing second head finds in
      // its record is never stored.)
      auto score = [&](int tw, int ts, int one, auto diagonal) {  // one: the only head, or -1
        floatx4 m = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
          m = FR::mma(FR::row(lb, row16[kt], ts * ROW * K), FR::row(lc, row16[kt], tw * ROW * K), m);
        const int to = TM::at(16 * tw + i, 16 * ts + 4 * g);
#pragma unroll
        for (int q = 0; q < HEADS; ++q) {
          if (one >= 0 && q > 0) break;
          const int hh = one >= 0 ? one : q;
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
              if (o > 0) f[e] = 0.f;
            }
          } else {
            const float et = __builtin_amdgcn_exp2f(r[kLocal + 16 * tw + i]) * r[kSkip + (tw - ts == 1 ? 0 : tw - ts == 3 ? 3 : ts + 1)];
            const float4 w4 = *reinterpret_cast<const float4*>(r + kPass + 16 * ts + 4 * g);
            f[0] = m[0] * et * w4.x; f[1] = m[1] * et * w4.y; f[2] = m[2] * et * w4.z; f[3] = m[3] * et * w4.w;
          }
          FR::store4(lm + hh * TM::kBytes, to, f[0], f[1], f[2], f[3]);
        }
      };
      score(wave, wave, -1, std::true_type{});
      score(wave == 0 ? 1 : wave == 1 ? 2 : 3, wave == 0 ? 0 : wave == 3 ? 2 : 1, -1, std::false_type{});
      if (HEADS == 2) score(2 + (wave & 1), 0, wave >> 1, std::false_type{});
      else if (wave < 2) score(2 + wave, 0, -1, std::false_type{});
    }
    F xt[4];  // columns of x by 16 tokens
#pragma unroll
    for (int st = 0; st < 4; ++st) xt[st] = FR::cols(lx, xcol, st * ROW * kValues);
    const float end = rec[kEnd], d = __builtin_amdgcn_exp2f(end);
    total += end;
    Weighted<IO> w[4];
    auto weigh = [&](int st) {
      Vec<8> ws;
      ws.load(rec + kLeft + 16 * st + 8 * h32);
      w[st].set(xt[st], ws.e);
    };
    if constexpr (!LOCAL) {
      // y: the state's part first, so that its products run while the scores settle
      floatx16 y[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) y[0][r] = y[1][r] = 0.f;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const F sk = FR::of(S[kt], 8 * j);
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) y[tt] = FR::mma(sk, FR::row(lc, row32[2 * kt + j], 2 * tt * ROW * K), y[tt]);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) S[kt][r] *= d;
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const float et = rec[kGate + 32 * tt + c32];
#pragma unroll
        for (int r = 0; r < 16; ++r) y[tt][r] *= et;
      }
      if (a.D) {  // in fp32: on the scores' diagonal it would be rounded with them
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const auto x = __builtin_bit_cast(Raw<IO, 8>, FR::row(lx, xrow[j], 2 * tt * ROW * kValues));
#pragma unroll
            for (int e = 0; e < 8; ++e) y[tt][8 * j + e] = fmaf(D, x.get(e), y[tt][8 * j + e]);
          }
      }
      lds_barrier();
      const int n = mine ? s.p1 - p : 0;
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int tt = st / 2; tt < 2; ++tt) y[tt] = FR::mma(xt[st], FR::row(lmh, mrow[st], 2 * tt * ROW * kChunk), y[tt]);
      auto rows = [&](auto all) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          if (!decltype(all)::value && 32 * tt + c32 >= n) continue;
#pragma unroll
          for (int j = 0; j < 2; ++j) {  // channels 16 j + 8 h32 ..
            Raw<IO, 8> o;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              if constexpr (sizeof(IO) == 2) o.w[e / 2] = bf16_pack2(y[tt][8 * j + e], y[tt][8 * j + e + 1]);
              else { o.e[e] = y[tt][8 * j + e]; o.e[e + 1] = y[tt][8 * j + e + 1]; }
            }
            o.store(reinterpret_cast<IO*>(py + tt * ny + oy) + 16 * j);
          }
        }
      };
      if (n >= kChunk) rows(std::true_type{});
      else rows(std::false_type{});
      py += 2 * ny;
    } else {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[kt][r] *= d;
    }
    __builtin_amdgcn_s_setprio(1);
    // the state: decayed already, now the chunk's tokens
    weigh(0);
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      if (st < 3) weigh(st + 1);
#pragma unroll
      for (int k = 0; k < Weighted<IO>::kParts; ++k)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[kt] = FR::mma(FR::cols(lb, bcol[kt], st * ROW * K), w[st].part(k), S[kt]);
    }
    __builtin_amdgcn_s_setprio(0);
  }

  if (!mine) return;
  if (LOCAL) {
    put_state(work_at(slot + 1));
    if (vbase == 0 && lane == 0) decays[(size_t)slot * a.H + h] = total;
  } else if (s.p1 == s.hi) {
    // S_out in place of S_in: other segments' workgroups may still read it, so that a later
    // segment leaves its state where only this workgroup reads, for a copy after the launch
    put_state(apart && s.k > 0 ? work_at(slot - a.seq.batch + 1) : a.S_out + ((size_t)s.b * a.H + h) * (V * K));
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

// Tokens of a segment: a fair share of all T tokens for each of the two workgroups that a CU
// holds, but not so few that joining a long sequence's states (about 1 us each) takes longer
// than its segments' chunks, twice (about 4 us each): sqrt(8 T) balances the two.  In whole
// chunks, long ones in whole gates; two chunks are not worth a second launch.  It follows from
// T alone, since the workspace is sized before the lengths are known.
// Measured against segments of 256 at least, one sequence: 300 tokens, 20 heads of 64 x 64, fp32, 54 -> 22 us;
// 16384 tokens, 16 heads of 128 x 64, 111 -> 81 us; 65536 tokens, 2 heads, 242 -> 123 us.
int scan_parts(int H, int G, int V) { return G * ((H / G + kValues / V - 1) / (kValues / V)); }
int scan_segment(const Sequences& q, int parts) {
  constexpr int64_t want = 512;
  if (q.tokens <= 2 * kChunk) return 2 * kChunk;
  int64_t seg = ((int64_t)q.tokens * parts + want - 1) / want;
  const int64_t joined = (int64_t)sqrt(8.0 * q.tokens);
  if (seg < joined) seg = joined;
  if (seg > q.tokens) seg = q.tokens;  // (as much: none is split)
  return (int)(seg <= kGates / 2 ? (seg + kChunk - 1) / kChunk * kChunk : (seg + kGates - 1) / kGates * kGates);
}
// Windows that may hold a later segment's start; none where no sequence is split.
int scan_windows(const Sequences& q, int seg) { return seg < (q.offsets ? q.tokens : q.each) ? q.tokens / seg : 0; }

size_t scan_workspace(int batch, int tokens, int H, int G, int K, int V) {
  Sequences q{};
  q.offsets = reinterpret_cast<const int32_t*>(4);  // lengths unknown
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
  constexpr size_t local = Tile<IO, K>::kBytes + Tile<IO, kValues>::kBytes;
  constexpr size_t full = local + Tile<IO, K>::kBytes + heads * Tile<IO, kChunk>::kBytes;
  if (windows)
    hipLaunchKernelGGL((scan_kernel<IO, K, V, true>), dim3((unsigned)windows * (unsigned)parts), dim3(256),
                       2 * (local + heads * 4 * kLocalRecord * sizeof(float)), s, a, seg, false);
  // (batch times heads is less than 2^23, windows times parts at most 512: every launch fits)
  if (windows && !taken()) return 0;
  hipLaunchKernelGGL((scan_kernel<IO, K, V, false>), dim3((unsigned)(a.seq.batch + windows) * (unsigned)parts), dim3(256),
                     full + heads * 4 * kRecord * sizeof(float), s, a, seg, apart);
  if (apart && taken()) hipLaunchKernelGGL(scan_states_kernel, dim3((unsigned)windows * (unsigned)a.H), dim3(256), 0, s, a, seg, V * K);
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
