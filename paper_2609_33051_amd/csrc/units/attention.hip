// Attention of the new tokens over a paged cache in 4 bits.
//
// A wave holds QT tiles of 16 query rows (a row is one head of one new token; the heads that share a key
// head lie together) and goes over the keys 32 at a time:
//     S^T = K Q^T, P^T = 2^(c S^T - m), O^T += V^T P^T      (16 x 16 x 32 matrix products)
// Both products take the cache as their left operand, so that a query row is one column, one lane in each of
// the wave's four rows of lanes: the running maximum and every weight are a lane's own, and P^T comes out of
// the first product in the registers in which the second one takes it (the order in which the 32
// keys are summed is free, and the cache's records hold the values in the order it leaves).  The weights never pass
// through LDS; the cache's operands do where a workgroup's waves share them (prompt_kernel).  A row of ones beside V^T
// sums the weights as the products see them.
//
// The maximum that the weights are taken over moves only where the weights' sum has grown past 2^16; until then no
// score is compared with another and nothing is rescaled (one prompt of 8192 tokens, with the registers that this
// frees: 2000 -> 607 us).  The limit is one for any number of keys: a wave whose sum is past it with scores that do not
// grow takes the maximum every step (2100 tokens over 130000 keys of equal scores 8.98 ms, of random ones 7.67).
//
// Single tokens are bound by the cache's bytes: 64 over contexts of up to 8192, 32 heads on 8 of 128 channels, in 59
// us (5.6 TB/s; with weights in one part 56, as long as the loads alone), one over 131072 keys in 27 (5.2).  Prompts are bound by the vector
// units (exponentials, the cache's conversion) and the matrix units, which hardly overlap: one of 8192 tokens in 524
// to 543 us, 1.0 PFLOP/s.
#include <type_traits>

#include "../attention.h"

namespace skssm {

namespace {

#define INLINE __attribute__((always_inline))

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kStep = 32;         // keys a step
constexpr float kMost = 65536.f;  // sum of weights from which on the maximum is taken again
constexpr int kCUs = 256;
constexpr int kApart = 8;         // rounds that a tile apart costs
constexpr int kMostRounds = (1 << 30) - 1;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <bool NT, typename T> __device__ __forceinline__ T read(const T* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  else return *p;
}

// N consecutive words of a record, 4-byte aligned at least (8 where N is even).
template <int N> struct Words {
  uint32_t w[N];
  template <bool NT> __device__ __forceinline__ void load(const uint8_t* p) {
    typedef uint32_t w2 __attribute__((ext_vector_type(2), aligned(8)));
    typedef uint32_t w3 __attribute__((ext_vector_type(3), aligned(4)));
    typedef uint32_t w4 __attribute__((ext_vector_type(4), aligned(8)));
    if constexpr (N == 3) {
      const w3 t = read<NT>(reinterpret_cast<const w3*>(p));
      w[0] = t.x; w[1] = t.y; w[2] = t.z;
    } else {
#pragma unroll
      for (int i = 0; i + 4 <= N; i += 4) {
        const w4 t = read<NT>(reinterpret_cast<const w4*>(p + 4 * i));
        w[i] = t.x; w[i + 1] = t.y; w[i + 2] = t.z; w[i + 3] = t.w;
      }
      if constexpr (N % 4 == 2) {
        const w2 t = read<NT>(reinterpret_cast<const w2*>(p + 4 * (N - 2)));
        w[N - 2] = t.x; w[N - 1] = t.y;
      }
    }
  }
};

// Byte i of w as the exponent of an fp32 number.  The conversions take their scale's exponent and nothing else of it.
template <int N> __device__ __forceinline__ float exponent(const Words<N>& w, int i) {
  const uint32_t x = w.w[i >> 2];
  return __uint_as_float((i & 3) == 3 ? x >> 1 : x << (23 - 8 * (i & 3)));
}

__device__ __forceinline__ uint32_t two(uint32_t w, float scale, int byte) {
  switch (byte) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  }
}

// One record of 16 tokens as a lane (r = lane % 16, a = lane / 16) takes it: channels a D/4 .. of token r's key,
// bytes r of every block of the values of tokens 4 a .. 4 a + 3.
template <int D, bool NT> struct Tile {
  static constexpr int N = D / 32;
  Words<N> k, v, vs;
  uint32_t ks[2];  // exponents of the key's blocks that the channels lie in
  // rec is one address for the wave; unsigned offsets of a lane are added to it by the load itself.
  __device__ __forceinline__ void load_keys(const uint8_t* rec, uint32_t lane, uint32_t bad) {
    const uint32_t r = lane & 15, a = lane >> 4, g = a * (D / 4) / 32;
    k.template load<NT>(rec + (r * (D / 2) + a * (D / 8)));
    ks[0] = rec[16 * D + r * N + g] | bad;
    if constexpr (D != 64 && D != 128) ks[1] = rec[16 * D + r * N + (g + 1 < N ? g + 1 : g)] | bad;
  }
  __device__ __forceinline__ void load_values(const uint8_t* rec, uint32_t lane) {
    v.template load<NT>(rec + (8 * D + lane * (D / 8)));
    vs.template load<NT>(rec + (16 * D + D / 2 + (lane >> 4) * (D / 8)));
  }
  // The key's 8 channels a D/4 + 8 j ..
  __device__ __forceinline__ bf16x8 key(int j, int lane) const {
    uint32_t e = ks[0];
    if constexpr (D == 256) e = j < 4 ? ks[0] : ks[1];
    if constexpr (D == 96 || D == 192) {
      const int c = (lane >> 4) * (D / 4);
      e = (c + 8 * j) / 32 == c / 32 ? ks[0] : ks[1];
    }
    const float s = __uint_as_float(e << 23);
    const uint4 t = make_uint4(two(k.w[j], s, 0), two(k.w[j], s, 1), two(k.w[j], s, 2), two(k.w[j], s, 3));
    return __builtin_bit_cast(bf16x8, t);
  }
};

// Channels 32 g + r and 32 g + r + 16 of the values of eight tokens, four of each record.
template <int D, bool NT> __device__ __forceinline__ void values(const Tile<D, NT>& x, const Tile<D, NT>& y, int g, bf16x8& lo, bf16x8& hi) {
  constexpr int N = D / 32;
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = two(x.v.w[g], exponent(x.vs, i * N + g), i);
    c[i + 4] = two(y.v.w[g], exponent(y.vs, i * N + g), i);
  }
  uint32_t l[4], h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    l[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
    h[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
  }
  lo = __builtin_bit_cast(bf16x8, make_uint4(l[0], l[1], l[2], l[3]));
  hi = __builtin_bit_cast(bf16x8, make_uint4(h[0], h[1], h[2], h[3]));
}

// Eight fp32 values as bf16, or as three parts that keep their 24 bits.
template <int PARTS> __device__ __forceinline__ void parts(const float (&x)[8], bf16x8 (&out)[PARTS]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = bf16_pack2(r[2 * i], r[2 * i + 1]);
      if (p + 1 < PARTS) { r[2 * i] -= bf16_lo(w[i]); r[2 * i + 1] -= bf16_hi(w[i]); }
    }
    out[p] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
  }
}

__device__ __forceinline__ float across_rows_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

// Weights 2^(c (s - m)) of scores s under a maximum m, c = scale log2 e.  EXACT: to fp32's last places, with what c's own
// rounding leaves out; otherwise the product c m is rounded, by the same for every weight under m.
template <bool EXACT> struct Weight {
  float c, low;
  __device__ __forceinline__ explicit Weight(float scale) {
    c = scale * 1.44269504f;
    low = EXACT ? fmaf(scale, 1.92596299e-8f, fmaf(scale, 1.44269504f, -c)) : 0.f;
  }
  __device__ __forceinline__ float under(float m) const { return m == -INFINITY ? 0.f : EXACT ? m : m * c; }  // -inf: nothing seen yet
  __device__ __forceinline__ float operator()(float s, float under) const {
    if constexpr (EXACT) {
      const float d = s - under, x = fmaf(d, c, d * low);
      return __builtin_amdgcn_exp2f(d == -INFINITY ? d : x);
    } else {
      return __builtin_amdgcn_exp2f(fmaf(s, c, -under));
    }
  }
  // What sums under the maximum m are multiplied by under a larger one: between the same rounded products that the weights are
  // taken over (scores past 2^22 have them whole numbers: with m c itself sums of different maxima were 19 % apart).
  __device__ __forceinline__ float from(float m, float to) const {
#pragma clang fp contract(off)  // a fused m c would not be the rounded one
    if constexpr (EXACT) {
      return m == to ? 1.f : (*this)(m, under(to));
    } else {
      const float x = m * c - to * c;  // -inf of a maximum that is
      return __builtin_amdgcn_exp2f(m == to ? 0.f : x);
    }
  }
};

// ---- what a workgroup takes

// Rows of a sequence's new tokens (tiles of ROWS) and the keys that they can see.
struct Extent { int first, n, length, tiles, steps; };
template <int ROWS> __device__ __forceinline__ Extent extent(const AttentionArgs& a, int b) {
  Extent e;
  e.first = a.tok.seq.start(b);
  e.n = a.tok.seq.start(b + 1) - e.first;
  e.n = e.n < 0 ? 0 : e.n;
  const int length = a.tok.lengths[b];
  e.length = length < -(1 << 30) ? -(1 << 30) : length < 1 << 30 ? length : 1 << 30;
  const int most = a.tok.columns << (a.cache.shift + 4);
  const int seen = e.length < 0 ? 0 : e.length < most ? e.length : most;
  e.tiles = (e.n * a.group + ROWS - 1) / ROWS;
  e.steps = (seen + kStep - 1) / kStep;
  return e;
}

// Where a position among the sequences' weights lies: each thread sums the weights of a run of sequences, and
// `upto` [kThreads] holds the sums up to and with each run.  Sums end at kMostRounds, which none reaches whose offsets
// rise: others may, and a sum that wrapped would lead out of the arrays.
__device__ __forceinline__ int held(int x) { return x < kMostRounds ? x : kMostRounds; }
template <typename F> __device__ __forceinline__ int lay_out(int batch, F weight, int* upto) {
  if (batch == 1) return weight(0);
  __shared__ int waves[kWaves];
  const int run = (batch + kThreads - 1) / kThreads, tid = threadIdx.x;
  int x = 0;
  for (int b = tid * run; b < (tid + 1) * run && b < batch; ++b) x = held(x + weight(b));
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d);
    x = held(x + ((tid & 63) >= d ? y : 0));
  }
  if ((tid & 63) == 63) waves[tid >> 6] = x;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < tid >> 6) x = held(x + waves[w]);
    total = held(total + waves[w]);
  }
  upto[tid] = x;
  __syncthreads();
  return total;
}
// The sequence that holds position x of the total, and x's place in it.
template <typename F> __device__ __forceinline__ int seek(int batch, F weight, const int* upto, int x, int& at) {
  at = x;
  if (batch == 1) return 0;
  const int run = (batch + kThreads - 1) / kThreads;
  int first = 0;
  for (int j = 0; j < kWaves; ++j) {
    const unsigned long long hit = __builtin_amdgcn_ballot_w64(upto[64 * j + (threadIdx.x & 63)] > x);
    if (hit) {
      first = 64 * j + __builtin_ctzll(hit);
      break;
    }
  }
  if (first) at -= upto[first - 1];
  int b = first * run;
  while (b + 1 < batch) {
    const int w = weight(b);
    if (at < w) break;
    at -= w;
    ++b;
  }
  at = uniform(at);
  return uniform(b);
}

// Split sequences.  The steps of a tile of rows are counted in rounds, one step of each wave, one round at least. A
// key head's rounds of all sequences and tiles lie one after the other and are shared out evenly: workgroup u has
// rounds u each .. of them, whatever tiles they are of.  A tile that one workgroup has whole is written by it; of
// others it leaves the sums in one of its two slots, the second where the tile begins behind the workgroup's own first
// round.
//
// Where there are no more tiles than workgroups and the longest is not much longer than an even share, every tile is
// one workgroup's: a share that ends inside a tile costs a second start and the join of its parts, some kApart rounds
// (us, even shares and whole tiles: 256 requests of up to 1500 keys, 2 key heads of 256 channels 42.7 and 34.4, of up
// to 1000, 128 channels 23.3 and 19.6; 64 of 1500, 8 key heads 24.0 and 22.1).
__device__ __forceinline__ int rounds(const Extent& e) { return e.steps <= kWaves ? 1 : (e.steps + kWaves - 1) / kWaves; }
template <int ROWS> struct Rounds {
  const AttentionArgs& a;
  __device__ __forceinline__ int operator()(int b) const {
    const Extent e = extent<ROWS>(a, b);
    return e.tiles * rounds(e);
  }
};
template <int ROWS> struct Tiles {
  const AttentionArgs& a;
  __device__ __forceinline__ int operator()(int b) const { return extent<ROWS>(a, b).tiles; }
};
// The most rounds of a tile, over all sequences.
template <int ROWS> __device__ __forceinline__ int longest(const AttentionArgs& a) {
  __shared__ int most[kWaves];
  int x = 0;
  for (int b = threadIdx.x; b < a.tok.seq.batch; b += kThreads) {
    const Extent e = extent<ROWS>(a, b);
    x = e.tiles > 0 && rounds(e) > x ? rounds(e) : x;
  }
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_xor(x, d);
    x = y > x ? y : x;
  }
  if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x = most[w] > x ? most[w] : x;
  return uniform(x);
}

// ---- outputs

// Eight consecutive channels of a row; 16 lanes of a DPP row hold a block of 128 columns.
template <typename IO, bool FP8> __device__ __forceinline__ void put(const AttentionArgs& a, int token, int column, const float (&y)[8]) {
  if constexpr (FP8) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t m = __float_as_uint(y[i]) & 0x7FFFFFFFu;
      top = m > top ? m : top;
    }
    const float most = __uint_as_float(row_max16(top)) / 448.f;
    const float s = most < 0x1p-64f ? 0x1p-64f : most;  // a NaN stays
    const float inv = 1.f / s;
    uint32_t lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inv, y[1] * inv, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inv, y[3] * inv, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * inv, y[5] * inv, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * inv, y[7] * inv, hi, true);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.out) + (size_t)token * a.ld_out + column) = make_uint2(lo, hi);
    if ((column & 127) == 0) a.scales[(size_t)(column >> 7) * a.ld_scales + token] = s;
  } else {
    IO* dst = static_cast<IO*>(a.out) + (size_t)token * a.ld_out + column;
    st_elem4(dst, y[0], y[1], y[2], y[3]);
    st_elem4(dst + 4, y[4], y[5], y[6], y[7]);
  }
}

// ---- the kernel

// A wave's query rows: QT tiles of 16, with the sums over the keys so far.
template <typename IO, int D, int QT, bool SPLIT, bool FP8> struct Rows {
  // bf16 parts of a query and of a weight.  Three keep what an fp32 result has to (the scales of an 8-bit output among
  // them).  Under a bf16 result a weight's rounding to one is as large as the result's own: over many rows 1.2 to 1.35
  // times its error, of a few rows, where weights may lie in one part of their binade, up to 1.6 times.  Few rows have
  // two, and with them the result's own rounding alone (us, one part and two: 64 requests 60.8 and 62.2, 64 with 64
  // channels 40.8 and 44.6, one of 131072 keys 31.6 and 32.4; 512 new tokens over 32768 keys 325 and 415).
  static constexpr int N = D / 32, QP = sizeof(IO) == 2 ? 1 : 3, WP = FP8 || QP == 3 ? 3 : SPLIT && QT == 1 ? 2 : 1;
  Weight<WP == 3> weight;
  bf16x8 q[QT][N][QP];
  floatx4 o[QT][2 * N], l[QT];  // of channels 16 j + 4 (lane / 16) .., and of the weights
  float m[QT];
  bool unset = true;            // some row's maximum is -inf yet: it sees no keys so far, or its scores overflowed to that
  int lim[QT];                  // the last key that a lane's row sees
  __device__ __forceinline__ explicit Rows(float scale) : weight(scale) {}

  template <typename F> __device__ __forceinline__ void start(const AttentionArgs& a, const Extent& e, int h, int row0, int rows, int lane, F limit) {
    const int r = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const bool in = 16 * t + r < rows;
      const int row = in ? row0 + 16 * t + r : 0, i = a.by_group(row);
      lim[t] = in ? limit(row) : -1;
      const IO* src = static_cast<const IO*>(a.q) + (in ? (size_t)(e.first + i) * a.ldq + (size_t)(h * a.group + row - i * a.group) * a.q_head : 0) + kg * (D / 4);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        Raw<IO, 8> x;
        x.zero();
        if (in) x.load(src + 8 * j);
        if constexpr (QP == 1) {
          q[t][j][0] = __builtin_bit_cast(bf16x8, make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]));
        } else {
          float f[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) f[k] = x.get(k);
          parts<QP>(f, q[t][j]);
        }
      }
      m[t] = -INFINITY;
      l[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 2 * N; ++j) o[t][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Keys first .. first + 31, of two records: keys(i, j) are channels 8 j .. (of a lane's quarter) of record i's,
  // values(g, lo, hi) block g of both records' values.  EDGE: some row does not see all of them; spoil() then has
  // bit i of a lane's eight keys for values that are not finite.  used: called when keys have been read.
  template <bool EDGE, typename K, typename U, typename S, typename V>
  __device__ __forceinline__ void step(int first, int lane, K keys, U used, S spoil, V values) {
    const int kg = lane >> 4;
    floatx4 z[QT][2];
#pragma unroll
    for (int t = 0; t < QT; ++t) z[t][0] = z[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bf16x8 k = keys(i, j);
#pragma unroll
        for (int p = 0; p < QP; ++p)
#pragma unroll
          for (int t = 0; t < QT; ++t) z[t][i] = mfma(k, q[t][j][p], z[t][i]);
      }
    used();
    float w[QT][8];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) w[t][i] = z[t][i >> 2][i & 3];
    uint32_t spoilt = 0;
    if constexpr (EDGE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = first + (i >> 2) * 16 + kg * 4 + (i & 3);
#pragma unroll
        for (int t = 0; t < QT; ++t) w[t][i] = key <= lim[t] ? w[t][i] : -INFINITY;
      }
      spoilt = spoil();
    }
    const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
    bf16x8 p[QT][WP];
    auto weigh = [&](int t) INLINE {
      const float under = weight.under(m[t]);
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = weight(w[t][i], under);
      if (EDGE && __builtin_amdgcn_ballot_w64(spoilt != 0)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (spoilt >> i & 1) && w[t][i] != -INFINITY ? __builtin_nanf("") : f[i];
      }
      parts<WP>(f, p[t]);
      floatx4 sum = l[t];
#pragma unroll
      for (int k = 0; k < WP; ++k) sum = mfma(ones, p[t][k], sum);
      return sum;
    };
    floatx4 sum[QT];
    bool fine = !unset;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      sum[t] = weigh(t);
      fine = fine && sum[t][0] <= kMost;
    }
    if (__builtin_amdgcn_ballot_w64(!fine)) {
      unset = false;
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float top = m[t];
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, w[t][i]);
        top = across_rows_max(top);
        const float f = weight.from(m[t], top);
        m[t] = top;
        unset = unset || __builtin_amdgcn_ballot_w64(top == -INFINITY);
        l[t] *= f;
#pragma unroll
        for (int j = 0; j < 2 * N; ++j) o[t][j] *= f;
        sum[t] = weigh(t);
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) l[t] = sum[t];
#pragma unroll
    for (int g = 0; g < N; ++g) {
      bf16x8 lo, hi;
      values(g, lo, hi);
#pragma unroll
      for (int k = 0; k < WP; ++k)
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          o[t][2 * g] = mfma(lo, p[t][k], o[t][2 * g]);
          o[t][2 * g + 1] = mfma(hi, p[t][k], o[t][2 * g + 1]);
        }
    }
  }

  // The rows' results, a tile at a time through 16 x (D + 4) floats of LDS that are this wave's.
  __device__ __forceinline__ void finish(const AttentionArgs& a, const Extent& e, int h, int row0, int rows, int lane, float* so) {
    constexpr int PITCH = D + 4;
    const int r = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float inv = l[t][0] == 0.f ? 0.f : 1.f / l[t][0];
#pragma unroll
      for (int j = 0; j < 2 * N; ++j) *reinterpret_cast<floatx4*>(so + r * PITCH + 16 * j + 4 * kg) = o[t][j] * inv;
      wave_lds_sync();
      const int left = rows - 16 * t < 16 ? rows - 16 * t : 16;
      for (int i = lane; i < left * (D / 8); i += 64) {
        const int row = i / (D / 8), c = (i - row * (D / 8)) * 8;
        Vec<8> v;
        v.load(so + row * PITCH + c);
        const int at_row = row0 + 16 * t + row, tok = a.by_group(at_row);
        put<IO, FP8>(a, e.first + tok, (h * a.group + at_row - tok * a.group) * D + c, v.e);
      }
      wave_lds_sync();
    }
  }
};

// Zero weights may meet nothing but numbers: what lies behind the sequence (key >= n) may be anything, and values
// that are not finite (an exponent of 255; of 252 to 254 only where nothing was appended) are to reach the rows that
// see them by their weights.  Takes both out of the values of a lane's four tokens from `key`; bit i of the result:
// token i's were not finite.
template <int D, bool NT> __device__ __forceinline__ uint32_t cleaned(Tile<D, NT>& x, int key, int n) {
  constexpr int N = D / 32;
  uint32_t spoilt = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t nan = 0;
#pragma unroll
    for (int g = 0; g < N; ++g) {
      const int at = i * N + g, sh = 8 * (at & 3);
      nan |= (x.vs.w[at >> 2] >> sh & 255u) >= 252u;
    }
    const bool gone = key + i >= n;
    spoilt |= gone ? 0u : nan << i;
    if (gone || nan) {
#pragma unroll
      for (int g = 0; g < N; ++g) {
        const int at = i * N + g, sh = 8 * (at & 3);
        uint32_t& word = x.vs.w[at >> 2];
        word = (word & ~(255u << sh)) | 127u << sh;
      }
    }
  }
  return spoilt;
}
// Whether a byte of a lane's exponents is 252 or more.
template <int D, bool NT> __device__ __forceinline__ bool any_nan(const Tile<D, NT>& x) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const uint32_t y = ~x.vs.w[i] & 0xFCFCFCFCu;
    any |= (y - 0x01010101u) & ~y & 0x80808080u;  // a byte of y is 0
  }
  return any != 0;
}

// Tiles of rows that a wave takes at most, and waves a SIMD that its registers are held to.
constexpr int most_tiles_held(size_t io, int D, bool split) {
  return io == 4 ? (D > (split ? 64 : 96) ? 1 : 2) : D == 256 || (split && D == 192) ? 1 : !split && D == 96 ? 3 : 2;
}
constexpr int waves_held(size_t io, int D) { return io == 4 && D == 256 ? 1 : 2; }

// SPLIT: the workgroup's waves share the keys of one piece of a sequence for one tile of rows; its rows are
// written where the sequence is one piece, else left in `work` for join_kernel.  Otherwise each wave has
// a tile of rows of its own and all their keys.
template <typename IO, int D, int QT, bool SPLIT, bool FP8, bool NT>
__global__ __launch_bounds__(kThreads, waves_held(sizeof(IO), D)) void attention_kernel(AttentionArgs a) {
  constexpr int N = D / 32, ROWS = 16 * QT, PITCH = D + 4;
  __shared__ float shared[SPLIT ? kWaves * ROWS * PITCH + 2 * kWaves * ROWS : kWaves * 16 * PITCH];
  const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.cache.heads, h = blockIdx.x % G, u = blockIdx.x / G;

  __shared__ int upto[kThreads];
  const int batch = a.tok.seq.batch;
  const Rounds<ROWS> weight_of{a};
  auto blocks_of = [&](int b) INLINE { return extent<ROWS * kWaves>(a, b).tiles; };
  int x = u, x1 = u + 1, each = 1, place = 0, total;
  int b;
  bool entire = false;
  if constexpr (SPLIT) {
    total = lay_out(batch, weight_of, upto);
    total = total < a.most ? total : a.most;
    each = (int)(((uint32_t)total + a.share - 1) / a.share);
    if (batch > 1 && batch <= a.share && longest<ROWS>(a) <= each + kApart) {  // as many tiles as there are rows for
      __syncthreads();
      const int tiles = lay_out(batch, Tiles<ROWS>{a}, upto);
      entire = tiles <= a.share;
      if (entire) {
        total = tiles;
        each = 1;
      } else {
        __syncthreads();
        lay_out(batch, weight_of, upto);
      }
    }
    x = u * each;
    x1 = total - x < each ? total : x + each;
    if (a.plan && blockIdx.x == 0) {  // for join_kernel
      if (threadIdx.x == 0) a.plan[0] = entire ? 1 << 30 : each;  // nothing ends inside a tile
      const int run = (batch + kThreads - 1) / kThreads;
      int before = batch == 1 || threadIdx.x == 0 ? 0 : upto[threadIdx.x - 1];
      for (int i = threadIdx.x * run; i < (int)(threadIdx.x + 1) * run && i < batch; ++i) {
        a.plan[1 + i] = before;
        before = held(before + weight_of(i));
      }
    }
    if (x >= total) return;
    b = entire ? seek(batch, Tiles<ROWS>{a}, upto, x, place) : seek(batch, weight_of, upto, x, place);
  } else {
    total = lay_out(batch, blocks_of, upto);
    if (x >= total) return;
    b = seek(batch, blocks_of, upto, x, place);
  }
  // a tile, or a part of one, after the other
  for (; x < x1;) {
    Extent e = extent<ROWS>(a, b);
    e.first = uniform(e.first);
    e.n = uniform(e.n);
    e.length = uniform(e.length);
    e.tiles = uniform(e.tiles);
    e.steps = uniform(e.steps);
    const int all = rounds(e);
    // the last rows see the most keys: they go first
    const int tile = entire ? place : SPLIT ? place / all : ((e.tiles + kWaves - 1) / kWaves - 1 - place) * kWaves + wave;
    const int r0 = SPLIT && !entire ? place - tile * all : 0, r1 = SPLIT && !entire && x1 - x < all - r0 ? r0 + x1 - x : all;
    const bool whole_tile = !SPLIT || (r0 == 0 && r1 == all);
    const int row0 = tile * ROWS, rows = e.n * a.group - row0 < ROWS ? e.n * a.group - row0 : ROWS;
    if (!SPLIT && rows <= 0) return;
    const int most = a.tok.columns << (a.cache.shift + 4);
    auto limit = [&](int row) INLINE {  // the last key that a row sees; of keys past the table one, which reads as NaN
      const int place = e.length - e.n + a.by_group(row);
      return place < most ? place : most;
    };
    const int low = limit(row0), high = limit(row0 + rows - 1);
    Rows<IO, D, QT, SPLIT, FP8> mine(a.scale);
    mine.start(a, e, h, row0, rows, lane, limit);

    const int stride = SPLIT ? kWaves : 1;
    const int last = high < 0 ? 0 : high / kStep + 1;
    const int s1 = SPLIT && r1 < all && r1 * kWaves < last ? r1 * kWaves : last, s0 = SPLIT ? r0 * kWaves + wave : 0;

    // 64 entries of the sequence's row of the table, one a lane: a step's pages are a lane's value, with no load
    // between a step and the next one's records.
    const int32_t* row_of_table = a.tok.table + (size_t)b * a.tok.ld_table;
    int window = 0, entries = 0;
    auto look = [&](int j) INLINE {
      window = j;
      const int at = j + lane;
      entries = row_of_table[at < a.tok.columns ? at : a.tok.columns - 1];
      __builtin_amdgcn_s_waitcnt(0x0F70);  // here, where it is rare, and not at every use
    };
    struct Pages { int p0, p1; };
    auto pages = [&](int s) INLINE {
      const int j0 = 2 * s >> a.cache.shift, j1 = (2 * s + 1) >> a.cache.shift;
      if (j1 - window >= 64) look(j0);
      return Pages{__builtin_amdgcn_readlane(entries, j0 - window), __builtin_amdgcn_readlane(entries, j1 - window)};
    };
    using Two = Tile<D, NT>;
    struct Records { const uint8_t *r0, *r1; uint32_t b0, b1; };
    auto records = [&](int s, const Pages& p) INLINE {
      auto good = [&](int tile, int page) INLINE { return tile >> a.cache.shift < a.tok.columns && (unsigned)page < (unsigned)a.cache.pages; };
      const bool g0 = good(2 * s, p.p0), g1 = good(2 * s + 1, p.p1), used = kStep * s + 16 <= high;  // whether a row sees the second record
      Records x;
      x.r0 = record<D>(a.cache, g0 ? p.p0 : 0, h, 2 * s);
      x.r1 = used ? record<D>(a.cache, g1 ? p.p1 : 0, h, 2 * s + 1) : x.r0;
      x.b0 = g0 ? 0u : 255u;
      x.b1 = g1 || !used ? 0u : 255u;
      return x;
    };
    auto load_keys = [&](Two (&x)[2], const Records& r) INLINE {
      x[0].load_keys(r.r0, lane, r.b0);
      x[1].load_keys(r.r1, lane, r.b1);
    };
    auto load_values = [&](Two (&x)[2], const Records& r) INLINE {
      x[0].load_values(r.r0, lane);
      x[1].load_values(r.r1, lane);
    };
    const int n = e.length < most ? e.length : most + 1;  // keys there are
    auto compute = [&](Two (&x)[2], int s, auto at_edge, auto keys_used, auto values_used) INLINE {
      auto spoil = [&]() INLINE {
        if (kStep * s + kStep <= n && !__builtin_amdgcn_ballot_w64(any_nan(x[0]) || any_nan(x[1]))) return 0u;
        const uint32_t lo = cleaned(x[0], kStep * s + 4 * kg, n);
        return lo | cleaned(x[1], kStep * s + 16 + 4 * kg, n) << 4;
      };
      mine.template step<decltype(at_edge)::value>(kStep * s, lane, [&](int i, int j) INLINE { return x[i].key(j, lane); }, keys_used, spoil,
                                                   [&](int g, bf16x8& lo, bf16x8& hi) INLINE { values(x[0], x[1], g, lo, hi); });
      values_used();
    };

    if (s0 < s1) {
      const int whole = low < 0 ? 0 : (low + 1) / kStep, end = whole < s1 ? whole : s1;  // steps that every row sees all of
      // the last round loads what it has again: loads under a condition would be waited for
      auto after = [&](int s) INLINE { return s + stride < s1 ? s + stride : s; };
      Two now[2];
      look(2 * s0 >> a.cache.shift);
      Records r = records(s0, pages(s0));
      load_keys(now, r);
      load_values(now, r);
      int s = s0;
      if constexpr (SPLIT) {
        // a step ahead in registers of its own: the cache comes from memory
        Two next[2];
        auto one = [&](Two (&x)[2], Two (&y)[2], auto at_edge) INLINE {
          const int s2 = after(s);
          r = records(s2, pages(s2));
          load_keys(y, r);
          load_values(y, r);
          compute(x, s, at_edge, [] {}, [] {});
          s += stride;
        };
        while (s + stride < end) {  // two steps a round, so that the buffers change places without moves
          one(now, next, std::false_type{});
          one(next, now, std::false_type{});
        }
        if (s < end) {
          one(now, next, std::false_type{});
          now[0] = next[0];
          now[1] = next[1];
        }
        while (s < s1) {
          one(now, next, std::true_type{});
          now[0] = next[0];
          now[1] = next[1];
        }
      } else {
        // keys and values of the next step as soon as the registers are free: the cache comes from L2
        auto one = [&](auto at_edge) INLINE {
          const int s2 = after(s);
          r = records(s2, pages(s2));
          compute(now, s, at_edge, [&]() INLINE { load_keys(now, r); }, [&]() INLINE { load_values(now, r); });
          s += stride;
        };
        while (s < end) one(std::false_type{});
        while (s < s1) one(std::true_type{});
      }
    }

    if constexpr (SPLIT) {
      float* so = shared;                               // [waves][ROWS][PITCH]
      float* sm = shared + kWaves * ROWS * PITCH;       // [waves][ROWS] maxima, then sums
      float* sl = sm + kWaves * ROWS;
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const int row = wave * ROWS + 16 * t + r;
#pragma unroll
        for (int j = 0; j < 2 * N; ++j) *reinterpret_cast<floatx4*>(so + row * PITCH + 16 * j + 4 * kg) = mine.o[t][j];
        if (kg == 0) { sm[row] = mine.m[t]; sl[row] = mine.l[t][0]; }
      }
      __syncthreads();
      for (int i = threadIdx.x; i < rows * (D / 8); i += kThreads) {
        const int row = i / (D / 8), c = (i - row * (D / 8)) * 8;
        float to = -INFINITY, sum = 0.f, y[8] = {};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) to = fmaxf(to, sm[k * ROWS + row]);
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
          const float mk = sm[k * ROWS + row], f = mine.weight.from(mk, to);
          sum = fmaf(f, sl[k * ROWS + row], sum);
          Vec<8> v;
          v.load(so + (k * ROWS + row) * PITCH + c);
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = fmaf(f, v.e[j], y[j]);
        }
        if (whole_tile) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] *= inv;
          const int tok = a.by_group(row0 + row);
          put<IO, FP8>(a, e.first + tok, (h * a.group + row0 + row - tok * a.group) * D + c, y);
        } else {
          float* slot = a.work + ((size_t)blockIdx.x * 2 + (x == u * each ? 0 : 1)) * (ROWS * (D + 2));
          st_elem4(slot + row * D + c, y[0], y[1], y[2], y[3]);
          st_elem4(slot + row * D + c + 4, y[4], y[5], y[6], y[7]);
          if (c == 0) {
            slot[ROWS * D + row] = to;
            slot[ROWS * D + ROWS + row] = sum;
          }
        }
      }
      x += entire ? 1 : r1 - r0;
      place += r1 - r0;
      if (x < x1) {
        __syncthreads();  // `shared` is written again
        while (place >= e.tiles * rounds(e) && b + 1 < batch) {  // the next sequence that has rows
          e = extent<ROWS>(a, ++b);
          e.tiles = uniform(e.tiles);
          e.steps = uniform(e.steps);
          place = 0;
        }
      }
    } else {
      mine.finish(a, e, h, row0, rows, lane, shared + wave * 16 * PITCH);
      x = x1;
    }
  }
}

// Prompts: each of a workgroup's waves has a tile of rows, and all of them go over the keys together, 64 a step.  Each
// wave turns one of the step's four records into the products' operands, which all read from LDS: alone, every wave
// would turn all four.  Two buffers: a step's operands are made while the one before is summed, a barrier a step.  Past
// 128 channels one (48 and 64 KB), between two barriers, so that a CU holds two workgroups, one of which sums while the
// other turns (us, each wave for itself and this: 8192 tokens of 32 heads of 192 channels 816 -> 767, 2048 behind 14336
// 820 -> 712; 16 heads of 256 channels, 4096 tokens 225 -> 204, 32 heads, 2048 behind 14336 1459 -> 1272.  Two buffers
// and one workgroup a CU: 183 for the 158 of 4096 tokens of 16 heads of 192 channels, which take 166 with one).
template <typename IO, int D, int QT, bool FP8> __global__ __launch_bounds__(kThreads, 2) void prompt_kernel(AttentionArgs a) {
  constexpr int N = D / 32, ROWS = 16 * QT, PITCH = D + 4, KEYS = 16 * kWaves, BUFFERS = D > 128 ? 1 : 2;
  struct Operands { uint4 k[kWaves][N][64], v[kWaves / 2][2 * N][64]; };
  __shared__ union { Operands x[BUFFERS]; float so[kWaves * 16 * PITCH]; } shared;
  __shared__ uint32_t spoil[2][kWaves][4];
  __shared__ int upto[kThreads];
  const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  const int G = a.cache.heads, h = blockIdx.x % G, u = blockIdx.x / G;
  auto blocks_of = [&](int b) INLINE { return extent<ROWS * kWaves>(a, b).tiles; };
  if (u >= lay_out(a.tok.seq.batch, blocks_of, upto)) return;
  int place;
  const int b = seek(a.tok.seq.batch, blocks_of, upto, u, place);
  Extent e = extent<ROWS * kWaves>(a, b);
  e.first = uniform(e.first);
  e.n = uniform(e.n);
  e.length = uniform(e.length);
  e.tiles = uniform(e.tiles);
  // the last rows see the most keys: they go first
  const int block0 = (e.tiles - 1 - place) * (ROWS * kWaves), left = e.n * a.group - block0, row0 = block0 + wave * ROWS;
  const int rows = left - wave * ROWS < ROWS ? left - wave * ROWS : ROWS;
  const int most = a.tok.columns << (a.cache.shift + 4);
  auto limit = [&](int row) INLINE {  // the last key that a row sees; of keys past the table one, which reads as NaN
    const int place = e.length - e.n + a.by_group(row);
    return place < most ? place : most;
  };
  const int low = limit(block0), high = limit(block0 + (left < ROWS * kWaves ? left : ROWS * kWaves) - 1);  // of the workgroup
  const int mine_high = rows > 0 ? limit(row0 + rows - 1) : -1;
  Rows<IO, D, QT, false, FP8> mine(a.scale);
  mine.start(a, e, h, row0, rows, lane, limit);
  const int n = e.length < most ? e.length : most + 1;  // keys there are
  const int steps = high < 0 ? 0 : high / KEYS + 1, whole = low < 0 ? 0 : (low + 1) / KEYS;

  const int32_t* row_of_table = a.tok.table + (size_t)b * a.tok.ld_table;
  int window = 0, entries = 0;
  auto look = [&](int j) INLINE {  // 64 entries of the table's row, one a lane
    window = j;
    const int at = j + lane;
    entries = row_of_table[at < a.tok.columns ? at : a.tok.columns - 1];
    __builtin_amdgcn_s_waitcnt(0x0F70);  // here, where it is rare, and not at every use
  };
  Tile<D, false> x;
  auto load = [&](int s) INLINE {
    const int t = s * kWaves + wave, tile = t * 16 <= high ? t : high >> 4;  // behind the last key any row sees: that one's record
    const int j = tile >> a.cache.shift;
    if (j - window >= 64) look(j);
    const int page = __builtin_amdgcn_readlane(entries, j - window);
    const bool good = j < a.tok.columns && (unsigned)page < (unsigned)a.cache.pages;
    const uint8_t* rec = record<D>(a.cache, good ? page : 0, h, tile);
    x.load_keys(rec, lane, good ? 0u : 255u);
    x.load_values(rec, lane);
  };
  auto turn = [&](int s) INLINE {
    Operands& to = shared.x[s & (BUFFERS - 1)];
    if (s >= whole) {
      const uint32_t bad = cleaned(x, s * KEYS + wave * 16 + 4 * kg, n);
      if (r == 0) spoil[s & 1][wave][kg] = bad;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) to.k[wave][j][lane] = __builtin_bit_cast(uint4, x.key(j, lane));
#pragma unroll
    for (int g = 0; g < N; ++g) {
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = two(x.v.w[g], exponent(x.vs, i * N + g), i);
      uint2 lo, hi;
      lo.x = __builtin_amdgcn_perm(c[1], c[0], 0x05040100u);
      lo.y = __builtin_amdgcn_perm(c[3], c[2], 0x05040100u);
      hi.x = __builtin_amdgcn_perm(c[1], c[0], 0x07060302u);
      hi.y = __builtin_amdgcn_perm(c[3], c[2], 0x07060302u);
      reinterpret_cast<uint2*>(&to.v[wave >> 1][2 * g][lane])[wave & 1] = lo;
      reinterpret_cast<uint2*>(&to.v[wave >> 1][2 * g + 1][lane])[wave & 1] = hi;
    }
  };
  auto sum = [&](int s, auto at_edge) INLINE {
    const Operands& from = shared.x[s & (BUFFERS - 1)];
#pragma unroll
    for (int p = 0; p < kWaves / 2; ++p) {
      if (s * KEYS + 32 * p > mine_high) break;
      mine.template step<decltype(at_edge)::value>(
          s * KEYS + 32 * p, lane, [&](int i, int j) INLINE { return __builtin_bit_cast(bf16x8, from.k[2 * p + i][j][lane]); }, [] {},
          [&]() INLINE { return spoil[s & 1][2 * p][kg] | spoil[s & 1][2 * p + 1][kg] << 4; },
          [&](int g, bf16x8& lo, bf16x8& hi) INLINE {
            lo = __builtin_bit_cast(bf16x8, from.v[p][2 * g][lane]);
            hi = __builtin_bit_cast(bf16x8, from.v[p][2 * g + 1][lane]);
          });
    }
  };
  if (steps > 0) {
    look(0);
    load(0);
    turn(0);
    load(steps > 1 ? 1 : 0);
    lds_barrier();
    int s = 0;
    auto one = [&](auto at_edge) INLINE {
      if constexpr (BUFFERS == 1) {
        sum(s, at_edge);
        lds_barrier();
      }
      if (s + 1 < steps) {
        turn(s + 1);
        load(s + 2 < steps ? s + 2 : s + 1);
      }
      if constexpr (BUFFERS == 2) sum(s, at_edge);
      lds_barrier();
    };
    for (; s < whole && s < steps; ++s) one(std::false_type{});
    for (; s < steps; ++s) one(std::true_type{});
  }
  if (rows > 0) mine.finish(a, e, h, row0, rows, lane, shared.so + wave * 16 * PITCH);
}

// Joins what workgroups left of a tile.  A token's rows of a key head are pieces of 8 channels; a workgroup has `span`
// (a power of two from 16, a block of 128 columns, to 256) of them, and its groups of lanes take the slots in turn.
template <typename IO, int D, int QT, bool FP8> __global__ __launch_bounds__(kThreads) void join_kernel(AttentionArgs a) {
  constexpr int ROWS = 16 * QT;
  __shared__ float so[kThreads][8], sm[kThreads], sl[kThreads];
  const int G = a.cache.heads, spans = (a.group * (D / 8) + a.span - 1) / a.span;
  const int item = blockIdx.x / spans, t = item / G, h = item - t * G, tid = threadIdx.x;
  const int each = a.plan[0];
  const int b = uniform(a.tok.seq.of(t));
  const int before = a.plan[1 + b];
  const Extent e = extent<ROWS>(a, b);
  if (t < e.first || t >= e.first + e.n) return;
  const int all = rounds(e), groups = kThreads / a.span, group = tid / a.span;
  const int piece = (blockIdx.x - item * spans) * a.span + (tid & (a.span - 1)), g = piece / (D / 8), c = (piece - g * (D / 8)) * 8;
  const int row = (t - e.first) * a.group + g, tile = row / ROWS, in = row - tile * ROWS;
  const int i0 = before + tile * all, w0 = i0 / each, w1 = (i0 + all - 1) / each;
  const bool mine = g < a.group && w0 != w1;  // the others are written already
  const Weight<sizeof(IO) == 4 || FP8> weight(a.scale);
  float to = -INFINITY, sum = 0.f, y[8] = {};
  if (mine) {
    for (int w = w0 + group; w <= w1 && w < a.share; w += groups) {
      const float* slot = a.work + (((size_t)w * G + h) * 2 + (w == w0 && i0 != w0 * each ? 1 : 0)) * (ROWS * (D + 2));
      const float mk = slot[ROWS * D + in], lk = slot[ROWS * D + ROWS + in];
      Vec<8> v;
      v.load(slot + in * D + c);
      const float next = fmaxf(to, mk), f = weight.from(to, next), f2 = weight.from(mk, next);
      to = next;
      sum = fmaf(sum, f, lk * f2);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = fmaf(y[j], f, v.e[j] * f2);
    }
  }
  if (groups > 1) {
#pragma unroll
    for (int j = 0; j < 8; ++j) so[tid][j] = y[j];
    sm[tid] = to;
    sl[tid] = sum;
    __syncthreads();
    if (group == 0 && mine) {
      const int n = w1 - w0 + 1 < groups ? w1 - w0 + 1 : groups;
      const float own = to;
#pragma unroll 4
      for (int k = 1; k < n; ++k) to = fmaxf(to, sm[tid + k * a.span]);
      const float f = weight.from(own, to);
      sum *= f;
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] *= f;
#pragma unroll 4
      for (int k = 1; k < n; ++k) {
        const float f2 = weight.from(sm[tid + k * a.span], to);
        sum = fmaf(f2, sl[tid + k * a.span], sum);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = fmaf(f2, so[tid + k * a.span][j], y[j]);
      }
    }
  }
  if (group == 0 && mine) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] *= inv;
    put<IO, FP8>(a, t, (h * a.group + g) * D + c, y);
  }
}

// ---- the host's side

// Tiles of `rows` rows that a call has at most, whatever its offsets are.
int64_t most_tiles(int batch, int tokens, int group, int rows) {
  const int64_t whole = (int64_t)tokens * group / rows + batch, apart = (int64_t)tokens * ((group + rows - 1) / rows);
  return whole < apart ? whole : apart;
}
// The plan that join_kernel reads: rounds a workgroup has, then those before each sequence.
int64_t plan_words(int batch) { return ((int64_t)batch + 1 + 3) / 4 * 4; }
// Whether keys are split, by the rows that a sequence has on average, the workgroups of 128 rows that they would fill
// and the keys that the table has room for.  In us, split and by rows: one prompt of 128 tokens 6.3 and 9.2, of 256
// 11.8 and 12.4, of 512 26 and 19, of 2048 105 and 62, 100 prompts of 20 tokens 32 and 18; 64 requests of 16 tokens
// over up to 4000 keys 119 and 115, of 1000 71 and 41; 128 of 8 tokens (32 rows) 96 and 147, 65 and 52; few
// workgroups over many keys: 512 tokens over 1024 keys 23 and 30, over 4096 52 and 101, 1024 over 4096 96 and 103, 4
// x 256 over 16000 270 and 421.
bool splits(int batch, int tokens, int group, int G, int64_t capacity) {
  const int64_t rows = (int64_t)tokens * group / batch, workgroups = (int64_t)batch * ((rows + 127) / 128) * G;
  if (rows < (capacity > 1024 ? 64 : 32)) return true;
  const int64_t enough = capacity / 4 < kCUs / 2 ? kCUs / 2 : capacity / 4 < 2 * kCUs ? capacity / 4 : 2 * kCUs;
  return workgroups < enough;
}
// Workgroups a key head's rounds are shared out to: as many as are at work at once (by the registers of
// attention_kernel), and no more than there can be rounds.
int64_t most_rounds(int batch, int tokens, int group, int QT, int64_t capacity) {
  return most_tiles(batch, tokens, group, 16 * QT) * ((capacity + kStep * kWaves - 1) / (kStep * kWaves));
}
int shares(int batch, int tokens, int group, int G, int D, int QT, int64_t capacity) {
  const int held = kCUs * (QT == 2 ? (D == 64 ? 3 : 2) : D == 64 ? 4 : D <= 128 ? 3 : 2);
  const int64_t most = most_rounds(batch, tokens, group, QT, capacity);
  const int64_t n = held / G < 1 ? 1 : held / G;
  return (int)(n < most ? n : most);
}

// Tiles of rows a wave: two where the sequences' rows fill them and there is more than a round or so of work for
// every workgroup; with less, what counts is the time of one.  In us, one tile and two: a prompt of 128 tokens 6.3
// and 7.7, of 256 11.8 and 15.7, 4 of 100 behind 900 32.6 and 33.0, behind 7900 90 and 73, one of 512 behind 512 35
// and 23.
int split_tiles(int batch, int tokens, int group, int G, int64_t capacity) {
  return (int64_t)tokens * group > (int64_t)16 * batch && most_rounds(batch, tokens, group, 2, capacity) * G > 16 * kCUs ? 2 : 1;
}

template <typename IO, int D, bool FP8> int launch(const AttentionArgs& a, hipStream_t s) {
  const int batch = a.tok.seq.batch, tokens = a.tok.seq.tokens, G = a.cache.heads;
  const int64_t capacity = (int64_t)a.tok.columns << (a.cache.shift + 4);
  if (splits(batch, tokens, a.group, G, capacity)) {
    auto run = [&](auto qt) {
      constexpr int QT = decltype(qt)::value;
      AttentionArgs b = a;
      b.most = (int)most_rounds(batch, tokens, a.group, QT, capacity);
      b.share = shares(batch, tokens, a.group, G, D, QT, capacity);
      const int64_t workgroups = (int64_t)b.share * G;
      const bool join = capacity > kStep * kWaves && b.share > 1;  // a round is never split
      // few pieces a workgroup, so that many lanes share a tile's slots, until there are workgroups enough
      const int pieces = a.group * (D / 8);
      b.span = 16;
      while (b.span < 256 && b.span < pieces && (int64_t)tokens * G * ((pieces + b.span - 1) / b.span) > 4 * kCUs) b.span *= 2;
      const int64_t joins = (int64_t)tokens * G * ((pieces + b.span - 1) / b.span);
      if (!fits(workgroups, kThreads) || !fits(joins, kThreads) || most_rounds(batch, tokens, a.group, QT, capacity) >= kMostRounds) return -3;
      if (join) {
        b.plan = reinterpret_cast<int*>(a.work);
        b.work = reinterpret_cast<float*>(b.plan + plan_words(batch));
      }
      // Past the caches where the pool is larger than the last-level one.  One layer's cache read over and over: 64
      // requests of up to 8192 tokens 61.3 -> 56.8 us (pool 330 MB); 32 of 4096 with 16 key heads, out of that cache, 40.3
      // -> 45.7.  It is the pool that counts and not the part of it that a call can reach: a large pool is that of a model
      // whose layers pass in turn (eight of 1.1 GB, without and with: 32 of 4096 39.6 and 36.6 us a layer, 64 of 2000 34.7
      // and 31.0, 64 of 3500 56.8 and 50.6, one of 16384 14.5 and 14.8; one layer alone 34.4 and 35.6, 30.2 and 30.2, 48.0
      // and 50.4, 14.1 and 14.5).  Records of 128 channels only, where every load takes whole lines: of 64, 41.4 -> 54.4.
      constexpr bool CAN = D == 128 && QT == 1;
      const bool past = CAN && (int64_t)a.cache.pages * G * (17 * D) << a.cache.shift > (int64_t)256 << 20;
      if (past) hipLaunchKernelGGL((attention_kernel<IO, D, QT, true, FP8, CAN>), dim3((unsigned)workgroups), dim3(kThreads), 0, s, b);
      else hipLaunchKernelGGL((attention_kernel<IO, D, QT, true, FP8, false>), dim3((unsigned)workgroups), dim3(kThreads), 0, s, b);
      if (join && taken()) hipLaunchKernelGGL((join_kernel<IO, D, QT, FP8>), dim3((unsigned)joins), dim3(kThreads), 0, s, b);
      return 0;
    };
    if constexpr (most_tiles_held(sizeof(IO), D, true) > 1)
      if (split_tiles(batch, tokens, a.group, G, capacity) == 2) return run(std::integral_constant<int, 2>{});
    return run(std::integral_constant<int, 1>{});
  }
  constexpr int QT = most_tiles_held(sizeof(IO), D, false);
  const int64_t workgroups = most_tiles(batch, tokens, a.group, 16 * QT * kWaves) * G;
  if (!fits(workgroups, kThreads)) return -3;
  if constexpr (sizeof(IO) == 2) hipLaunchKernelGGL((prompt_kernel<IO, D, QT, FP8>), dim3((unsigned)workgroups), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((attention_kernel<IO, D, QT, false, FP8, false>), dim3((unsigned)workgroups), dim3(kThreads), 0, s, a);
  return 0;
}

template <typename IO, int D> int launch(const AttentionArgs& a, bool fp8, hipStream_t s) {
  if constexpr (D == 96 || D == 192) {
    return fp8 ? -2 : launch<IO, D, false>(a, s);
  } else {
    return fp8 ? launch<IO, D, true>(a, s) : launch<IO, D, false>(a, s);
  }
}

template <int D> int launch(const AttentionArgs& a, int io, bool fp8, hipStream_t s) {
  return io == 0 ? launch<float, D>(a, fp8, s) : launch<bf16_t, D>(a, fp8, s);
}

}  // namespace

int run_attention(const AttentionArgs& a, int D, int io, bool fp8, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (D) {
    case 64: return launch<64>(a, io, fp8, s);
    case 96: return launch<96>(a, io, fp8, s);
    case 128: return launch<128>(a, io, fp8, s);
    case 192: return launch<192>(a, io, fp8, s);
    case 256: return launch<256>(a, io, fp8, s);
  }
  return -2;
}

size_t attention_workspace(int batch, int tokens, int H, int G, int D, int columns, int page) {
  const int group = H / G;
  const int64_t capacity = (int64_t)columns * page;
  if (!splits(batch, tokens, group, G, capacity) || capacity <= kStep * kWaves) return 0;
  size_t most = 0;  // whichever tiles the type's kernel takes
  for (int QT = 1; QT <= 2; ++QT) {
    const size_t n = (size_t)shares(batch, tokens, group, G, D, QT, capacity) * G * 2 * (16 * QT) * (D + 2) * 4;
    most = n > most ? n : most;
  }
  return most + (size_t)plan_words(batch) * 4;
}

}  // namespace skssm
