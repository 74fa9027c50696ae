// The selective scan of packed prompts (Mamba-2 form), by chunks of 64 tokens on
// the matrix cores.  With g_t the sum of log decays from the chunk's start and
// S the state before it,
//     y_t = e^{g_t} S C_t + sum_{s <= t} e^{g_t - g_s} dt_s <B_s, C_t> x_s + D x_t,
//     S' = e^{g_L} S + sum_s (e^{g_L - g_s} dt_s x_s) B_s^T,
// every exponent <= 0.  A workgroup of four waves owns a head and a run of tokens
// and goes through it chunk by chunk; the state stays in its registers (V / 4
// value channels a wave) and each input is read once.
//
// Fragments.  Both operands of a product hold, per lane, 8 consecutive indices of
// a 32-deep reduction (lane group g = lane / 16: 8 g .. 8 g + 7) of the row or
// column lane % 16.  The state's accumulator tiles are assigned to channels so
// that two of them are such a fragment as they lie: tile kt, row m is channel
// 32 (kt / 2) + 8 (m / 4) + 4 (kt % 2) + m % 4.
//
// Few sequences: a sequence is split into segments of `seg` tokens.  A first
// launch runs the state part of every segment but a sequence's last, from zero
// (the first: from S_in), and keeps its end state and total decay; the second
// begins each segment from the states before it, joined.
#include "../mixer.h"

namespace skssm {

constexpr int kChunk = 64;
constexpr int kGates = 4 * kChunk;  // tokens whose gates are computed together, a chunk per wave

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// 64 rows of COLS elements in LDS.  16-byte chunks of a row are permuted by the
// row, so that rows read together (16 lanes, the same columns) and the four rows
// of a transposed read lie in different banks.
template <typename IO, int COLS> struct Tile {
  static constexpr int kBytes = kChunk * COLS * (int)sizeof(IO), kChunks = COLS * (int)sizeof(IO) / 16;
  static constexpr int kPer = 16 / (int)sizeof(IO);  // elements of a chunk
  static __device__ __forceinline__ int at(int row, int col) {  // byte offset
    const int c = col / kPer;
    const int key = kChunks >= 16 ? ((row & 3) << 2) | ((row >> 2) & 3) : ((row & 3) << 1) | ((row >> 2) & 1);
    return row * (COLS * (int)sizeof(IO)) + ((c ^ key) << 4) + (col % kPer) * (int)sizeof(IO);
  }
};

struct FragF32 { float e[8]; };

template <typename IO> struct Frags;
template <> struct Frags<bf16_t> {
  using F = bf16x8;
  // 8 consecutive columns of one row
  template <int COLS> static __device__ __forceinline__ F row(const char* t, int row, int col) {
    return __builtin_bit_cast(F, *reinterpret_cast<const uint4*>(t + Tile<bf16_t, COLS>::at(row, col)));
  }
  // 8 consecutive rows (row0 ..) of the column that the lane's place i = lane % 16 stands
  // for, where places 4 p .. 4 p + 3 are columns col(p) .. col(p) + 3: a transposed read takes,
  // from the lanes of a group, four rows of four 8-byte pieces
  template <int COLS, class Col> static __device__ __forceinline__ F cols(const char* t, int row0, int i, Col col) {
    typedef __attribute__((address_space(3))) shortx4* lds4;
    const int r = row0 + (i >> 2), c = col(i & 3);
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(t + Tile<bf16_t, COLS>::at(r, c)));
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(t + Tile<bf16_t, COLS>::at(r + 4, c)));
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
  template <int COLS> static __device__ __forceinline__ F row(const char* t, int row, int col) {
    F f;
    const float4 a = *reinterpret_cast<const float4*>(t + Tile<float, COLS>::at(row, col));
    const float4 b = *reinterpret_cast<const float4*>(t + Tile<float, COLS>::at(row, col + 4));
    f.e[0] = a.x; f.e[1] = a.y; f.e[2] = a.z; f.e[3] = a.w;
    f.e[4] = b.x; f.e[5] = b.y; f.e[6] = b.z; f.e[7] = b.w;
    return f;
  }
  template <int COLS, class Col> static __device__ __forceinline__ F cols(const char* t, int row0, int i, Col col) {
    F f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.e[e] = *reinterpret_cast<const float*>(t + Tile<float, COLS>::at(row0 + e, col(i >> 2) + (i & 3)));
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

// x weighted per token, as the state's update takes it: fp32, or two bf16 parts that
// hold 16 bits of the product (what enters the state is not rounded to one bf16).
template <typename IO> struct Weighted;
template <> struct Weighted<float> {
  FragF32 f;
  __device__ __forceinline__ void set(const FragF32& x, const float* w) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.e[e] = x.e[e] * w[e];
  }
  __device__ __forceinline__ floatx4 mma(const FragF32& a, floatx4 c) const { return Frags<float>::mma(a, f, c); }
};
template <> struct Weighted<bf16_t> {
  bf16x8 hi, lo;
  __device__ __forceinline__ void set(bf16x8 x, const float* w) {
    const uint4 u = __builtin_bit_cast(uint4, x);
    const uint32_t in[4] = {u.x, u.y, u.z, u.w};
    uint32_t h[4], l[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float a = bf16_lo(in[p]) * w[2 * p], b = bf16_hi(in[p]) * w[2 * p + 1];
      h[p] = bf16_pack2(a, b);
      l[p] = bf16_pack2(a - bf16_lo(h[p]), b - bf16_hi(h[p]));
    }
    hi = __builtin_bit_cast(bf16x8, make_uint4(h[0], h[1], h[2], h[3]));
    lo = __builtin_bit_cast(bf16x8, make_uint4(l[0], l[1], l[2], l[3]));
  }
  __device__ __forceinline__ floatx4 mma(bf16x8 a, floatx4 c) const {
    return Frags<bf16_t>::mma(a, lo, Frags<bf16_t>::mma(a, hi, c));
  }
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

// LOCAL: the state part alone, over the segment before the slot's (first launch).
template <typename IO, int K, int V, bool LOCAL>
__global__ __launch_bounds__(256) void scan_kernel(ScanArgs a, int seg, bool apart) {
  using FR = Frags<IO>;
  using F = typename FR::F;
  using TB = Tile<IO, K>;
  using TX = Tile<IO, V>;
  using TM = Tile<IO, kChunk>;
  constexpr int KT = K / 16, KF = K / 32, VT = V / 64, PER = TB::kPer;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % a.H, slot = blockIdx.x / a.H, grp = h / (a.H / a.G);

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
  char* const lm = lc + TB::kBytes;
  float* const gates = reinterpret_cast<float*>(LOCAL ? lc : lm + TM::kBytes);
  float* const ghi = gates;             // g of the chunk in two parts, log2
  float* const glo = gates + kGates;
  float* const gdt = gates + 2 * kGates;
  float* const get = gates + 3 * kGates;  // 2^{g_t}
  float* const gws = gates + 4 * kGates;  // dt_s 2^{g_L - g_s}
  float* const gend = gates + 5 * kGates; // g_L of the four chunks

  // channels of the lane's pieces: value channels of place 4 p, key channels of tile kt
  auto vcol = [&](int u, int p) { return VT == 2 ? 32 * wave + 8 * p + 4 * u : 16 * wave + 4 * p; };
  auto kcol = [&](int kt, int p) { return 32 * (kt >> 1) + 8 * p + 4 * (kt & 1); };
  // the lane's four values (v = place i, channels of group g) of tile (u, kt) in a tile-major state
  auto state_at = [&](int u, int kt) {
    const int v = vcol(u, i >> 2) + (i & 3), k = kcol(kt, g);
    return ((v >> 4) * (K / 16) + (k >> 4)) * 256 + 4 * ((v & 15) + 16 * ((k & 15) >> 2));
  };
  auto work_at = [&](int j) { return a.work + ((size_t)(j - 1) * a.H + h) * (V * K); };  // before segment start j
  float* const decays = a.work ? a.work + (size_t)(a.seq.tokens / seg) * a.H * (V * K) : nullptr;
  auto own_at = [&](int u, int kt) { return (((wave * VT + u) * KT + kt) * 64 + lane) * 4; };

  floatx4 S[VT][KT];
  if (s.k == 0) {
    const float* in = a.S_in ? a.S_in + ((size_t)s.b * a.H + h) * (V * K) : nullptr;
#pragma unroll
    for (int u = 0; u < VT; ++u)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) S[u][kt] = in ? *reinterpret_cast<const floatx4*>(in + state_at(u, kt)) : floatx4{0.f, 0.f, 0.f, 0.f};
  } else {
#pragma unroll
    for (int u = 0; u < VT; ++u)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) S[u][kt] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (!LOCAL) {
      for (int k = 0; k < s.k; ++k) {  // the segments before this one, in order
        const int j = (int)(((int64_t)s.lo + (int64_t)(k + 1) * seg) / seg);
        const float* w = work_at(j);
        const float d = k ? __builtin_amdgcn_exp2f(decays[(size_t)(j - 1) * a.H + h]) : 0.f;
#pragma unroll
        for (int u = 0; u < VT; ++u)
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            const floatx4 t = *reinterpret_cast<const floatx4*>(w + own_at(u, kt));
#pragma unroll
            for (int e = 0; e < 4; ++e) S[u][kt][e] = k ? fmaf(S[u][kt][e], d, t[e]) : t[e];
          }
      }
    }
  }

  // a chunk's rows in registers on their way to LDS: 16-byte pieces, zero past the segment
  constexpr int NB = kChunk * TB::kChunks / 256, NX = kChunk * TX::kChunks / 256;
  uint4 pb[NB], pc[NB], px[NX];
  auto fetch = [&](int p) {
    const int n = s.p1 - p;
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      const int at = q * 256 + tid, row = at / TB::kChunks, c = (at % TB::kChunks) * PER;
      pb[q] = make_uint4(0, 0, 0, 0);
      if (!LOCAL) pc[q] = make_uint4(0, 0, 0, 0);
      if (row < n) {
        pb[q] = *reinterpret_cast<const uint4*>(static_cast<const IO*>(a.b) + (size_t)(p + row) * a.ldb + grp * K + c);
        if (!LOCAL) pc[q] = *reinterpret_cast<const uint4*>(static_cast<const IO*>(a.c) + (size_t)(p + row) * a.ldc + grp * K + c);
      }
    }
#pragma unroll
    for (int q = 0; q < NX; ++q) {
      const int at = q * 256 + tid, row = at / TX::kChunks, c = (at % TX::kChunks) * PER;
      px[q] = make_uint4(0, 0, 0, 0);
      if (row < n) px[q] = *reinterpret_cast<const uint4*>(static_cast<const IO*>(a.x) + (size_t)(p + row) * a.ldx + (size_t)h * V + c);
    }
  };
  auto put = [&]() {
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      const int at = q * 256 + tid, row = at / TB::kChunks, c = (at % TB::kChunks) * PER;
      *reinterpret_cast<uint4*>(lb + TB::at(row, c)) = pb[q];
      if (!LOCAL) *reinterpret_cast<uint4*>(lc + TB::at(row, c)) = pc[q];
    }
#pragma unroll
    for (int q = 0; q < NX; ++q) {
      const int at = q * 256 + tid, row = at / TX::kChunks, c = (at % TX::kChunks) * PER;
      *reinterpret_cast<uint4*>(lx + TX::at(row, c)) = px[q];
    }
  };
  // step sizes and decays of four chunks.  Sums of log decays run in 64 bits: a token that
  // forgets everything (held to 2^-150, which is 0 in fp32) must not blur the differences
  // of those after it.
  const float A2 = a.A[h] * 1.44269504f, bias = a.dt_bias ? a.dt_bias[h] : 0.f;
  auto gate = [&](int p) {
    const int t = p + tid;
    float dt = 0.f, la = 0.f;
    if (t < s.p1) {
      dt = softplus(ld_elem(static_cast<const IO*>(a.dt) + (size_t)t * a.lddt + h) + bias);
      la = fmaxf(dt * A2, -150.f);
    }
    double sum = (double)la;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double up = __shfl_up(sum, o);
      if (lane >= o) sum += up;
    }
    const double end = __shfl(sum, 63);
    const float hi = (float)sum;
    ghi[tid] = hi;
    glo[tid] = (float)(sum - (double)hi);
    gdt[tid] = dt;
    get[tid] = __builtin_amdgcn_exp2f(hi);
    gws[tid] = dt * __builtin_amdgcn_exp2f((float)(end - sum));
    if (lane == 0) gend[wave] = (float)end;
  };

  float total = 0.f;
  if (s.p0 < s.p1) fetch(s.p0);
  int part = 0;
  for (int p = s.p0; p < s.p1; p += kChunk, part = (part + 1) & 3) {
    __syncthreads();
    put();
    if (part == 0) gate(p);
    __syncthreads();
    if (p + kChunk < s.p1) fetch(p + kChunk);
    const int go = part * kChunk, n = s.p1 - p;

    if constexpr (!LOCAL) {
      // scores of the wave's 16 tokens t (place i) against s <= t, with decay and step: rows of M
      const int t = 16 * wave + i;
      F ct[KF];
#pragma unroll
      for (int kf = 0; kf < KF; ++kf) ct[kf] = FR::template row<K>(lc, t, 32 * kf + 8 * g);
      const float th = ghi[go + t], tl = glo[go + t];
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        if (st > (wave | 1)) continue;  // (pairs of tiles: a fragment of M is 32 tokens deep)
        floatx4 m = {0.f, 0.f, 0.f, 0.f};
        if (st <= wave) {
#pragma unroll
          for (int kf = 0; kf < KF; ++kf) m = FR::mma(FR::template row<K>(lb, 16 * st + i, 32 * kf + 8 * g), ct[kf], m);
          const int s0 = 16 * st + 4 * g;
          const float4 sh = *reinterpret_cast<const float4*>(ghi + go + s0), sl = *reinterpret_cast<const float4*>(glo + go + s0),
                       sd = *reinterpret_cast<const float4*>(gdt + go + s0);
          const float h4[4] = {sh.x, sh.y, sh.z, sh.w}, l4[4] = {sl.x, sl.y, sl.z, sl.w}, d4[4] = {sd.x, sd.y, sd.z, sd.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            m[e] = s0 + e <= t ? m[e] * d4[e] * __builtin_amdgcn_exp2f((th - h4[e]) + (tl - l4[e])) : 0.f;
        }
        FR::store4(lm, TM::at(t, 16 * st + 4 * g), m[0], m[1], m[2], m[3]);
      }
    }
    F xt[VT][2];
#pragma unroll
    for (int u = 0; u < VT; ++u)
#pragma unroll
      for (int sf = 0; sf < 2; ++sf) xt[u][sf] = FR::template cols<V>(lx, 32 * sf + 8 * g, i, [&](int q) { return vcol(u, q); });
    if constexpr (!LOCAL) {
      __syncthreads();
      F sk[VT][KF];
#pragma unroll
      for (int u = 0; u < VT; ++u)
#pragma unroll
        for (int kf = 0; kf < KF; ++kf) sk[u][kf] = FR::of(S[u][2 * kf], S[u][2 * kf + 1]);
      const float D = a.D ? a.D[h] : 0.f;
#pragma unroll
      for (int tt = 0; tt < 4; ++tt) {
        const int t = 16 * tt + i;
        floatx4 off[VT], y[VT];
#pragma unroll
        for (int u = 0; u < VT; ++u) off[u] = y[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kf = 0; kf < KF; ++kf) {
          const F ct = FR::template row<K>(lc, t, 32 * kf + 8 * g);
#pragma unroll
          for (int u = 0; u < VT; ++u) off[u] = FR::mma(sk[u][kf], ct, off[u]);
        }
#pragma unroll
        for (int sf = 0; sf <= tt / 2; ++sf) {
          const F mt = FR::template row<kChunk>(lm, t, 32 * sf + 8 * g);
#pragma unroll
          for (int u = 0; u < VT; ++u) y[u] = FR::mma(xt[u][sf], mt, y[u]);
        }
        const float et = get[go + t];
        if (t < n) {
          IO* dst = static_cast<IO*>(a.y) + (size_t)(p + t) * a.ldy + (size_t)h * V;
#pragma unroll
          for (int u = 0; u < VT; ++u) {
            const int v = vcol(u, g);
            Raw<IO, 4> x;
            x.load(reinterpret_cast<const IO*>(lx + TX::at(t, v)));
#pragma unroll
            for (int e = 0; e < 4; ++e) y[u][e] = fmaf(off[u][e], et, y[u][e]) + D * x.get(e);
            st_elem4(dst + v, y[u][0], y[u][1], y[u][2], y[u][3]);
          }
        }
      }
    }
    // the state: decay, then the chunk's tokens
    const float end = gend[part], d = __builtin_amdgcn_exp2f(end);
    total += end;
#pragma unroll
    for (int u = 0; u < VT; ++u)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) S[u][kt] *= d;
#pragma unroll
    for (int sf = 0; sf < 2; ++sf) {
      Weighted<IO> w[VT];
      Vec<8> ws;
      ws.load(gws + go + 32 * sf + 8 * g);
#pragma unroll
      for (int u = 0; u < VT; ++u) w[u].set(xt[u][sf], ws.e);
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const F bt = FR::template cols<K>(lb, 32 * sf + 8 * g, i, [&](int q) { return kcol(kt, q); });
#pragma unroll
        for (int u = 0; u < VT; ++u) S[u][kt] = w[u].mma(bt, S[u][kt]);
      }
    }
  }

  if (LOCAL) {
    float* w = work_at(slot + 1);
#pragma unroll
    for (int u = 0; u < VT; ++u)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) *reinterpret_cast<floatx4*>(w + own_at(u, kt)) = S[u][kt];
    if (tid == 0) decays[(size_t)slot * a.H + h] = total;
  } else if (s.p1 == s.hi && a.S_out) {
    // S_out in place of S_in: other segments' workgroups may still read it, so that a later
    // segment leaves its state where only this workgroup reads, for a copy after the launch
    const bool keep = apart && s.k > 0;
    float* out = keep ? work_at(slot - a.seq.batch + 1) : a.S_out + ((size_t)s.b * a.H + h) * (V * K);
#pragma unroll
    for (int u = 0; u < VT; ++u)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) *reinterpret_cast<floatx4*>(out + (keep ? own_at(u, kt) : state_at(u, kt))) = S[u][kt];
  }
}

// The end states that a launch in place left in the workspace, into S_out.
template <int K, int V>
__global__ __launch_bounds__(256) void scan_states_kernel(ScanArgs a, int seg) {
  constexpr int KT = K / 16, VT = V / 64;
  const int h = blockIdx.x % a.H, j = blockIdx.x / a.H + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i = lane & 15, g = lane >> 4;
  Segment s;
  if (!s.later(a.seq, j, seg) || s.p1 != s.hi) return;
  const float* w = a.work + ((size_t)(j - 1) * a.H + h) * (V * K);
  float* out = a.S_out + ((size_t)s.b * a.H + h) * (V * K);
  for (int u = 0; u < VT; ++u)
    for (int kt = 0; kt < KT; ++kt) {
      const int v = (VT == 2 ? 32 * wave + 8 * (i >> 2) + 4 * u : 16 * wave + 4 * (i >> 2)) + (i & 3);
      const int k = 32 * (kt >> 1) + 8 * g + 4 * (kt & 1);
      const int at = ((v >> 4) * (K / 16) + (k >> 4)) * 256 + 4 * ((v & 15) + 16 * ((k & 15) >> 2));
      *reinterpret_cast<floatx4*>(out + at) = *reinterpret_cast<const floatx4*>(w + (((wave * VT + u) * KT + kt) * 64 + lane) * 4);
    }
}

// Tokens of a segment: long enough to leave about `kWant` workgroups where one
// per sequence and head would be fewer, and a multiple of the gates' 256 tokens.
constexpr int kWant = 1024;
int scan_segment(int batch, int tokens, int H) {
  const int64_t items = (int64_t)batch * H;
  if (items >= kWant) return tokens > 0 ? tokens : 1;
  int64_t seg = ((int64_t)tokens * H + kWant - 1) / kWant;
  seg = (seg + kGates - 1) / kGates * kGates;
  return seg < kGates ? kGates : seg > tokens ? (tokens > 0 ? tokens : 1) : (int)seg;
}

size_t scan_workspace(int batch, int tokens, int H, int K, int V) {
  const int seg = scan_segment(batch, tokens, H);
  if (seg >= tokens) return 0;
  return (size_t)(tokens / seg) * H * ((size_t)V * K + 1) * sizeof(float);
}

template <typename IO, int K, int V>
int launch_scan(const ScanArgs& a, hipStream_t s) {
  const int seg = scan_segment(a.seq.batch, a.seq.tokens, a.H);
  const int windows = seg < a.seq.tokens ? a.seq.tokens / seg : 0;
  const bool apart = windows && a.S_in && a.S_in == a.S_out;
  constexpr size_t gates = (5 * kGates + 4) * sizeof(float);
  constexpr size_t local = Tile<IO, K>::kBytes + Tile<IO, V>::kBytes + gates;
  constexpr size_t full = local + Tile<IO, K>::kBytes + Tile<IO, kChunk>::kBytes;
  if (windows)
    hipLaunchKernelGGL((scan_kernel<IO, K, V, true>), dim3((unsigned)windows * (unsigned)a.H), dim3(256), local, s, a, seg, false);
  hipLaunchKernelGGL((scan_kernel<IO, K, V, false>), dim3((unsigned)(a.seq.batch + windows) * (unsigned)a.H), dim3(256), full, s, a,
                     seg, apart);
  if (apart) hipLaunchKernelGGL((scan_states_kernel<K, V>), dim3((unsigned)windows * (unsigned)a.H), dim3(256), 0, s, a, seg);
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
