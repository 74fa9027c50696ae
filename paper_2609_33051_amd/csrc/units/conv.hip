// The short depthwise causal convolution: packed prompts, and one token of
// every request into the replay buffer.
//
// y[t][c] = act(bias[c] + sum_j taps[c][j] x[t - (w-1) + j][c]): 2 w operations
// for four bytes moved (bf16), so both kernels are bound by memory.  A thread
// owns 16 bytes of channels.
#include "../mixer.h"

namespace skssm {

// A thread's channels: 16 bytes of io, their taps and bias.
template <typename IO, int W> struct Taps {
  static constexpr int CH = 16 / sizeof(IO);
  float t[W][CH], b[CH];
  __device__ __forceinline__ void load(const float* taps, const float* bias, int c) {
    Raw<float, CH * W> r;
    r.load(taps + (size_t)c * W);
    Raw<float, CH> rb;
    if (bias) rb.load(bias + c); else rb.zero();
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      b[i] = rb.get(i);
#pragma unroll
      for (int j = 0; j < W; ++j) t[j][i] = r.get(i * W + j);
    }
  }
  // The same for the 64 lanes of a wave whose first channel is c0, by `threads` threads through LDS: lanes
  // lie 128 bytes apart in the array (bf16, four taps), and an instruction that loads 16 of each would
  // take the 64 lines one after the other.  A lane's place in LDS is an odd number of 16 bytes.
  static constexpr int NT = CH * W / 4, NB = CH / 4, ST = NT | 1, SB = NB | 1, kShared = 64 * (ST + SB);  // in 16 bytes
  static __device__ __forceinline__ void share(uint4* lds, const float* taps, const float* bias, int c0, int C, int tid, int threads) {
    const int n = min(64 * CH, C - c0) / CH;  // lanes that have channels
    for (int j = tid; j < n * NT; j += threads) lds[j / NT * ST + j % NT] = reinterpret_cast<const uint4*>(taps + (size_t)c0 * W)[j];
    for (int j = tid; j < n * NB; j += threads)
      lds[64 * ST + j / NB * SB + j % NB] = bias ? reinterpret_cast<const uint4*>(bias + c0)[j] : make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void load(const uint4* lds, int lane) {
    float r[4 * NT], rb[4 * NB];
#pragma unroll
    for (int j = 0; j < NT; ++j) __builtin_memcpy(r + 4 * j, lds + lane * ST + j, 16);
#pragma unroll
    for (int j = 0; j < NB; ++j) __builtin_memcpy(rb + 4 * j, lds + 64 * ST + lane * SB + j, 16);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      b[i] = rb[i];
#pragma unroll
      for (int j = 0; j < W; ++j) t[j][i] = r[i * W + j];
    }
  }
  // z of the window's W inputs, oldest first
  __device__ __forceinline__ float sum(const Raw<IO, CH>* win, int i) const {
    float z = b[i];
#pragma unroll
    for (int j = 0; j < W; ++j) z = fmaf(t[j][i], win[j].get(i), z);
    return z;
  }
};

template <typename IO, int CH> __device__ __forceinline__ void set_pair(Raw<IO, CH>& r, int i, float a, float b) {
  if constexpr (sizeof(IO) == 2) r.w[i / 2] = bf16_pack2(a, b);
  else { r.e[i] = a; r.e[i + 1] = b; }
}

template <typename IO, int W, bool SILU>
__device__ __forceinline__ Raw<IO, 16 / sizeof(IO)> conv_row(const Taps<IO, W>& k, const Raw<IO, 16 / sizeof(IO)>* win) {
  constexpr int CH = 16 / sizeof(IO);
  Raw<IO, CH> y;
#pragma unroll
  for (int i = 0; i < CH; i += 2) {
    float a = k.sum(win, i), b = k.sum(win, i + 1);
    if constexpr (SILU) { a *= sigmoid<IO>(a); b *= sigmoid<IO>(b); }
    set_pair<IO, CH>(y, i, a, b);
  }
  return y;
}

// Tokens of a wave, loaded together, and waves of a workgroup, one below the other on the
// same 64 lanes of channels, so that they share their taps: 12, or 4 where there would be fewer than ten for
// each SIMD.  Measured, rows of 10240 bf16, four taps, 12 / 4 (us): 16384 tokens 119 / 128 (5.7 TB/s, 92 % of what the
// same loads and stores reach without the sums, 110; 16 tokens 119, 8 125), 4096 36.8 / 38.0,
// 512 6.8 / 7.8, 256 6.2 / 5.3; 777 x 1792 fp32 7.6 / 5.3.  Each thread loading its own taps took 10 more for the
// first.
// Rows are loaded and stored past the caches: a stream larger than them gains by it, one that the scan finds there loses
// less.  Stored past them / not, alone: 16384 tokens 119 / 137, 4096 36.3 / 37.3; with the
// scan behind it: 16384 446 / 448, 8192 244 / 241, 4096 151 / 145, 2048 88 / 84, 1024 62 / 62.
constexpr int kConvRows = 12, kConvFew = 4, kDown = 4;

template <typename IO, int CH> __device__ __forceinline__ void store_nt(const Raw<IO, CH>& r, IO* p) {
  static_assert(sizeof(r) == 16, "one store");
  __builtin_nontemporal_store(__builtin_bit_cast(uintx4, r), reinterpret_cast<uintx4*>(p));
}

// The new state of one sequence and 16 bytes of channels: rows of the old one
// where the sequence is shorter than w - 1 (row j comes from row j + length, so
// ascending order never reads a row that was written).
template <typename IO, int W>
__device__ __forceinline__ void conv_state(const ConvArgs& a, int b, int c) {
  constexpr int CH = 16 / sizeof(IO);
  const int lo = a.seq.start(b), hi = a.seq.start(b + 1), len = hi > lo ? hi - lo : 0;
  const IO* x = static_cast<const IO*>(a.x) + c;
  const IO* in = static_cast<const IO*>(a.state_in);
  const size_t base = (size_t)b * (W - 1) * a.C + c;
  for (int j = 0; j < W - 1; ++j) {
    const int past = j + len;  // row of state ++ sequence
    Raw<IO, CH> r;
    if (past >= W - 1) r.load(x + (size_t)(lo + past - (W - 1)) * a.ldx);
    else if (in) r.load(in + base + (size_t)past * a.C);
    else r.zero();
    r.store(static_cast<IO*>(a.state_out) + base + (size_t)j * a.C);
  }
}

template <typename IO, int W, bool SILU, int ROWS>
__global__ __launch_bounds__(64 * kDown) void conv_kernel(ConvArgs a, int cols, int tiles, int states) {
  constexpr int CH = 16 / sizeof(IO);
  __shared__ uint4 shared[Taps<IO, W>::kShared];
  const int lane = threadIdx.x & 63, c0 = (blockIdx.x % cols) * 64 * CH, c = c0 + lane * CH;
  const int part = blockIdx.x / cols * kDown + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int T = a.seq.tokens, t0 = part * ROWS;
  const bool work = part < tiles && c < a.C;
  const IO* x = static_cast<const IO*>(a.x) + c;
  IO* y = static_cast<IO*>(a.y) + c;
  const IO* in = static_cast<const IO*>(a.state_in);

  // the window, then the rows: loaded before the sequence is known, which takes loads of its own
  Raw<IO, CH> win[W - 1 + ROWS];
  if (work) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) win[W - 1 + i].load_nt(x + (size_t)min(t0 + i, T - 1) * a.ldx);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) win[j].load(x + (size_t)max(t0 - (W - 1) + j, 0) * a.ldx);
  }
  // lo is held to the row (offsets that do not start at 0), so that a state's row index stays in 0..W-2
  int b = 0, lo = 0, hi = 0;
  if (part < tiles) {
    b = a.seq.of(t0);
    lo = min(t0, a.seq.start(b));
    hi = a.seq.start(b + 1);
  }
  // row p < lo: one of the state's
  auto past = [&](Raw<IO, CH>& r, int p) {
    if (in) r.load(in + ((size_t)b * (W - 1) + (p - lo + (W - 1))) * a.C + c);
    else r.zero();
  };
  const bool whole = work && t0 + ROWS <= min(T, hi);  // all of one sequence
  if (whole) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
      if (t0 - (W - 1) + j < lo) past(win[j], t0 - (W - 1) + j);
  }
  Taps<IO, W>::share(shared, a.taps, a.bias, c0, a.C, threadIdx.x, 64 * kDown);
  lds_barrier();
  if (!work) {
    if (part >= tiles && part - tiles < states && c < a.C) conv_state<IO, W>(a, part - tiles, c);
    return;
  }
  Taps<IO, W> k;
  k.load(shared, lane);
  if (whole) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) store_nt<IO, CH>(conv_row<IO, W, SILU>(k, win + i), y + (size_t)(t0 + i) * a.ldy);
    return;
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int t = t0 + i;
    if (t >= T) break;
    if (t >= hi && b + 1 < a.seq.batch) {  // the next sequence that has tokens (or the last one)
      do {
        ++b;
        hi = a.seq.start(b + 1);
      } while (t >= hi && b + 1 < a.seq.batch);
      lo = min(t, a.seq.start(b));
    }
    Raw<IO, CH> w[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      if (t - (W - 1) + j >= lo) w[j] = win[i + j];
      else past(w[j], t - (W - 1) + j);
    }
    store_nt<IO, CH>(conv_row<IO, W, SILU>(k, w), y + (size_t)t * a.ldy);
  }
}

template <typename IO, int W, bool SILU, int ROWS>
int launch_conv_rows(const ConvArgs& a, bool apart, hipStream_t s) {
  constexpr int CH = 16 / sizeof(IO);
  const int cols = (a.C / CH + 63) / 64, tiles = (a.seq.tokens + ROWS - 1) / ROWS;
  const int states = a.state_out ? a.seq.batch : 0, with = apart ? 0 : states;
  const int64_t first = cols * (((int64_t)tiles + with + kDown - 1) / kDown), then = apart ? cols * (((int64_t)states + kDown - 1) / kDown) : 0;
  if (!fits(first, 64 * kDown) || !fits(then, 64 * kDown)) return -3;
  if (first) hipLaunchKernelGGL((conv_kernel<IO, W, SILU, ROWS>), dim3((unsigned)first), dim3(64 * kDown), 0, s, a, cols, tiles, with);
  // the new states in place of the old ones: after the outputs, which read those
  if (then && taken())
    hipLaunchKernelGGL((conv_kernel<IO, W, SILU, ROWS>), dim3((unsigned)then), dim3(64 * kDown), 0, s, a, cols, 0, states);
  return 0;
}

template <typename IO, int W, bool SILU>
int launch_conv(const ConvArgs& a, bool apart, hipStream_t s) {
  const int64_t cols = (a.C / (16 / (int)sizeof(IO)) + 63) / 64;
  return cols * a.seq.tokens >= 10 * 1024 ? launch_conv_rows<IO, W, SILU, kConvRows>(a, apart, s)
                                          : launch_conv_rows<IO, W, SILU, kConvFew>(a, apart, s);
}

template <typename IO, int W>
int launch_conv(const ConvArgs& a, int silu, bool apart, hipStream_t s) {
  return silu ? launch_conv<IO, W, true>(a, apart, s) : launch_conv<IO, W, false>(a, apart, s);
}

template <typename IO>
int launch_conv(const ConvArgs& a, int width, int silu, bool apart, hipStream_t s) {
  switch (width) {
    case 2: return launch_conv<IO, 2>(a, silu, apart, s);
    case 3: return launch_conv<IO, 3>(a, silu, apart, s);
    case 4: return launch_conv<IO, 4>(a, silu, apart, s);
    default: return -2;
  }
}

int run_conv(const ConvArgs& a, int width, int io, int silu, bool states_apart, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return io == 1 ? launch_conv<bf16_t>(a, width, silu, states_apart, s) : launch_conv<float>(a, width, silu, states_apart, s);
}

// One token of every request.  Workgroups of RB requests: first those of the x
// channels (256 threads of 16 bytes each, into ring.v), which also do the
// gates; then one per group, which convolves the group's B and C once, leaves
// them in LDS and writes them to every head of the group (ring.k and q): those
// writes, H (V + 2 K) values a request against the H V + 2 G K that are read, are
// half of what the call moves.  A thread's taps and bias, 10 bytes for each byte of x,
// serve RB requests.  10240 channels bf16, 8 groups of 16 heads, RB = 1 / 4 (us): 32 requests 4.5 / 5.5,
// 128 8.7 / 9.2, 170 12.0 / 9.9, 256 15.9 / 11.5 (5.0 TB/s), 1024 69 / 64 (3.6: past the caches the
// slots' 128 and 256 byte pieces cost).
template <typename IO, int W, int RB>
__global__ __launch_bounds__(256) void conv_token_kernel(ConvTokenArgs a, int xparts) {
  constexpr int CH = 16 / sizeof(IO);
  const int parts = xparts + a.G, b0 = blockIdx.x / parts * RB, part = blockIdx.x % parts, tid = threadIdx.x;
  const int HV = a.H * a.V, GK = a.G * a.K, C = HV + 2 * GK;
  auto x = [&](int b) { return static_cast<const IO*>(a.x) + (size_t)b * a.ldx; };
  auto state = [&](int b) { return static_cast<IO*>(a.state) + (size_t)b * (W - 1) * C; };
  if (part < xparts) {
    const int c = (part * 256 + tid) * CH;
    if (c < HV) {
      Taps<IO, W> k;
      Raw<IO, CH> win[RB][W];
#pragma unroll
      for (int q = 0; q < RB; ++q) {
        const int b = min(b0 + q, a.B - 1);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) win[q][j].load(state(b) + (size_t)j * C + c);
        win[q][W - 1].load(x(b) + c);
      }
      k.load(a.taps, a.bias, c);
      const int h = c / a.V;
#pragma unroll
      for (int q = 0; q < RB; ++q) {
        const int b = b0 + q;
        if (b >= a.B) break;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) win[q][j + 1].store(state(b) + (size_t)j * C + c);
        conv_row<IO, W, true>(k, win[q]).store(static_cast<IO*>(a.rv) + (((size_t)b * a.H + h) * a.W + a.n) * a.V + (c - h * a.V));
      }
    }
    for (int i = part * 256 + tid; i < RB * a.H; i += xparts * 256) {
      const int b = b0 + i / a.H, h = i % a.H;
      if (b >= a.B) break;
      const float r = ld_elem(static_cast<const IO*>(a.dt) + (size_t)b * a.lddt + h) + (a.dt_bias ? a.dt_bias[h] : 0.f);
      const float beta = softplus(r);
      const size_t at = ((size_t)b * a.H + h) * a.W + a.n;
      a.rbeta[at] = beta;
      a.rla[at] = beta * a.A[h];
    }
    return;
  }
  __shared__ uint4 row[RB][2 * 128 / CH];
  const int g = part - xparts, chunks = a.K / CH, rep = a.H / a.G, count = min(RB, a.B - b0);
  for (int i = tid; i < count * 2 * chunks; i += 256) {
    const int q = i / (2 * chunks), j = i % (2 * chunks), side = j / chunks, c = HV + side * GK + g * a.K + (j - side * chunks) * CH;
    Taps<IO, W> k;
    Raw<IO, CH> win[W];
#pragma unroll
    for (int t = 0; t < W - 1; ++t) win[t].load(state(b0 + q) + (size_t)t * C + c);
    win[W - 1].load(x(b0 + q) + c);
    k.load(a.taps, a.bias, c);
#pragma unroll
    for (int t = 0; t < W - 1; ++t) win[t + 1].store(state(b0 + q) + (size_t)t * C + c);
    conv_row<IO, W, true>(k, win).store(reinterpret_cast<IO*>(&row[q][j]));
  }
  __syncthreads();
  for (int i = tid; i < count * 2 * rep * chunks; i += 256) {
    const int at = i % chunks, hh = i / chunks % rep, qs = i / chunks / rep, side = qs & 1, q = qs >> 1;
    const size_t item = (size_t)(b0 + q) * a.H + g * rep + hh;
    IO* dst = side ? static_cast<IO*>(a.q) + item * a.K : static_cast<IO*>(a.rk) + (item * a.W + a.n) * a.K;
    reinterpret_cast<uint4*>(dst)[at] = row[q][side * chunks + at];
  }
}

template <typename IO, int W>
int launch_conv_token(const ConvTokenArgs& a, hipStream_t s) {
  constexpr int CH = 16 / sizeof(IO);
  const int xparts = (a.H * a.V / CH + 255) / 256;
  const unsigned parts = (unsigned)(xparts + a.G);
  // four requests a workgroup where that leaves seven workgroups for four CUs
  if ((int64_t)parts * a.B >= 4 * 448)
    hipLaunchKernelGGL((conv_token_kernel<IO, W, 4>), dim3(parts * (unsigned)((a.B + 3) / 4)), dim3(256), 0, s, a, xparts);
  else
    hipLaunchKernelGGL((conv_token_kernel<IO, W, 1>), dim3(parts * (unsigned)a.B), dim3(256), 0, s, a, xparts);
  return 0;
}

template <typename IO>
int launch_conv_token(const ConvTokenArgs& a, int width, hipStream_t s) {
  switch (width) {
    case 2: return launch_conv_token<IO, 2>(a, s);
    case 3: return launch_conv_token<IO, 3>(a, s);
    case 4: return launch_conv_token<IO, 4>(a, s);
    default: return -2;
  }
}

int run_conv_token(const ConvTokenArgs& a, int width, int io, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return io == 1 ? launch_conv_token<bf16_t>(a, width, s) : launch_conv_token<float>(a, width, s);
}

}  // namespace skssm
