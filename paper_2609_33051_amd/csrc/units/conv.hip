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
    if constexpr (SILU) { a *= sigmoid(a); b *= sigmoid(b); }
    set_pair<IO, CH>(y, i, a, b);
  }
  return y;
}

// Tokens of a workgroup, loaded together: 16, or 8 where 16 would leave less than
// four workgroups a CU.  16384 x 10240 bf16 (four taps): 127.7 us, 5.26 TB/s, what a copy
// of its size reaches (5.1 to 5.4); two loads of 8 133, 32 tokens as four loads of 8 139,
// 64 154, and 32 with ordinary loads and stores 150 (nothing here is read twice but
// the w - 1 tokens before a workgroup's).  777 x 1792 fp32: 6.5 us with 16, 5.4 with 8.
constexpr int kConvRows = 16, kConvFew = 8;

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
__global__ __launch_bounds__(256) void conv_kernel(ConvArgs a, int cols, int tiles) {
  constexpr int CH = 16 / sizeof(IO);
  const int c = ((blockIdx.x % cols) * 256 + threadIdx.x) * CH;
  const int part = blockIdx.x / cols;
  if (c >= a.C) return;
  if (part >= tiles) {
    conv_state<IO, W>(a, part - tiles, c);
    return;
  }
  const int T = a.seq.tokens, t0 = part * ROWS, t1 = min(T, t0 + ROWS);
  Taps<IO, W> k;
  k.load(a.taps, a.bias, c);
  const IO* x = static_cast<const IO*>(a.x) + c;
  IO* y = static_cast<IO*>(a.y) + c;
  const IO* in = static_cast<const IO*>(a.state_in);

  // lo is held to the row (offsets that do not start at 0), so that a state's row index stays in 0..W-2
  int b = a.seq.of(t0), lo = min(t0, a.seq.start(b)), hi = a.seq.start(b + 1);
  Raw<IO, CH> win[W - 1 + ROWS];  // the window, then the rows
  // the W - 1 inputs before row t of sequence b
  auto before = [&](int t) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int p = t - (W - 1) + j, s = p - lo + (W - 1);  // row of x; row of the state
      if (p >= lo) win[j].load(x + (size_t)p * a.ldx);
      else if (in) win[j].load(in + ((size_t)b * (W - 1) + s) * a.C + c);
      else win[j].zero();
    }
  };
  if (t0 + ROWS <= min(T, hi)) {  // all of one sequence
#pragma unroll
    for (int i = 0; i < ROWS; ++i) win[W - 1 + i].load_nt(x + (size_t)(t0 + i) * a.ldx);
    before(t0);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) store_nt<IO, CH>(conv_row<IO, W, SILU>(k, win + i), y + (size_t)(t0 + i) * a.ldy);
    return;
  }
  before(t0);
  for (int t = t0; t < t1;) {
    if (t >= hi && b + 1 < a.seq.batch) {  // the next sequence that has tokens (or the last one)
      do {
        ++b;
        lo = a.seq.start(b);
        hi = a.seq.start(b + 1);
      } while (t >= hi && b + 1 < a.seq.batch);
      lo = min(t, lo);
      before(t);
    }
    const int end = t >= hi ? t1 : min(t1, hi);  // of this sequence here
    for (; t < end; ++t) {
      win[W - 1].load(x + (size_t)t * a.ldx);
      store_nt<IO, CH>(conv_row<IO, W, SILU>(k, win), y + (size_t)t * a.ldy);
#pragma unroll
      for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
    }
  }
}

template <typename IO, int W, bool SILU, int ROWS>
int launch_conv_rows(const ConvArgs& a, bool apart, hipStream_t s) {
  constexpr int CH = 16 / sizeof(IO);
  const int cols = (a.C / CH + 255) / 256, tiles = (a.seq.tokens + ROWS - 1) / ROWS;
  const int states = a.state_out ? a.seq.batch : 0;
  const unsigned first = (unsigned)cols * (unsigned)(tiles + (apart ? 0 : states));
  if (first) hipLaunchKernelGGL((conv_kernel<IO, W, SILU, ROWS>), dim3(first), dim3(256), 0, s, a, cols, tiles);
  // the new states in place of the old ones: after the outputs, which read those
  if (apart && states)
    hipLaunchKernelGGL((conv_kernel<IO, W, SILU, ROWS>), dim3((unsigned)cols * (unsigned)states), dim3(256), 0, s, a, cols, 0);
  return 0;
}

template <typename IO, int W, bool SILU>
int launch_conv(const ConvArgs& a, bool apart, hipStream_t s) {
  const int64_t cols = (a.C / (16 / (int)sizeof(IO)) + 255) / 256;
  return cols * a.seq.tokens >= 4 * 256 * kConvRows ? launch_conv_rows<IO, W, SILU, kConvRows>(a, apart, s)
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
