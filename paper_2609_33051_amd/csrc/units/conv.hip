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

constexpr int kConvRows = 32;   // tokens of a workgroup
constexpr int kConvBatch = 8;   // rows loaded together

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

template <typename IO, int W, bool SILU>
__global__ __launch_bounds__(256) void conv_kernel(ConvArgs a, int cols, int tiles) {
  constexpr int CH = 16 / sizeof(IO);
  const int c = ((blockIdx.x % cols) * 256 + threadIdx.x) * CH;
  const int part = blockIdx.x / cols;
  if (c >= a.C) return;
  if (part >= tiles) {
    conv_state<IO, W>(a, part - tiles, c);
    return;
  }
  const int T = a.seq.tokens, t0 = part * kConvRows, t1 = min(T, t0 + kConvRows);
  Taps<IO, W> k;
  k.load(a.taps, a.bias, c);
  const IO* x = static_cast<const IO*>(a.x) + c;
  IO* y = static_cast<IO*>(a.y) + c;
  const IO* in = static_cast<const IO*>(a.state_in);

  // lo is held to the row (offsets that do not start at 0), so that a state's row index stays in 0..W-2
  int b = a.seq.of(t0), lo = min(t0, a.seq.start(b)), hi = a.seq.start(b + 1);
  Raw<IO, CH> win[W - 1 + kConvBatch];  // the window, then the batch's rows
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
  before(t0);
  int t = t0;
  while (t < t1) {
    if (t >= hi && b + 1 < a.seq.batch) {  // the next sequence that has tokens (or the last one)
      do {
        ++b;
        lo = a.seq.start(b);
        hi = a.seq.start(b + 1);
      } while (t >= hi && b + 1 < a.seq.batch);
      lo = min(t, lo);
      before(t);
    }
    const int run = (t >= hi ? t1 : min(t1, hi)) - t;  // rows of this sequence here
    if (run >= kConvBatch) {
#pragma unroll
      for (int i = 0; i < kConvBatch; ++i) win[W - 1 + i].load(x + (size_t)(t + i) * a.ldx);
#pragma unroll
      for (int i = 0; i < kConvBatch; ++i) conv_row<IO, W, SILU>(k, win + i).store(y + (size_t)(t + i) * a.ldy);
#pragma unroll
      for (int j = 0; j < W - 1; ++j) win[j] = win[kConvBatch + j];
      t += kConvBatch;
    } else {
      for (int i = 0; i < run; ++i, ++t) {
        win[W - 1].load(x + (size_t)t * a.ldx);
        conv_row<IO, W, SILU>(k, win).store(y + (size_t)t * a.ldy);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
      }
    }
  }
}

template <typename IO, int W, bool SILU>
int launch_conv(const ConvArgs& a, bool apart, hipStream_t s) {
  constexpr int CH = 16 / sizeof(IO);
  const int cols = (a.C / CH + 255) / 256, tiles = (a.seq.tokens + kConvRows - 1) / kConvRows;
  const int states = a.state_out ? a.seq.batch : 0;
  const unsigned first = (unsigned)cols * (unsigned)(tiles + (apart ? 0 : states));
  if (first) hipLaunchKernelGGL((conv_kernel<IO, W, SILU>), dim3(first), dim3(256), 0, s, a, cols, tiles);
  if (apart && states)
    hipLaunchKernelGGL((conv_kernel<IO, W, SILU>), dim3((unsigned)cols * (unsigned)states), dim3(256), 0, s, a, cols, 0);
  return 0;
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

// One token of every request.  Workgroups of request b: first those of the x
// channels (256 threads of 16 bytes each, into ring.v), which also do the
// gates; then one per group, which convolves the group's B and C once, leaves
// them in LDS and writes them to every head of the group (ring.k and q): those
// writes, H (V + 2 K) values a request against the H V + 2 G K that are read, are
// what the call moves.
template <typename IO, int W>
__global__ __launch_bounds__(256) void conv_token_kernel(ConvTokenArgs a, int xparts) {
  constexpr int CH = 16 / sizeof(IO);
  const int parts = xparts + a.G, b = blockIdx.x / parts, part = blockIdx.x % parts, tid = threadIdx.x;
  const int HV = a.H * a.V, GK = a.G * a.K, C = HV + 2 * GK;
  const IO* x = static_cast<const IO*>(a.x) + (size_t)b * a.ldx;
  IO* state = static_cast<IO*>(a.state) + (size_t)b * (W - 1) * C;
  auto conv = [&](int c) {
    Taps<IO, W> k;
    Raw<IO, CH> win[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) win[j].load(state + (size_t)j * C + c);
    win[W - 1].load(x + c);
    k.load(a.taps, a.bias, c);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) win[j + 1].store(state + (size_t)j * C + c);
    return conv_row<IO, W, true>(k, win);
  };
  if (part < xparts) {
    const int c = (part * 256 + tid) * CH;
    if (c < HV) {
      const int h = c / a.V;
      conv(c).store(static_cast<IO*>(a.rv) + (((size_t)b * a.H + h) * a.W + a.n) * a.V + (c - h * a.V));
    }
    for (int h = part * 256 + tid; h < a.H; h += xparts * 256) {
      const float r = ld_elem(static_cast<const IO*>(a.dt) + (size_t)b * a.lddt + h) + (a.dt_bias ? a.dt_bias[h] : 0.f);
      const float beta = softplus(r);
      const size_t at = ((size_t)b * a.H + h) * a.W + a.n;
      a.rbeta[at] = beta;
      a.rla[at] = beta * a.A[h];
    }
    return;
  }
  __shared__ uint4 row[2 * 128 / CH];
  const int g = part - xparts, chunks = a.K / CH, rep = a.H / a.G;
  if (tid < 2 * chunks) {
    const int side = tid / chunks, c = HV + side * GK + g * a.K + (tid - side * chunks) * CH;
    conv(c).store(reinterpret_cast<IO*>(&row[tid]));
  }
  __syncthreads();
  for (int i = tid; i < 2 * rep * chunks; i += 256) {
    const int side = i / (rep * chunks), j = i - side * rep * chunks, hh = j / chunks, at = j - hh * chunks;
    const size_t item = (size_t)b * a.H + g * rep + hh;
    IO* dst = side ? static_cast<IO*>(a.q) + item * a.K : static_cast<IO*>(a.rk) + (item * a.W + a.n) * a.K;
    reinterpret_cast<uint4*>(dst)[at] = row[side * chunks + at];
  }
}

template <typename IO>
int launch_conv_token(const ConvTokenArgs& a, int width, hipStream_t s) {
  constexpr int CH = 16 / sizeof(IO);
  const int xparts = (a.H * a.V / CH + 255) / 256;
  const dim3 grid((unsigned)a.B * (unsigned)(xparts + a.G));
  switch (width) {
    case 2: hipLaunchKernelGGL((conv_token_kernel<IO, 2>), grid, dim3(256), 0, s, a, xparts); return 0;
    case 3: hipLaunchKernelGGL((conv_token_kernel<IO, 3>), grid, dim3(256), 0, s, a, xparts); return 0;
    case 4: hipLaunchKernelGGL((conv_token_kernel<IO, 4>), grid, dim3(256), 0, s, a, xparts); return 0;
    default: return -2;
  }
}

int run_conv_token(const ConvTokenArgs& a, int width, int io, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return io == 1 ? launch_conv_token<bf16_t>(a, width, s) : launch_conv_token<float>(a, width, s);
}

}  // namespace skssm
