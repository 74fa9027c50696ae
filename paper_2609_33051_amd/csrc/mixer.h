// Argument blocks and device helpers of the operators around the recurrence
// (convolution, scan, norm, 8-bit products).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "args.h"
#include "device.h"

namespace skssm {

// Packed sequences: sequence b is rows start(b) .. start(b + 1) - 1 of `tokens`.
// Offsets come from device memory and are held to 0..tokens here, so that no
// access leaves the arrays whatever they hold.
struct Sequences {
  const int32_t* offsets;  // [batch + 1], or NULL: equal lengths
  int batch, tokens, each; // each = tokens / batch (offsets NULL)
  __device__ __forceinline__ int start(int b) const {
    if (!offsets) return b * each;
    const int o = offsets[b];
    return o < 0 ? 0 : o > tokens ? tokens : o;
  }
  // The sequence that holds row t: the last one that starts at or before it.
  __device__ __forceinline__ int of(int t) const {
    if (!offsets) return t / each;
    int lo = 0, hi = batch;  // start(lo) <= t (or lo = 0), start(hi) > t (or hi = batch)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start(mid) <= t) lo = mid; else hi = mid;
    }
    return lo;
  }
};

// e^x of x <= 0, as 2^p 2^l with p = x log2 e rounded and l what p leaves out (the product's own rounding
// and that of log2 e); 2^l = 1 + l ln 2.  The instruction's 2^p alone is |x| 2^-24 off, which step
// sizes of 1e-3 and less would show: they and their decays are stored in fp32 whatever io is.
// Held to x = -104, where 2^p is 0 already, for l of an infinity; a NaN stays.
__device__ __forceinline__ float exp_down(float x) {
  x = x < -104.f ? -104.f : x;
  const float p = x * 1.44269504f, l = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269504f, -p)), e = __builtin_amdgcn_exp2f(p);
  return fmaf(e, l * 0.693147181f, e);
}
// For results of type IO: under bf16 (and e4m3 beside it) the plain exponential's |z| 2^-24, 2^-17 at
// the most, is nothing, and the exact one costs 6 to 13 % (convolution of 16384 and 4096 tokens, 119.7 -> 127.5
// and 36.9 -> 41.7 us; gated norm of 8192 rows 68.8 -> 72.2).  In fp32 it is nearly free (8192
// tokens 116.1 -> 117.0, 777 4.9 -> 5.3, gated norm of 4096 rows 73.8 -> 73.6).
template <typename IO> __device__ __forceinline__ float sigmoid(float z) {
  if constexpr (sizeof(IO) == 2) {
    return __builtin_amdgcn_rcpf(1.f + fast_exp(-z));
  } else {
    const float e = exp_down(-fabsf(z));
    return __builtin_amdgcn_rcpf(1.f + e) * (z < 0.f ? e : 1.f);
  }
}
// log(1 + e^r) = max(r, 0) + log(1 + e), e = e^{-|r|}, to a few units of fp32 also where e is
// small: log(1 + e) = 2 artanh(z), z = e / (2 + e) <= 1/3,
// by its series 2 z (1 + z^2 / 3 + z^4 / 5 + ..), whose ninth term is below 2^-28.
__device__ __forceinline__ float softplus(float r) {
  const float e = exp_down(-fabsf(r)), z = e * __builtin_amdgcn_rcpf(2.f + e), q = z * z;
  float t = 1.f / 15.f;
#pragma unroll
  for (int k = 13; k >= 1; k -= 2) t = fmaf(t, q, 1.f / (float)k);
  return fmaf(2.f * z, t, fmaxf(r, 0.f));
}

// What a launch can hold: fewer than 2^32 threads.  A call whose launches do not all fit makes none and returns -3.
inline bool fits(int64_t workgroups, int threads) { return workgroups * threads < (int64_t)1 << 32; }
// Whether the launches so far were taken: one that follows from them is not made where they were not.
inline bool taken() { return hipPeekAtLastError() == hipSuccess; }

struct ConvArgs {
  Sequences seq;
  int C;                  // channels
  const void* x;          // rows ldx elements apart
  size_t ldx;
  const float* taps;      // [C][w]
  const float* bias;      // [C] or NULL
  const void* state_in;   // [batch][w-1][C] or NULL
  void* state_out;        // or NULL
  void* y;
  size_t ldy;
};
// `states_apart`: the new states are written by a launch of their own, after the outputs'
int run_conv(const ConvArgs& a, int width, int io, int silu, bool states_apart, void* stream);

struct ConvTokenArgs {
  int B, H, G, W, n, K, V;
  const void* x;          // [B][H V + 2 G K], rows ldx apart
  size_t ldx;
  const float* taps;
  const float* bias;
  void* state;            // [B][w-1][C]
  const void* dt;         // [B][H], rows lddt apart
  size_t lddt;
  const float* dt_bias;
  const float* A;
  void* rk;               // ring fields [B][H][W][..], slot n
  void* rv;
  float* rbeta;
  float* rla;
  void* q;                // [B][H][K]
};
int run_conv_token(const ConvTokenArgs& a, int width, int io, void* stream);

struct NormArgs {
  int rows, columns, group;
  int skip_width;
  float eps;
  const void* x;
  size_t ldx;
  const void* residual;
  size_t ld_residual;
  void* residual_out;
  size_t ld_residual_out;
  const void* gate;
  size_t ld_gate;
  const void* skip;
  size_t ld_skip, skip_head;
  const float* D;
  const float* weight;
  void* out;
  size_t ld_out;
  float* scales;
  size_t ld_scales;
};
int run_norm(const NormArgs& a, int x_dtype, int io, int out, void* stream);

struct MatmulArgs {
  int M, N, K;
  const uint8_t* a;
  size_t lda;
  const float* sa;
  size_t ldsa;
  const uint8_t* w;
  size_t ldw;
  const float* sw;
  void* y;
  size_t ldy;
  float* part;            // split products, [splits][M][N]
};
int run_matmul_fp8(const MatmulArgs& a, int out, void* stream);
size_t matmul_fp8_workspace(int M, int N, int K);

struct ScanArgs {
  Sequences seq;
  int H, G;
  const void* x;
  size_t ldx;
  const void* b;
  size_t ldb;
  const void* c;
  size_t ldc;
  const void* dt;
  size_t lddt;
  const float* dt_bias;
  const float* A;
  const float* D;
  const float* S_in;
  float* S_out;
  void* y;
  size_t ldy;
  float* work;
};
int run_scan(const ScanArgs& a, int K, int V, int io, void* stream);
size_t scan_workspace(int batch, int tokens, int H, int G, int K, int V);

}  // namespace skssm
