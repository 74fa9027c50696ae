// Root-mean-square norm over groups of columns, with the residual's addition
// or the gate (and skip term) before it and 8-bit blocks with scales after it.
//
// One pass: a workgroup holds a group's values in registers between the sum of
// squares and the output, so every array moves once and the kernel is bound by
// memory.  A lane owns 8 consecutive columns at a time, 16 lanes (one DPP row)
// a block of 128, whose largest value is a reduction inside the row.
#include "../mixer.h"

namespace skssm {

enum NormForm { PLAIN = 0, RESIDUAL = 1, GATED = 2, GATED_SKIP = 3 };

// Largest of a row's 16 values, by their bits: magnitudes order as integers, NaN above all.
__device__ __forceinline__ uint32_t row_max16(uint32_t x) {
  auto step = [](uint32_t v, uint32_t w) { return v > w ? v : w; };
  x = step(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));
  x = step(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));
  x = step(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true));
  x = step(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, true));
  return x;
}

template <typename TX, typename IO, bool FP8, int FORM, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormArgs a) {
  const int groups = a.columns / a.group, row = blockIdx.x / groups, g = blockIdx.x - row * groups, tid = threadIdx.x;
  const int first = g * a.group, n = a.group;
  const TX* x = static_cast<const TX*>(a.x) + (size_t)row * a.ldx + first;
  float u[NV][8];
  float ss = 0.f;
  Raw<TX, 8> rx[NV];
  Raw<IO, 8> r1[NV], r2[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * THREADS + tid) * 8;
    rx[v].zero();
    if (c < n) {
      rx[v].load(x + c);
      if constexpr (FORM == RESIDUAL) r1[v].load(static_cast<const IO*>(a.residual) + (size_t)row * a.ld_residual + first + c);
      if constexpr (FORM >= GATED) r1[v].load(static_cast<const IO*>(a.gate) + (size_t)row * a.ld_gate + first + c);
      if constexpr (FORM == GATED_SKIP) {
        const int h = (first + c) / a.skip_width;
        r2[v].load(static_cast<const IO*>(a.skip) + (size_t)row * a.ld_skip + (size_t)h * a.skip_head + (first + c - h * a.skip_width));
      }
    }
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * THREADS + tid) * 8;
    const bool in = c < n;
    float d = 0.f;
    if constexpr (FORM == GATED_SKIP) d = in ? a.D[(first + c) / a.skip_width] : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float t = rx[v].get(i);
      if constexpr (FORM == RESIDUAL) t += r1[v].get(i);
      if constexpr (FORM == GATED_SKIP) t = fmaf(d, r2[v].get(i), t);
      if constexpr (FORM >= GATED) { const float z = r1[v].get(i); t *= z * sigmoid<IO>(z); }
      u[v][i] = in ? t : 0.f;
      ss = fmaf(u[v][i], u[v][i], ss);
    }
    if constexpr (FORM == RESIDUAL) {
      if (in && a.residual_out) {
        IO* dst = static_cast<IO*>(a.residual_out) + (size_t)row * a.ld_residual_out + first + c;
        st_elem4(dst, u[v][0], u[v][1], u[v][2], u[v][3]);
        st_elem4(dst + 4, u[v][4], u[v][5], u[v][6], u[v][7]);
      }
    }
  }
  ss = wave_sum(ss);
  if constexpr (THREADS > 64) {
    __shared__ float part[THREADS / 64];
    if ((tid & 63) == 0) part[tid >> 6] = ss;
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) ss += part[i];
  }
  const float scale = rsqrtf(ss / (float)n + a.eps);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * THREADS + tid) * 8;
    const bool in = c < n;
    Vec<8> w;
    if (in) w.load(a.weight + first + c);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u[v][i] = in ? u[v][i] * scale * w.e[i] : 0.f;
      const uint32_t m = __float_as_uint(u[v][i]) & 0x7FFFFFFFu;
      top = m > top ? m : top;
    }
    if constexpr (FP8) {
      const float most = __uint_as_float(row_max16(top)) / 448.f;
      const float s = most < 0x1p-64f ? 0x1p-64f : most;  // a NaN stays
      const float inv = 1.f / s;
      if (in) {
        uint32_t lo = 0, hi = 0;
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(u[v][0] * inv, u[v][1] * inv, lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(u[v][2] * inv, u[v][3] * inv, lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(u[v][4] * inv, u[v][5] * inv, hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(u[v][6] * inv, u[v][7] * inv, hi, true);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.out) + (size_t)row * a.ld_out + first + c) = make_uint2(lo, hi);
        if ((tid & 15) == 0) a.scales[(size_t)((first + c) >> 7) * a.ld_scales + row] = s;
      }
    } else if (in) {
      IO* dst = static_cast<IO*>(a.out) + (size_t)row * a.ld_out + first + c;
      st_elem4(dst, u[v][0], u[v][1], u[v][2], u[v][3]);
      st_elem4(dst + 4, u[v][4], u[v][5], u[v][6], u[v][7]);
    }
  }
}

template <typename TX, typename IO, bool FP8, int FORM, int THREADS, int NV>
int launch_norm(const NormArgs& a, hipStream_t s) {
  const int64_t workgroups = (int64_t)a.rows * (a.columns / a.group);
  if (!fits(workgroups, THREADS)) return -3;
  hipLaunchKernelGGL((norm_kernel<TX, IO, FP8, FORM, THREADS, NV>), dim3((unsigned)workgroups), dim3(THREADS), 0, s, a);
  return 0;
}

// Threads and 8-column pieces a thread, by the group's width.  8192 rows with the residual into
// 8 bits, bf16 (us; the best copy moves 6.4 TB/s): 1024 columns 11.7, 2048 23.2 to 25 (5.0 TB/s; 256
// threads 26.4), 4096 46.6 (5.0), 8192 90 (5.2; 1024 threads 92.8); 16384 columns of
// an ordinary norm 93.9 (4.3; 1024 threads 108); gated, 8192 columns by groups of 1024 67.3 (5.0).  Into bf16: 4096 columns
// with the residual 47.7 (5.6), 16384 of an ordinary norm 101 (5.3).
// Reads past the caches move these by -4 % to +18 %, reads and writes past them by -9 % to +9 %:
// they gain where nothing is used again soon and lose where it is, and a norm's output is.
template <typename TX, typename IO, bool FP8, int FORM>
int launch_norm(const NormArgs& a, hipStream_t s) {
  const int n = a.group;
  if (n <= 512) return launch_norm<TX, IO, FP8, FORM, 64, 1>(a, s);
  if (n <= 1024) return launch_norm<TX, IO, FP8, FORM, 64, 2>(a, s);
  if (n <= 2048) return launch_norm<TX, IO, FP8, FORM, 128, 2>(a, s);
  if (n <= 4096) return launch_norm<TX, IO, FP8, FORM, 256, 2>(a, s);
  if (n <= 8192) return launch_norm<TX, IO, FP8, FORM, 256, 4>(a, s);
  if (n <= 16384) return launch_norm<TX, IO, FP8, FORM, 512, 4>(a, s);
  if (n <= 32768) return launch_norm<TX, IO, FP8, FORM, 1024, 4>(a, s);
  return -2;
}

template <typename TX, typename IO, bool FP8>
int launch_norm(const NormArgs& a, hipStream_t s) {
  if (a.gate) return a.skip ? launch_norm<TX, IO, FP8, GATED_SKIP>(a, s) : launch_norm<TX, IO, FP8, GATED>(a, s);
  return a.residual ? launch_norm<TX, IO, FP8, RESIDUAL>(a, s) : launch_norm<TX, IO, FP8, PLAIN>(a, s);
}

template <typename TX, typename IO>
int launch_norm(const NormArgs& a, bool fp8, hipStream_t s) {
  return fp8 ? launch_norm<TX, IO, true>(a, s) : launch_norm<TX, IO, false>(a, s);
}

int run_norm(const NormArgs& a, int x_dtype, int io, int out, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool fp8 = out == 2;
  if (io == 0) return launch_norm<float, float>(a, fp8, s);
  return x_dtype == 0 ? launch_norm<float, bf16_t>(a, fp8, s) : launch_norm<bf16_t, bf16_t>(a, fp8, s);
}

}  // namespace skssm
