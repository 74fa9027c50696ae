// y = a w^T of e4m3 matrices, with a scale per row and 128 columns of a and per
// 128 x 128 of w.  The matrix cores sum a block of 128 columns for a 16 x 16 tile, the
// vector units scale its four results a lane and add them to fp32 sums.  w is
// the first operand, so that a lane's results are consecutive columns n of one
// row m and one factor a_scale w_scale serves all of them.  The order of k inside
// an instruction is free as long as both operands share it: a lane takes two
// 16-byte chunks of its row.
//
// Which instruction: v_mfma_f32_16x16x128_f8f6f4 takes the block in one, at the
// 8-bit rate, but shifts the products it adds to the largest of them and keeps some
// 13 bits (measured over random blocks: within 2^-11.8 of the largest product,
// 5e-5 of the result where the exponents vary most; 16x16x32_fp8_fp8 the same).
// Under an output stored in bf16 (2^-8) that is nothing.  An fp32 output is computed
// from the same values as bf16, which holds e4m3 exactly, by four 16x16x32_bf16
// (7.5e-8 on the same blocks) at half the rate.
#include "../mixer.h"

namespace skssm {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ intx8 join(uint4 x, uint4 y) {
  return intx8{(int)x.x, (int)x.y, (int)x.z, (int)x.w, (int)y.x, (int)y.y, (int)y.z, (int)y.w};
}

// A lane's 32 values of a block, as the products of an OUT take them.
template <typename OUT> struct Operand;
template <> struct Operand<bf16_t> {
  intx8 v;
  __device__ __forceinline__ void set(intx8 x) { v = x; }
};
template <> struct Operand<float> {
  bf16x8 v[4];
  __device__ __forceinline__ void set(intx8 x) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t lo = (uint32_t)x[2 * q], hi = (uint32_t)x[2 * q + 1];
      const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                   c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
      v[q] = bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
  }
};
// The sum over a block.
__device__ __forceinline__ floatx4 block_product(const Operand<bf16_t>& a, const Operand<bf16_t>& b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ floatx4 block_product(const Operand<float>& a, const Operand<float>& b) {
  floatx4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < 4; ++q) t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[q], b.v[q], t, 0, 0, 0);
  return t;
}

// ---- few rows: the weights' bytes bound the call.  A workgroup owns 16 columns
// n; its waves split the K blocks, read their weights straight into registers
// (each byte once) and join their sums in LDS.

template <typename OUT, int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void matmul_few_kernel(MatmulArgs p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, nb = n0 >> 7, blocks = (p.K + 127) >> 7;
  const uint8_t* w = p.w + (size_t)min(n0 + r, p.N - 1) * p.ldw;
  floatx4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  const uint8_t* a[MT];
  int m[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    m[i] = min(16 * i + r, p.M - 1);
    a[i] = p.a + (size_t)m[i] * p.lda;
  }
  for (int kb = wave; kb < blocks; kb += WAVES) {
    // chunks past the end read the row's last one; a's are then zero, so that they add nothing
    // (a NaN among w's is a value of the same row n, whose results it makes NaN anyway)
    const int last = p.K / 16 - 1, c0 = kb * 8 + 2 * g, c1 = c0 + 1;
    const bool in0 = c0 <= last, in1 = c1 <= last;
    const size_t o0 = (size_t)min(c0, last) * 16, o1 = (size_t)min(c1, last) * 16;
    Operand<OUT> wf;
    wf.set(join(ld_nt(reinterpret_cast<const uint4*>(w + o0)), ld_nt(reinterpret_cast<const uint4*>(w + o1))));
    const float sw = p.sw[(size_t)nb * blocks + kb];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      uint4 x = *reinterpret_cast<const uint4*>(a[i] + o0), y = *reinterpret_cast<const uint4*>(a[i] + o1);
      if (!in0) x = make_uint4(0, 0, 0, 0);
      if (!in1) y = make_uint4(0, 0, 0, 0);
      const float s = p.sa[(size_t)kb * p.ldsa + m[i]] * sw;
      Operand<OUT> af;
      af.set(join(x, y));
      const floatx4 t = block_product(wf, af);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(s, t[e], acc[i][e]);
    }
  }
  __shared__ floatx4 sums[WAVES][MT][64];
  if constexpr (WAVES > 1) {
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
  }
  // the tiles of rows are joined and stored by the waves in turn
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    if (i % WAVES != wave) continue;
    floatx4 t = acc[i];
    if constexpr (WAVES > 1) {
      t = sums[0][i][lane];
#pragma unroll
      for (int v = 1; v < WAVES; ++v) t += sums[v][i][lane];
    }
    const int row = 16 * i + r;
    if (row < p.M) {
      OUT* y = static_cast<OUT*>(p.y) + (size_t)row * p.ldy + n0 + 4 * g;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n0 + 4 * g + e < p.N) st_elem(y + e, t[e]);
    }
  }
}

// ---- many rows: tiles of BM x BN, K in blocks of 128 through LDS.  A row of a
// tile is 128 bytes in 8 chunks of 16; chunk c of a row lies at slot c ^ key(row), so
// that the 8 rows a read takes at once lie in different banks.  Rows of w are
// taken in the order that leaves a lane 16 consecutive columns of its output row.

__device__ __forceinline__ int key_a(int row) { return row & 7; }
__device__ __forceinline__ int key_w(int row) { return (row & 3) | ((row >> 2) & 4); }

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;
__device__ __forceinline__ void to_lds16(const void* src, void* dst) {  // dst: the wave's first lane's
  __builtin_amdgcn_global_load_lds((global_void*)src, (lds_void*)dst, 16, 0, 0);
}

template <typename OUT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void matmul_tile_kernel(MatmulArgs p) {
  constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;  // 16 x 16 tiles of a wave
  static_assert(TN % 4 == 0, "a lane's 16 consecutive columns come from 4 tiles");
  __shared__ __attribute__((aligned(16))) uint8_t la[2][BM * 128], lw[2][BN * 128];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
  const int mt = (p.M + BM - 1) / BM;
  const int m0 = (blockIdx.x % mt) * BM, n0 = (blockIdx.x / mt) * BN;
  const int wm = wave % WM, wn = wave / WM, blocks = (p.K + 127) >> 7, last = p.K / 16 - 1;
  floatx4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};

  auto stage = [&](int kb, int buf) {  // a wave moves 8 rows at a time
#pragma unroll
    for (int s = 0; s < BM / 8 / WAVES; ++s) {
      const int row = (s * WAVES + wave) * 8 + (lane >> 3);
      const int c = min(kb * 8 + ((lane & 7) ^ key_a(row)), last);
      to_lds16(p.a + (size_t)min(m0 + row, p.M - 1) * p.lda + (size_t)c * 16, &la[buf][(s * WAVES + wave) * 1024]);
    }
#pragma unroll
    for (int s = 0; s < BN / 8 / WAVES; ++s) {
      const int row = (s * WAVES + wave) * 8 + (lane >> 3);
      const int c = min(kb * 8 + ((lane & 7) ^ key_w(row)), last);
      to_lds16(p.w + (size_t)min(n0 + row, p.N - 1) * p.ldw + (size_t)c * 16, &lw[buf][(s * WAVES + wave) * 1024]);
    }
  };
  auto frag = [&](const uint8_t* tile, int row, int key) {
    const uint8_t* at = tile + row * 128;
    return join(*reinterpret_cast<const uint4*>(at + ((g ^ key) << 4)), *reinterpret_cast<const uint4*>(at + (((g + 4) ^ key) << 4)));
  };
  float sa[TM];
  auto scales = [&](int kb) {
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = p.sa[(size_t)kb * p.ldsa + min(m0 + (wm * TM + i) * 16 + r, p.M - 1)];
  };
  stage(0, 0);
  for (int kb = 0; kb < blocks; ++kb) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (kb + 1 < blocks) stage(kb + 1, (kb + 1) & 1);
    scales(kb);
    const uint8_t* ta = la[kb & 1];
    const uint8_t* tw = lw[kb & 1];
    Operand<OUT> fa[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int row = (wm * TM + i) * 16 + r;
      intx8 x = frag(ta, row, key_a(row));
      if (kb * 8 + 7 > last) {  // chunks past the end of K add nothing
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (kb * 8 + g + (e & 4) > last) x[e] = 0;
      }
      fa[i].set(x);
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      // rows of tile j: lane row 4 x + y is column 16 x + 4 (j % 4) + y of 64
      const int row = wn * TN * 16 + (j >> 2) * 64 + (r >> 2) * 16 + (j & 3) * 4 + (r & 3);
      Operand<OUT> fw;
      fw.set(frag(tw, row, key_w(row)));
      const int nb = min((n0 + wn * TN * 16 + (j >> 2) * 64) >> 7, (p.N - 1) >> 7);
      const float sw = p.sw[(size_t)nb * blocks + kb];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const floatx4 t = block_product(fw, fa[i]);
        const float s = sa[i] * sw;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][i][e] = fmaf(s, t[e], acc[j][i][e]);
      }
    }
  }
  const bool wide = (p.ldy * sizeof(OUT)) % 16 == 0 && (p.N & 15) == 0;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = m0 + (wm * TM + i) * 16 + r;
    if (m >= p.M) continue;
#pragma unroll
    for (int q = 0; q < TN / 4; ++q) {
      const int n = n0 + wn * TN * 16 + q * 64 + g * 16;
      OUT* y = static_cast<OUT*>(p.y) + (size_t)m * p.ldy + n;
      if (wide) {
        if (n < p.N) {
          Raw<OUT, 16> o;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const float x0 = acc[q * 4 + j][i][e], x1 = acc[q * 4 + j][i][e + 1];
              if constexpr (sizeof(OUT) == 2) o.w[(j * 4 + e) / 2] = bf16_pack2(x0, x1);
              else { o.e[j * 4 + e] = x0; o.e[j * 4 + e + 1] = x1; }
            }
          o.store(y);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + j * 4 + e < p.N) st_elem(y + j * 4 + e, acc[q * 4 + j][i][e]);
      }
    }
  }
}

template <typename OUT>
int launch_matmul(const MatmulArgs& p, hipStream_t s) {
  const int mt = (p.M + 15) / 16;
  const dim3 few((unsigned)((p.N + 15) / 16));
  if (mt <= 1) hipLaunchKernelGGL((matmul_few_kernel<OUT, 1, 8>), few, dim3(512), 0, s, p);
  else if (mt <= 2) hipLaunchKernelGGL((matmul_few_kernel<OUT, 2, 8>), few, dim3(512), 0, s, p);
  else if (mt <= 4) hipLaunchKernelGGL((matmul_few_kernel<OUT, 4, 8>), few, dim3(512), 0, s, p);
  else if (mt <= 8) hipLaunchKernelGGL((matmul_few_kernel<OUT, 8, 8>), few, dim3(512), 0, s, p);
  else
    hipLaunchKernelGGL((matmul_tile_kernel<OUT, 128, 128, 2, 2>), dim3((unsigned)(((p.M + 127) / 128) * ((p.N + 127) / 128))),
                       dim3(256), 0, s, p);
  return 0;
}

int run_matmul_fp8(const MatmulArgs& p, int out, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return out == 1 ? launch_matmul<bf16_t>(p, s) : launch_matmul<float>(p, s);
}

size_t matmul_fp8_workspace(int, int, int) { return 0; }

}  // namespace skssm
