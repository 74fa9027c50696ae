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
#include <type_traits>

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

// 16 bytes a lane from base + at into LDS, the wave's 64 lanes one after the other
// from `lds`.  In assembly, as the compiler would wait for every such load before the next
// LDS read, whatever it reads; the caller waits (vmcnt) before the barrier that
// publishes a stage.  No register is written.
__device__ __forceinline__ void to_lds16(const uint8_t* base, uint32_t at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(at), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

template <typename OUT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void matmul_tile_kernel(MatmulArgs p, int mt, int nt) {
  constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;  // 16 x 16 tiles of a wave
  constexpr int SA = BM / 8 / WAVES, SW = BN / 8 / WAVES;              // 8-row pieces a wave stages
  static_assert(TN % 4 == 0, "a lane's 16 consecutive columns come from 4 tiles");
  __shared__ __attribute__((aligned(16))) uint8_t la[2][BM * 128], lw[2][BN * 128];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  // Workgroups go round the eight XCDs: each XCD takes a run of tiles, in columns of 8
  // tiles of rows, so that what runs at once on it shares rows of a and of w in its L2.
  int tile = blockIdx.x;
  {
    const int n = mt * nt, per = n / 8, rest = n % 8, x = tile % 8, i = tile / 8;
    tile = x * per + min(x, rest) + i;
  }
  constexpr int BAND = 8;
  const int band = tile / (BAND * nt), rows = min(BAND, mt - band * BAND), in = tile - band * BAND * nt;
  const int m0 = (band * BAND + in % rows) * BM, n0 = (in / rows) * BN;
  const int wm = wave % WM, wn = wave / WM, blocks = (p.K + 127) >> 7, full = p.K >> 7;
  floatx4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};

  const uint8_t* const a0 = p.a + (size_t)m0 * p.lda;
  const uint8_t* const w0 = p.w + (size_t)n0 * p.ldw;
  const uint32_t lds_a = lds_address(la), lds_w = lds_address(lw);
  // a wave moves 8 rows at a time; rows past the end repeat the last one, chunks past the end of K the last chunk
  uint32_t va[SA], vw[SW];
  auto places = [&](int chunks) {
#pragma unroll
    for (int s = 0; s < SA; ++s) {
      const int row = (s * WAVES + wave) * 8 + (lane >> 3), c = min((lane & 7) ^ key_a(row), chunks - 1);
      va[s] = (uint32_t)(min(row, p.M - 1 - m0) * (uint32_t)p.lda) + c * 16;
    }
#pragma unroll
    for (int s = 0; s < SW; ++s) {
      const int row = (s * WAVES + wave) * 8 + (lane >> 3), c = min((lane & 7) ^ key_w(row), chunks - 1);
      vw[s] = (uint32_t)(min(row, p.N - 1 - n0) * (uint32_t)p.ldw) + c * 16;
    }
  };
  auto stage = [&](int kb, int buf) {
    if (kb == full) places((p.K >> 4) & 7);
#pragma unroll
    for (int s = 0; s < SA; ++s) to_lds16(a0 + (size_t)kb * 128, va[s], lds_a + buf * BM * 128 + (s * WAVES + wave) * 1024);
#pragma unroll
    for (int s = 0; s < SW; ++s) to_lds16(w0 + (size_t)kb * 128, vw[s], lds_w + buf * BN * 128 + (s * WAVES + wave) * 1024);
  };
  // the lane's two chunks of its row in the wave's first tile of a and of w; tile i of a lies
  // 16 rows on, and tile j of w takes lane row 4 x + y from row 16 x + 4 (j % 4) + y of 64:
  // neither changes the key
  const uint32_t oa = (wm * TM * 16 + r) * 128, ow = (wn * TN * 16 + (r >> 2) * 16 + (r & 3)) * 128;
  const int ka = key_a(r), kw = (r & 3) | (r & 4);
  const uint32_t oa0 = oa + ((g ^ ka) << 4), oa1 = oa + (((g + 4) ^ ka) << 4);
  const uint32_t ow0 = ow + ((g ^ kw) << 4), ow1 = ow + (((g + 4) ^ kw) << 4);
  auto frag = [&](const uint8_t* t0, const uint8_t* t1, int at) {
    return join(*reinterpret_cast<const uint4*>(t0 + at), *reinterpret_cast<const uint4*>(t1 + at));
  };
  // the block's factors: a_scale of the lane's rows, w_scale of the wave's 64-column parts
  float sa[TM], sw[TN / 4], na[TM], nw[TN / 4];
  auto scales = [&](int kb) {
#pragma unroll
    for (int i = 0; i < TM; ++i) na[i] = p.sa[(size_t)kb * p.ldsa + min(m0 + (wm * TM + i) * 16 + r, p.M - 1)];
#pragma unroll
    for (int q = 0; q < TN / 4; ++q) nw[q] = p.sw[(size_t)min((n0 + wn * TN * 16 + q * 64) >> 7, (p.N - 1) >> 7) * blocks + kb];
  };
  auto compute = [&](int kb, auto tail) {
    const uint8_t* ta = la[kb & 1];
    const uint8_t* tw = lw[kb & 1];
    // w's fragments are read a tile ahead, and between the products of a tile the
    // vector units scale the sums of the tile before: 4 FMA in the shadow of an
    // instruction of 32 cycles (in a block of their own after the tile's products
    // they cost 7 %: 654 us against 609 at 8192 x 18560 x 4096)
    auto weights = [&](int j) { return frag(tw + ow0, tw + ow1, ((j >> 2) * 64 + (j & 3) * 4) * 128); };
    intx8 ahead = weights(0);
    Operand<OUT> fa[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      intx8 x = frag(ta + oa0, ta + oa1, i * 16 * 128);
      if constexpr (decltype(tail)::value) {  // chunks past the end of K add nothing
        const int chunks = (p.K >> 4) & 7;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (g + (e & 4) >= chunks) x[e] = 0;
      }
      fa[i].set(x);
    }
    floatx4 t[2][TM];
#pragma unroll
    for (int j = 0; j <= TN; ++j) {
      Operand<OUT> fw;
      if (j < TN) fw.set(ahead);
      if (j + 1 < TN) ahead = weights(j + 1);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (j < TN) t[j & 1][i] = block_product(fw, fa[i]);
        if (j > 0) {
          const float s = sa[i] * sw[(j - 1) >> 2];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j - 1][i][e] = fmaf(s, t[(j - 1) & 1][i][e], acc[j - 1][i][e]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  auto next = [&](int kb) {  // block kb's stage has come; block kb + 1's starts
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = na[i];
#pragma unroll
    for (int q = 0; q < TN / 4; ++q) sw[q] = nw[q];
    if (kb + 1 < blocks) {
      stage(kb + 1, (kb + 1) & 1);
      scales(kb + 1);
    }
  };
  places(8);
  stage(0, 0);
  scales(0);
  for (int kb = 0; kb < full; ++kb) {
    next(kb);
    compute(kb, std::false_type{});
  }
  if (full < blocks) {
    next(full);
    compute(full, std::true_type{});
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

template <typename OUT, int BM, int BN, int WM, int WN>
void launch_tiles(const MatmulArgs& p, hipStream_t s) {
  const int mt = (p.M + BM - 1) / BM, nt = (p.N + BN - 1) / BN;
  hipLaunchKernelGGL((matmul_tile_kernel<OUT, BM, BN, WM, WN>), dim3((unsigned)mt * (unsigned)nt), dim3(64 * WM * WN), 0, s, p, mt, nt);
}

template <typename OUT>
int launch_matmul(const MatmulArgs& p, hipStream_t s) {
  const int mt = (p.M + 15) / 16;
  const dim3 few((unsigned)((p.N + 15) / 16));
  if (mt <= 1) hipLaunchKernelGGL((matmul_few_kernel<OUT, 1, 8>), few, dim3(512), 0, s, p);
  else if (mt <= 2) hipLaunchKernelGGL((matmul_few_kernel<OUT, 2, 8>), few, dim3(512), 0, s, p);
  else if (mt <= 4) hipLaunchKernelGGL((matmul_few_kernel<OUT, 4, 8>), few, dim3(512), 0, s, p);
  else if (mt <= 8) hipLaunchKernelGGL((matmul_few_kernel<OUT, 8, 8>), few, dim3(512), 0, s, p);
  else if (sizeof(OUT) == 4 || (int64_t)((p.M + 255) / 256) * ((p.N + 255) / 256) < 256) launch_tiles<OUT, 128, 128, 2, 2>(p, s);
  else launch_tiles<bf16_t, 256, 256, 4, 2>(p, s);
  return 0;
}

int run_matmul_fp8(const MatmulArgs& p, int out, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return out == 1 ? launch_matmul<bf16_t>(p, s) : launch_matmul<float>(p, s);
}

size_t matmul_fp8_workspace(int, int, int) { return 0; }

}  // namespace skssm
