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
// (7.5e-8 on the same blocks) at half the rate: 8192 x 18560 x 4096 558 us for bf16 outputs (2.2 PFLOP/s), 1140 for
// fp32 (1.1), 1024 x 4096 x 4096 27 and 42, 1 x 18560 x 4096 15 and 20.
#include <algorithm>
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

// Tiles of BM x BN, K in blocks of 128 through LDS, STAGES of them at
// once (STAGES - 1 on their way while one is multiplied).  A row of a tile is 128
// bytes in 8 chunks of 16; chunk c of a row lies at slot c ^ key(row), so that the 8 rows a
// read takes at once lie in different banks.  Rows of w are taken in the order that
// leaves a lane RUN = 16 (8) consecutive columns of its output row.  Few tiles: the K axis is
// split over workgroups too (gridDim.y), which leave fp32 sums for a second launch to join.

__device__ __forceinline__ int key_a(int row) { return row & 7; }
// the 8 rows of a read are 4 x + y, x = 0, 1, at RUN x + y
template <int RUN> __device__ __forceinline__ int key_w(int row) { return (row & 3) | ((row >> (RUN == 16 ? 2 : 1)) & 4); }

// 16 (4) bytes a lane from base + at into LDS, the wave's 64 lanes one after the other
// from `lds`.  In assembly, as the compiler would wait for every such load before the next
// LDS read, whatever it reads; the caller waits (vmcnt) before the barrier that
// publishes a stage.  The load takes M0 one wait state after it is written.
__device__ __forceinline__ void to_lds16(const void* base, uint32_t at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(at), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void to_lds4(const void* base, uint32_t at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(at), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

template <typename OUT, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN, 2) void matmul_tile_kernel(MatmulArgs p, int mt, int nt) {
  constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;  // 16 x 16 tiles of a wave
  constexpr int SA = BM / 8 / WAVES, SW = BN / 8 / WAVES;              // 8-row pieces a wave stages
  constexpr int QT = TN < 4 ? TN : 4, RUN = 4 * QT;                    // tiles, and columns, of a lane's run
  constexpr int AT_W = BM < 64 ? 64 : BM, SCALES = AT_W + 64;          // a's factors (64 a load), then w's by 64 columns
  static_assert(TN % QT == 0 && QT >= 2 && SA >= 1 && SW >= 1 && BM / 64 < WAVES, "shape");
  __shared__ __attribute__((aligned(16))) uint8_t la[STAGES][BM * 128], lw[STAGES][BN * 128];
  __shared__ float ls[STAGES][SCALES];
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
  const int blocks = (p.K + 127) >> 7, full = p.K >> 7;
  const int first = (int)((int64_t)blocks * blockIdx.y / gridDim.y), end = (int)((int64_t)blocks * (blockIdx.y + 1) / gridDim.y);
  const int wm = wave % WM, wn = wave / WM;
  floatx4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};

  const uint8_t* const a0 = p.a + (size_t)m0 * p.lda;
  const uint8_t* const w0 = p.w + (size_t)n0 * p.ldw;
  const uint32_t lds_a = lds_address(la), lds_w = lds_address(lw), lds_s = lds_address(ls);
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
      const int row = (s * WAVES + wave) * 8 + (lane >> 3), c = min((lane & 7) ^ key_w<RUN>(row), chunks - 1);
      vw[s] = (uint32_t)(min(row, p.N - 1 - n0) * (uint32_t)p.ldw) + c * 16;
    }
  };
  // the block's factors, one load a wave: the first BM / 64 waves a's rows, the others (all the
  // same) w's, for column n0 + 64 lane
  const bool rows_of_a = wave < BM / 64 || BM < 64 && wave == 0;
  const float* const s0 = rows_of_a ? p.sa + m0 : p.sw;
  const uint32_t vs = rows_of_a ? 4 * min(wave * 64 + lane, p.M - 1 - m0)
                                : 4 * (uint32_t)(min((n0 + 64 * min(lane, BN / 64)) >> 7, (p.N - 1) >> 7) * blocks);
  const size_t next_s = rows_of_a ? p.ldsa : 1;
  const uint32_t to_s = lds_s + 4 * (rows_of_a ? wave * 64 : AT_W);
  constexpr int LOADS = SA + SW + 1;  // of a wave, a stage
  auto stage = [&](int kb, int buf) {
    if (kb == full) places((p.K >> 4) & 7);
#pragma unroll
    for (int s = 0; s < SA; ++s) to_lds16(a0 + (size_t)kb * 128, va[s], lds_a + buf * BM * 128 + (s * WAVES + wave) * 1024);
#pragma unroll
    for (int s = 0; s < SW; ++s) to_lds16(w0 + (size_t)kb * 128, vw[s], lds_w + buf * BN * 128 + (s * WAVES + wave) * 1024);
    to_lds4(s0 + (size_t)kb * next_s, vs, to_s + buf * SCALES * 4);
  };
  // the lane's two chunks of its row in the wave's first tile of a and of w; tile i of a lies
  // 16 rows on, and tile j of w takes lane row 4 x + y from row RUN x + 4 (j % QT) + y of its
  // 16 QT: neither changes the key
  const int x0 = (r >> 2) * RUN + (r & 3);
  const uint32_t oa = (wm * TM * 16 + r) * 128, ow = (wn * TN * 16 + x0) * 128;
  const int ka = key_a(r), kw = key_w<RUN>(x0);
  const uint32_t oa0 = oa + ((g ^ ka) << 4), oa1 = oa + (((g + 4) ^ ka) << 4);
  const uint32_t ow0 = ow + ((g ^ kw) << 4), ow1 = ow + (((g + 4) ^ kw) << 4);
  auto frag = [&](const uint8_t* t0, const uint8_t* t1, int at) {
    return join(*reinterpret_cast<const uint4*>(t0 + at), *reinterpret_cast<const uint4*>(t1 + at));
  };
  auto compute = [&](int buf, auto tail) {
    const uint8_t* ta = la[buf];
    const uint8_t* tw = lw[buf];
    // w's fragments are read a tile ahead, and between the products of a tile the
    // vector units scale the sums of the tile before: 4 FMA in the shadow of an
    // instruction of 32 cycles (in a block of their own after the tile's products
    // they cost 7 %: 654 us against 609 at 8192 x 18560 x 4096)
    auto weights = [&](int j) { return frag(tw + ow0, tw + ow1, ((j / QT) * 16 * QT + (j % QT) * 4) * 128); };
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
    float sa[TM], sw[(TN + 3) / 4];
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = ls[buf][(wm * TM + i) * 16 + r];
#pragma unroll
    for (int q = 0; q < (TN + 3) / 4; ++q) sw[q] = ls[buf][AT_W + ((wn * TN * 16 + q * 64) >> 6)];
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
          const float s = sa[i] * sw[(j - 1) / 4];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j - 1][i][e] = fmaf(s, t[(j - 1) & 1][i][e], acc[j - 1][i][e]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  places(8);
  for (int q = 0; q < STAGES - 1; ++q)
    if (first + q < end) stage(first + q, q);
  int buf = 0;
  auto next = [&](int kb) {
    // block kb's stage has come (the STAGES - 2 younger ones may be on their way, but near the
    // end, where there are fewer), and every wave is done with the buffer of block kb - 1,
    // where block kb + STAGES - 1 goes
    if (STAGES == 2 || kb + STAGES - 2 >= end) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 2) * LOADS) : "memory");
    lds_barrier();
    if (kb + STAGES - 1 < end) stage(kb + STAGES - 1, buf == 0 ? STAGES - 1 : buf - 1);
  };
  const int stop = min(end, full);
  for (int kb = first; kb < stop; ++kb) {
    next(kb);
    compute(buf, std::false_type{});
    buf = buf == STAGES - 1 ? 0 : buf + 1;
  }
  if (end > full) {
    next(full);
    compute(buf, std::true_type{});
  }
  if (gridDim.y > 1) {
    float* part = p.part + (size_t)blockIdx.y * p.M * p.N;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = m0 + (wm * TM + i) * 16 + r;
      if (m >= p.M) continue;
#pragma unroll
      for (int q = 0; q < TN / QT; ++q) {
        const int n = n0 + wn * TN * 16 + q * 16 * QT + g * RUN;
        float* y = part + (size_t)m * p.N + n;
#pragma unroll
        for (int j = 0; j < QT; ++j)
          if ((p.N & 3) == 0) {
            if (n + j * 4 < p.N) *reinterpret_cast<floatx4*>(y + j * 4) = acc[q * QT + j][i];
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (n + j * 4 + e < p.N) y[j * 4 + e] = acc[q * QT + j][i][e];
          }
      }
    }
    return;
  }
  const bool wide = (p.ldy * sizeof(OUT)) % 16 == 0 && p.N % RUN == 0;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = m0 + (wm * TM + i) * 16 + r;
    if (m >= p.M) continue;
#pragma unroll
    for (int q = 0; q < TN / QT; ++q) {
      const int n = n0 + wn * TN * 16 + q * 16 * QT + g * RUN;
      OUT* y = static_cast<OUT*>(p.y) + (size_t)m * p.ldy + n;
      if (wide) {
        if (n < p.N) {
          Raw<OUT, RUN> o;
#pragma unroll
          for (int j = 0; j < QT; ++j)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const float x0 = acc[q * QT + j][i][e], x1 = acc[q * QT + j][i][e + 1];
              if constexpr (sizeof(OUT) == 2) o.w[(j * 4 + e) / 2] = bf16_pack2(x0, x1);
              else { o.e[j * 4 + e] = x0; o.e[j * 4 + e + 1] = x1; }
            }
          o.store(y);
        }
      } else {
#pragma unroll
        for (int j = 0; j < QT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + j * 4 + e < p.N) st_elem(y + j * 4 + e, acc[q * QT + j][i][e]);
      }
    }
  }
}

// The sums of `splits` parts, in order.
template <typename OUT>
__global__ __launch_bounds__(256) void matmul_join_kernel(MatmulArgs p, int splits) {
  const int quads = (p.N + 3) >> 2;
  const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(at / quads), n = 4 * (int)(at % quads);
  if (m >= p.M) return;
  const float* x = p.part + (size_t)m * p.N + n;
  floatx4 t = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s, x += (size_t)p.M * p.N) {
    if ((p.N & 3) == 0) t += *reinterpret_cast<const floatx4*>(x);
    else
      for (int e = 0; e < 4; ++e) t[e] += n + e < p.N ? x[e] : 0.f;
  }
  OUT* y = static_cast<OUT*>(p.y) + (size_t)m * p.ldy + n;
  for (int e = 0; e < 4; ++e)
    if (n + e < p.N) st_elem(y + e, t[e]);
}

template <typename OUT, int BM, int BN, int WM, int WN, int STAGES>
int launch_tiles(const MatmulArgs& p, int splits, hipStream_t s) {
  const int mt = (p.M + BM - 1) / BM, nt = (p.N + BN - 1) / BN;
  if (!fits((int64_t)mt * nt, 64 * WM * WN)) return -3;
  hipLaunchKernelGGL((matmul_tile_kernel<OUT, BM, BN, WM, WN, STAGES>), dim3((unsigned)mt * (unsigned)nt, (unsigned)splits), dim3(64 * WM * WN), 0,
                     s, p, mt, nt);
  if (splits > 1 && taken()) {  // (of fewer tiles than the card runs at once)
    const size_t quads = (size_t)p.M * ((p.N + 3) / 4);
    hipLaunchKernelGGL((matmul_join_kernel<OUT>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, p, splits);
  }
  return 0;
}

// Which tiles, and over how many workgroups the K axis is split.
//   wide   tiles of 256 x 256 cover the first `wide` columns (a multiple of 256; 0: none)
//   rest   the others: 0 none, 1: 128 x 128, 2: 128 x 64, 3: 64 x 64, 4: 32 x 64
// Measured on one MI355X (us):
//   M x N x K             256    128   128x64  64x64  32x64
//   8192 x 18560 x 4096   616    693     906      -      -     256 over 18432 columns, then 128x64: 592
//   1024 x 18560 x 4096   116    108     130      -      -     256 over 16384, then 128: 95
//    300 x 18560 x 4096     -   38.0    52.5   50.3      -
//   1024 x  4096 x 4096     -   28.4    26.9   33.6      -
//    600 x  4096 x 8192     -   46.4    40.4   52.0      -
//    128 x 18560 x 4096     -   27.8    23.6   28.9      -
//    200 x  4096 x 4096     -   24.5    18.5   14.2      -
//    100 x  2048 x 2048     -   13.6    10.2    8.1    9.3
//     64 x 18560 x 4096     -   25.2    22.1   17.1   19.3
//      1 x 18560 x 4096     -      -       -   16.0   15.1     (weights straight into registers: 19.5)
// so: the largest tiles of which there is one for each CU, but for 256 x 256, of which a
// round of all CUs has to be full -- what is left over goes to smaller ones -- and half a tile's rows
// have to be there: 131072 x 4096, of 1 / 64 / 100 / 128 / 129 rows, 256 x 256: 142 / 147 / 152 / 154 / 152, without:
// 98 / 117 / 139 / 142 / -.
// K split (not / by 2 / by 4): 77 x 4096 x 8192, 64x64: 23.7 / 17.5 / 15.5; 16 x 4096 x 8192 23.1 / 16.0 / 11.4; 16 x
// 4096 x 4096 12.1 / 10.4 / 9.6; 200 x 2048 x 4096 13.8 / 13.2 / 13.6; 100 x 2048 x 2048 8.1 / 8.7 / 8.7: over what fills the
// CUs in parts of 8 blocks at least, or twice that in parts of 16.
struct MatmulPlan { int wide, rest, splits; };
MatmulPlan matmul_plan(int M, int N, int K, bool narrow) {  // M, N, K >= 1
  constexpr int64_t cus = 256;
  auto tiles = [&](int bm, int bn, int n) { return (int64_t)((M + bm - 1) / bm) * ((n + bn - 1) / bn); };
  if (narrow && M > 128 && tiles(256, 256, N) >= cus) {
    const int64_t all = tiles(256, 256, N), rounds = all / cus, over = all % cus;
    if (over == 0 || over > cus / 2) return {(N + 255) / 256 * 256, 0, 1};
    const int64_t rows = (M + 255) / 256, columns = rounds * cus / rows;
    if (columns > 0) {
      const int wide = (int)columns * 256;
      return {wide, tiles(128, 128, N - wide) > cus / 2 ? 1 : 2, 1};
    }
  }
  if (M > 64 && tiles(128, 128, N) > cus) return {0, 1, 1};
  const int rest = M > 64 && tiles(128, 64, N) >= cus ? 2 : M > 32 ? 3 : 4;
  const int64_t t = rest == 2 ? tiles(128, 64, N) : rest == 3 ? tiles(64, 64, N) : tiles(32, 64, N);
  const int blocks = (K + 127) / 128;
  const int64_t once = std::min<int64_t>(blocks / 8, cus / t), twice = std::min<int64_t>(blocks / 16, 2 * cus / t);
  return {0, rest, (int)std::max<int64_t>({1, once, twice})};
}

template <typename OUT>
int launch_matmul(const MatmulArgs& p, hipStream_t s) {
  const MatmulPlan plan = matmul_plan(p.M, p.N, p.K, sizeof(OUT) == 2);
  MatmulArgs q = p;
  if constexpr (sizeof(OUT) == 2) {
    if (plan.wide) {
      if (plan.rest && !fits((int64_t)((p.M + 127) / 128) * ((p.N - plan.wide + 63) / 64), 256)) return -3;  // (128 x 64, the most tiles)
      q.N = std::min(p.N, plan.wide);
      const int rc = launch_tiles<OUT, 256, 256, 4, 2, 2>(q, 1, s);
      if (rc || !plan.rest || !taken()) return rc;
      q.N = p.N - plan.wide;
      q.w = p.w + (size_t)plan.wide * p.ldw;
      q.sw = p.sw + (size_t)(plan.wide / 128) * ((p.K + 127) / 128);
      q.y = static_cast<OUT*>(p.y) + plan.wide;
    }
  }
  switch (plan.rest) {
    case 1: return launch_tiles<OUT, 128, 128, 2, 2, 2>(q, plan.splits, s);
    case 2: return launch_tiles<OUT, 128, 64, 2, 2, 3>(q, plan.splits, s);
    case 3: return launch_tiles<OUT, 64, 64, 2, 2, 3>(q, plan.splits, s);
    case 4: return launch_tiles<OUT, 32, 64, 2, 2, 4>(q, plan.splits, s);
    default: return -2;
  }
}

int run_matmul_fp8(const MatmulArgs& p, int out, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return out == 1 ? launch_matmul<bf16_t>(p, s) : launch_matmul<float>(p, s);
}

size_t matmul_fp8_workspace(int M, int N, int K) {
  const int splits = std::max(matmul_plan(M, N, K, false).splits, matmul_plan(M, N, K, true).splits);
  return splits > 1 ? (size_t)splits * M * N * sizeof(float) : 0;
}

}  // namespace skssm
