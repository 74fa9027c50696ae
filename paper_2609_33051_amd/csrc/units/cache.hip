// Rotary positions and the 4-bit cache: the rotation of queries and keys, the
// append of keys and values, and the cache's values back as numbers.
//
// Every array moves once, so the kernels are bound by memory: 16384 tokens of 40 heads of 128 channels turned in 60
// us (5.7 TB/s), of 32 + 2 x 8 heads turned and appended in 74 (4.8; 71 without the byte stores of the values), read
// back in 21 (4.0).  A lane owns 8 channels of a token (16 or 32 bytes) and keeps their cosines and sines in
// registers while it goes over the token's heads; four lanes (a DPP quad) hold the 32 channels that share an
// exponent.
#include <type_traits>

#include "../attention.h"

namespace skssm {

namespace {

constexpr int kThreads = 256;

// How the rotated channels pair up: channel i with i + R / 2 where that leaves lanes' pieces whole, or any i, or 2 i with 2 i + 1.
enum Pairs { NONE = 0, HALVES = 1, HALVES_ANY = 2, INTERLEAVED = 3 };

__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  auto step = [](uint32_t v, uint32_t w) { return v > w ? v : w; };
  x = step(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));
  return step(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));
}

// A lane's part of the rotation: y_i = x_i co_i + partner_i si_i.
template <typename IO, int PAIRS> struct Turn {
  float co[8], si[8];
  uint32_t turned;  // bit i: channel i of the lane's eight is rotated
  __device__ __forceinline__ void load(const Rotation& r, int row, int c0) {
    turned = 0;
    if constexpr (PAIRS != NONE) {
      const int half = r.rotated >> 1;
      const bool in = (unsigned)row < (unsigned)r.places;
      const float* at = r.angles + (size_t)(in ? row : 0) * r.rotated;
      if constexpr (PAIRS == HALVES) {
        if (c0 < r.rotated) {
          const bool low = c0 < half;
          const int i0 = low ? c0 : c0 - half;
          Vec<8> c, s;
          c.load(at + i0);
          s.load(at + half + i0);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            co[i] = in ? c.e[i] : __builtin_nanf("");
            si[i] = low ? -s.e[i] : s.e[i];
          }
          turned = 0xFF;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = c0 + i;
          if (c < r.rotated) {
            const bool low = PAIRS == INTERLEAVED ? !(c & 1) : c < half;
            const int j = PAIRS == INTERLEAVED ? c >> 1 : low ? c : c - half;
            co[i] = in ? at[j] : __builtin_nanf("");
            si[i] = low ? -at[half + j] : at[half + j];
            turned |= 1u << i;
          }
        }
      }
    }
  }
  // The partners of a lane's channels, where another piece holds them.
  __device__ __forceinline__ void partners(Raw<IO, 8>& p, const IO* x, int c0, int half) const {
    if constexpr (PAIRS == HALVES) {
      if (turned) p.load(x + (c0 < half ? c0 + half : c0 - half));
    }
  }
  __device__ __forceinline__ void apply(const Raw<IO, 8>& x, const Raw<IO, 8>& p, const IO* row, int c0, int half, float (&y)[8]) const {
#pragma clang fp contract(off)  // as the definition has it: each product and sum rounded
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = x.get(i);
      if constexpr (PAIRS != NONE) {
        if (PAIRS == HALVES ? turned != 0 : (turned >> i & 1) != 0) {
          float b;
          if constexpr (PAIRS == HALVES) b = p.get(i);
          else if constexpr (PAIRS == INTERLEAVED) b = x.get(i ^ 1);
          else b = ld_elem(row + (c0 + i < half ? c0 + i + half : c0 + i - half));
          const float u = y[i] * co[i], w = b * si[i];
          y[i] = u + w;
        }
      }
    }
  }
};

// Eight values over their block's power of two, in 4 bits (the first in the lowest); the block's exponent + 127.
__device__ __forceinline__ uint32_t encode(const float (&y)[8], int& exponent) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = __float_as_uint(y[i]) & 0x7FFFFFFFu;
    top = m > top ? m : top;
  }
  top = quad_max(top);
  // 7 = 1.75 * 4: one more where the mantissa is past 1.75
  const int e = (int)((top + 0x1FFFFFu) >> 23) - 2;
  exponent = top > 0x7EE00000u ? 255 : e < 63 ? 63 : e;  // past 7 2^124, or not a number
  const float scale = __uint_as_float((uint32_t)exponent << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
  return w;
}

// A workgroup takes 2^LT tokens; 2^lanes lanes (at least D / 8) hold a head, so that a head's lanes are of
// one wave and y may be x: a wave's loads of a head have come back before its stores go out.
template <typename IO, int PAIRS, int LT>
__global__ __launch_bounds__(kThreads) void append_kernel(CacheAppendArgs a, int lanes) {
  constexpr int U = 4;  // heads in flight
  const int tid = threadIdx.x, c0 = (tid & ((1 << lanes) - 1)) * 8;
  const int t = (int)((blockIdx.x << LT) + (tid >> lanes & ((1 << LT) - 1)));
  const int h0 = tid >> (lanes + LT), step = kThreads >> (lanes + LT);
  if (c0 >= a.D || t >= a.tok.seq.tokens) return;
  int b = 0, place = t;
  if (a.tok.lengths) {
    b = a.tok.seq.of(t);
    const int first = a.tok.seq.start(b), n = a.tok.seq.start(b + 1) - first;
    if (t < first || t >= first + n) return;  // behind the last sequence
    place = a.tok.place(b, n, t - first);
  }
  Turn<IO, PAIRS> turn;
  const int half = a.rot.rotated >> 1;
  if (PAIRS != NONE && (place >= 0 || a.rot.positions)) turn.load(a.rot, a.rot.positions ? a.rot.positions[t] : place, c0);
  else turn.turned = 0;

  // over the heads of x: their values, rotated where TURNED, to f(head, y)
  auto heads = [&](const void* xs, size_t ld, size_t head, int n, auto turned, auto f) {
    const IO* x = static_cast<const IO*>(xs) + (size_t)t * ld;
    for (int h = h0; h < n; h += U * step) {
      Raw<IO, 8> v[U], p[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (h + u * step < n) {
          const IO* at = x + (size_t)(h + u * step) * head;
          v[u].load(at + c0);
          if constexpr (turned.value) turn.partners(p[u], at, c0, half);
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (h + u * step < n) {
          float y[8];
          if constexpr (turned.value) {
            turn.apply(v[u], p[u], x + (size_t)(h + u * step) * head, c0, half, y);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[u].get(i);
          }
          f(h + u * step, y);
        }
    }
  };

  // where the token goes, looked up while the queries are turned
  const int tile = place >> 4, r = place & 15, D = a.D, blocks = D >> 5;
  const int page = a.tok.lengths && place >= 0 ? a.tok.page(a.cache, b, tile) : -1;
  heads(a.q, a.ldq, a.q_head, a.H, std::true_type{}, [&](int h, const float (&y)[8]) {
    IO* dst = static_cast<IO*>(a.y) + (size_t)t * a.ldy + (size_t)h * a.y_head + c0;
    st_elem4(dst, y[0], y[1], y[2], y[3]);
    st_elem4(dst + 4, y[4], y[5], y[6], y[7]);
  });
  if (page < 0) return;
  const size_t stride = (size_t)(17 * D) << a.cache.shift;  // from head to head
  uint8_t* rec = a.cache.data + (size_t)page * a.cache.heads * stride + (size_t)(tile & ((1 << a.cache.shift) - 1)) * (17 * D);
  heads(a.k, a.ldk, a.k_head, a.cache.heads, std::true_type{}, [&](int h, const float (&y)[8]) {
    int e;
    const uint32_t w = encode(y, e);
    uint8_t* at = rec + (size_t)h * stride;
    *reinterpret_cast<uint32_t*>(at + r * (D >> 1) + (c0 >> 1)) = w;
    if ((c0 & 31) == 0) at[16 * D + r * blocks + (c0 >> 5)] = (uint8_t)e;
  });
  heads(a.v, a.ldv, a.v_head, a.cache.heads, std::false_type{}, [&](int h, const float (&y)[8]) {
    int e;
    const uint32_t w = encode(y, e);
    uint8_t* at = rec + (size_t)h * stride;
    if ((c0 & 31) == 0) at[16 * D + (D >> 1) + r * blocks + (c0 >> 5)] = (uint8_t)e;
    // byte c of a block holds channels c and c + 16: the quad's lane l and l ^ 2; the lower lane takes the even bytes of its eight
    const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, 0x4E, 0xF, 0xF, true);
    const bool upper = (c0 & 16) != 0;
    const uint32_t lo = upper ? o : w, hi = upper ? w : o;
    const uint32_t bytes = upper ? (lo >> 4 & 0x0F0F0F0Fu) | (hi & 0xF0F0F0F0u) : (lo & 0x0F0F0F0Fu) | (hi & 0x0F0F0F0Fu) << 4;
    uint8_t* dst = at + 8 * D + (((r >> 2) * 16 + (c0 & 8) + (upper ? 1 : 0)) * blocks + (c0 >> 5)) * 4 + (r & 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[2 * i * blocks * 4] = (uint8_t)(bytes >> (8 * i));
  });
}

template <typename IO, int PAIRS, int LT> int launch_append(const CacheAppendArgs& a, hipStream_t s) {
  int lanes = 0;
  while (8 << lanes < a.D) ++lanes;
  const int64_t workgroups = ((int64_t)a.tok.seq.tokens + (1 << LT) - 1) >> LT;
  if (!fits(workgroups, kThreads)) return -3;
  hipLaunchKernelGGL((append_kernel<IO, PAIRS, LT>), dim3((unsigned)workgroups), dim3(kThreads), 0, s, a, lanes);
  return 0;
}

template <typename IO, int PAIRS> int launch_append(const CacheAppendArgs& a, hipStream_t s) {
  // Four tokens a workgroup (64 lanes each at most), or one, in us for the append and the read back of 32 + 2 x 8
  // heads of 128 channels: 64 tokens 10.2 and 8.7, 1024 12.1 and 11.8, 2048 17.3 and 18.4, 4096 25.7 and 28.2;
  // 16384 74 (two a workgroup 81, eight 77).
  return a.tok.seq.tokens > 1024 ? launch_append<IO, PAIRS, 2>(a, s) : launch_append<IO, PAIRS, 0>(a, s);
}

template <typename IO> int launch_append(const CacheAppendArgs& a, hipStream_t s) {
  if (!a.rot.angles) return launch_append<IO, NONE>(a, s);
  if (a.rot.interleaved) return launch_append<IO, INTERLEAVED>(a, s);
  return a.rot.rotated % 16 ? launch_append<IO, HALVES_ANY>(a, s) : launch_append<IO, HALVES>(a, s);
}

// A lane owns 16 channels of a token's head: keys 8 p .. and 8 p + D / 2 .., and the values that eight bytes of a record hold.
template <typename IO> __global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a) {
  const int D = a.D, pieces = D >> 4, blocks = D >> 5, G = a.cache.heads;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t item = i / pieces;
  const int p = (int)(i - item * pieces), t = (int)(item / G), h = (int)(item - (int64_t)t * G);
  if (t >= a.tok.seq.tokens) return;
  const int b = a.tok.seq.of(t), first = a.tok.seq.start(b), n = a.tok.seq.start(b + 1) - first;
  if (t < first || t >= first + n) return;
  const int place = a.tok.place(b, n, t - first), tile = place >> 4, r = place & 15;
  const int page = place < 0 ? 0 : a.tok.page(a.cache, b, tile);
  const uint8_t* rec = a.cache.data + ((((size_t)(page < 0 ? 0 : page) * G + h) << a.cache.shift) + (tile & ((1 << a.cache.shift) - 1))) * (17 * D);
  auto give = [&](void* out, int c0, uint32_t w, uint32_t e) {
    e = page < 0 ? 255 : e;
    const float scale = __uint_as_float(e << 23);
    IO* dst = static_cast<IO*>(out) + ((size_t)t * G + h) * D + c0;
    uint32_t x[4];
    x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = place < 0 ? 0 : x[j];
    if constexpr (sizeof(IO) == 2) {
      *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
    } else {
      st_elem4(dst, bf16_lo(x[0]), bf16_hi(x[0]), bf16_lo(x[1]), bf16_hi(x[1]));
      st_elem4(dst + 4, bf16_lo(x[2]), bf16_hi(x[2]), bf16_lo(x[3]), bf16_hi(x[3]));
    }
  };
  if (a.k) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c0 = 8 * p + j * (D >> 1);
      give(a.k, c0, *reinterpret_cast<const uint32_t*>(rec + r * (D >> 1) + (c0 >> 1)), rec[16 * D + r * blocks + (c0 >> 5)]);
    }
  }
  if (a.v) {
    const int g = p >> 1, c = (p & 1) * 8;  // bytes c .. c + 7 of block g
    const uint8_t* at = rec + 8 * D + (((r >> 2) * 16 + c) * blocks + g) * 4 + (r & 3);
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t x = at[j * blocks * 4];
      lo |= (x & 15) << (4 * j);
      hi |= (x >> 4) << (4 * j);
    }
    const uint32_t e = rec[16 * D + (D >> 1) + r * blocks + g];
    give(a.v, 32 * g + c, lo, e);
    give(a.v, 32 * g + c + 16, hi, e);
  }
}

}  // namespace

int run_append(const CacheAppendArgs& a, int io, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return io == 0 ? launch_append<float>(a, s) : launch_append<bf16_t>(a, s);
}

int run_cache_read(const ReadArgs& a, int io, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t workgroups = ((int64_t)a.tok.seq.tokens * a.cache.heads * (a.D / 16) + kThreads - 1) / kThreads;
  if (!fits(workgroups, kThreads)) return -3;
  if (io == 0) hipLaunchKernelGGL((read_kernel<float>), dim3((unsigned)workgroups), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((read_kernel<bf16_t>), dim3((unsigned)workgroups), dim3(kThreads), 0, s, a);
  return 0;
}

}  // namespace skssm
