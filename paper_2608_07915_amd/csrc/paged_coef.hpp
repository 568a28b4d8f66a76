// Records of a page as fp16 coefficients in LDS, and the matrix products of the paged attention
// kernels. A slot tile holds one kept group of 64 slots: [slot][32 places], keys and values alike.
#pragma once
#include "attn_common.hpp"
#include "code_operands.hpp"
#include "paged_dev.hpp"

namespace spectra_dev {

constexpr int CA_TILE = TILE * 64;     // bytes of a slot tile: 64 slots x 32 fp16
constexpr float CA_SLACK = 3.0f;       // log2: the running maximum moves when passed by more
constexpr float CA_LIFT = 12.0f;       // log2: weights are kept 2^12 above their share
constexpr float CA_LO = 2048.0f;       // the second fp16 part of a number is scaled by 2^11

// LDS byte of 16-byte piece `piece` of slot `t` in a slot tile. Slots 4 apart lie 2 pieces apart, so
// that transposed reads of eight neighbouring slots use all banks.
__device__ __forceinline__ int piece_at(int t, int piece) { return t * 64 + ((piece ^ ((t >> 1) & 2) ^ ((t >> 3) & 1)) << 4); }

// A token's metadata word of a b-bit group, made finite: NaN or infinite scales count as 0, and
// the scale is lowered where z + s (2^b - 1) would pass fp16's largest number.
__device__ __forceinline__ uint32_t finite_meta(uint32_t m, int b) {
  m = finite_or_zero(m);
  const float s = h2f(m), z = h2f(m >> 16), top = (float)((1 << b) - 1);
  if (__builtin_fabsf(__builtin_fmaf(s, top, z)) > 65504.0f)
    m = (m & 0xFFFF0000u) | f2h_sat((__builtin_copysignf(65472.0f, s) - z) / top);
  return m;
}

// One slot's group as fp16 coefficients z + s code into its LDS row (parts: the low parts'
// tiles are `lo` bytes further).
template <int B, bool PRECISE>
__device__ __forceinline__ void write_coefficients(const uint32_t (&w)[8], uint32_t meta, uint8_t* tile, int t, int lo,
                                                   uint32_t magic) {
  uint32_t Z[8];
  join_halves<B>(w, Z);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f16x8 c = codes_f16<B, false>(Z, k, magic);
    const _Float16 s = __builtin_bit_cast(_Float16, (uint16_t)meta), z = __builtin_bit_cast(_Float16, (uint16_t)(meta >> 16));
    if constexpr (!PRECISE) {
      u32x4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        r[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(f16x2{s, s}, f16x2{c[2 * i], c[2 * i + 1]}, f16x2{z, z}));
      *reinterpret_cast<u32x4*>(tile + piece_at(t, k)) = r;
    } else {
      u32x4 rh, rl;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 x = f32x2{__builtin_fmaf((float)s, (float)c[2 * i], (float)z), __builtin_fmaf((float)s, (float)c[2 * i + 1], (float)z)};
        const f16x2 hi = __builtin_convertvector(x, f16x2);
        const f32x2 d = f32x2{(x[0] - (float)hi[0]) * CA_LO, (x[1] - (float)hi[1]) * CA_LO};
        rh[i] = __builtin_bit_cast(uint32_t, hi);
        rl[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(d, f16x2));
      }
      *reinterpret_cast<u32x4*>(tile + piece_at(t, k)) = rh;
      *reinterpret_cast<u32x4*>(tile + lo + piece_at(t, k)) = rl;
    }
  }
}

typedef __fp16 h16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ u32x2 read_transposed(const uint8_t* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
}
__device__ __forceinline__ f16x8 as_f16x8(u32x4 v) { return __builtin_bit_cast(f16x8, v); }
__device__ __forceinline__ f32x16 mfma_f16(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}
// Eight fp32 numbers as NP bf16 parts.
template <int NP>
__device__ __forceinline__ void split8(const float (&v)[8], bf16x8 (&p)[NP]) {
  uint32_t a[NP][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float r = v[i];
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      a[q][i] = f2bf(r);
      r -= bf2f(a[q][i]);
    }
  }
#pragma unroll
  for (int q = 0; q < NP; ++q)
    p[q] = as_bf16x8(u32x4{pack2(a[q][0], a[q][1]), pack2(a[q][2], a[q][3]), pack2(a[q][4], a[q][5]), pack2(a[q][6], a[q][7])});
}

// The same by the conversion instruction, two numbers at a time (a third of the instructions; finite
// numbers alike).
template <int NP>
__device__ __forceinline__ void split8_pairs(const float (&v)[8], bf16x8 (&p)[NP]) {
  u32x4 w[NP];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x2 r = f32x2{v[2 * i], v[2 * i + 1]};
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_convertvector(r, bf16x2));
      w[q][i] = b;
      r = f32x2{r[0] - __uint_as_float(b << 16), r[1] - __uint_as_float(b & 0xFFFF0000u)};
    }
  }
#pragma unroll
  for (int q = 0; q < NP; ++q) p[q] = as_bf16x8(w[q]);
}

}  // namespace spectra_dev
