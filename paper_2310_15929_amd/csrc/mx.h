// Microscaled (MX) numbers on the device: 32 consecutive channels of a row share a scale 2^(E - 127), E one byte.
//   E = max(floor(log2(largest magnitude)) - emax, -127) + 127, emax = 2 (4 bits: E2M1, up to 6) or 8 (8 bits: E4M3, up to 448);
//   an element is value / 2^(E - 127), rounded to the nearest number of its format (ties to even) and no further than the largest.
// 255 in the place of E marks a block that holds an infinity or a NaN: it reads as NaN throughout.
// The division and the rounding are one conversion instruction of gfx950 for two values, exact for every 16-bit input and
// every scale (checked over all of them); it takes magnitudes beyond 464 of a scale to the NaN code of E4M3, hence mx_saturate_fp8.
#pragma once
#include "intrinsics.h"

typedef short esp_short2 __attribute__((ext_vector_type(2)));
typedef _Float16 esp_half2 __attribute__((ext_vector_type(2)));
typedef __bf16 esp_bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short esp_ushort2 __attribute__((ext_vector_type(2)));
typedef float esp_float2 __attribute__((ext_vector_type(2)));

// E of a block from the bits of its largest magnitude (type DT, sign cleared)
template <int DT, int FMT>
__device__ __forceinline__ unsigned mx_exponent(uint32_t a) {
  constexpr int emax = FMT == ESPARSE_MX_FP4 ? 2 : 8;
  if (DT == ESPARSE_F16) {
    if (a >= 0x7c00u) return 255u;
    if (a == 0u) return 0u;
    const int e = a >= 0x400u ? (int)(a >> 10) - 15 : 7 - (int)__builtin_clz(a);  // subnormal: a 2^-24
    return (unsigned)(e - emax + 127);
  } else {
    const unsigned e = DT == ESPARSE_BF16 ? a >> 7 : a >> 23;
    if (e == 255u) return 255u;
    return e > (unsigned)emax ? e - emax : 0u;
  }
}

// 2^(E - 127) as a float (E = 0: the subnormal 2^-127; 255: NaN)
__device__ __forceinline__ float mx_scale(unsigned e) {
  return __builtin_bit_cast(float, e == 0u ? 0x00400000u : (e == 255u ? 0x7fc00000u : e << 23));
}

// codes of E4M3 beyond 448 (0x7f: the conversion's NaN) down to 448 (0x7e), four at a time
__device__ __forceinline__ uint32_t mx_saturate_fp8(uint32_t w) {
  return w - ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7);
}

// a lane's neighbours: the other lanes of its quad, and of its row of 16 by rotation
template <int CTRL>
__device__ __forceinline__ uint32_t lane_move(uint32_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
#else
  return v;
#endif
}
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  uint32_t o = lane_move<0xB1>(v);  // lanes 1 0 3 2
  v = o > v ? o : v;
  o = lane_move<0x4E>(v);  // lanes 2 3 0 1
  return o > v ? o : v;
}

// Four lanes hold a block, eight values each.  mx_block_exponent: E of the block (all four lanes get it).
__device__ __forceinline__ uint32_t mx_max_pair(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(esp_ushort2, a), __builtin_bit_cast(esp_ushort2, b)));
}
template <int DT, int FMT>
__device__ __forceinline__ unsigned mx_block_exponent(const uint32_t (&v)[4]) {  // eight 16-bit values
  constexpr uint32_t mag = 0x7fff7fffu;
  const uint32_t m = mx_max_pair(mx_max_pair(v[0] & mag, v[1] & mag), mx_max_pair(v[2] & mag, v[3] & mag));
  const uint32_t lo = m & 0xffffu, hi = m >> 16;
  return mx_exponent<DT, FMT>(quad_max(lo > hi ? lo : hi));
}
template <int FMT>
__device__ __forceinline__ unsigned mx_block_exponent(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const uint32_t a = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
    m = a > m ? a : m;
  }
  return mx_exponent<ESPARSE_F32, FMT>(quad_max(m));
}

// the eight codes: 4 bits in lo alone, 8 bits in lo and hi
struct MxCodes {
  uint32_t lo, hi;
};
template <int DT, int FMT>
__device__ __forceinline__ MxCodes mx_encode(const uint32_t (&v)[4], unsigned e) {
  MxCodes r = {0u, 0u};
#if defined(__HIP_DEVICE_COMPILE__)
  const float s = mx_scale(e);
  if constexpr (FMT == ESPARSE_MX_FP4) {
    if constexpr (DT == ESPARSE_F16) {
      r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r.lo, __builtin_bit_cast(esp_half2, v[0]), s, 0);
      r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r.lo, __builtin_bit_cast(esp_half2, v[1]), s, 1);
      r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r.lo, __builtin_bit_cast(esp_half2, v[2]), s, 2);
      r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r.lo, __builtin_bit_cast(esp_half2, v[3]), s, 3);
    } else {
      r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r.lo, __builtin_bit_cast(esp_bf16x2, v[0]), s, 0);
      r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r.lo, __builtin_bit_cast(esp_bf16x2, v[1]), s, 1);
      r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r.lo, __builtin_bit_cast(esp_bf16x2, v[2]), s, 2);
      r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r.lo, __builtin_bit_cast(esp_bf16x2, v[3]), s, 3);
    }
  } else {
    esp_short2 a = {0, 0}, b = {0, 0};
    if constexpr (DT == ESPARSE_F16) {
      a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(a, __builtin_bit_cast(esp_half2, v[0]), s, false);
      a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(a, __builtin_bit_cast(esp_half2, v[1]), s, true);
      b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(b, __builtin_bit_cast(esp_half2, v[2]), s, false);
      b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(b, __builtin_bit_cast(esp_half2, v[3]), s, true);
    } else {
      a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(esp_bf16x2, v[0]), s, false);
      a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(esp_bf16x2, v[1]), s, true);
      b = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(b, __builtin_bit_cast(esp_bf16x2, v[2]), s, false);
      b = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(b, __builtin_bit_cast(esp_bf16x2, v[3]), s, true);
    }
    r.lo = mx_saturate_fp8(__builtin_bit_cast(uint32_t, a));
    r.hi = mx_saturate_fp8(__builtin_bit_cast(uint32_t, b));
  }
  if (e == 255u) r.lo = r.hi = 0u;
#endif
  return r;
}
template <int FMT>
__device__ __forceinline__ MxCodes mx_encode(const float (&v)[8], unsigned e) {
  MxCodes r = {0u, 0u};
#if defined(__HIP_DEVICE_COMPILE__)
  const float s = mx_scale(e);
  if constexpr (FMT == ESPARSE_MX_FP4) {
    r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.lo, v[0], v[1], s, 0);
    r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.lo, v[2], v[3], s, 1);
    r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.lo, v[4], v[5], s, 2);
    r.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.lo, v[6], v[7], s, 3);
  } else {
    esp_short2 a = {0, 0}, b = {0, 0};
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, v[0], v[1], s, false);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, v[2], v[3], s, true);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, v[4], v[5], s, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, v[6], v[7], s, true);
    r.lo = mx_saturate_fp8(__builtin_bit_cast(uint32_t, a));
    r.hi = mx_saturate_fp8(__builtin_bit_cast(uint32_t, b));
  }
  if (e == 255u) r.lo = r.hi = 0u;
#endif
  return r;
}

// the four scales of 16 lanes (128 channels), as the 32-bit word they are stored as; every lane of the 16 gets it
__device__ __forceinline__ uint32_t mx_scale_word(unsigned e, unsigned lane) {
  uint32_t w = e << (8u * ((lane >> 2) & 3u));
  w |= lane_move<0x128>(w);  // the row of 16 rotated by 8
  w |= lane_move<0x124>(w);  // and by 4
  return w;
}
// stores a lane's codes (row: first byte of the row's data, chunk: number of the eight channels) and, from every 16th lane, the scale word
template <int FMT>
__device__ __forceinline__ void mx_store(unsigned char* row, unsigned chunk, MxCodes c, uint32_t* scale, unsigned e, unsigned lane) {
  if constexpr (FMT == ESPARSE_MX_FP4) __builtin_nontemporal_store(c.lo, reinterpret_cast<uint32_t*>(row + 4ull * chunk));
  else store_stream_8(row + 8ull * chunk, &c);
  const uint32_t w = mx_scale_word(e, lane);
  if ((lane & 15u) == 0u) *scale = w;
}

// eight consecutive values from an address of any alignment that suits one of them; `left`: how many there are
template <class T>
__device__ __forceinline__ void load_8(const T* p, long long left, uint32_t (&v)[4]) {
  static_assert(sizeof(T) == 2, "16-bit values");
  if (left >= 8) {
    __builtin_memcpy(v, p, 16);
  } else {
    // all eight loads under way at once: places behind the last repeat it
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 8; i++) t[i] = 0;
    if (left > 0) {
#pragma unroll
      for (int i = 0; i < 8; i++) t[i] = p[i < left ? i : left - 1];
    }
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = (2 * i < left ? t[2 * i] : 0u) | (2 * i + 1 < left ? t[2 * i + 1] : 0u) << 16;
  }
}
