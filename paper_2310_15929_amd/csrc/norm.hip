// The norm in front of a linear layer: h = x + residual (rounded to the type, as it is kept for the next layer), y = h w / sqrt(mean(h^2) + eps),
// y rounded once, to 16 bits or to microscaled 8 or 4 bits as the product of csrc/mx_matmul.hip takes them.
// Bound by memory: a row stays in registers between the sum of its squares (64 bits) and its output, so that every value is read and written
// once.  NT threads work on a row, C pieces of eight channels each; 64 threads (a wave) need no barrier.  Measured, cold, with a residual: 1 x 4096 3.4 us,
// 2048 x 4096 12.3 us (5.5 TB/s), to 8 bits 14.0, 2048 x 8192 27.7 us (4.8 TB/s), to 8 bits 26.5 (4.4 TB/s), without a residual 12.7 (5.3 TB/s).
#include <hip/hip_runtime.h>

#include "mx.h"

namespace {

constexpr int OUT_16 = -1;  // the output in the type of the input

struct NormArgs {
  const uint16_t* x;
  const uint16_t* residual;  // or null
  const uint16_t* weight;
  uint16_t* sum_out;  // h, or null; may be x or residual
  uint16_t* y;
  unsigned char* data;
  uint32_t* scales;
  long long ldx, ldr, R, K;
  unsigned steps;
  double eps;
};

template <int DT>
__device__ __forceinline__ uint32_t add_pair(uint32_t a, uint32_t b) {
  const float lo = esp_to_float<DT>((uint16_t)a) + esp_to_float<DT>((uint16_t)b);
  const float hi = esp_to_float<DT>((uint16_t)(a >> 16)) + esp_to_float<DT>((uint16_t)(b >> 16));
  return esp_from_float<DT>(lo) | (uint32_t)esp_from_float<DT>(hi) << 16;
}
__device__ __forceinline__ void store_8(uint16_t* p, long long left, const uint32_t (&v)[4]) {
  if (left >= 8) {
    store_stream_16(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < left) p[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
  }
}
// s + the squares of eight values, in 64 bits: rows of 16-bit numbers of any size, sums that no output can tell from exact ones
template <int DT>
__device__ __forceinline__ double squares(const uint32_t (&v)[4], double s) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const double lo = esp_to_float<DT>((uint16_t)v[i]), hi = esp_to_float<DT>((uint16_t)(v[i] >> 16));
    s = __builtin_fma(lo, lo, s);
    s = __builtin_fma(hi, hi, s);
  }
  return s;
}

// 1 / sqrt(mean of the squares + eps) = (hi + lo) 2^up, right to 2^-47, and K times the mean and eps, times 2^(2 up)
struct RowInverse {
  float hi, lo;
  int up;
  double sum;
};
// ... from the threads' sums; every thread of the row gets it.  `buf`: one double per wave.  hi is from 1 to 2, or 0, infinite or NaN with up = 0: rows of bf16
// numbers (and an eps of any size) have inverses from far below to 2^149, and h weight may pass fp32 where y does not, so that h takes the factor 2^up before the
// weight (in all rows: a test for those that need it costs as much, 0.1 us a launch)
template <int NT>
__device__ __forceinline__ RowInverse row_inverse(double own, double* buf, long long K, double eps) {
  double v = own;
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if constexpr (NT > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) buf[wave] = v;
    __syncthreads();
    v = 0.;
#pragma unroll
    for (int i = 0; i < NT / 64; i++) v += buf[i];
  }
  double inv = 1. / __builtin_sqrt(v / (double)K + eps);
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, inv);
  const unsigned top = (unsigned)(bits >> 32), exponent = top >> 20;
  int up = 0;
  if (exponent - 1u < 2046u) {
    up = (int)exponent - 1023;
    inv = __builtin_bit_cast(double, (unsigned long long)((top & 0xfffffu) | 0x3ff00000u) << 32 | (unsigned)bits);
  }
  const float hi = (float)inv;
  return RowInverse{hi, __builtin_isfinite(hi) ? (float)(inv - (double)hi) : 0.f, up, __builtin_ldexp(__builtin_fma(eps, (double)K, v), 2 * up)};
}

// p (hi + lo), rounded once
__device__ __forceinline__ float times(float p, const RowInverse& by) {
  return __builtin_copysignf(__builtin_fmaf(p, by.hi, p * by.lo), p);  // (-0 (hi + lo) with lo < 0 would be +0)
}
// v = times(p, by), not 0, to an odd last bit where it is not exact: rounding that again to 8 or 4 bits gives what rounding the exact value would.  Which side of v the
// exact value is on, or whether it is v (rows of one magnitude, and others with a rational norm, put results right on the middle of two codes), the squares tell
// without a root or a division: those of p (times K, below 2^21) and of v are exact in 64 bits
__device__ __forceinline__ float to_odd(float v, float p, const RowInverse& by, long long K) {
  const double rest = __builtin_fma(-(double)v * (double)v, by.sum, (double)p * (double)p * (double)K);
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  if ((b & 1u) || !(rest < 0. || rest > 0.)) return v;
  return __builtin_bit_cast(float, rest > 0. ? b + 1u : b - 1u);
}

// output of one piece of eight channels (a product of two 16-bit numbers and a power of two is exact within fp32: y = h w / sqrt(..) is
// rounded once).  Lanes of pieces
// behind the row's last channel take part (zeros in the padding of a microscaled row); `chunk` differs by one between neighbouring lanes and starts at a
// multiple of 16
template <int DT, int OUT>
__device__ __forceinline__ void norm_out(const NormArgs& a, long long row, unsigned chunk, const uint32_t (&h)[4], const uint32_t (&w)[4], const RowInverse& inv) {
  float v[8], p[8];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    p[2 * i] = __builtin_ldexpf(esp_to_float<DT>((uint16_t)h[i]), inv.up) * esp_to_float<DT>((uint16_t)w[i]);
    p[2 * i + 1] = __builtin_ldexpf(esp_to_float<DT>((uint16_t)(h[i] >> 16)), inv.up) * esp_to_float<DT>((uint16_t)(w[i] >> 16));
  }
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] = times(p[i], inv);
  if constexpr (OUT != OUT_16) {
    // The middle between two codes, and a power of two, has at most five of the 24 significant bits: only a value with the others zero can have been
    // rounded onto one (one in 2^19)
    uint32_t low = ~0u;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const uint32_t b = __builtin_bit_cast(uint32_t, v[i]) << 13;
      low = b < low ? b : low;
    }
    if (low == 0u) {  // (those of the eight, one after the other: all eight in a row are so much code that 2048 x 4096 to 8 bits takes 15.1 us instead of 13.9)
      unsigned todo = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) todo |= (__builtin_bit_cast(uint32_t, v[i]) << 13 == 0u && v[i] != 0.f ? 1u : 0u) << i;
      for (; todo; todo &= todo - 1u) {
        const unsigned at = (unsigned)__builtin_ctz(todo);
        float one = v[0], of = p[0];
#pragma unroll
        for (unsigned i = 1; i < 8; i++) {
          one = at == i ? v[i] : one;
          of = at == i ? p[i] : of;
        }
        one = to_odd(one, of, inv, a.K);
#pragma unroll
        for (unsigned i = 0; i < 8; i++) v[i] = at == i ? one : v[i];
      }
    }
  }
  if constexpr (OUT == OUT_16) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = esp_from_float<DT>(v[2 * i]) | (uint32_t)esp_from_float<DT>(v[2 * i + 1]) << 16;
    store_8(a.y + row * a.K + (long long)chunk * 8, a.K - (long long)chunk * 8, o);
  } else {
    if (chunk >= a.steps * 16) return;  // (whole groups of 16 lanes)
#pragma unroll
    for (int i = 0; i < 8; i++)
      if ((long long)chunk * 8 + i >= a.K) v[i] = 0.f;  // (0 times an infinite 1 / norm is no 0)
    const unsigned e = mx_block_exponent<OUT>(v);
    mx_store<OUT>(a.data + row * ((long long)a.steps * (OUT == ESPARSE_MX_FP4 ? 64 : 128)), chunk, mx_encode<OUT>(v, e),
                  a.scales + (long long)(chunk >> 4) * a.R + row, e, threadIdx.x);
  }
}

template <int DT, int OUT, int NT, int C>
__global__ void __launch_bounds__(NT < 256 ? 256 : NT) k_rms_norm(const NormArgs a) {
  constexpr int ROWS = NT < 256 ? 256 / NT : 1;
  __shared__ double buf[NT > 64 ? NT / 64 : 1];
  const unsigned t = threadIdx.x % NT;
  const long long row = (long long)blockIdx.x * ROWS + threadIdx.x / NT;
  if (row >= a.R) return;  // (whole waves, and no barrier where a workgroup has several rows)
  uint32_t h[C][4], r[C][4], w[C][4];
#pragma unroll
  for (int j = 0; j < C; j++) load_8(a.x + row * a.ldx + (long long)(j * NT + t) * 8, a.K - (long long)(j * NT + t) * 8, h[j]);
  if (a.residual) {
#pragma unroll
    for (int j = 0; j < C; j++) load_8(a.residual + row * a.ldr + (long long)(j * NT + t) * 8, a.K - (long long)(j * NT + t) * 8, r[j]);
  }
#pragma unroll
  for (int j = 0; j < C; j++) load_8(a.weight + (long long)(j * NT + t) * 8, a.K - (long long)(j * NT + t) * 8, w[j]);
  double s = 0.;
#pragma unroll
  for (int j = 0; j < C; j++) {
    if (a.residual) {
#pragma unroll
      for (int i = 0; i < 4; i++) h[j][i] = add_pair<DT>(h[j][i], r[j][i]);
    }
    if (a.sum_out) store_8(a.sum_out + row * a.K + (long long)(j * NT + t) * 8, a.K - (long long)(j * NT + t) * 8, h[j]);
    s = squares<DT>(h[j], s);
  }
  const RowInverse inv = row_inverse<NT>(s, buf, a.K, a.eps);
#pragma unroll
  for (int j = 0; j < C; j++) norm_out<DT, OUT>(a, row, j * NT + t, h[j], w[j], inv);
}

// rows that do not fit the registers of a workgroup are read twice
template <int DT, int OUT>
__global__ void __launch_bounds__(1024) k_rms_norm_long(const NormArgs a) {
  __shared__ double buf[16];
  const long long row = blockIdx.x;
  const unsigned chunks = a.steps * 16, t = threadIdx.x;
  double s = 0.;
  uint32_t h[4], r[4], w[4];
  for (unsigned c = t; c < chunks; c += 1024) {
    const long long at = (long long)c * 8, left = a.K - at;
    load_8(a.x + row * a.ldx + at, left, h);
    if (a.residual) {
      load_8(a.residual + row * a.ldr + at, left, r);
#pragma unroll
      for (int i = 0; i < 4; i++) h[i] = add_pair<DT>(h[i], r[i]);
    }
    if (a.sum_out) store_8(a.sum_out + row * a.K + at, left, h);
    s = squares<DT>(h, s);
  }
  const RowInverse inv = row_inverse<1024>(s, buf, a.K, a.eps);
  for (unsigned c0 = 0; c0 < chunks; c0 += 1024) {
    const unsigned c = c0 + t;
    const long long at = (long long)c * 8, left = a.K - at;
    if (a.sum_out) {  // this thread's own stores (x or the residual may be gone)
      load_8(a.sum_out + row * a.K + at, left, h);
    } else {
      load_8(a.x + row * a.ldx + at, left, h);
      if (a.residual) {
        load_8(a.residual + row * a.ldr + at, left, r);
#pragma unroll
        for (int i = 0; i < 4; i++) h[i] = add_pair<DT>(h[i], r[i]);
      }
    }
    load_8(a.weight + at, left, w);
    norm_out<DT, OUT>(a, row, c, h, w, inv);
  }
}

template <int DT, int OUT>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  const unsigned chunks = a.steps * 16;
#define GO(NT, C) \
  hipLaunchKernelGGL((k_rms_norm<DT, OUT, NT, C>), dim3((unsigned)((a.R + (NT < 256 ? 256 / NT : 1) - 1) / (NT < 256 ? 256 / NT : 1))), dim3(NT < 256 ? 256 : NT), 0, st, a)
  if (chunks <= 64) GO(64, 1);
  else if (chunks <= 256) GO(256, 1);
  else if (chunks <= 512) GO(256, 2);
  else if (chunks <= 1024) GO(256, 4);
  else if (chunks <= 2048) GO(1024, 2);
  else if (chunks <= 4096) GO(1024, 4);
  else hipLaunchKernelGGL((k_rms_norm_long<DT, OUT>), dim3((unsigned)a.R), dim3(1024), 0, st, a);
#undef GO
  return hipGetLastError();
}

}  // namespace

int esp_rms_norm_device(esparse_ctx* ctx, const void* x, long long ldx, const void* residual, long long ldr, const void* weight, long long R, long long K,
                        double eps, int dtype, void* sum_out, void* y, int fmt, void* data, void* scales) {
  const NormArgs a = {(const uint16_t*)x, (const uint16_t*)residual, (const uint16_t*)weight, (uint16_t*)sum_out, (uint16_t*)y, (unsigned char*)data,
                      (uint32_t*)scales, ldx, ldr, R, K, (unsigned)((K + 127) / 128), eps};
  if (dtype == ESPARSE_F16) {
    if (y) ESP_HIP(ctx, (launch<ESPARSE_F16, OUT_16>(a, ctx->stream)));
    else if (fmt == ESPARSE_MX_FP4) ESP_HIP(ctx, (launch<ESPARSE_F16, ESPARSE_MX_FP4>(a, ctx->stream)));
    else ESP_HIP(ctx, (launch<ESPARSE_F16, ESPARSE_MX_FP8>(a, ctx->stream)));
  } else {
    if (y) ESP_HIP(ctx, (launch<ESPARSE_BF16, OUT_16>(a, ctx->stream)));
    else if (fmt == ESPARSE_MX_FP4) ESP_HIP(ctx, (launch<ESPARSE_BF16, ESPARSE_MX_FP4>(a, ctx->stream)));
    else ESP_HIP(ctx, (launch<ESPARSE_BF16, ESPARSE_MX_FP8>(a, ctx->stream)));
  }
  return ESPARSE_OK;
}
