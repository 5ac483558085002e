// Quantisation to microscaled numbers, reading them back, and the order in which the product streams 4-bit weights.
// All three are bound by memory: a value is read and written once, about ten vector operations for each two of them.  Measured, cold (a copy of 1 GiB:
// 5.1 TB/s): 11008 x 4096 16-bit values to 4 bits 21.6 us (5.3 TB/s), to 8 bits 26.1 (5.2), back 18.0 (6.3) and 24.1 (5.7); 11008 x 13824 to 4 bits 64.5 (6.0),
// back 56.9 (6.8).  Small ones are launches: 333 x 5003 to 8 bits 4.4 us, back 3.6.
#include <hip/hip_runtime.h>

#include "mx.h"

namespace {

// One workgroup of 256 threads takes 16 rows x 512 channels: a wave 512 channels of one row (runs of 1 KiB are read, of 256 or 512 bytes written) and four
// rows, 64 bytes a lane under way; 16 lanes hold 128 channels (eight values a lane, four lanes a block).  The scale words of the 16 rows meet in the L2.
constexpr int TILE_ROWS = 16, TILE_STEPS = 4;

template <int DT, int FMT>
__global__ void __launch_bounds__(256) k_mx_quantize(const void* __restrict__ X, long long ldx, long long R, long long K, unsigned steps, unsigned spans,
                                                     unsigned char* __restrict__ data, uint32_t* __restrict__ scales) {
  const unsigned tile = blockIdx.x / spans, span = blockIdx.x % spans, lane = threadIdx.x & 63u;
  const long long row0 = (long long)tile * TILE_ROWS + (threadIdx.x >> 6);
  const unsigned chunk = span * (TILE_STEPS * 16) + lane, step = chunk >> 4;
  if (step >= steps) return;  // (whole groups of 16 lanes)
  const long long at = (long long)chunk * 8, left = K - at;
  const long long row_bytes = (long long)steps * (FMT == ESPARSE_MX_FP4 ? 64 : 128);
  if constexpr (DT == ESPARSE_F32) {
    float v[TILE_ROWS / 4][8];
#pragma unroll
    for (int j = 0; j < TILE_ROWS / 4; j++) {
      const float* x = reinterpret_cast<const float*>(X) + (row0 + 4 * j < R ? row0 + 4 * j : R - 1) * ldx + at;
      if (left >= 8) {
        __builtin_memcpy(v[j], x, 32);
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          v[j][i] = 0.f;
          if (i < left) v[j][i] = x[i];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < TILE_ROWS / 4; j++) {
      const long long row = row0 + 4 * j;
      if (row >= R) break;
      const unsigned e = mx_block_exponent<FMT>(v[j]);
      mx_store<FMT>(data + row * row_bytes, chunk, mx_encode<FMT>(v[j], e), scales + (long long)step * R + row, e, lane);
    }
  } else {
    uint32_t v[TILE_ROWS / 4][4];
#pragma unroll
    for (int j = 0; j < TILE_ROWS / 4; j++)
      load_8(reinterpret_cast<const uint16_t*>(X) + (row0 + 4 * j < R ? row0 + 4 * j : R - 1) * ldx + at, left, v[j]);
#pragma unroll
    for (int j = 0; j < TILE_ROWS / 4; j++) {
      const long long row = row0 + 4 * j;
      if (row >= R) break;
      const unsigned e = mx_block_exponent<DT, FMT>(v[j]);
      mx_store<FMT>(data + row * row_bytes, chunk, mx_encode<DT, FMT>(v[j], e), scales + (long long)step * R + row, e, lane);
    }
  }
}

// the same split of the work; a lane reads the codes of eight channels and its block's scale
template <int FMT, int DT>
__global__ void __launch_bounds__(256) k_mx_dequantize(const unsigned char* __restrict__ data, const unsigned char* __restrict__ scales, long long R,
                                                       long long K, unsigned steps, unsigned spans, void* __restrict__ out) {
  const unsigned tile = blockIdx.x / spans, span = blockIdx.x % spans, lane = threadIdx.x & 63u;
  const long long row0 = (long long)tile * TILE_ROWS + (threadIdx.x >> 6);
  const long long at = (long long)span * (TILE_STEPS * 128) + lane * 8, left = K - at;
  if (left <= 0) return;
  const unsigned step = span * TILE_STEPS + (lane >> 4);
  const long long row_bytes = (long long)steps * (FMT == ESPARSE_MX_FP4 ? 64 : 128);
  uint32_t c[TILE_ROWS / 4][2];
  unsigned e[TILE_ROWS / 4];
#pragma unroll
  for (int j = 0; j < TILE_ROWS / 4; j++) {
    const long long row = row0 + 4 * j < R ? row0 + 4 * j : R - 1;
    if constexpr (FMT == ESPARSE_MX_FP4) c[j][0] = *reinterpret_cast<const uint32_t*>(data + row * row_bytes + at / 2);
    else __builtin_memcpy(c[j], data + row * row_bytes + at, 8);
    e[j] = scales[((long long)step * R + row) * 4 + ((lane >> 2) & 3u)];
  }
#pragma unroll
  for (int j = 0; j < TILE_ROWS / 4; j++) {
    const long long row = row0 + 4 * j;
    if (row >= R) break;
    float f[8];
#if defined(__HIP_DEVICE_COMPILE__)
    const float s = mx_scale(e[j]);
#define PAIR(i, call)                   \
  {                                     \
    const esp_float2 p = call;          \
    f[2 * (i)] = p[0];                  \
    f[2 * (i) + 1] = p[1];              \
  }
    if constexpr (FMT == ESPARSE_MX_FP4) {
      PAIR(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[j][0], s, 0))
      PAIR(1, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[j][0], s, 1))
      PAIR(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[j][0], s, 2))
      PAIR(3, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[j][0], s, 3))
    } else {
      PAIR(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[j][0], s, false))
      PAIR(1, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[j][0], s, true))
      PAIR(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[j][1], s, false))
      PAIR(3, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[j][1], s, true))
    }
#undef PAIR
    if (e[j] == 255u) {
#pragma unroll
      for (int i = 0; i < 8; i++) f[i] = __builtin_nanf("");
    }
#endif
    if constexpr (DT == ESPARSE_F32) {
      float* o = reinterpret_cast<float*>(out) + row * K + at;
      if (left >= 8) {
        store_stream_16(o, f);
        store_stream_16(o + 4, f + 4);
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
          if (i < left) o[i] = f[i];
      }
    } else {
      uint16_t* o = reinterpret_cast<uint16_t*>(out) + row * K + at;
      uint16_t h[8];
#pragma unroll
      for (int i = 0; i < 8; i++) h[i] = esp_from_float<DT>(f[i]);
      if (left >= 8) {
        store_stream_16(o, h);
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
          if (i < left) o[i] = h[i];
      }
    }
  }
}

// 4-bit weights in the order the product streams them (include/esparse.h).  A wave takes 64 rows x 128 channels.
__global__ void __launch_bounds__(256) k_mx_pack(const unsigned char* __restrict__ data, const unsigned char* __restrict__ scales, long long N, unsigned steps,
                                                 long long groups, uint4* __restrict__ values, uint32_t* __restrict__ out_scales) {
  const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= groups * steps) return;
  const long long grp = item / steps;
  const unsigned ks = (unsigned)(item % steps), lane = threadIdx.x & 63u, c = lane & 15u, g = lane >> 4;
  uint32_t w = 0;
#pragma unroll
  for (int b = 0; b < 4; b++) {
    const long long row = grp * 64 + b * 16 + c;
    uint4 v = {0u, 0u, 0u, 0u};
    if (row < N) {
      v = *reinterpret_cast<const uint4*>(data + row * ((long long)steps * 64) + ks * 64ull + g * 16);
      w |= (uint32_t)scales[((long long)ks * N + row) * 4 + g] << (8 * b);
    }
    values[((grp * 4 + b) * steps + ks) * 64 + lane] = v;
  }
  out_scales[(grp * steps + ks) * 64 + lane] = w;
}

}  // namespace

int esp_mx_quantize_device(esparse_ctx* ctx, const void* X, long long R, long long K, long long ldx, int dtype, int fmt, void* data, void* scales) {
  const unsigned steps = (unsigned)((K + 127) / 128), spans = (steps + TILE_STEPS - 1) / TILE_STEPS;
  const long long blocks = (R + TILE_ROWS - 1) / TILE_ROWS * spans;
#define GO(D, F)                                                                                                                                 \
  hipLaunchKernelGGL((k_mx_quantize<D, F>), dim3((unsigned)blocks), dim3(256), 0, ctx->stream, X, ldx, R, K, steps, spans, (unsigned char*)data, \
                     (uint32_t*)scales)
  if (fmt == ESPARSE_MX_FP4) {
    if (dtype == ESPARSE_F16) GO(ESPARSE_F16, ESPARSE_MX_FP4);
    else if (dtype == ESPARSE_BF16) GO(ESPARSE_BF16, ESPARSE_MX_FP4);
    else GO(ESPARSE_F32, ESPARSE_MX_FP4);
  } else {
    if (dtype == ESPARSE_F16) GO(ESPARSE_F16, ESPARSE_MX_FP8);
    else if (dtype == ESPARSE_BF16) GO(ESPARSE_BF16, ESPARSE_MX_FP8);
    else GO(ESPARSE_F32, ESPARSE_MX_FP8);
  }
#undef GO
  ESP_HIP(ctx, hipGetLastError());
  return ESPARSE_OK;
}

int esp_mx_dequantize_device(esparse_ctx* ctx, const void* data, const void* scales, long long R, long long K, int fmt, int dtype, void* out) {
  const unsigned steps = (unsigned)((K + 127) / 128), spans = (steps + TILE_STEPS - 1) / TILE_STEPS;
  const long long blocks = (R + TILE_ROWS - 1) / TILE_ROWS * spans;
#define GO(F, D)                                                                                                                            \
  hipLaunchKernelGGL((k_mx_dequantize<F, D>), dim3((unsigned)blocks), dim3(256), 0, ctx->stream, (const unsigned char*)data,                \
                     (const unsigned char*)scales, R, K, steps, spans, out)
  if (fmt == ESPARSE_MX_FP4) {
    if (dtype == ESPARSE_F16) GO(ESPARSE_MX_FP4, ESPARSE_F16);
    else if (dtype == ESPARSE_BF16) GO(ESPARSE_MX_FP4, ESPARSE_BF16);
    else GO(ESPARSE_MX_FP4, ESPARSE_F32);
  } else {
    if (dtype == ESPARSE_F16) GO(ESPARSE_MX_FP8, ESPARSE_F16);
    else if (dtype == ESPARSE_BF16) GO(ESPARSE_MX_FP8, ESPARSE_BF16);
    else GO(ESPARSE_MX_FP8, ESPARSE_F32);
  }
#undef GO
  ESP_HIP(ctx, hipGetLastError());
  return ESPARSE_OK;
}

int esp_mx_pack_device(esparse_ctx* ctx, const void* data, const void* scales, long long N, long long K, void* packed) {
  const unsigned steps = (unsigned)((K + 127) / 128);
  const long long groups = (N + 63) / 64;
  hipLaunchKernelGGL(k_mx_pack, dim3((unsigned)((groups * steps + 3) / 4)), dim3(256), 0, ctx->stream, (const unsigned char*)data,
                     (const unsigned char*)scales, N, steps, groups, (uint4*)packed,
                     reinterpret_cast<uint32_t*>((unsigned char*)packed + groups * 64 * steps * 64));
  ESP_HIP(ctx, hipGetLastError());
  return ESPARSE_OK;
}
