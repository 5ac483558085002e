// Products Y[M,N] = X[M,K] . W[N,K]^T with weights in microscaled 4 bits (csrc/mx.h) and activations in 16 bits or microscaled
// 8 or 4 bits, on gfx950.
//
// Operand layouts of the matrix instructions (wave of 64 lanes, lane l, c = l % 16, g = l / 16), measured with one-hot operands:
//   v_mfma_scale_f32_16x16x128_f8f6f4  A (row c) and B (column c):  4 bits: k = 32 g + e, the 16 bytes of a lane in order
//                                        8 bits: e < 16: k = 16 g + e;  e >= 16: k = 64 + 16 g + (e - 16)
//                                      scales: the byte of lane l that op_sel names belongs to row / column c, k = 32 g .. 32 g + 31
//                                      sums: 4 x 4 bits exact up to the fp32 sum; with 8-bit B the products of k = 8 i .. 8 i + 7 are cut to multiples of
//                                        2^(p - 13), p the exponent of the largest of them, before they are added (measured).  Kept: it is far below the
//                                        rounding of the operands (2^-4), and the 16-bit instruction, which would not, has under half the rate
//   v_mfma_f32_16x16x32_{f16,bf16}     A (row c), B (column c): k = 8 g + e
//   both                               D: column c, rows 4 g + j (j = 0..3)
// W is the A operand (rows of D = output features), tokens are the columns of D.  A NaN scale (255) makes its products NaN.
//
// Memory formats (include/esparse.h)
//   weights: 16-byte unit (rt * nks + ks) * 64 + l = row 16 rt + c, channels 128 ks + 32 g .. + 31: lane l's A operand of the scaled
//     instruction.  For 16-bit activations the unit is turned into four A operands of the 16-bit instruction, the j-th from its j-th
//     32-bit word (channels 128 ks + 32 g + 8 j .. + 7, scale included by the conversion); lane l's B operand is then the 16 bytes of
//     token c at those same channels.  Which k of the instruction a channel takes does not matter as long as both operands agree.
//   scales: 32-bit word (grp * nks + ks) * 64 + l = the scales of rows 64 grp + 16 b + c, channels 128 ks + 32 g .. + 31, b = byte 0..3.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "intrinsics.h"
#include "mx.h"

namespace {

typedef int esp_int8v __attribute__((ext_vector_type(8)));

constexpr int ACT_FP4 = ESPARSE_MX_FP4, ACT_FP8 = ESPARSE_MX_FP8, ACT_16 = 2;

struct MxGemmArgs {
  const unsigned char* x;    // rows of codes or of 16-bit values
  const uint32_t* xs;        // scale words [nks][M] (microscaled activations)
  const uint4* w;
  const uint32_t* ws;
  void* y;
  long long ldx;             // bytes from row to row of x
  long long M, N, K;
  unsigned nks;              // steps of 128 channels
  unsigned nrt;              // row tiles of 16 (a multiple of 4)
  int out;                   // type of y
};

// B operand of one token tile and 128 channels: 16 bytes (4 bits), 32 (8 bits), 4 x 16 (16 bits, one for each j)
template <int ACT>
struct MxB {
  uint4 v[ACT == ACT_FP4 ? 1 : (ACT == ACT_FP8 ? 2 : 4)];
  uint32_t s;  // the scale, in the lowest byte
};

template <int ACT, int B>
__device__ __forceinline__ floatx4_t mx_mfma(uint4 a, uint32_t as, const MxB<ACT>& b, floatx4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
  const esp_int8v av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  if constexpr (ACT == ACT_FP8) {
    const esp_int8v bv = {(int)b.v[0].x, (int)b.v[0].y, (int)b.v[0].z, (int)b.v[0].w, (int)b.v[1].x, (int)b.v[1].y, (int)b.v[1].z, (int)b.v[1].w};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4, 0, B, (int)as, 0, (int)b.s);
  } else {
    const esp_int8v bv = {(int)b.v[0].x, (int)b.v[0].y, (int)b.v[0].z, (int)b.v[0].w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4, 4, B, (int)as, 0, (int)b.s);
  }
#else
  (void)a;
  (void)as;
  (void)b;
  return c;
#endif
}

// one 32-bit word of a weight unit (eight channels) as the A operand of the 16-bit instruction, times 2^(E - 127).  bf16: exact.  f16: rounded
// where the scaled number is no f16 (below 2^-24 or beyond 65504)
template <int DT>
__device__ __forceinline__ uint4 mx_widen(uint32_t w, float s) {
  uint4 r = {0u, 0u, 0u, 0u};
#if defined(__HIP_DEVICE_COMPILE__)
  if (DT == ESPARSE_F16) {
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3));
  } else {
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
  }
#endif
  return r;
}

__device__ __forceinline__ uint16_t to_16(float f, int out) { return out == ESPARSE_F16 ? esp_from_float<ESPARSE_F16>(f) : esp_from_float<ESPARSE_BF16>(f); }
// four neighbouring output features of a token
__device__ __forceinline__ void store_4(const MxGemmArgs& a, long long t, long long n, floatx4_t v) {
  if (t >= a.M || n >= a.N) return;
  if (a.out == ESPARSE_F32) {
    float* y = reinterpret_cast<float*>(a.y) + t * a.N + n;
    if ((a.N & 3) == 0) {
      *reinterpret_cast<floatx4_t*>(y) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++)
        if (n + i < a.N) y[i] = v[i];
    }
  } else {
    uint16_t* y = reinterpret_cast<uint16_t*>(a.y) + t * a.N + n;
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; i++) h[i] = to_16(v[i], a.out);
    if ((a.N & 3) == 0) {
      uint2 p;
      __builtin_memcpy(&p, h, 8);
      *reinterpret_cast<uint2*>(y) = p;
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++)
        if (n + i < a.N) y[i] = h[i];
    }
  }
}

// ------------------------------------------------------------------------------------------------
// rows kernel: a workgroup of NW waves owns RT row tiles and one token tile of 16; wave w takes the steps w, w + NW, ... of K straight
// from memory into registers; the NW sums of an output are added in the order of the waves.
// ------------------------------------------------------------------------------------------------
template <int ACT, int DT, int RT, int NW>
__global__ void __launch_bounds__(NW * 64) k_mx_rows(const MxGemmArgs a) {
  __shared__ floatx4_t s_acc[NW * RT * 64];
  const unsigned lane = threadIdx.x & 63u, wave = (unsigned)wave_uniform((int)(threadIdx.x >> 6)), c = lane & 15u, g = lane >> 4;
  const unsigned rt0 = blockIdx.x * RT;
  const long long t0 = (long long)blockIdx.y * 16;
  const bool real = t0 + c < a.M;
  const long long tok = real ? t0 + c : a.M - 1;
  const unsigned char* x = a.x + tok * a.ldx;
  const uint4* w = a.w + (long long)rt0 * a.nks * 64 + lane;
  const uint32_t* ws = a.ws + (long long)(rt0 >> 2) * a.nks * 64 + lane;
  const unsigned shift = 8u * (rt0 & 3u);
  floatx4_t acc[RT];
#pragma unroll
  for (int i = 0; i < RT; i++) acc[i] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  for (unsigned ks = wave; ks < a.nks; ks += NW) {
    uint4 wv[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) wv[i] = load_stream_16(w + ((long long)i * a.nks + ks) * 64);
    const uint32_t sc = ws[(long long)ks * 64] >> shift;
    MxB<ACT> b;
    if constexpr (ACT == ACT_16) {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const long long k = 128ll * ks + 32 * g + 8 * j;  // (K is a multiple of 8)
        b.v[j] = uint4{0u, 0u, 0u, 0u};
        if (k < a.K) b.v[j] = *reinterpret_cast<const uint4*>(x + 2 * k);
      }
#pragma unroll
      for (int i = 0; i < RT; i++) {
        const float s = mx_scale((sc >> (8 * i)) & 255u);
        acc[i] = mfma16<DT>(mx_widen<DT>(wv[i].x, s), b.v[0], acc[i]);
        acc[i] = mfma16<DT>(mx_widen<DT>(wv[i].y, s), b.v[1], acc[i]);
        acc[i] = mfma16<DT>(mx_widen<DT>(wv[i].z, s), b.v[2], acc[i]);
        acc[i] = mfma16<DT>(mx_widen<DT>(wv[i].w, s), b.v[3], acc[i]);
      }
    } else {
      if constexpr (ACT == ACT_FP4) {
        b.v[0] = *reinterpret_cast<const uint4*>(x + 64ull * ks + 16 * g);
      } else {
        b.v[0] = *reinterpret_cast<const uint4*>(x + 128ull * ks + 16 * g);
        b.v[1] = *reinterpret_cast<const uint4*>(x + 128ull * ks + 64 + 16 * g);
      }
      b.s = a.xs[(long long)ks * a.M + tok] >> (8 * g);
      acc[0] = mx_mfma<ACT, 0>(wv[0], sc, b, acc[0]);
      if constexpr (RT > 1) acc[1] = mx_mfma<ACT, 1>(wv[1], sc, b, acc[1]);
      if constexpr (RT > 2) {
        acc[2] = mx_mfma<ACT, 2>(wv[2], sc, b, acc[2]);
        acc[3] = mx_mfma<ACT, 3>(wv[3], sc, b, acc[3]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RT; i++) s_acc[(wave * RT + i) * 64 + lane] = acc[i];
  __syncthreads();
  for (unsigned o = threadIdx.x; o < RT * 64; o += NW * 64) {
    floatx4_t v = s_acc[o];
#pragma unroll
    for (int k = 1; k < NW; k++) v += s_acc[k * RT * 64 + o];
    const unsigned i = o >> 6, l = o & 63u;
    store_4(a, t0 + (l & 15u), (long long)(rt0 + i) * 16 + 4 * (l >> 4), v);
  }
}

// rows of 16-bit activations that the kernels cannot read as they are, into rows of 128 nks values, zero padded
__global__ void __launch_bounds__(256) k_mx_pad_rows(const uint16_t* __restrict__ x, long long ldx, long long M, long long K, unsigned chunks, uint4* __restrict__ out) {
  const long long u = (long long)blockIdx.x * 256 + threadIdx.x;
  if (u >= M * chunks) return;
  const long long t = u / chunks, at = (u % chunks) * 8;
  uint32_t v[4];
  load_8(x + t * ldx + at, K - at, v);
  out[u] = uint4{v[0], v[1], v[2], v[3]};
}

// 16-bit rows that are read where they are: whole 16-byte pieces of them
bool readable(const void* X, long long ldx, long long K) { return K % 8 == 0 && ldx % 8 == 0 && esp_aligned16(X); }

template <int ACT, int DT>
hipError_t launch_rows(const MxGemmArgs& a, hipStream_t st) {
  const dim3 grid(a.nrt, (unsigned)((a.M + 15) / 16));
  hipLaunchKernelGGL((k_mx_rows<ACT, DT, 1, 16>), grid, dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace

bool esp_mx_gemm_in_place(const void* X, long long ldx, long long K, int act) { return act != ACT_16 || readable(X, ldx, K); }

size_t esp_mx_gemm_workspace_bytes(long long M, long long N, long long K, int act, bool in_place) {
  (void)N;
  (void)act;
  return in_place ? 0 : (size_t)M * (size_t)((K + 127) / 128) * 256;
}

int esp_mx_gemm_device(esparse_ctx* ctx, const void* X, const void* xs, long long M, long long ldx, int act, int dtype, const void* packed, long long N,
                       long long K, int out, void* Y, void* workspace) {
  MxGemmArgs a = {};
  a.nks = (unsigned)((K + 127) / 128);
  const long long groups = (N + 63) / 64;
  a.nrt = (unsigned)(groups * 4);
  a.w = reinterpret_cast<const uint4*>(packed);
  a.ws = reinterpret_cast<const uint32_t*>(reinterpret_cast<const unsigned char*>(packed) + groups * 64 * (long long)a.nks * 64);
  a.x = reinterpret_cast<const unsigned char*>(X);
  a.xs = reinterpret_cast<const uint32_t*>(xs);
  a.y = Y;
  a.M = M;
  a.N = N;
  a.K = K;
  a.out = out;
  a.ldx = act == ACT_FP4 ? 64ll * a.nks : (act == ACT_FP8 ? 128ll * a.nks : 2 * ldx);
  if (act == ACT_16 && !readable(X, ldx, K)) {
    const unsigned chunks = a.nks * 16;
    hipLaunchKernelGGL(k_mx_pad_rows, dim3((unsigned)((M * chunks + 255) / 256)), dim3(256), 0, ctx->stream, (const uint16_t*)X, ldx, M, K, chunks, (uint4*)workspace);
    ESP_HIP(ctx, hipGetLastError());
    a.x = reinterpret_cast<const unsigned char*>(workspace);
    a.ldx = 256ll * a.nks;
    a.K = 128ll * a.nks;
  }
  if (act == ACT_FP4) ESP_HIP(ctx, (launch_rows<ACT_FP4, ESPARSE_F16>(a, ctx->stream)));
  else if (act == ACT_FP8) ESP_HIP(ctx, (launch_rows<ACT_FP8, ESPARSE_F16>(a, ctx->stream)));
  else if (dtype == ESPARSE_F16) ESP_HIP(ctx, (launch_rows<ACT_16, ESPARSE_F16>(a, ctx->stream)));
  else ESP_HIP(ctx, (launch_rows<ACT_16, ESPARSE_BF16>(a, ctx->stream)));
  return ESPARSE_OK;
}
