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
#include <cstdlib>
#include <type_traits>

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

struct MxTilePlan {
  float* partial;
  unsigned nrb, ntb, nsplit, per_split, band;  // row and token blocks, ranges of K and their stages, row blocks of a band
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

// The scale of the widening conversions, from the low byte of e: they take its exponent alone (tested for all 256), with 0 for 2^-127 and 255 for NaN
__device__ __forceinline__ float mx_widen_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

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
        const float s = mx_widen_scale(sc >> (8 * i));
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

// ------------------------------------------------------------------------------------------------
// tile kernel: a workgroup of NWR x NWC waves owns RTM = NWR TR row tiles x NTT = NWC TC token tiles, a wave TR x TC of them.
// K runs in stages of 128 channels, software pipelined: weights (1 KiB a row tile), activations (16 RB bytes a token tile) and
// scales are copied from memory straight into rings of three LDS buffers; a wave holds its A operands of the stage in registers
// and reads those of the next during it, B operands stream from LDS one token tile ahead.
//   stage k:  copies of B(k+2) and its scales into the buffers of stage k-1 and of A(k+3) into that of A(k) (in registers by then);
//             all token tiles but the last; counted wait (only this stage's copies may be under way) and barrier; then the first
//             B operand and the A scales of stage k+1 are read while the last token tile is multiplied.
// Activations stay in rows: a stage's RB bytes of a token are consecutive in memory (64, 128 or 256) and in LDS, where the
// 16-byte pieces of a token are exchanged by an exclusive or with its number, so that the 16 tokens of an operand read hit all banks.
// 16-bit activations: a unit of weights is expanded to 16 bits once per wave and stage, one stage ahead, between the multiplies.
// nsplit > 1: K is cut, a workgroup stores an fp32 partial tile, k_mx_reduce adds them in ascending order.
// ------------------------------------------------------------------------------------------------
template <int ACT>
constexpr int kRowBytes = ACT == ACT_FP4 ? 64 : (ACT == ACT_FP8 ? 128 : 256);  // of a token and stage

template <int ACT, int TR, int TC, int NWR, int NWC>
struct MxTile {
  static constexpr int NW = NWR * NWC, RTM = NWR * TR, NTT = NWC * TC, RB = kRowBytes<ACT>;
  static constexpr int AU = RTM * 64, BU = NTT * RB;                            // 16-byte units of a stage
  static constexpr int SA = RTM / 4, SB = ACT == ACT_16 ? 0 : NTT / 4;          // runs of 64 scale words
  static constexpr int AC = (RTM + NW - 1) / NW, BC = (BU / 64 + NW - 1) / NW, SC = (SA + SB + NW - 1) / NW;  // copies of a wave
  static constexpr int OPS = AC + BC + SC, SW = (SA + SB) * 64;
  static_assert(3 * ((AU + BU) * 16 + SW * 4) <= 160 * 1024, "the rings fit the LDS");
  static constexpr int BV = ACT == ACT_FP4 ? 1 : (ACT == ACT_FP8 ? 2 : 4);      // B reads of a token tile
  static constexpr int AV = ACT == ACT_16 ? 4 : 1;                              // A operands of a row tile
  static_assert(TR % 4 == 0 && NTT % 4 == 0, "scale words hold four row tiles, a run of them four token tiles");
};

template <int ACT, int TR>
struct MxA {
  uint4 a[TR][ACT == ACT_16 ? 4 : 1];
};

// Copies into LDS go through buffer descriptors: a 64-bit base and a uniform offset in scalar registers, 32 bits of each lane's own.  (A 64-bit address a
// lane and copy took 14 more vector registers and spilled.)
struct MxSource {
#if defined(__HIP_DEVICE_COMPILE__)
  __amdgpu_buffer_rsrc_t r;
#endif
};
__device__ __forceinline__ MxSource mx_source(const void* base) {
  MxSource s;
#if defined(__HIP_DEVICE_COMPILE__)
  s.r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, 0xffffffff, 0x00027000);
#endif
  return s;
}
template <int BYTES>
__device__ __forceinline__ void mx_copy(const MxSource& s, unsigned lane_off, unsigned uniform_off, void* lds_wave_base) {
#if defined(__HIP_DEVICE_COMPILE__)
  auto* to = (__attribute__((address_space(3))) void*)lds_wave_base;
  if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(s.r, to, 16, (int)lane_off, (int)uniform_off, 0, 0);
  else __builtin_amdgcn_raw_ptr_buffer_load_lds(s.r, to, 4, (int)lane_off, (int)uniform_off, 0, 0);
#else
  (void)s;
  (void)lane_off;
  (void)uniform_off;
  (void)lds_wave_base;
#endif
}

template <int ACT, int DT, int TR, int TC, int NWR, int NWC>
struct MxTileWave {
  using T = MxTile<ACT, TR, TC, NWR, NWC>;
  floatx4_t acc[TR][TC];
  MxSource a_src, x_src, s_src[T::SC];
  unsigned a_off[T::AC], s_step[T::SC];           // uniform
  unsigned x_off[T::BC], s_off[T::SC], lane16;    // of the lane
  unsigned lane, wave, wr, wc, b_off, shift;
  unsigned k0, k1;

  __device__ __forceinline__ void copy_a(uint4* sa, unsigned k) {
#pragma unroll
    for (int p = 0; p < T::AC; p++) mx_copy<16>(a_src, lane16, a_off[p] + k * 1024u, sa + ((p * T::NW + wave) % T::RTM) * 64);
  }
  __device__ __forceinline__ void copy_b(uint4* sb, unsigned k) {
#pragma unroll
    for (int p = 0; p < T::BC; p++) mx_copy<16>(x_src, x_off[p], k * (unsigned)T::RB, sb + ((p * T::NW + wave) % (T::BU / 64)) * 64);
  }
  __device__ __forceinline__ void copy_s(uint32_t* ss, unsigned k) {
#pragma unroll
    for (int p = 0; p < T::SC; p++) mx_copy<4>(s_src[p], s_off[p], k * s_step[p], ss + ((p * T::NW + wave) % (T::SA + T::SB)) * 64);
  }
  __device__ __forceinline__ void read_scales(const uint32_t* ss, uint32_t (&as)[TR / 4]) {
#pragma unroll
    for (int i = 0; i < TR / 4; i++) as[i] = ss[(wr * (TR / 4) + i) * 64 + lane];
  }
  __device__ __forceinline__ void read_a(const uint4* sa, const uint32_t (&as)[TR / 4], MxA<ACT, TR>& r) {
#pragma unroll
    for (int i = 0; i < TR; i++) {
      const uint4 u = sa[(wr * TR + i) * 64 + lane];
      if constexpr (ACT == ACT_16) {
        const float s = mx_widen_scale(as[i / 4] >> (8 * (i % 4)));
        r.a[i][0] = mx_widen<DT>(u.x, s);
        r.a[i][1] = mx_widen<DT>(u.y, s);
        r.a[i][2] = mx_widen<DT>(u.z, s);
        r.a[i][3] = mx_widen<DT>(u.w, s);
      } else {
        r.a[i][0] = u;
      }
    }
  }
  __device__ __forceinline__ void read_b(const uint4* sb, const uint32_t* ss, int j, MxB<ACT>& b) {
    const unsigned char* p = reinterpret_cast<const unsigned char*>(sb) + (wc * TC + j) * (16u * T::RB);
    b.v[0] = *reinterpret_cast<const uint4*>(p + b_off);
    if constexpr (ACT == ACT_FP8) b.v[1] = *reinterpret_cast<const uint4*>(p + (b_off ^ 64u));
    if constexpr (ACT == ACT_16) {
#pragma unroll
      for (unsigned v = 1; v < 4; v++) b.v[v] = *reinterpret_cast<const uint4*>(p + (b_off ^ (v * 16u)));
    } else {
      b.s = ss[T::SA * 64 + (wc * TC + j) * 16 + (lane & 15u)] >> shift;
    }
  }
  __device__ __forceinline__ void multiply(const MxA<ACT, TR>& r, const uint32_t (&as)[TR / 4], const MxB<ACT>& b, int j) {
    if constexpr (ACT == ACT_16) {
#pragma unroll
      for (int v = 0; v < 4; v++)
#pragma unroll
        for (int i = 0; i < TR; i++) acc[i][j] = mfma16<DT>(r.a[i][v], b.v[v], acc[i][j]);
    } else {
#pragma unroll
      for (int i = 0; i < TR; i += 4) {
        acc[i][j] = mx_mfma<ACT, 0>(r.a[i][0], as[i / 4], b, acc[i][j]);
        acc[i + 1][j] = mx_mfma<ACT, 1>(r.a[i + 1][0], as[i / 4], b, acc[i + 1][j]);
        acc[i + 2][j] = mx_mfma<ACT, 2>(r.a[i + 2][0], as[i / 4], b, acc[i + 2][j]);
        acc[i + 3][j] = mx_mfma<ACT, 3>(r.a[i + 3][0], as[i / 4], b, acc[i + 3][j]);
      }
    }
  }
};

__device__ __forceinline__ unsigned uniform(unsigned v) { return (unsigned)wave_uniform((int)v); }
// LDS that lanes of one wave exchange: in order in the hardware, kept in order by the compiler
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// all of this wave's copies but the newest N have landed, its LDS reads are back; then the other waves
template <int N>
__device__ __forceinline__ void mx_arrive() {
  sched_fence();
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);
  __builtin_amdgcn_s_barrier();
#endif
  sched_fence();
}

// cur: A(k) in registers; nxt receives A(k+1).  as: scales of stage k (16-bit activations: of k+1, which nxt is expanded with)
template <int ACT, int DT, int TR, int TC, int NWR, int NWC>
__device__ __forceinline__ void mx_stage(MxTileWave<ACT, DT, TR, TC, NWR, NWC>& st, const MxA<ACT, TR>& cur, MxA<ACT, TR>& nxt, uint32_t (&as)[TR / 4], MxB<ACT>& bq,
                                         const uint4* b_cur, const uint32_t* s_cur, const uint4* a_nxt, const uint4* b_nxt, const uint32_t* s_nxt, const uint32_t* s_nxt2,
                                         uint4* a_pre, uint4* b_pre, uint32_t* s_pre, unsigned k) {
  using T = MxTile<ACT, TR, TC, NWR, NWC>;
  constexpr int TH = TC > 1 ? TC - 1 : 1;  // token tiles ahead of the barrier
  constexpr int MM = TR * T::AV;           // multiplies of a token tile
  constexpr int READS = T::BV + (ACT == ACT_16 ? 0 : 1) + (TR + TH - 1) / TH;
  const unsigned last = st.k1 - 1;
  st.copy_b(b_pre, k + 2 < st.k1 ? k + 2 : last);
  st.copy_s(s_pre, ACT == ACT_16 ? (k + 3 < st.k1 ? k + 3 : last) : (k + 2 < st.k1 ? k + 2 : last));
  st.copy_a(a_pre, k + 3 < st.k1 ? k + 3 : last);
  st.read_a(a_nxt, as, nxt);
#pragma unroll
  for (int j = 0; j < TC - 1; j++) {
    MxB<ACT> b;
    st.read_b(b_cur, s_cur, j + 1, b);
    st.multiply(cur, as, bq, j);
    bq = b;
  }
  if constexpr (TC > 1) {
#pragma unroll
    for (int j = 0; j < TH; j++) sched_spread<MM, (T::OPS + TH - 1) / TH, READS, true>();
  }
  mx_arrive<T::OPS>();
  MxB<ACT> b;
  uint32_t an[TR / 4];
  st.read_b(b_nxt, s_nxt, 0, b);
  st.read_scales(ACT == ACT_16 ? s_nxt2 : s_nxt, an);
  st.multiply(cur, as, bq, TC - 1);
  bq = b;
#pragma unroll
  for (int i = 0; i < TR / 4; i++) as[i] = an[i];
  sched_group<0x100, T::BV + 1 + TR / 4>();
  sched_group<0x008, MM>();
  sched_fence();
}

template <int ACT, int DT, int TR, int TC, int NWR, int NWC>
__device__ __attribute__((always_inline)) void mx_tile_pipeline(uint4* __restrict__ a0, uint4* __restrict__ a1, uint4* __restrict__ a2, uint4* __restrict__ b0,
                                                                uint4* __restrict__ b1, uint4* __restrict__ b2, uint32_t* __restrict__ s0, uint32_t* __restrict__ s1,
                                                                uint32_t* __restrict__ s2, const MxGemmArgs& a, const MxTilePlan& p) {
  using T = MxTile<ACT, TR, TC, NWR, NWC>;
  MxTileWave<ACT, DT, TR, TC, NWR, NWC> st;
  const unsigned tid = threadIdx.x;
  st.lane = tid & 63u;
  st.wave = (unsigned)wave_uniform((int)(tid >> 6));
  st.wr = st.wave / NWC;
  st.wc = st.wave % NWC;
  // XCD x (= blockIdx % 8) works through the items [x per, (x + 1) per): neighbouring macro tiles share operands in its L2
  const unsigned items = p.nrb * p.ntb * p.nsplit, per = (items + 7) / 8, item = (blockIdx.x & 7u) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || item >= items) return;
  const unsigned tile = uniform(item / p.nsplit), split = item - tile * p.nsplit;
  st.k0 = split * p.per_split;
  st.k1 = st.k0 + p.per_split < a.nks ? st.k0 + p.per_split : a.nks;
  // bands of `band` row blocks, the token blocks outermost within one
  const unsigned bt = p.band * p.ntb, bi = uniform(tile / bt), in = tile - bi * bt, gh = p.nrb - bi * p.band < p.band ? p.nrb - bi * p.band : p.band;
  const unsigned tb = uniform(in / gh), rb = bi * p.band + in - tb * gh;
  const unsigned rt0 = rb * T::RTM;
  const long long t0 = (long long)tb * (T::NTT * 16);
  st.a_src = mx_source(a.w + (long long)rt0 * a.nks * 64);
#pragma unroll
  for (int c = 0; c < T::AC; c++) {
    const unsigned i = (c * T::NW + st.wave) % T::RTM;
    st.a_off[c] = (rt0 + i < a.nrt ? i : a.nrt - 1 - rt0) * a.nks * 1024u;  // past the end: duplicate work, not stored
  }
  st.x_src = mx_source(a.x + t0 * a.ldx);
  const unsigned tokens = (unsigned)(a.M - t0 < T::NTT * 16 ? a.M - t0 : T::NTT * 16);
#pragma unroll
  for (int c = 0; c < T::BC; c++) {
    constexpr unsigned U = T::RB / 16;  // pieces of a token
    const unsigned u = ((c * T::NW + st.wave) % (T::BU / 64)) * 64 + st.lane, t = u / U, slot = u % U;
    const unsigned piece = slot ^ (ACT == ACT_FP4 ? (t >> 2) & 3u : (ACT == ACT_FP8 ? (t >> 1) & 7u : t & 15u));
    st.x_off[c] = (t < tokens ? t : tokens - 1) * (unsigned)a.ldx + piece * 16u;
  }
#pragma unroll
  for (int c = 0; c < T::SC; c++) {
    const unsigned q = (c * T::NW + st.wave) % (T::SA + T::SB), t = (q - T::SA) * 64 + st.lane, grp = rt0 / 4 + q, most = a.nrt / 4 - 1;
    const bool of_weights = q < (unsigned)T::SA;
    st.s_src[c] = mx_source(of_weights ? a.ws + (long long)(grp < most ? grp : most) * a.nks * 64 : a.xs + t0);
    st.s_off[c] = of_weights ? st.lane * 4u : (t < tokens ? t : tokens - 1) * 4u;
    st.s_step[c] = of_weights ? 256u : 4u * (unsigned)a.M;
  }
  st.lane16 = st.lane * 16;
  const unsigned c = st.lane & 15u, g = st.lane >> 4;
  st.shift = 8u * g;
  st.b_off = c * T::RB + (ACT == ACT_FP4 ? g ^ (c >> 2) : (ACT == ACT_FP8 ? g ^ (c >> 1) : (4u * g) ^ c)) * 16u;
#pragma unroll
  for (int i = 0; i < TR; i++)
#pragma unroll
    for (int j = 0; j < TC; j++) st.acc[i][j] = floatx4_t{0.f, 0.f, 0.f, 0.f};

  const unsigned last = st.k1 - 1, kb = st.k0;
  auto at = [&](unsigned k) { return k < st.k1 ? k : last; };
  st.copy_b(b0, kb);
  st.copy_s(s0, kb);
  st.copy_a(a0, kb);
  st.copy_b(b1, at(kb + 1));
  st.copy_s(s1, at(kb + 1));
  st.copy_a(a1, at(kb + 1));
  if constexpr (ACT == ACT_16) st.copy_s(s2, at(kb + 2));
  st.copy_a(a2, at(kb + 2));
  mx_arrive<0>();
  MxA<ACT, TR> r0, r1;
  uint32_t as[TR / 4];
  MxB<ACT> bq;
  st.read_scales(s0, as);
  st.read_a(a0, as, r0);
  if constexpr (ACT == ACT_16) st.read_scales(s1, as);
  st.read_b(b0, s0, 0, bq);
  mx_arrive<0>();  // every wave has its first A operands before the first stage's copies take their place
  // 16-bit activations: the scales of stage k are used with A(k), a stage ahead of B(k): they are copied three stages ahead, into the buffer of A(k)'s
#define STAGE(R, N, B0, S0, A1, B1, S1, S2, AP, BP, SP, K) mx_stage<ACT, DT, TR, TC, NWR, NWC>(st, R, N, as, bq, B0, S0, A1, B1, S1, S2, AP, BP, SP, K)
  unsigned k = kb;
  for (; k + 3 <= st.k1; k += 3) {
    if constexpr (ACT == ACT_16) {
      STAGE(r0, r1, b0, s0, a1, b1, s1, s2, a0, b2, s0, k);
      STAGE(r1, r0, b1, s1, a2, b2, s2, s0, a1, b0, s1, k + 1);
      STAGE(r0, r1, b2, s2, a0, b0, s0, s1, a2, b1, s2, k + 2);
    } else {
      STAGE(r0, r1, b0, s0, a1, b1, s1, s2, a0, b2, s2, k);
      STAGE(r1, r0, b1, s1, a2, b2, s2, s0, a1, b0, s0, k + 1);
      STAGE(r0, r1, b2, s2, a0, b0, s0, s1, a2, b1, s1, k + 2);
    }
    r0 = r1;
  }
  if (k < st.k1) {
    if constexpr (ACT == ACT_16) STAGE(r0, r1, b0, s0, a1, b1, s1, s2, a0, b2, s0, k);
    else STAGE(r0, r1, b0, s0, a1, b1, s1, s2, a0, b2, s2, k);
  }
  if (k + 1 < st.k1) {
    if constexpr (ACT == ACT_16) STAGE(r1, r0, b1, s1, a2, b2, s2, s0, a1, b0, s1, k + 1);
    else STAGE(r1, r0, b1, s1, a2, b2, s2, s0, a1, b0, s0, k + 1);
  }
#undef STAGE
  mx_arrive<0>();  // nothing is on its way into the rings
  __syncthreads();  // and every wave is done with them

  const long long t_wave = t0 + (long long)st.wc * TC * 16, n_wave = ((long long)rt0 + st.wr * TR) * 16;
  if (p.nsplit > 1) {
    // partial tile: [split][token][Np rows]
    const long long Np = (long long)a.nrt * 16;
#pragma unroll
    for (int j = 0; j < TC; j++) {
      const long long t = t_wave + 16 * j + c;
#pragma unroll
      for (int i = 0; i < TR; i++) {
        const long long n = n_wave + 16 * i + 4 * g;
        if (t < a.M && n < Np) *reinterpret_cast<floatx4_t*>(p.partial + ((long long)split * a.M + t) * Np + n) = st.acc[i][j];
      }
    }
    return;
  }
  // Outputs through LDS: a wave transposes one token tile after the other (32 bits: half of it) in a slice of its own and stores 16-byte pieces of rows of Y
  constexpr unsigned ROW = TR * 32 + 16, SLICE = 16 * ROW;  // 16 tokens; the padding puts them into different banks
  constexpr unsigned PER_A = T::AU * 16 / SLICE;
  static_assert(3 * PER_A >= T::NW, "the weight buffers hold a slice for every wave");
  unsigned char* slice = reinterpret_cast<unsigned char*>(st.wave < PER_A ? a0 : (st.wave < 2 * PER_A ? a1 : a2)) + st.wave % PER_A * SLICE;
#pragma unroll
  for (int j = 0; j < TC; j++) {
    if (a.out == ESPARSE_F32) {
#pragma unroll
      for (int h = 0; h < 2; h++) {
#pragma unroll
        for (int i = 0; i < TR / 2; i++) *reinterpret_cast<floatx4_t*>(slice + c * ROW + (16 * i + 4 * g) * 4) = st.acc[h * (TR / 2) + i][j];
        wave_fence();
#pragma unroll
        for (int q = 0; q < TR / 2; q++) {
          const unsigned u = q * 64 + st.lane, tl = u / (2 * TR), piece = u % (2 * TR);
          const floatx4_t v = *reinterpret_cast<const floatx4_t*>(slice + tl * ROW + piece * 16);
          const long long t = t_wave + 16 * j + tl, n = n_wave + h * (8 * TR) + 4 * piece;
          float* y = reinterpret_cast<float*>(a.y) + t * a.N + n;
          if (t < a.M) {
            if (n + 4 <= a.N) {
              __builtin_memcpy(y, &v, 16);
            } else {
#pragma unroll
              for (int e = 0; e < 4; e++)
                if (n + e < a.N) y[e] = v[e];
            }
          }
        }
        wave_fence();
      }
    } else {
      auto put = [&](auto type) {
        constexpr int OT = decltype(type)::value;
#pragma unroll
        for (int i = 0; i < TR; i++) {
          const floatx4_t v = st.acc[i][j];
          *reinterpret_cast<uint2*>(slice + c * ROW + (16 * i + 4 * g) * 2) =
              uint2{esp_from_float<OT>(v[0]) | (uint32_t)esp_from_float<OT>(v[1]) << 16, esp_from_float<OT>(v[2]) | (uint32_t)esp_from_float<OT>(v[3]) << 16};
        }
      };
      if (a.out == ESPARSE_F16) put(std::integral_constant<int, ESPARSE_F16>{});
      else put(std::integral_constant<int, ESPARSE_BF16>{});
      wave_fence();
#pragma unroll
      for (int q = 0; q < TR / 2; q++) {
        const unsigned u = q * 64 + st.lane, tl = u / (2 * TR), piece = u % (2 * TR);
        const uint4 v = *reinterpret_cast<const uint4*>(slice + tl * ROW + piece * 16);
        const long long t = t_wave + 16 * j + tl, n = n_wave + 8 * piece;
        uint16_t* y = reinterpret_cast<uint16_t*>(a.y) + t * a.N + n;
        if (t < a.M) {
          if (n + 8 <= a.N) {
            __builtin_memcpy(y, &v, 16);
          } else {
            const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; e++)
              if (n + e < a.N) y[e] = (uint16_t)(d[e / 2] >> (16 * (e & 1)));
          }
        }
      }
      wave_fence();
    }
  }
}

template <int ACT, int DT, int TR, int TC, int NWR, int NWC>
__global__ void __launch_bounds__(NWR * NWC * 64) k_mx_tile(const MxGemmArgs a, const MxTilePlan p) {
  using T = MxTile<ACT, TR, TC, NWR, NWC>;
  // separate arrays handed on as __restrict__ pointers: the compiler sees that reading one buffer does not have to wait for the copies into another
  __shared__ uint4 a0[T::AU], a1[T::AU], a2[T::AU];
  __shared__ uint4 b0[T::BU], b1[T::BU], b2[T::BU];
  __shared__ uint32_t s0[T::SW], s1[T::SW], s2[T::SW];
  mx_tile_pipeline<ACT, DT, TR, TC, NWR, NWC>(a0, a1, a2, b0, b1, b2, s0, s1, s2, a, p);
}

// the partial tiles of a product that K was cut for, four features a thread
__global__ void __launch_bounds__(256) k_mx_reduce(const MxGemmArgs a, const float* __restrict__ partial, unsigned nsplit) {
  const long long Np = (long long)a.nrt * 16, u = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long t = u / (Np / 4), n = u % (Np / 4) * 4;
  if (t >= a.M || n >= a.N) return;
  floatx4_t v = *reinterpret_cast<const floatx4_t*>(partial + t * Np + n);
  for (unsigned s = 1; s < nsplit; s++) v += *reinterpret_cast<const floatx4_t*>(partial + ((long long)s * a.M + t) * Np + n);
  store_4(a, t, n, v);
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

template <int ACT, int DT, int TR, int TC, int NWR, int NWC>
hipError_t launch_tile(const MxGemmArgs& a, float* partial, unsigned nsplit, hipStream_t st) {
  using T = MxTile<ACT, TR, TC, NWR, NWC>;
  MxTilePlan p = {};
  p.partial = partial;
  p.nrb = (a.nrt + T::RTM - 1) / T::RTM;
  p.ntb = (unsigned)((a.M + T::NTT * 16 - 1) / (T::NTT * 16));
  p.per_split = (a.nks + nsplit - 1) / nsplit;
  p.nsplit = (a.nks + p.per_split - 1) / p.per_split;
  p.band = p.ntb > 8 ? 8 : 1;
  const unsigned items = p.nrb * p.ntb * p.nsplit;
  hipLaunchKernelGGL((k_mx_tile<ACT, DT, TR, TC, NWR, NWC>), dim3((items + 7) / 8 * 8), dim3(NWR * NWC * 64), 0, st, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  const long long units = a.M * ((long long)a.nrt * 4);
  hipLaunchKernelGGL(k_mx_reduce, dim3((unsigned)((units + 255) / 256)), dim3(256), 0, st, a, partial, p.nsplit);
  return hipGetLastError();
}

template <int ACT, int DT>
hipError_t launch(const MxGemmArgs& a, float* partial, hipStream_t st) {
  const char* e = getenv("MXV");
  const int v = e ? atoi(e) : 0;
  if (a.M <= 64 && v == 0) return launch_rows<ACT, DT>(a, st);
  if constexpr (ACT != ACT_16) {
    if (v == 1) return launch_tile<ACT, DT, 4, 2, 2, 2>(a, partial, 1, st);   // 128 x 64, 4 waves
    if (v == 2) return launch_tile<ACT, DT, 4, 4, 2, 2>(a, partial, 1, st);   // 128 x 128, 4 waves
    if (v == 3) return launch_tile<ACT, DT, 4, 4, 2, 4>(a, partial, 1, st);   // 128 x 256, 8 waves
    if (v == 4) return launch_tile<ACT, DT, 8, 2, 2, 4>(a, partial, 1, st);   // 256 x 128, 8 waves
    if (v == 5) return launch_tile<ACT, DT, 4, 2, 2, 4>(a, partial, 1, st);   // 128 x 128, 8 waves
    if (v == 6) return launch_tile<ACT, DT, 4, 8, 4, 2>(a, partial, 1, st);
    return launch_tile<ACT, DT, 8, 4, 2, 4>(a, partial, 1, st);               // 256 x 256, 8 waves
  } else {
    if (v == 1) return launch_tile<ACT, DT, 4, 2, 2, 2>(a, partial, 1, st);   // 128 x 64, 4 waves
    if (v == 2) return launch_tile<ACT, DT, 4, 4, 2, 2>(a, partial, 1, st);   // 128 x 128, 4 waves
    if (v == 5) return launch_tile<ACT, DT, 4, 2, 2, 4>(a, partial, 1, st);   // 128 x 128, 8 waves
    return launch_tile<ACT, DT, 4, 4, 4, 2>(a, partial, 1, st);               // 256 x 128, 8 waves
  }
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
  if (act == ACT_FP4) ESP_HIP(ctx, (launch<ACT_FP4, ESPARSE_F16>(a, nullptr, ctx->stream)));
  else if (act == ACT_FP8) ESP_HIP(ctx, (launch<ACT_FP8, ESPARSE_F16>(a, nullptr, ctx->stream)));
  else if (dtype == ESPARSE_F16) ESP_HIP(ctx, (launch<ACT_16, ESPARSE_F16>(a, nullptr, ctx->stream)));
  else ESP_HIP(ctx, (launch<ACT_16, ESPARSE_BF16>(a, nullptr, ctx->stream)));
  return ESPARSE_OK;
}
