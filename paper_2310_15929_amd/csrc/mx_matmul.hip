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
#include <type_traits>
#include <utility>

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

template <int ACT>
constexpr int kRowBytes = ACT == ACT_FP4 ? 64 : (ACT == ACT_FP8 ? 128 : 256);  // of a token and 128 channels

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
// rows kernel (few tokens, bound by reading the weights): a workgroup of NW waves owns RT row tiles and MT token tiles over all of K; wave w takes
// the groups w, w + NW, ... of U steps straight from memory into registers, the loads of a group under way while the one before it is
// multiplied; the NW sums of an output are added in the order of the waves.  Measured, cold weights: 1 x 11008 x 4096 6.9 - 7.2 us whatever the activations
// (24 MB; an empty launch takes 2.3), 16 x 22016 x 8192 (96 MB) 17.7 us with 8-bit activations on one card (5.4 TB/s), on another
// 21.2, 20.2 with 4-bit and 24.0 with 16-bit ones.
// ------------------------------------------------------------------------------------------------
template <int ACT, int MT, int RT, int U>
struct MxGroup {
  uint4 w[U][RT];
  uint32_t s[U][(RT + 3) / 4];
  MxB<ACT> b[U][MT];
};

template <int ACT, int DT, int MT, int RT, int NW, int U>
__global__ void __launch_bounds__(NW * 64) k_mx_rows(const MxGemmArgs a) {
  __shared__ floatx4_t s_acc[NW * RT * MT * 64];
  const unsigned lane = threadIdx.x & 63u, wave = (unsigned)wave_uniform((int)(threadIdx.x >> 6)), c = lane & 15u, g = lane >> 4;
  // row groups that share scale words run on one XCD (= blockIdx % 8)
  const unsigned groups = (a.nrt + RT - 1) / RT, per = (groups + 7) / 8, grp = (blockIdx.x & 7u) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || grp >= groups) return;
  const unsigned rt0 = grp * RT;
  const long long t0 = (long long)blockIdx.y * (16 * MT);
  const unsigned char* x[MT];
  const uint32_t* xs[MT];
  bool real[MT];
#pragma unroll
  for (int j = 0; j < MT; j++) {
    const long long t = t0 + 16 * j + c;
    real[j] = t < a.M;
    const long long tok = real[j] ? t : a.M - 1;
    x[j] = a.x + tok * a.ldx + (ACT == ACT_16 ? 64u : 16u) * g;
    xs[j] = a.xs + tok;
  }
  const uint4* w = a.w + (long long)rt0 * a.nks * 64 + lane;
  const uint32_t* ws = a.ws + (long long)(rt0 >> 2) * a.nks * 64 + lane;
  const unsigned shift = 8u * (rt0 & 3u);
  floatx4_t acc[RT][MT];
#pragma unroll
  for (int i = 0; i < RT; i++)
#pragma unroll
    for (int j = 0; j < MT; j++) acc[i][j] = floatx4_t{0.f, 0.f, 0.f, 0.f};

  auto load_step = [&](MxGroup<ACT, MT, RT, U>& r, int u, unsigned ks) {
#pragma unroll
    for (int i = 0; i < RT; i++) r.w[u][i] = load_stream_16(w + ((long long)(RT <= 4 || rt0 + i < a.nrt ? i : 0) * a.nks + ks) * 64);
#pragma unroll
    for (int i = 0; i < RT; i += 4) r.s[u][i / 4] = ws[((long long)(RT <= 4 || rt0 + i < a.nrt ? i / 4 : 0) * a.nks + ks) * 64];
#pragma unroll
    for (int j = 0; j < MT; j++) {
      MxB<ACT>& b = r.b[u][j];
      if constexpr (ACT == ACT_16) {
#pragma unroll
        for (int v = 0; v < 4; v++) b.v[v] = uint4{0u, 0u, 0u, 0u};
        if (real[j]) {
#pragma unroll
          for (int v = 0; v < 4; v++)
            if (128ll * ks + 32 * g + 8 * v < a.K) b.v[v] = *reinterpret_cast<const uint4*>(x[j] + 256ull * ks + 16 * v);  // (K is a multiple of 8)
        }
      } else {
        b.v[0] = *reinterpret_cast<const uint4*>(x[j] + (unsigned long long)ks * kRowBytes<ACT>);
        if constexpr (ACT == ACT_FP8) b.v[1] = *reinterpret_cast<const uint4*>(x[j] + (unsigned long long)ks * kRowBytes<ACT> + 64);
        b.s = xs[j][(long long)ks * a.M];
      }
    }
  };
  auto multiply_step = [&](const MxGroup<ACT, MT, RT, U>& r, int u) {
    if constexpr (ACT == ACT_16) {
#pragma unroll
      for (int i = 0; i < RT; i++) {
        const float s = mx_widen_scale((r.s[u][i / 4] >> shift) >> (8 * (i % 4)));
        const uint32_t word[4] = {r.w[u][i].x, r.w[u][i].y, r.w[u][i].z, r.w[u][i].w};
#pragma unroll
        for (int v = 0; v < 4; v++) {
          const uint4 wide = mx_widen<DT>(word[v], s);
#pragma unroll
          for (int j = 0; j < MT; j++) acc[i][j] = mfma16<DT>(wide, r.b[u][j].v[v], acc[i][j]);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < MT; j++) {
        MxB<ACT> b = r.b[u][j];
        b.s >>= 8 * g;
#pragma unroll
        for (int i = 0; i < RT; i += 4) {
          const uint32_t sc = r.s[u][i / 4] >> shift;
          acc[i][j] = mx_mfma<ACT, 0>(r.w[u][i], sc, b, acc[i][j]);
          if constexpr (RT > 1) acc[i + 1][j] = mx_mfma<ACT, 1>(r.w[u][i + 1], sc, b, acc[i + 1][j]);
          if constexpr (RT > 2) {
            acc[i + 2][j] = mx_mfma<ACT, 2>(r.w[u][i + 2], sc, b, acc[i + 2][j]);
            acc[i + 3][j] = mx_mfma<ACT, 3>(r.w[u][i + 3], sc, b, acc[i + 3][j]);
          }
        }
      }
    }
  };
  const unsigned full = a.nks / U;  // whole groups
  unsigned k = wave;
  if (k < full) {
    MxGroup<ACT, MT, RT, U> cur, next;
#pragma unroll
    for (int u = 0; u < U; u++) load_step(cur, u, k * U + u);
    for (; k + NW < full; k += NW) {
#pragma unroll
      for (int u = 0; u < U; u++) load_step(next, u, (k + NW) * U + u);
#pragma unroll
      for (int u = 0; u < U; u++) multiply_step(cur, u);
      cur = next;
    }
#pragma unroll
    for (int u = 0; u < U; u++) multiply_step(cur, u);
    k += NW;
  }
  if constexpr (U > 1) {
    if (k == full) {  // the steps behind the last whole group
      MxGroup<ACT, MT, RT, U> cur;
      for (unsigned ks = full * U; ks < a.nks; ks++) {
        load_step(cur, 0, ks);
        multiply_step(cur, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RT; i++)
#pragma unroll
    for (int j = 0; j < MT; j++) s_acc[((wave * RT + i) * MT + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (unsigned o = threadIdx.x; o < RT * MT * 64; o += NW * 64) {
    floatx4_t v = s_acc[o];
#pragma unroll
    for (int n = 1; n < NW; n++) v += s_acc[n * (RT * MT * 64) + o];
    const unsigned i = o / (MT * 64), j = o / 64 % MT, l = o & 63u;
    store_4(a, t0 + 16 * j + (l & 15u), (long long)(rt0 + i) * 16 + 4 * (l >> 4), v);
  }
}

// ------------------------------------------------------------------------------------------------
// tile kernel: a workgroup of NWR x NWC waves owns RTM = NWR TR row tiles x NTT = NWC TC token tiles, a wave TR x TC of them.
// K runs in stages of 128 channels, software pipelined: weights (1 KiB a row tile), activations (16 RB bytes a token tile) and
// scales are copied from memory straight into rings of RING LDS buffers; a wave holds its A operands of the stage in registers
// and reads those of the next during it, B operands stream from LDS one token tile ahead.
//   stage k:  copies of B(k+RING-1) and its scales into the buffers of stage k-1 and of A(k+RING) into that of A(k) (in registers by then);
//             all token tiles but the last; counted wait (only the newest RING - 2 stages' copies may be under way) and barrier; then the first
//             B operand and the A scales of stage k+1 are read while the last token tile is multiplied.
// Activations stay in rows: a stage's RB bytes of a token are consecutive in memory (64, 128 or 256) and in LDS, where the
// 16-byte pieces of a token are exchanged by an exclusive or with its number, so that the 16 tokens of an operand read hit all banks.
// 16-bit activations: a unit of weights is expanded to 16 bits once per wave and stage, one stage ahead, between the multiplies.
// Bound by the matrix pipe and its power at prompts: 2048 x 13824 x 5120 takes 104 - 108 us with 8-bit activations (2.7 - 2.8 PFLOP/s; the instruction alone,
// in registers on random data, 4.3), 79 with 4-bit (3.7; alone 7.3), 218 with 16-bit ones (1.33; alone 1.75); 2048 x 22016 x 8192 252 - 270, 175 - 190 and 520 - 530 us
// and on zeros, which draw less power, 216, 155 and 411.  8192 x 8192 x 8192: 3.1, 4.5 and 1.44 PFLOP/s, on zeros 4.0, 6.0 and 1.8.  So what the stage does beside
// the multiplies hardly counts: rings of 4 (4 bits: 181 - 183 us), wave tiles of 4 x 8 (187 - 190) and 8 x 8 (245 and more: registers spilled), two stages
// between two barriers (no less) are not kept.
// nsplit > 1: K is cut, a workgroup stores an fp32 partial tile, k_mx_reduce adds them in ascending order.
// KG = 2: two groups of NWR x NWC waves, each with rings of its own, take half of the stages each; at the end each group hands half of its sums to the other.
//   A compute unit keeps a bounded number of lines on their way, whatever the depth of the rings (fp8, 128 x 64 tiles: 0.28 us a stage with 4 as with 6 buffers
//   and with two groups; 0.2 with weights in the last cache), so for tens to hundreds of tokens it is smaller tiles - more compute units at work - that pay
//   (fp8, 256 x 4096 x 4096: 12.2 us with 128 x 64, 9.8 with 64 x 64, 13.9 with 32 x 64).  In 16 bits expanding the weights stands between the multiplies: a
//   second group does it meanwhile (256 x 4096 x 4096, 64 x 64: 14.9 us with one group and 6 buffers, 13.5 with two groups of 3).
// ------------------------------------------------------------------------------------------------
template <int ACT, int TR, int TC, int NWR, int NWC, int RING, int KG>
struct MxTile {
  static constexpr int NW = NWR * NWC, RTM = NWR * TR, NTT = NWC * TC, RB = kRowBytes<ACT>;
  static constexpr int AU = RTM * 64, BU = NTT * RB;                            // 16-byte units of a stage
  static constexpr bool ALIGNED = TR % 4 == 0;                                  // a wave's rows start with a scale word
  static constexpr int SW_TR = (TR + 3) / 4;                                    // scale words of a wave
  static constexpr int SA = (RTM + (RTM % 4 == 0 ? 0 : (RTM % 2 == 0 ? 2 : 3)) + 3) / 4, SB = ACT == ACT_16 ? 0 : NTT / 4;          // runs of 64 scale words
  static constexpr int AC = (RTM + NW - 1) / NW, BC = (BU / 64 + NW - 1) / NW, SC = (SA + SB + NW - 1) / NW;  // copies of a wave
  static constexpr int OPS = AC + BC + SC, SW = (SA + SB) * 64;
  static constexpr int LDS = KG * RING * ((AU + BU) * 16 + SW * 4);
  static_assert(LDS <= 160 * 1024, "the rings fit the LDS");
  static constexpr int WAVES = KG * NW >= 8 || 2 * LDS <= 160 * 1024 ? 2 : 1;        // of a SIMD: what the registers are shared among
  static constexpr int BV = ACT == ACT_FP4 ? 1 : (ACT == ACT_FP8 ? 2 : 4);      // B reads of a token tile
  static constexpr int AV = ACT == ACT_16 ? 4 : 1;                              // A operands of a row tile
  static_assert(NTT % 4 == 0, "a run of scale words holds four token tiles");
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

template <int ACT, int DT, int TR, int TC, int NWR, int NWC, int RING, int KG>
struct MxTileWave {
  using T = MxTile<ACT, TR, TC, NWR, NWC, RING, KG>;
  floatx4_t acc[TR][TC];
  MxSource a_src, x_src, s_src[T::SC];
  unsigned a_off[T::AC], s_step[T::SC];           // uniform
  unsigned x_off[T::BC], s_off[T::SC], lane16;    // of the lane
  unsigned lane, wave, wr, wc, b_off, shift, s_word, s_shift;
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
  // byte i of the words: the scale of the wave's row tile i
  __device__ __forceinline__ void read_scales(const uint32_t* ss, uint32_t (&as)[T::SW_TR]) {
    if constexpr (T::ALIGNED) {
#pragma unroll
      for (int i = 0; i < T::SW_TR; i++) as[i] = ss[(s_word + i) * 64 + lane];
    } else {
      uint32_t w[T::SW_TR + 1];
#pragma unroll
      for (int i = 0; i <= T::SW_TR; i++) w[i] = ss[(s_word + i < (unsigned)T::SA ? s_word + i : T::SA - 1) * 64 + lane];
#pragma unroll
      for (int i = 0; i < T::SW_TR; i++) as[i] = (uint32_t)(((unsigned long long)w[i + 1] << 32 | w[i]) >> s_shift);
    }
  }
  __device__ __forceinline__ void read_a(const uint4* sa, const uint32_t (&as)[MxTile<ACT, TR, TC, NWR, NWC, RING, KG>::SW_TR], MxA<ACT, TR>& r) {
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
  __device__ __forceinline__ void multiply(const MxA<ACT, TR>& r, const uint32_t (&as)[MxTile<ACT, TR, TC, NWR, NWC, RING, KG>::SW_TR], const MxB<ACT>& b, int j) {
    if constexpr (ACT == ACT_16) {
#pragma unroll
      for (int v = 0; v < 4; v++)
#pragma unroll
        for (int i = 0; i < TR; i++) acc[i][j] = mfma16<DT>(r.a[i][v], b.v[v], acc[i][j]);
    } else {
#pragma unroll
      for (int i = 0; i < TR; i++) {
        if (i % 4 == 0) acc[i][j] = mx_mfma<ACT, 0>(r.a[i][0], as[i / 4], b, acc[i][j]);
        if (i % 4 == 1) acc[i][j] = mx_mfma<ACT, 1>(r.a[i][0], as[i / 4], b, acc[i][j]);
        if (i % 4 == 2) acc[i][j] = mx_mfma<ACT, 2>(r.a[i][0], as[i / 4], b, acc[i][j]);
        if (i % 4 == 3) acc[i][j] = mx_mfma<ACT, 3>(r.a[i][0], as[i / 4], b, acc[i][j]);
      }
    }
  }
};

__device__ __forceinline__ unsigned uniform(unsigned v) { return (unsigned)wave_uniform((int)v); }
// LDS that the lanes of one wave exchange: the hardware keeps its order, the fences keep the compiler's, and the barrier (no instruction) keeps all lanes
// together: with fences alone the lanes that skip the conditional stores between two passes were sent ahead to write the next one
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int N, class F, int... I>
__device__ __forceinline__ void each_stage_of(F& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each_stage(F& f) {
  each_stage_of<N>(f, std::make_integer_sequence<int, N>{});
}

// this wave's LDS reads are back; then the other waves
__device__ __forceinline__ void mx_meet() {
  sched_fence();
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt = 0 alone
  __builtin_amdgcn_s_barrier();
#endif
  sched_fence();
}
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
template <int ACT, int DT, int TR, int TC, int NWR, int NWC, int RING, int KG>
__device__ __forceinline__ void mx_stage(MxTileWave<ACT, DT, TR, TC, NWR, NWC, RING, KG>& st, const MxA<ACT, TR>& cur, MxA<ACT, TR>& nxt, uint32_t (&as)[MxTile<ACT, TR, TC, NWR, NWC, RING, KG>::SW_TR], MxB<ACT>& bq,
                                         const uint4* b_cur, const uint32_t* s_cur, const uint4* a_nxt, const uint4* b_nxt, const uint32_t* s_nxt, const uint32_t* s_nxt2,
                                         uint4* a_pre, uint4* b_pre, uint32_t* s_pre, unsigned k) {
  using T = MxTile<ACT, TR, TC, NWR, NWC, RING, KG>;
  constexpr int TH = TC > 1 ? TC - 1 : 1;  // token tiles ahead of the barrier
  constexpr int MM = TR * T::AV;           // multiplies of a token tile
  constexpr int READS = T::BV + (ACT == ACT_16 ? 0 : 1) + (TR + TH - 1) / TH;
  // B RING - 1 stages ahead, A (in registers a stage early) RING
  const unsigned last = st.k1 - 1, kb = k + RING - 1 < st.k1 ? k + RING - 1 : last, ka = k + RING < st.k1 ? k + RING : last;
  st.copy_b(b_pre, kb);
  st.copy_s(s_pre, ACT == ACT_16 ? ka : kb);
  st.copy_a(a_pre, ka);
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
  mx_arrive<(RING - 2) * T::OPS>();
  MxB<ACT> b;
  uint32_t an[T::SW_TR];
  st.read_b(b_nxt, s_nxt, 0, b);
  st.read_scales(ACT == ACT_16 ? s_nxt2 : s_nxt, an);
  st.multiply(cur, as, bq, TC - 1);
  bq = b;
#pragma unroll
  for (int i = 0; i < T::SW_TR; i++) as[i] = an[i];
  sched_group<0x100, T::BV + 1 + T::SW_TR + (T::ALIGNED ? 0 : 1)>();
  sched_group<0x008, MM>();
  sched_fence();
}

// the I-th of the buffers of a ring
template <int I, class P>
__device__ __forceinline__ P ring_at(P b0, P b1, P b2, P b3, P b4, P b5) {
  return I == 0 ? b0 : (I == 1 ? b1 : (I == 2 ? b2 : (I == 3 ? b3 : (I == 4 ? b4 : b5))));
}

template <int ACT, int DT, int TR, int TC, int NWR, int NWC, int RING, int KG>
__device__ __attribute__((always_inline)) void mx_tile_pipeline(uint4* __restrict__ a0, uint4* __restrict__ a1, uint4* __restrict__ a2, uint4* __restrict__ a3,
                                                                uint4* __restrict__ a4, uint4* __restrict__ a5, uint4* __restrict__ b0, uint4* __restrict__ b1,
                                                                uint4* __restrict__ b2, uint4* __restrict__ b3, uint4* __restrict__ b4, uint4* __restrict__ b5,
                                                                uint32_t* __restrict__ s0, uint32_t* __restrict__ s1, uint32_t* __restrict__ s2,
                                                                uint32_t* __restrict__ s3, uint32_t* __restrict__ s4, uint32_t* __restrict__ s5,
                                                                const MxGemmArgs& a, const MxTilePlan& p) {
  using T = MxTile<ACT, TR, TC, NWR, NWC, RING, KG>;
  MxTileWave<ACT, DT, TR, TC, NWR, NWC, RING, KG> st;
  const unsigned tid = threadIdx.x;
  st.lane = tid & 63u;
  st.wave = (unsigned)wave_uniform((int)(tid >> 6));
  const unsigned group = KG > 1 ? st.wave / T::NW : 0;  // of waves: its own rings, its own half of the stages
  st.wave -= group * T::NW;
  st.wr = st.wave / NWC;
  st.wc = st.wave % NWC;
  // XCD x (= blockIdx % 8) works through the items [x per, (x + 1) per): neighbouring macro tiles share operands in its L2
  const unsigned items = p.nrb * p.ntb * p.nsplit, per = (items + 7) / 8, item = (blockIdx.x & 7u) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || item >= items) return;
  const unsigned tile = uniform(item / p.nsplit), split = item - tile * p.nsplit;
  st.k0 = split * p.per_split;
  st.k1 = st.k0 + p.per_split < a.nks ? st.k0 + p.per_split : a.nks;
  const unsigned stages = (st.k1 - st.k0 + KG - 1) / KG;  // of the first group; the second has as many or one less
  if constexpr (KG > 1) {
    if (group == 0) st.k1 = st.k0 + stages;
    else st.k0 += stages;
  }
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
  st.s_word = (rt0 % 4 + st.wr * TR) / 4;
  st.s_shift = (rt0 % 4 + st.wr * TR) % 4 * 8;
  st.b_off = c * T::RB + (ACT == ACT_FP4 ? g ^ (c >> 2) : (ACT == ACT_FP8 ? g ^ (c >> 1) : (4u * g) ^ c)) * 16u;
#pragma unroll
  for (int i = 0; i < TR; i++)
#pragma unroll
    for (int j = 0; j < TC; j++) st.acc[i][j] = floatx4_t{0.f, 0.f, 0.f, 0.f};

#define A_AT(i) (ring_at<(i) % RING>(a0, a1, a2, a3, a4, a5) + group * T::AU)
#define B_AT(i) (ring_at<(i) % RING>(b0, b1, b2, b3, b4, b5) + group * T::BU)
#define S_AT(i) (ring_at<(i) % RING>(s0, s1, s2, s3, s4, s5) + group * T::SW)
  // what the stages ahead of the first would have copied, in their order: their waits hold from the start
  const unsigned last = st.k1 - 1, first = KG > 1 && st.k0 > last ? last : st.k0;
  if constexpr (ACT == ACT_16) st.copy_s(S_AT(0), first);
  st.copy_a(A_AT(0), first);
  auto fill = [&](auto stage) {
    constexpr int I = decltype(stage)::value;
    const unsigned kb = st.k0 + I < st.k1 ? st.k0 + I : last, ka = st.k0 + I + 1 < st.k1 ? st.k0 + I + 1 : last;
    st.copy_b(B_AT(I), kb);
    if constexpr (ACT == ACT_16) st.copy_s(S_AT(I + 1), ka);
    else st.copy_s(S_AT(I), kb);
    st.copy_a(A_AT(I + 1), ka);
  };
  each_stage<RING - 1>(fill);
  mx_arrive<(RING - 2) * T::OPS>();
  MxA<ACT, TR> r0, r1;
  uint32_t as[T::SW_TR];
  MxB<ACT> bq;
  st.read_scales(S_AT(0), as);
  st.read_a(A_AT(0), as, r0);
  if constexpr (ACT == ACT_16) st.read_scales(S_AT(1), as);
  st.read_b(B_AT(0), S_AT(0), 0, bq);
  sched_fence();
  mx_meet();  // every wave has its first A operands before the first stage's copies take their place
  // 16-bit activations: the scales of stage k are used with A(k), a stage ahead of B(k): they are copied with A, into the buffer of stage k's
  unsigned k = st.k0;
  auto stage = [&](auto index) {
    constexpr int I = decltype(index)::value;
    mx_stage<ACT, DT, TR, TC, NWR, NWC, RING, KG>(st, I % 2 ? r1 : r0, I % 2 ? r0 : r1, as, bq, B_AT(I), S_AT(I), A_AT(I + 1), B_AT(I + 1), S_AT(I + 1), S_AT(I + 2), A_AT(I),
                                              B_AT(I + RING - 1), ACT == ACT_16 ? S_AT(I) : S_AT(I + RING - 1), k + I);
  };
  for (; k + RING <= st.k1; k += RING) {
    each_stage<RING>(stage);
    if constexpr (RING % 2) r0 = r1;
  }
  auto rest = [&](auto index) {
    if (k + decltype(index)::value < st.k1) stage(index);
  };
  each_stage<RING - 1>(rest);
  if (KG > 1 && st.k1 - st.k0 < stages) mx_meet();  // the barrier of the first group's last stage
#undef A_AT
#undef B_AT
#undef S_AT
  mx_arrive<0>();  // nothing is on its way into the rings
  __syncthreads();  // and every wave is done with them

  constexpr int TJ = TC / KG;  // token tiles of a wave from here on
  if constexpr (KG > 1) {
    // the groups' sums: each hands half of its token tiles to the other, through its larger buffers, and adds what it gets to the rest
    constexpr bool IN_B = T::BU > T::AU;
    constexpr unsigned UNITS = IN_B ? T::BU : T::AU;
    static_assert(KG == 2 && TC % 2 == 0 && T::NW * TR * TJ <= RING * (int)UNITS / 64, "the rings hold half the sums");
    auto chunk = [&](unsigned of, int q) {
      const unsigned ch = st.wave * (TR * TJ) + q, buf = ch / (UNITS / 64);
      uint4* ring = IN_B ? (buf == 0 ? b0 : (buf == 1 ? b1 : (buf == 2 ? b2 : (buf == 3 ? b3 : (buf == 4 ? b4 : b5)))))
                         : (buf == 0 ? a0 : (buf == 1 ? a1 : (buf == 2 ? a2 : (buf == 3 ? a3 : (buf == 4 ? a4 : a5)))));
      return reinterpret_cast<floatx4_t*>(ring + of * UNITS + ch % (UNITS / 64) * 64 + st.lane);
    };
#pragma unroll
    for (int i = 0; i < TR; i++)
#pragma unroll
      for (int j = 0; j < TJ; j++) *chunk(group, i * TJ + j) = group ? st.acc[i][j] : st.acc[i][j + TJ];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TR; i++)
#pragma unroll
      for (int j = 0; j < TJ; j++) st.acc[i][j] = (group ? st.acc[i][j + TJ] : st.acc[i][j]) + *chunk(group ^ 1u, i * TJ + j);
    __syncthreads();
  }
  const long long t_wave = t0 + (long long)(st.wc * TC + group * TJ) * 16, n_wave = ((long long)rt0 + st.wr * TR) * 16;
  if (p.nsplit > 1) {
    // partial tile: [split][token][Np rows]
    const long long Np = (long long)a.nrt * 16;
#pragma unroll
    for (int j = 0; j < TJ; j++) {
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
  constexpr int HT = (TR + 1) / 2;  // row tiles of a half
  constexpr unsigned ROW = HT * 64 + 16, SLICE = 16 * ROW;  // 16 tokens; the padding puts them into different banks
  constexpr unsigned PER_A = T::AU * 16 / SLICE, PER_B = T::BU * 16 / SLICE;  // of a buffer
  constexpr unsigned BUFS = RING < 3 ? RING : 3;
  static_assert(BUFS * (PER_A + PER_B) >= T::NW, "the rings hold a slice for every wave");
  unsigned char* slice;
  if (st.wave < BUFS * PER_A) {
    const unsigned buf = st.wave / (PER_A ? PER_A : 1);
    slice = reinterpret_cast<unsigned char*>((buf == 0 ? a0 : (buf == 1 ? a1 : a2)) + group * T::AU) + st.wave % (PER_A ? PER_A : 1) * SLICE;
  } else {
    const unsigned w = st.wave - BUFS * PER_A, buf = w / (PER_B ? PER_B : 1);
    slice = reinterpret_cast<unsigned char*>((buf == 0 ? b0 : (buf == 1 ? b1 : b2)) + group * T::BU) + w % (PER_B ? PER_B : 1) * SLICE;
  }
#pragma unroll
  for (int j = 0; j < TJ; j++) {
    if (a.out == ESPARSE_F32) {
#pragma unroll
      for (int h = 0; h < 2; h++) {
#pragma unroll
        for (int i = 0; i < HT; i++)
          if (h * HT + i < TR) *reinterpret_cast<floatx4_t*>(slice + c * ROW + (16 * i + 4 * g) * 4) = st.acc[h * HT + i < TR ? h * HT + i : 0][j];
        wave_fence();
#pragma unroll
        for (int q = 0; q < HT; q++) {
          const unsigned u = q * 64 + st.lane, tl = u / (4 * HT), piece = u % (4 * HT);
          const floatx4_t v = *reinterpret_cast<const floatx4_t*>(slice + tl * ROW + piece * 16);
          const long long t = t_wave + 16 * j + tl, n = n_wave + h * (16 * HT) + 4 * piece;
          float* y = reinterpret_cast<float*>(a.y) + t * a.N + n;
          if (t < a.M && (TR % 2 == 0 || h == 0 || piece < 4 * (TR - HT))) {
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
      for (int q = 0; q < HT; q++) {
        const unsigned u = q * 64 + st.lane, tl = u / (2 * TR), piece = u % (2 * TR);
        if (TR % 2 && tl >= 16) break;
        const uint4 v = *reinterpret_cast<const uint4*>(slice + tl * ROW + piece * 16);
        const long long t = t_wave + 16 * j + tl, n = n_wave + 8 * piece;
        uint16_t* y = reinterpret_cast<uint16_t*>(a.y) + t * a.N + n;
        if (t < a.M) {
          if (n + 8 <= a.N) {
            store_stream_16(y, &v);
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

template <int ACT, int DT, int TR, int TC, int NWR, int NWC, int RING, int KG>
__global__ void __launch_bounds__(NWR * NWC * KG * 64, (MxTile<ACT, TR, TC, NWR, NWC, RING, KG>::WAVES)) k_mx_tile(const MxGemmArgs a, const MxTilePlan p) {
  using T = MxTile<ACT, TR, TC, NWR, NWC, RING, KG>;
  // separate arrays handed on as __restrict__ pointers: the compiler sees that reading one buffer does not have to wait for the copies into another
#define RING_OF(type, b, size) __shared__ type b##0[size], b##1[size], b##2[RING > 2 ? size : 1], b##3[RING > 3 ? size : 1], b##4[RING > 4 ? size : 1], b##5[RING > 5 ? size : 1]
  RING_OF(uint4, a, KG * T::AU);
  RING_OF(uint4, b, KG * T::BU);
  RING_OF(uint32_t, s, KG * T::SW);
#undef RING_OF
  mx_tile_pipeline<ACT, DT, TR, TC, NWR, NWC, RING, KG>(a0, a1, a2, a3, a4, a5, b0, b1, b2, b3, b4, b5, s0, s1, s2, s3, s4, s5, a, p);
}

// the partial tiles of a product that K was cut for, four features a thread
constexpr unsigned MOST_PIECES = 8;
__global__ void __launch_bounds__(256) k_mx_reduce(const MxGemmArgs a, const float* __restrict__ partial, unsigned nsplit) {
  // (at most 2^24 units: MOST_PARTIAL_BYTES)
  const unsigned u = blockIdx.x * 256u + threadIdx.x, row = u / (a.nrt * 4u);
  const long long Np = (long long)a.nrt * 16, t = row, n = (u - row * (a.nrt * 4u)) * 4u;
  if (t >= a.M || n >= a.N) return;
  floatx4_t v[MOST_PIECES];
#pragma unroll
  for (unsigned s = 0; s < MOST_PIECES; s++)  // all of them under way at once (pieces behind the last repeat it)
    v[s] = *reinterpret_cast<const floatx4_t*>(partial + ((long long)(s < nsplit ? s : nsplit - 1) * a.M + t) * Np + n);
#pragma unroll
  for (unsigned s = 1; s < MOST_PIECES; s++)
    if (s < nsplit) v[0] += v[s];
  store_4(a, t, n, v[0]);
}

// rows of 16-bit activations that the kernels cannot read as they are, into rows of 128 nks values, zero padded
__global__ void __launch_bounds__(256) k_mx_pad_rows(const uint16_t* __restrict__ x, long long ldx, long long M, long long K, unsigned chunks, uint4* __restrict__ out) {
  const unsigned u = blockIdx.x * 256u + threadIdx.x, row = u / chunks;  // (fewer than 2^32 units: at most 2^34 values, rows padded by 15 units at most)
  const long long t = row, at = (u - row * chunks) * 8u;
  if (t >= M) return;
  uint32_t v[4];
  load_8(x + t * ldx + at, K - at, v);
  out[u] = uint4{v[0], v[1], v[2], v[3]};
}

template <int ACT, int DT, int MT, int RT, int NW, int U>
hipError_t launch_rows(const MxGemmArgs& a, hipStream_t st) {
  const dim3 grid(((a.nrt + RT - 1) / RT + 7) / 8 * 8, (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
  hipLaunchKernelGGL((k_mx_rows<ACT, DT, MT, RT, NW, U>), grid, dim3(NW * 64), 0, st, a);
  return hipGetLastError();
}

template <int ACT, int DT, int TR, int TC, int NWR, int NWC, int RING, int KG>
hipError_t launch_tile(const MxGemmArgs& a, float* partial, unsigned nsplit, hipStream_t st) {
  using T = MxTile<ACT, TR, TC, NWR, NWC, RING, KG>;
  MxTilePlan p = {};
  p.partial = partial;
  p.nrb = (a.nrt + T::RTM - 1) / T::RTM;
  p.ntb = (unsigned)((a.M + T::NTT * 16 - 1) / (T::NTT * 16));
  p.per_split = (a.nks + nsplit - 1) / nsplit;
  p.nsplit = (a.nks + p.per_split - 1) / p.per_split;
  p.band = p.ntb > 8 ? 8 : 1;
  const unsigned items = p.nrb * p.ntb * p.nsplit;
  hipLaunchKernelGGL((k_mx_tile<ACT, DT, TR, TC, NWR, NWC, RING, KG>), dim3((items + 7) / 8 * 8), dim3(NWR * NWC * KG * 64), 0, st, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  const long long units = a.M * ((long long)a.nrt * 4);
  hipLaunchKernelGGL(k_mx_reduce, dim3((unsigned)((units + 255) / 256)), dim3(256), 0, st, a, partial, p.nsplit);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// The choice of a kernel: the smallest estimate of its time in microseconds, a function of the sizes and of the kind of the activations alone.
//   rows   t0 + steps (c L + b x) (1 - d + d q)                     L, x: workgroups per compute unit, whole and as they are; q: filled part of the token tiles
//   tile   t0 + e L + c stages max(1, u L) + (K cut: r0 + r MB of partial tiles)      L: workgroups per compute unit (256 of them)
// The constants are a least-squares fit of the logarithm of estimate / time, kernels near the fastest weighted most, to the times of 20 kernels of each kind on 13 weight
// shapes (512 x 512 to 36864 x 9216, ragged ones among them) and 1 to 2048 tokens, weights cold, K cut up to eight times.  Over those 234 products of each kind the kernel so
// chosen takes 1.007 (8 bits), 1.011 (4 bits) and 1.005 (16 bits) of the fastest one's time on average, 1.22 at most (8.1 us against 6.6); without any one of the 15 kernels
// the average would be worse.  (profiles/mx_kernel_choice.py makes these figures from the tables below and profiles/mx_kernel_choice_times.csv)
// ------------------------------------------------------------------------------------------------
// rows: token tiles, row tiles, waves, steps at a time; t0, c, b, d
#define MX_ROWS_FP8(X) \
  X(1, 1, 8, 2, 2.4, 0.0662, 0.0161, 0.378) \
  X(1, 2, 8, 2, 2.41, 0.0777, 0.0334, 0.243) \
  X(1, 8, 8, 1, 2.48, 0.181, 0.152, 0.0962) \
  X(2, 2, 8, 2, 2.41, 0.147, 0.0175, 0.495) \
  X(2, 4, 8, 1, 2.71, 0.155, 0.0691, 0.403) \
  X(4, 1, 8, 1, 2.44, 0.233, 0.00552, 0.495) \
  X(1, 4, 8, 2, 2.39, 0.108, 0.0843, 0.178) \
  X(1, 1, 16, 1, 2.55, 0.0609, 0.0206, 0.411)
#define MX_ROWS_FP4(X) \
  X(1, 1, 8, 2, 2.44, 0.0434, 0.0199, 0.296) \
  X(1, 2, 8, 2, 2.4, 0.0573, 0.0456, 0.161) \
  X(1, 8, 8, 1, 2.4, 0.163, 0.159, 0.0476) \
  X(2, 1, 16, 1, 2.49, 0.0717, 0.0241, 0.509) \
  X(2, 2, 8, 2, 2.4, 0.104, 0.0319, 0.509) \
  X(2, 4, 8, 1, 2.51, 0.123, 0.0803, 0.279) \
  X(4, 1, 8, 1, 2.41, 0.127, 0.0242, 0.511) \
  X(1, 4, 8, 2, 2.36, 0.0917, 0.0959, 0.131) \
  X(1, 1, 16, 2, 2.63, 0.0381, 0.0268, 0.335)
#define MX_ROWS_16(X) \
  X(1, 1, 8, 2, 2.53, 0.13, 0.0287, 0.608) \
  X(1, 2, 8, 2, 2.52, 0.142, 0.0557, 0.499) \
  X(1, 4, 8, 1, 2.45, 0.177, 0.0917, 0.368) \
  X(1, 8, 8, 1, 2.52, 0.255, 0.136, 0.091) \
  X(2, 1, 16, 1, 2.33, 0.255, 0.0306, 0.573) \
  X(4, 1, 8, 1, 2.36, 0.469, 0.0101, 0.756)
// tile: row and token tiles of a wave, waves along both, buffers of a ring, groups of waves along K; t0, e, c, u, r0, r
#define MX_TILES_FP8(X) \
  X(4, 2, 2, 2, 3, 1, 2.69, 0.0319, 0.374, 0.675, 2.09, 0.64) \
  X(4, 4, 2, 2, 3, 1, 3.87, 0, 0.427, 0.887, 2.36, 0.47) \
  X(8, 4, 2, 2, 2, 1, 4.26, 0, 0.954, 0.695, 4.18, 0.364) \
  X(4, 2, 2, 2, 6, 1, 2.61, 0.968, 0.265, 1.04, 1.85, 0.634) \
  X(8, 4, 2, 4, 3, 1, 0, 6.88, 0.849, 1.21, 6.94, 0.27) \
  X(2, 2, 2, 2, 6, 1, 2.99, 0.28, 0.193, 0.934, 1.66, 0.72) \
  X(2, 1, 1, 4, 6, 1, 2.68, 0.424, 0.164, 0.913, 1.88, 0.654)
#define MX_TILES_FP4(X) \
  X(4, 4, 2, 2, 3, 1, 3.74, 0, 0.401, 0.793, 2.26, 0.494) \
  X(7, 4, 2, 2, 2, 1, 6.32, 0, 0.858, 0.617, 1.38, 0.403) \
  X(4, 2, 2, 2, 6, 1, 3.1, 0, 0.25, 0.934, 2.09, 0.681) \
  X(8, 4, 2, 4, 3, 1, 0, 6.2, 0.703, 1.02, 7.27, 0.265) \
  X(2, 2, 2, 2, 6, 1, 3.01, 0, 0.174, 0.942, 1.78, 0.754) \
  X(2, 1, 1, 4, 6, 1, 2.72, 0.185, 0.143, 0.895, 1.99, 0.654)
#define MX_TILES_16(X) \
  X(4, 4, 4, 2, 3, 1, 0.66, 3.72, 1.21, 1.08, 4.44, 0.407) \
  X(3, 4, 4, 2, 3, 1, 1.99, 3.32, 0.989, 1.01, 2.05, 0.43) \
  X(4, 4, 4, 1, 2, 1, 2.46, 0.0824, 1.06, 0.691, 3.25, 0.458) \
  X(4, 2, 2, 4, 3, 1, 1.99, 1.83, 0.731, 1.07, 2.88, 0.501) \
  X(2, 4, 4, 1, 3, 1, 2.99, 0.317, 0.483, 0.891, 2.15, 0.591) \
  X(2, 4, 4, 1, 3, 2, 1.06, 2.7, 0.407, 1.03, 2.61, 0.69) \
  X(2, 2, 2, 2, 3, 2, 1.52, 1.76, 0.31, 1.02, 2.46, 0.712) \
  X(1, 2, 2, 2, 3, 2, 1.34, 1.93, 0.145, 1.78, 2.36, 0.625) \
  X(2, 2, 4, 2, 3, 1, 2.14, 0.946, 0.484, 1.01, 2.54, 0.621)

struct MxChoice {
  int variant;  // rows kernels first, then tile kernels
  unsigned nsplit;
};
constexpr int COMPUTE_UNITS = 256;
constexpr long long MOST_PARTIAL_BYTES = 256ll << 20;

struct MxRows {
  int mt, rt;
  double t0, c, b, d;
};
struct MxTiles {
  int rows, tokens;
  double t0, e, c, u, r0, r;
};
#define ROWS_OF(MT, RT, NW, U, T0, C, B, D) {MT, RT, T0, C, B, D},
#define TILE_OF(TR, TC, NWR, NWC, RING, KG, T0, E, C, U, R0, R) {TR * NWR * 16, TC * NWC * 16, T0, E, C, U, R0, R},
constexpr MxRows kRowsFp8[] = {MX_ROWS_FP8(ROWS_OF)}, kRowsFp4[] = {MX_ROWS_FP4(ROWS_OF)}, kRows16[] = {MX_ROWS_16(ROWS_OF)};
constexpr MxTiles kTilesFp8[] = {MX_TILES_FP8(TILE_OF)}, kTilesFp4[] = {MX_TILES_FP4(TILE_OF)}, kTiles16[] = {MX_TILES_16(TILE_OF)};
#undef ROWS_OF
#undef TILE_OF

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

template <size_t NR, size_t NT>
MxChoice choose_from(const MxRows (&rows)[NR], const MxTiles (&tiles)[NT], long long M, long long N, long long K) {
  const long long nks = ceil_div(K, 128), nrt = ceil_div(N, 64) * 4;
  MxChoice best = {-1, 1};
  double least = 0;
  auto offer = [&](int v, unsigned ns, double t) {
    if (best.variant < 0 || t < least) {
      best = {v, ns};
      least = t;
    }
  };
  for (int v = 0; v < (int)NR; v++) {
    const MxRows& r = rows[v];
    // one workgroup along the tokens, up to twice 64 of them
    if (M <= (r.mt > 1 ? 8 * r.mt : 0) || M > (r.mt == 4 ? 128 : 16 * r.mt)) continue;
    const long long wgs = ceil_div(nrt, r.rt) * ceil_div(M, 16 * r.mt);
    const double q = (double)(M < 16 * r.mt ? M : 16 * r.mt) / (16 * r.mt);
    offer(v, 1, r.t0 + nks * (r.c * ceil_div(wgs, COMPUTE_UNITS) + r.b * wgs / COMPUTE_UNITS) * (1 - r.d + r.d * q));
  }
  if (M > 16) {
    for (int v = 0; v < (int)NT; v++) {
      const MxTiles& k = tiles[v];
      if (k.tokens > 64 && M <= k.tokens / 2) continue;
      for (unsigned ns : {1u, 2u, 3u, 4u, 6u, MOST_PIECES}) {
        if (ns > 1 && (nks < 2 * ns || ns * M * nrt * 64 > MOST_PARTIAL_BYTES)) break;
        const long long per = ceil_div(nks, ns), cut = ceil_div(nks, per), L = ceil_div(ceil_div(nrt * 16, k.rows) * ceil_div(M, k.tokens) * cut, COMPUTE_UNITS);
        offer((int)NR + v, ns, k.t0 + k.e * L + k.c * per * (k.u * L > 1 ? k.u * L : 1) + (cut > 1 ? k.r0 + cut * M * nrt * 64e-6 * k.r : 0));
      }
    }
  }
  return best;
}
MxChoice choose(long long M, long long N, long long K, int act) {
  if (act == ACT_FP8) return choose_from(kRowsFp8, kTilesFp8, M, N, K);
  if (act == ACT_FP4) return choose_from(kRowsFp4, kTilesFp4, M, N, K);
  return choose_from(kRows16, kTiles16, M, N, K);
}
size_t partial_bytes(const MxChoice& c, long long M, long long N) { return c.nsplit > 1 ? (size_t)c.nsplit * M * ceil_div(N, 64) * 64 * 4 : 0; }
bool is_tile(const MxChoice& c, int act) {
  return c.variant >= (int)(act == ACT_FP8 ? sizeof(kRowsFp8) / sizeof(MxRows) : (act == ACT_FP4 ? sizeof(kRowsFp4) / sizeof(MxRows) : sizeof(kRows16) / sizeof(MxRows)));
}
// Whether 16-bit rows are copied and padded first: the rows kernels read whole 16-byte pieces, the tile kernels whole runs of 128 channels (behind a row's
// last channel there are other values, and behind the last row none)
bool copies_rows(const MxChoice& c, long long K, int act, bool aligned) { return act == ACT_16 && (!aligned || K % (is_tile(c, act) ? 128 : 8) != 0); }
size_t padded_bytes(long long M, long long K) { return ((size_t)M * ceil_div(K, 128) * 256 + 255) / 256 * 256; }

template <int ACT, int DT>
hipError_t launch(const MxGemmArgs& a, const MxChoice& c, float* partial, hipStream_t st) {
  int i = 0;
#define ROWS_GO(MT, RT, NW, U, ...) \
  if (c.variant == i++) return launch_rows<ACT, DT, MT, RT, NW, U>(a, st);
#define TILE_GO(TR, TC, NWR, NWC, RING, KG, ...) \
  if (c.variant == i++) return launch_tile<ACT, DT, TR, TC, NWR, NWC, RING, KG>(a, partial, c.nsplit, st);
  if constexpr (ACT == ACT_FP8) {
    MX_ROWS_FP8(ROWS_GO) MX_TILES_FP8(TILE_GO)
  } else if constexpr (ACT == ACT_FP4) {
    MX_ROWS_FP4(ROWS_GO) MX_TILES_FP4(TILE_GO)
  } else {
    MX_ROWS_16(ROWS_GO) MX_TILES_16(TILE_GO)
  }
#undef ROWS_GO
#undef TILE_GO
  return hipErrorInvalidValue;
}

}  // namespace

size_t esp_mx_gemm_workspace_bytes(long long M, long long N, long long K, int act, bool aligned) {
  const MxChoice c = choose(M, N, K, act);
  return (copies_rows(c, K, act, aligned) ? padded_bytes(M, K) : 0) + partial_bytes(c, M, N);
}

int esp_mx_gemm_device(esparse_ctx* ctx, const void* X, const void* xs, long long M, long long ldx, int act, int dtype, const void* packed, long long N,
                       long long K, int out, void* Y, void* workspace, bool aligned) {
  MxGemmArgs a = {};
  a.nks = (unsigned)ceil_div(K, 128);
  const long long groups = ceil_div(N, 64);
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
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  const MxChoice c = choose(M, N, K, act);
  if (copies_rows(c, K, act, aligned)) {
    const unsigned chunks = a.nks * 16;
    hipLaunchKernelGGL(k_mx_pad_rows, dim3((unsigned)((M * chunks + 255) / 256)), dim3(256), 0, ctx->stream, (const uint16_t*)X, ldx, M, K, chunks, (uint4*)ws);
    ESP_HIP(ctx, hipGetLastError());
    a.x = ws;
    a.ldx = 256ll * a.nks;
    a.K = 128ll * a.nks;
    ws += padded_bytes(M, K);
  }
  float* partial = reinterpret_cast<float*>(ws);
  if (act == ACT_FP4) ESP_HIP(ctx, (launch<ACT_FP4, ESPARSE_F16>(a, c, partial, ctx->stream)));
  else if (act == ACT_FP8) ESP_HIP(ctx, (launch<ACT_FP8, ESPARSE_F16>(a, c, partial, ctx->stream)));
  else if (dtype == ESPARSE_F16) ESP_HIP(ctx, (launch<ACT_16, ESPARSE_F16>(a, c, partial, ctx->stream)));
  else ESP_HIP(ctx, (launch<ACT_16, ESPARSE_BF16>(a, c, partial, ctx->stream)));
  return ESPARSE_OK;
}
