// Heads between the q/k/v products and attention: each head of queries and keys normalised (if there are weights) and rotated by its token's position, queries
// written in 16 bits, keys in 16 bits and, with the values, into the pages of a cache in microscaled 4 bits (include/esparse.h).
//   y = x w / sqrt(mean(x^2) + eps);  (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position x frequency
// A row (a head of a token) belongs to DP / 8 lanes with eight channels each: the sum of squares goes over the lanes, the partners of a lane's channels are in a lane of the same row (where
// rotary / 2 is no multiple of eight they are read again).  Everything up to the rounding (for 16 bits by way of fp32, 2^-24 of a value more: a single rounding takes a few instructions more a number of a
// kernel that the vector unit bounds) is in 64 bits: the angles of far positions are lost in 32,
// and a number on the border of two 4-bit codes goes where the exact one would (sqrt and the corrected quotient are exact where the exact result is
// short enough to be such a border; what is rounded to 16 bits does without that).  The angles of a token are computed once per workgroup, whose
// rows all belong to one token, while its first row is on its way.
// Bound by the vector unit (80 % of its slots) rather than memory, with the start of a workgroup - positions, angles, factors: twice as many workgroups for the same rows take twice the time.
// Measured: 1 token of 32 + 32 + 32 heads of 128 channels 6 us, 4096 tokens of 64 + 8 + 8 heads 73 us (2.2 TB/s; 127 vector registers, 38 scalar ones spilled into lanes of those); with a division by the norm for each channel and
// its partner, without the row ahead, and with the library's sine and cosine 88; with five rows ahead (spilled registers) 93, with two 75.  k_cache_read: 4096 tokens of 8 heads of both kinds 5.6 us (4 TB/s).
#include <hip/hip_runtime.h>

#include "mx.h"

namespace {

constexpr int NT = 256;

struct RotateArgs {
  const uint16_t *q, *k, *v, *qw, *kw;
  uint16_t *q_out, *k_out;
  const int32_t* positions;
  const float* frequencies;
  const int32_t* slots;
  unsigned char *k_data, *k_scales, *v_data, *v_scales;
  long long ldq, ldk, ldv, T, tokens;  // tokens: places of the cache
  int Hq, Hkv, D, rotary, paired, page_bits;
  int rows, chunks;  // rows of a token, workgroups that share them
  double eps, per_channel;  // 1 / D
};

template <int DT>
__device__ __forceinline__ void widen_8(const uint32_t (&v)[4], double (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    y[2 * i] = esp_to_float<DT>((uint16_t)v[i]);
    y[2 * i + 1] = esp_to_float<DT>((uint16_t)(v[i] >> 16));
  }
}

// sine and cosine of f turns, |f| <= 1/2 (and a little), by their series within an eighth of a turn: the first terms left out are below 2^-54
__device__ __forceinline__ void turn_by(double f, double& s, double& c) {
  const double n = __builtin_rint(4. * f), x = (f - 0.25 * n) * 6.283185307179586, z = x * x;
  double a = -1. / 1307674368000., b = 1. / 20922789888000.;
  a = __builtin_fma(a, z, 1. / 6227020800.);
  b = __builtin_fma(b, z, -1. / 87178291200.);
  a = __builtin_fma(a, z, -1. / 39916800.);
  b = __builtin_fma(b, z, 1. / 479001600.);
  a = __builtin_fma(a, z, 1. / 362880.);
  b = __builtin_fma(b, z, -1. / 3628800.);
  a = __builtin_fma(a, z, -1. / 5040.);
  b = __builtin_fma(b, z, 1. / 40320.);
  a = __builtin_fma(a, z, 1. / 120.);
  b = __builtin_fma(b, z, -1. / 720.);
  a = __builtin_fma(a, z, -1. / 6.);
  b = __builtin_fma(b, z, 1. / 24.);
  b = __builtin_fma(b, z, -0.5);
  a = __builtin_fma(a * z, x, x);
  b = __builtin_fma(b, z, 1.);
  const int q = (int)n & 3;
  s = q & 1 ? b : a;
  c = q & 1 ? a : b;
  s = q & 2 ? -s : s;
  c = q == 1 || q == 2 ? -c : c;
}

// sum over the LN lanes of a row
template <int LN>
__device__ __forceinline__ double row_sum(double v) {
#pragma unroll
  for (int o = LN / 2; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// p / n, rounded once where n is finite (by = 1 / n, rest_n = n or 0)
__device__ __forceinline__ double over(double p, double by, double rest_n) {
  const double q = p * by;
  return __builtin_fma(__builtin_fma(-q, rest_n, p), by, q);
}

// 1 / sqrt(v), to 2^-46: the instruction's 24 bits and one step of Newton's
__device__ __forceinline__ double inverse_root(double v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const double r = __builtin_amdgcn_rsq(v);
#else
  const double r = v;
#endif
  return v == __builtin_inf() ? 0. : r * __builtin_fma(-0.5 * v * r, r, 1.5);
}

// to 24 bits with the last one odd where something was lost: rounding that to 4 bits gives what rounding v would
__device__ __forceinline__ float to_odd_24(double v) {
  unsigned long long b = __builtin_bit_cast(unsigned long long, v);
  const unsigned lost = (unsigned)b & 0x1fffffffu;
  b = (b & ~0x1fffffffull) | (lost ? 0x20000000ull : 0ull);
  return (float)__builtin_bit_cast(double, b);
}

// a row of a head in the cache: eight channels of this lane, the scales of the row's lanes.  Only lanes of the same row exchange anything: the neighbours may be of rows that are not kept, whose
// lanes are off here and give zeros.
template <int DP>
__device__ __forceinline__ void put_row(unsigned char* data, unsigned char* scales, long long row, unsigned lane, MxCodes c, unsigned e) {
  *reinterpret_cast<uint32_t*>(data + row * (DP / 2) + 4 * lane) = c.lo;
  if constexpr (DP == 64) {
    const uint32_t other = lane_move<0x141>(e);  // eight lanes in reverse: the first gets the second block's
    if (lane == 0) *reinterpret_cast<uint16_t*>(scales + row * 2) = (uint16_t)(e | other << 8);
  } else {
    const uint32_t w = mx_scale_word(e, threadIdx.x);  // four blocks of 16 lanes
    if ((lane & 15u) == 0u) *reinterpret_cast<uint32_t*>(scales + row * (DP / 32) + lane / 4) = w;
  }
}

template <int DT, int DP>
__global__ void __launch_bounds__(NT, 4) k_rotate_heads(const RotateArgs a) {
  constexpr int LN = DP / 8, ROWS = NT / LN;  // lanes of a row, rows of a pass
  __shared__ double turn[2][DP / 2];          // cos, sin
  const long long t = blockIdx.x / (unsigned)a.chunks;
  const int chunk = (int)(blockIdx.x % (unsigned)a.chunks);
  const unsigned lane = threadIdx.x % LN;
  const int c0 = (int)lane * 8, half = a.rotary / 2;
  const int first = (int)((long long)a.rows * chunk / a.chunks), end = (int)((long long)a.rows * (chunk + 1) / a.chunks);
  // a row is on its way while the one before it, or the angles, are computed
  uint32_t ahead[4];
  auto row_at = [&](int r, int& kind, int& head) {  // kind: 0 queries, 1 keys, 2 values
    kind = r < a.Hq ? 0 : (r < a.Hq + a.Hkv ? 1 : 2);
    head = kind == 0 ? r : (kind == 1 ? r - a.Hq : r - a.Hq - a.Hkv);
    return (kind == 0 ? a.q + t * a.ldq : (kind == 1 ? a.k + t * a.ldk : a.v + t * a.ldv)) + (long long)head * a.D;
  };
  auto fetch = [&](int r0) {
    const int r = r0 + (int)(threadIdx.x / LN);
    int kind, head;
    const uint16_t* x = row_at(r < end ? r : first, kind, head);
    load_8(x + c0, r < end ? a.D - c0 : 0, ahead);
  };
  fetch(first);
  uint32_t weight[2][4] = {};
  if (a.qw) load_8(a.qw + c0, a.D - c0, weight[0]);
  if (a.kw) load_8(a.kw + c0, a.D - c0, weight[1]);
  if ((int)threadIdx.x < half) {
    // position x frequency in turns, to 2^-50 of one: the product of a 31-bit and a 24-bit number and 1 / 2 pi in two pieces each
    const double p = a.positions[t], f = a.frequencies[threadIdx.x], angle = p * f;
    const double hi = 0.15915494309189535, lo = -9.839338337591243e-18;
    const double turns = angle * hi;
    const double rest = __builtin_fma(angle, hi, -turns) + (angle * lo + __builtin_fma(p, f, -angle) * hi);
    double s, c;
    turn_by((turns - __builtin_rint(turns)) + rest, s, c);
    turn[0][threadIdx.x] = c;
    turn[1][threadIdx.x] = s;
  }
  // The last of the tokens that are given one place has it: the slots of all later tokens are looked through, T^2 / 2 comparisons in all.  Of a prompt of 4096 tokens of 64 + 8 + 8 heads that is
  // 6 us of 79, of 65536 tokens 0.6 ms of 1.7, of 131072 tokens 2.1 of 4.3.  (A list of who has which place would need scratch memory of the size of the cache.)  Tokens that have no place look
  // for nothing.
  long long slot = -1;
  int later = 0;
  if (a.slots) {
    const int32_t mine = a.slots[t];
    if (mine >= 0 && mine < a.tokens) slot = mine;
    // (the waves that have no angles look through those behind it, sixteen of a thread at a time)
    if (slot >= 0 && threadIdx.x >= NT / 2) {
      for (long long j = t + 1 + 4 * (long long)(threadIdx.x - NT / 2); j < a.T; j += 8 * NT) {
        int32_t s[4][4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
          const long long i = j + u * 2 * NT;
          if (i + 4 <= a.T) {
            __builtin_memcpy(s[u], a.slots + i, 16);
          } else {
#pragma unroll
            for (int e = 0; e < 4; e++) s[u][e] = i + e < a.T ? a.slots[i + e] : -1;
          }
        }
#pragma unroll
        for (int u = 0; u < 4; u++)
#pragma unroll
          for (int e = 0; e < 4; e++) later |= s[u][e] == mine;
      }
    }
  }
  if (__syncthreads_or(later)) slot = -1;
  const long long place = slot < 0 ? 0 : ((slot >> a.page_bits) * a.Hkv << a.page_bits) + (slot & ((1ll << a.page_bits) - 1));
  // What this lane's channels and their partners (i +- half, or i +- 1) are multiplied with: cosine and sine, times the weights of the kind of head at hand, so that a channel takes
  // a product, a multiply-add and one division by the norm
  double own[8], other[8];
  // the partners of eight values v of a row x (0 where there is none)
  auto partners = [&](const uint32_t (&v)[4], const uint16_t* x, bool live, uint32_t (&p)[4]) {
#pragma unroll
    for (int i = 0; i < 4; i++) p[i] = 0u;
    if (a.paired) {
#pragma unroll
      for (int i = 0; i < 4; i++) p[i] = v[i] >> 16 | v[i] << 16;
    } else if ((half & 7) == 0) {  // a lane of the same row has them
      const int from = (int)(threadIdx.x & 63u) + (c0 < half ? half / 8 : -(half / 8));
#pragma unroll
      for (int i = 0; i < 4; i++) p[i] = (uint32_t)__shfl((int)v[i], c0 < a.rotary ? from : 0);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const int ch = c0 + i;
        if (live && ch < a.rotary) p[i / 2] |= (uint32_t)x[ch < half ? ch + half : ch - half] << (16 * (i & 1));
      }
    }
  };
  auto factors = [&](int kind) {
    const uint16_t* w = kind ? a.kw : a.qw;
    uint32_t g[4], p[4];
#pragma unroll
    for (int i = 0; i < 4; i++) g[i] = kind ? weight[1][i] : weight[0][i];
    if (w) partners(g, w, true, p);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int ch = c0 + i;
      const bool turned = ch < a.rotary, second = a.paired ? (i & 1) : ch >= half;
      const int at = !turned ? 0 : (a.paired ? ch >> 1 : (second ? ch - half : ch));
      own[i] = turned ? turn[0][at] : 1.;
      other[i] = turned ? (second ? turn[1][at] : -turn[1][at]) : 0.;
      if (w) {
        own[i] *= (double)esp_to_float<DT>((uint16_t)(g[i / 2] >> (16 * (i & 1))));
        other[i] *= (double)esp_to_float<DT>((uint16_t)(p[i / 2] >> (16 * (i & 1))));
      }
    }
  };
  int known = -1;  // the kind that they are of
  for (int r0 = first; r0 < end; r0 += ROWS) {
    const int r = r0 + (int)(threadIdx.x / LN);
    const bool live = r < end;
    int kind, head;
    const uint16_t* x = row_at(live ? r : first, kind, head);
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = ahead[i];
    if (r0 + ROWS < end) fetch(r0 + ROWS);
    const long long row = place + ((long long)head << a.page_bits);
    MxCodes codes = {0u, 0u};
    unsigned e = 0;
    if (kind == 2) {
      e = mx_block_exponent<DT, ESPARSE_MX_FP4>(v);
      codes = mx_encode<DT, ESPARSE_MX_FP4>(v, e);
    } else {
      const uint16_t* w = kind == 0 ? a.qw : a.kw;
      const bool exact = kind == 1 && a.slots;  // (what is rounded to 16 bits has no border that a last bit decides)
      double y[8], z[8];
      widen_8<DT>(v, y);
      double by = 1., n = 0.;
      if (w) {
        double s = 0.;
#pragma unroll
        for (int i = 0; i < 8; i++) s = __builtin_fma(y[i], y[i], s);
        s = row_sum<LN>(s);
        if (exact) {
          n = __builtin_sqrt(s / (double)a.D + a.eps);
          by = 1. / n;
          n = __builtin_isfinite(n) ? n : 0.;
        } else {
          by = inverse_root(__builtin_fma(s, a.per_channel, a.eps));
        }
      }
      if (half || w) {
        if (known != kind) factors(kind);
        known = kind;
        uint32_t p[4];
        partners(v, x, live, p);
        widen_8<DT>(p, z);
#pragma unroll
        for (int i = 0; i < 8; i++) {
          y[i] *= own[i];
          if (c0 + i < a.rotary) y[i] = __builtin_fma(z[i], other[i], y[i]);  // (a channel that is not turned keeps its value, whatever its partner holds)
        }
        if (w) {
#pragma unroll
          for (int i = 0; i < 8; i++) y[i] = exact ? over(y[i], by, n) : y[i] * by;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (c0 + i >= a.D) y[i] = 0.;  // (0 times an infinite 1 / norm is no 0)
      uint16_t* out = kind == 0 ? a.q_out : a.k_out;
      if (out && live) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; i++) o[i] = pack_2<DT>((float)y[2 * i], (float)y[2 * i + 1]);
        out += (t * (kind == 0 ? a.Hq : a.Hkv) + head) * a.D + c0;
        if (a.D - c0 >= 8) {
          store_stream_16(out, o);
        } else {
#pragma unroll
          for (int i = 0; i < 8; i++)
            if (c0 + i < a.D) out[i] = (uint16_t)(o[i / 2] >> (16 * (i & 1)));
        }
      }
      if (kind == 1 && a.slots) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const uint32_t h = (uint32_t)(__builtin_bit_cast(unsigned long long, y[i]) >> 32) & 0x7fffffffu;
          top = h > top ? h : top;
        }
        // floor(log2) of the block's largest, less 2, from its exponent
        const int lead = (int)(quad_max(top) >> 20);
        const int ex = lead - 1023 - 2 + 127;
        e = lead == 2047 ? 255u : (ex < 0 ? 0u : (ex > 254 ? 254u : (unsigned)ex));
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = to_odd_24(__builtin_ldexp(y[i], 127 - (int)e));
        codes = mx_encode<ESPARSE_MX_FP4>(f, e == 255u ? 255u : 127u);
      }
    }
    if (kind && live && slot >= 0) put_row<DP>(kind == 1 ? a.k_data : a.v_data, kind == 1 ? a.k_scales : a.v_scales, row, lane, codes, e);
  }
}

struct ReadArgs {
  const unsigned char *data[2], *scales[2];
  void* out[2];
  const int32_t* slots;
  long long T, tokens;
  int H, D, page_bits;
};

// rows of the cache as numbers: DP / 8 lanes for a row, keys in the first half of the grid's rows
template <int DT, int DP>
__global__ void __launch_bounds__(NT) k_cache_read(const ReadArgs a) {
  constexpr int LN = DP / 8;
  const long long r = (long long)blockIdx.x * (NT / LN) + threadIdx.x / LN;
  const int which = blockIdx.y;
  if (r >= a.T * a.H) return;
  const long long t = r / a.H;
  const int head = (int)(r % a.H), c0 = (int)(threadIdx.x % LN) * 8, left = a.D - c0;
  if (left <= 0) return;
  const int32_t slot = a.slots[t];
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; i++) f[i] = 0.f;
  if (slot >= 0 && slot < a.tokens) {
    const long long row = (((long long)(slot >> a.page_bits) * a.H + head) << a.page_bits) + (slot & ((1 << a.page_bits) - 1));
    const uint32_t w = *reinterpret_cast<const uint32_t*>(a.data[which] + row * (DP / 2) + c0 / 2);
    const unsigned e = a.scales[which][row * (DP / 32) + c0 / 32];
#if defined(__HIP_DEVICE_COMPILE__)
    const float s = mx_scale(e);
    const esp_float2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1),
                     p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    f[0] = p0[0], f[1] = p0[1], f[2] = p1[0], f[3] = p1[1], f[4] = p2[0], f[5] = p2[1], f[6] = p3[0], f[7] = p3[1];
#endif
    if (e == 255u) {
#pragma unroll
      for (int i = 0; i < 8; i++) f[i] = __builtin_nanf("");
    }
  }
  const long long at = r * a.D + c0;
  if constexpr (DT == ESPARSE_F32) {
    float* o = reinterpret_cast<float*>(a.out[which]) + at;
    if (left >= 8) {
      store_stream_16(o, f);
      store_stream_16(o + 4, f + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (i < left) o[i] = f[i];
    }
  } else {
    uint16_t* o = reinterpret_cast<uint16_t*>(a.out[which]) + at;
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

int log2_of(int page) { return __builtin_ctz((unsigned)page); }

}  // namespace

int esp_rotate_heads_device(esparse_ctx* ctx, const esparse_heads* h, long long T, int dtype, const void* q, long long ldq, const void* q_weight, const void* k,
                            long long ldk, const void* k_weight, const int32_t* positions, const float* frequencies, void* q_out, void* k_out, const void* v,
                            long long ldv, const esparse_cache* cache, const int32_t* slots) {
  RotateArgs a = {};
  a.q = (const uint16_t*)q, a.k = (const uint16_t*)k, a.v = (const uint16_t*)v, a.qw = (const uint16_t*)q_weight, a.kw = (const uint16_t*)k_weight;
  a.q_out = (uint16_t*)q_out, a.k_out = (uint16_t*)k_out;
  a.positions = positions, a.frequencies = frequencies;
  a.ldq = ldq, a.ldk = ldk, a.ldv = ldv, a.T = T;
  a.Hq = q ? h->q_heads : 0, a.Hkv = k ? h->kv_heads : 0, a.D = h->head_dim, a.rotary = h->rotary, a.paired = h->paired, a.eps = h->eps, a.per_channel = 1. / h->head_dim;
  if (cache) {
    a.slots = slots;
    a.k_data = (unsigned char*)cache->k_data, a.k_scales = (unsigned char*)cache->k_scales;
    a.v_data = (unsigned char*)cache->v_data, a.v_scales = (unsigned char*)cache->v_scales;
    a.page_bits = log2_of(cache->page);
    a.tokens = cache->pages << a.page_bits;
  }
  a.rows = a.Hq + a.Hkv * (cache ? 2 : 1);
  const int row = esp_cache_row(a.D), pass = NT / (row / 8), passes = (a.rows + pass - 1) / pass;
  // a workgroup for each pass over a few rows until they fill the chip, then one for all rows of a token (the angles are computed once)
  const long long want = (1024 + T - 1) / T;
  a.chunks = (int)(want < passes ? want : passes);
  const dim3 grid((unsigned)(T * a.chunks));
#define GO(DT, DP) hipLaunchKernelGGL((k_rotate_heads<DT, DP>), grid, dim3(NT), 0, ctx->stream, a)
  if (dtype == ESPARSE_F16) {
    if (row == 64) GO(ESPARSE_F16, 64);
    else if (row == 128) GO(ESPARSE_F16, 128);
    else GO(ESPARSE_F16, 256);
  } else {
    if (row == 64) GO(ESPARSE_BF16, 64);
    else if (row == 128) GO(ESPARSE_BF16, 128);
    else GO(ESPARSE_BF16, 256);
  }
#undef GO
  ESP_HIP(ctx, hipGetLastError());
  return ESPARSE_OK;
}

int esp_cache_read_device(esparse_ctx* ctx, const esparse_cache* cache, const int32_t* slots, long long T, int dtype, void* k_out, void* v_out) {
  ReadArgs a = {};
  const bool both = k_out && v_out;
  a.data[0] = (const unsigned char*)(k_out ? cache->k_data : cache->v_data), a.scales[0] = (const unsigned char*)(k_out ? cache->k_scales : cache->v_scales);
  a.data[1] = (const unsigned char*)cache->v_data, a.scales[1] = (const unsigned char*)cache->v_scales;
  a.out[0] = k_out ? k_out : v_out, a.out[1] = v_out;
  a.slots = slots, a.T = T, a.H = cache->heads, a.D = cache->head_dim, a.page_bits = log2_of(cache->page);
  a.tokens = cache->pages << a.page_bits;
  const int row = esp_cache_row(a.D), pass = NT / (row / 8);
  const dim3 grid((unsigned)((T * a.H + pass - 1) / pass), both ? 2 : 1);
#define GO(DT, DP) hipLaunchKernelGGL((k_cache_read<DT, DP>), grid, dim3(NT), 0, ctx->stream, a)
#define ROW(DT)                    \
  {                                \
    if (row == 64) GO(DT, 64);     \
    else if (row == 128) GO(DT, 128); \
    else GO(DT, 256);              \
  }
  if (dtype == ESPARSE_F16) ROW(ESPARSE_F16)
  else if (dtype == ESPARSE_BF16) ROW(ESPARSE_BF16)
  else ROW(ESPARSE_F32)
#undef ROW
#undef GO
  ESP_HIP(ctx, hipGetLastError());
  return ESPARSE_OK;
}
