// Attention over a cache held in microscaled 4 bits (include/esparse.h, csrc/heads.hip): o = sum_j p_j v_j, p = softmax(scale q.k_j), one pass over the tokens
// with the running maximum m and sum l of the softmax:  m' = max(m, x_j), l' = l 2^(c (m - m')) + sum 2^(c (x_j - m')), o' likewise, c = |scale| log2(e).
// x_j are the products q.k_j themselves (with a negative scale q has its sign turned, with none it is zeros) and their distances to the maximum are what is multiplied: a scale cannot take
// them out of fp32 but to minus infinity, where the exponential is 0 as it should be.
//
// The rows of a tile are the queries of one head of the cache, (token, query head of the group) in order: 16 of them are the columns of the 16-bit matrix
// instruction (lane l = 16 g + c: operands hold k = 8 g .. 8 g + 7 of row / column c, results rows 4 g + j of column c).
//   scores  X^T[token, row] = K Q^T.  Lane (c, g) loads 16 bytes of token c: channels 32 g .. 32 g + 31, one block with one scale, brought to 16 bits by the
//           conversion that takes the scale; its j-th word is the operand of step j (which k a channel takes does not matter as long as Q's agrees).
//   output  O^T[channel, row] += V^T P^T.  The lane holds the probabilities of tokens 4 g + j of two groups of 16 for its row: with the tokens of a step numbered that
//           way P^T is an operand as it stands.  V needs token and channel exchanged: it goes through LDS in 16 bits and comes back by the transposing read, which
//           hands a lane four tokens of one channel.  P is rounded to the 16 bits of the output's type, as V is held: the matrix instruction takes both so, and each number is off by at
//           most half a step of the type, which the output is rounded to as well; sums and statistics are in 32 bits.  The error against 64 bits is 1.1 to 1.2 of that of the rounded output
//           alone.  A second product with what P lost takes that to 1.0, and 122 us instead of 116 (48 sequences), 97 instead of 93 (drafts), 1842 instead of 1405 (a prompt of 8192 tokens).
//           f16 has few exponents: there P is 2^15 at the maximum, so that it keeps its bits down to 2^-29 and vanishes below 2^-40 (with 1 at the maximum a tail of 2^-26 and less was in l
//           but not in o).
// Bound by memory at one token a sequence where there is work for the chip: 48 sequences of 500 to 4096 tokens, 32 heads of 128 channels, 116 us (4.1 TB/s; a copy reaches 4.9), where
// four waves a SIMD (122 registers, 37 KB of LDS a workgroup) do not cover the latency of a strip (a third of a wave's time it waits for memory, a fifth for a slot of the vector unit, which is busy
// 55 %); 131072 tokens, 64 heads on 8, 32 us and 5 to join the pieces (3.8 TB/s).  256 channels take 208 registers, two waves a SIMD: 21 sequences of five tokens each, 16 heads on 4, 81 us (1.3 TB/s).
// The statistics of a row are those of a column of X^T: they stay in the lane but for two exchanges (lanes 16 and 32 apart) a strip of 32 tokens.
// A block of V that has no numbers in 16 bits (scale 255, or so large that some would be infinite) is left out of the product and makes the rows that see its token NaN afterwards, so that
// masked tokens cannot reach a row.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "intrinsics.h"
#include "mx.h"

namespace {

constexpr int STRIP = 32;      // tokens of a step
constexpr int ROWS = 16;       // rows of a tile
constexpr int WAVES = 4;
constexpr int LEAST = 8;       // strips of a piece, where a long sequence is cut
constexpr int MOST_PIECES = 512;
constexpr uint16_t NAN16 = 0x7fff;  // of both types

struct AttendArgs {
  const uint16_t* q;
  const unsigned char *k_data, *k_scales, *v_data, *v_scales;
  const int32_t *table, *lengths, *starts;
  uint16_t* out;
  float* lse;
  float* partial;  // [tile][head][piece]: 16 x DP sums, 16 maxima, 16 sums of probabilities
  long long ldq, T, pages;
  long long width;  // pages of a row of the table
  int B, Hkv, group, D, page_bits, tiles, pieces;
  int rows;  // of a tile that can be anything
  float c, natural;      // |scale| log2(e), 1 without scale; |scale|
  uint32_t flip, keep;   // of two 16-bit numbers of q: signs to turn, bits to keep
};

// where a tile is: the sequence, its first row, and what its rows see
struct Tile {
  int b, first, queries;  // sequence, first row of the tile among the sequence's, queries of the sequence
  long long start;        // first query of the sequence
  int length, end;        // tokens of the sequence; those that the tile's last row sees
};

__device__ __forceinline__ long long clamp_to(long long v, long long lo, long long hi) { return v < lo ? lo : (v > hi ? hi : v); }

// Tiles of sequence b begin at floor(starts[b] group / rows) + b: enough for all of its rows.  The last
// sequence that begins no later is looked for among 64 at a time
__device__ __forceinline__ Tile find_tile(const AttendArgs& a, int tile, int rows) {
  Tile t;
  if (!a.starts) {
    const int each = (a.group + rows - 1) / rows;
    t.b = tile / each;
    t.first = (tile % each) * rows;
    t.start = t.b;
    t.queries = 1;
  } else {
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, b = lo + (int)(threadIdx.x & 63u) * step;
      const bool yes = b < hi && clamp_to(a.starts[b < hi ? b : lo], 0, a.T) * a.group / rows + b <= tile;
      const int found = (int)__popcll(__ballot(yes));
      lo += found > 0 ? (found - 1) * step : 0;
      hi = lo + step < hi ? lo + step : hi;
    }
    t.b = wave_uniform(lo);
    t.start = clamp_to(a.starts[t.b], 0, a.T);
    const long long stop = clamp_to(a.starts[t.b + 1], t.start, a.T);
    t.queries = (int)(stop - t.start);
    t.first = (int)(tile - (t.start * a.group / rows + t.b)) * rows;
    if (t.first < 0) t.first = t.queries = 0;  // rows in front of the first sequence: of none
  }
  t.length = (int)clamp_to(a.lengths[t.b], 0, a.width << a.page_bits);
  const long long all = (long long)t.queries * a.group;
  const long long last = t.first + rows < all ? t.first + rows - 1 : all - 1;
  t.end = t.first >= all ? 0 : (int)clamp_to(t.length - t.queries + last / a.group + 1, 0, t.length);
  return t;
}
__device__ __forceinline__ int pieces_of(int end, int pieces) {
  const int strips = (end + STRIP - 1) / STRIP, most = (strips + LEAST - 1) / LEAST;
  return most < pieces ? (most > 0 ? most : 1) : pieces;
}

// c (x - base) is one instruction with c base as a rounded number, as long as that is off by less than a quarter (no more than what the products' own rounding makes of it); scores beyond that,
// which may leave fp32 when scaled, have the distance to base taken first
constexpr float NEAR = 0x1p22f;
// the exponent of the largest probability (with the rounding of base above it stays below 65504)
template <int DT>
constexpr float kOffset = DT == ESPARSE_F16 ? 15.f : 0.f;
// four 16-bit numbers to an address of any alignment that suits one of them.  (As a vector: the compiler makes four stores of a copy whose last number is stored on the other branch too, 5 % of a long
// prompt's time)
__device__ __forceinline__ void store_8(uint16_t* p, const uint32_t (&v)[2]) {
  const esp_u32x2_any w = {v[0], v[1]};
  *reinterpret_cast<esp_u32x2_any*>(p) = w;
}
// what 32 bits of a query (two numbers) take part as
__device__ __forceinline__ uint32_t oriented(const AttendArgs& a, uint32_t v) { return (v ^ a.flip) & a.keep; }
// the first of n tokens that is in a page (n: none); the lanes that are here look together
__device__ __forceinline__ int first_token(const AttendArgs& a, const int32_t* table, int n) {
  const int pages = (n + (1 << a.page_bits) - 1) >> a.page_bits;
  const unsigned long long here = __ballot(1);
  auto rank = [&](int lane) { return (int)__popcll(here & ((1ull << lane) - 1ull)); };
  for (int p0 = 0; p0 < pages; p0 += (int)__popcll(here)) {
    const int p = p0 + rank((int)(threadIdx.x & 63u)), page = p < pages ? table[p] : -1;
    const unsigned long long some = __ballot(page >= 0 && page < a.pages);
    if (some) return (p0 + rank((int)__builtin_ctzll(some))) << a.page_bits;
  }
  return n;
}
// What a row is divided by, inverted, and ln sum exp; a sum of nothing: 0 and minus infinity, as for a row that sees nothing
struct Sums {
  float by, lse;
};
template <int DT>
__device__ __forceinline__ Sums sums_of(const AttendArgs& a, float all, float top) {
  return {all == 0.f ? 0.f : 1.f / all, all == 0.f ? -__builtin_inff() : top * a.natural + (log2f(all) - kOffset<DT>) * 0.6931471805599453f};
}
// ... but a row that sees tokens, up to `sees` of the n that rows of the tile see, has a sum of nothing where all of its products are minus infinity in 32 bits: it has no number.  (Asked after the
// outputs are written, when their registers are free.)  The rows of the lanes that are here are of the sequence that `table` is of
__device__ __forceinline__ bool no_number(const AttendArgs& a, float all, const int32_t* table, int n, int sees) {
  if (!__ballot(all == 0.f && sees >= 0)) return false;
  return first_token(a, table, n) <= sees && all == 0.f;
}

// the largest scale with which all codes have numbers of the type: 6 x 2^13 and 6 x 2^125
template <int DT>
constexpr unsigned kLargest = DT == ESPARSE_F16 ? 140 : 252;

// channels of a lane's operand of step s (eight of them)
template <int DP>
__device__ __forceinline__ int channel_of(int s, int g) {
  return DP == 64 ? 16 * g + 8 * s : 128 * (s / 4) + 32 * g + 8 * (s % 4);
}
// a lane's codes and scales of its token in a group of 16
template <int DP>
struct Codes {
  uint32_t w[DP / 32];
  unsigned e[DP == 256 ? 2 : 1];
};
template <int DP>
__device__ __forceinline__ void load_codes(const unsigned char* data, const unsigned char* scales, long long row, int g, Codes<DP>& o) {
  if constexpr (DP == 64) {
    const uint2 v = *reinterpret_cast<const uint2*>(data + row * 32 + 8 * g);
    o.w[0] = v.x, o.w[1] = v.y;
    o.e[0] = scales[row * 2 + (g >> 1)];
  } else {
#pragma unroll
    for (int i = 0; i < DP / 128; i++) {
      const uint4 v = *reinterpret_cast<const uint4*>(data + row * (DP / 2) + 64 * i + 16 * g);
      o.w[4 * i] = v.x, o.w[4 * i + 1] = v.y, o.w[4 * i + 2] = v.z, o.w[4 * i + 3] = v.w;
      o.e[i] = scales[row * (DP / 32) + 4 * i + g];
    }
  }
}

// maximum and sum over the lanes that are 32, and 16 and 32, apart
#if defined(__HIP_DEVICE_COMPILE__)
#define HALVES(v, op)                                                                                                         \
  const auto w = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false); \
  v = op(__builtin_bit_cast(float, (unsigned)w[0]), __builtin_bit_cast(float, (unsigned)w[1]));
#define QUARTERS(v, op)                                                                                                       \
  const auto u = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false); \
  v = op(__builtin_bit_cast(float, (unsigned)u[0]), __builtin_bit_cast(float, (unsigned)u[1]));
#else
#define HALVES(v, op)
#define QUARTERS(v, op)
#endif
__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float half_max(float v) {
  HALVES(v, fmaxf)
  return v;
}
__device__ __forceinline__ float half_sum(float v) {
  HALVES(v, add)
  return v;
}
__device__ __forceinline__ float column_max(float v) {
  QUARTERS(v, fmaxf)
  return half_max(v);
}
__device__ __forceinline__ float column_sum(float v) {
  QUARTERS(v, add)
  return half_sum(v);
}
#undef HALVES
#undef QUARTERS

typedef short esp_short4 __attribute__((ext_vector_type(4)));
// four rows of 16-bit numbers, 16 columns: lane c of 16 hands in columns 4 (c % 4) .. + 3 of row c / 4 and gets column c of the four rows
__device__ __forceinline__ uint2 read_transposed(const uint16_t* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef __attribute__((address_space(3))) esp_short4 lds_short4;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)p));
#else
  return uint2{0u, 0u};
#endif
}
// what the lanes of a wave have written to LDS is read by others of the same wave
__device__ __forceinline__ void wave_fence() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#endif
}

// Results of matrix instructions are read from here on: 32 clocks, more than the longest of them needs.  The compiler counts these within a stretch of code without branches;
// behind a branch it has read the last number of a result a clock after its instruction.  Two results are named by one statement: their instructions are in front of the wait, what reads them is
// behind it, however the compiler orders the rest.
template <class V>
__device__ __forceinline__ void settle(V& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 15\n\ts_nop 15" : "+v"(v));
#else
  (void)v;
#endif
}
template <class V>
__device__ __forceinline__ void settle(V& v, V& w) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 15\n\ts_nop 15" : "+v"(v), "+v"(w));
#else
  (void)v, (void)w;
#endif
}

template <int DP>
constexpr int kHalf = DP == 256 ? 128 : DP;  // channels of V in LDS at a time
template <int DP>
constexpr int kVRow = kHalf<DP> + 16;  // 16-bit numbers from token to token in LDS: eight tokens' columns lie in different banks
template <int DP>
constexpr int kPartial = ROWS * DP + 2 * ROWS;

// the codes of a strip, and which of its groups of 16 tokens are in a page
template <int DP>
struct Strip {
  Codes<DP> k[2], v[2];
  bool there[2];
};

// One tile of 16 rows and a piece of its tokens: the waves take strips in turn, their results are joined in LDS.  A wave asks for its next strip, and for the pages of the one after that,
// before it works on one.
template <int DT, int DP>
__global__ void __launch_bounds__(64 * WAVES, DP == 256 ? 2 : 3) k_attend_few(const AttendArgs a) {
  constexpr int NS = DP / 32, ND = DP / 16, NH = DP / kHalf<DP>, NE = DP == 256 ? 2 : 1;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ float stat[2][WAVES][ROWS];
  const int wave = wave_uniform((int)(threadIdx.x >> 6)), lane = (int)(threadIdx.x & 63u), c = lane & 15, g = lane >> 4;
  uint16_t* vt = reinterpret_cast<uint16_t*>(lds) + wave * (STRIP * kVRow<DP>);
  const int piece = (int)(blockIdx.x % (unsigned)a.pieces);
  const int head = (int)(blockIdx.x / (unsigned)a.pieces % (unsigned)a.Hkv), tile = (int)(blockIdx.x / (unsigned)a.pieces / (unsigned)a.Hkv);
  const Tile t = find_tile(a, tile, ROWS);
  if (t.first >= (long long)t.queries * a.group) return;
  const int pieces = pieces_of(t.end, a.pieces);
  if (piece >= pieces) return;
  const int strips = (t.end + STRIP - 1) / STRIP;
  const int from = (int)((long long)strips * piece / pieces), to = (int)((long long)strips * (piece + 1) / pieces);
  const int32_t* table = a.table + (long long)t.b * a.width;

  auto pages_of = [&](int strip, int (&page)[2]) {
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const int at = strip * STRIP + 16 * u;
      page[u] = strip < to && at < t.end ? wave_uniform(table[at >> a.page_bits]) : -1;
    }
  };
  auto load = [&](int strip, const int (&page)[2], Strip<DP>& o) {
#pragma unroll
    for (int u = 0; u < 2; u++) {
      o.there[u] = page[u] >= 0 && page[u] < a.pages;
      if (o.there[u]) {
        const int at = strip * STRIP + 16 * u;
        const long long r = (((long long)page[u] * a.Hkv + head) << a.page_bits) + (at & ((1 << a.page_bits) - 1)) + c;
        load_codes<DP>(a.k_data, a.k_scales, r, g, o.k[u]);
        load_codes<DP>(a.v_data, a.v_scales, r, g, o.v[u]);
      } else {
        o.k[u] = Codes<DP>{};
        o.v[u] = Codes<DP>{};
      }
    }
  };
  Strip<DP> next;
  int page[2];
  pages_of(from + wave, page);
  load(from + wave, page, next);
  pages_of(from + wave + WAVES, page);

  const int row = t.first + c, query = row / a.group;
  const bool live = query < t.queries;
  const int sees = live ? t.length - t.queries + query : -1;  // the row's last token
  uint4 qv[NS];
#pragma unroll
  for (int s = 0; s < NS; s++) {
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    const int ch = channel_of<DP>(s, g);
    if (live) load_8(a.q + (t.start + query) * a.ldq + (long long)(head * a.group + row % a.group) * a.D + ch, a.D - ch, v);
    qv[s] = uint4{v[0], v[1], v[2], v[3]};
  }
  if (a.flip | ~a.keep) {  // (else the queries are still on their way)
#pragma unroll
    for (int s = 0; s < NS; s++) qv[s] = uint4{oriented(a, qv[s].x), oriented(a, qv[s].y), oriented(a, qv[s].z), oriented(a, qv[s].w)};
  }
  floatx4_t o[ND];
#pragma unroll
  for (int n = 0; n < ND; n++) o[n] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;
  bool beyond = false;  // (of some row of the wave)

  for (int strip = from + wave; strip < to; strip += WAVES) {
    Strip<DP> now = next;
    load(strip + WAVES, page, next);
    pages_of(strip + 2 * WAVES, page);
    // scores
    float x[2][4];
    floatx4_t acc[2];
#pragma unroll
    for (int u = 0; u < 2; u++) {
      acc[u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; s++) acc[u] = mfma16<DT>(mx_widen<DT>(now.k[u].w[s], mx_scale(now.k[u].e[DP == 256 ? s / 4 : 0])), qv[s], acc[u]);
    }
    settle(acc[0], acc[1]);
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int j = 0; j < 4; j++) x[u][j] = now.there[u] && strip * STRIP + 16 * u + 4 * g + j <= sees ? acc[u][j] : -__builtin_inff();
    float top = m;
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int j = 0; j < 4; j++) top = fmaxf(top, x[u][j]);
    top = column_max(top);
    const float base = top == -__builtin_inff() ? 0.f : top;
    float scaled = base * a.c;
    if (__ballot(top > m) || beyond) {  // (else all have kept their maxima)
      const float shrink = __builtin_amdgcn_exp2f((m - base) * a.c);
      l *= shrink;
#pragma unroll
      for (int n = 0; n < ND; n++)
#pragma unroll
        for (int j = 0; j < 4; j++) o[n][j] *= shrink;
      m = top;
      const bool row_beyond = !(fabsf(scaled) < NEAR);
      beyond = __ballot(row_beyond) != 0;
      if (__builtin_expect(beyond, 0)) {
        const float off = row_beyond ? base : 0.f;
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
          for (int j = 0; j < 4; j++) x[u][j] -= off;
        scaled = row_beyond ? 0.f : scaled;
      }
    }
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        x[u][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][j], a.c, kOffset<DT> - scaled));
        l += x[u][j];
      }
    const uint4 p = {pack_2<DT>(x[0][0], x[0][1]), pack_2<DT>(x[0][2], x[0][3]), pack_2<DT>(x[1][0], x[1][1]), pack_2<DT>(x[1][2], x[1][3])};
    // V through LDS
    unsigned long long odd[2][NE];
#pragma unroll
    for (int u = 0; u < 2; u++) {
      if (strip * STRIP + 16 * u + c >= t.end) now.v[u] = Codes<DP>{};  // tokens that no row sees: no numbers of theirs take part
#pragma unroll
      for (int i = 0; i < NE; i++) odd[u][i] = __ballot(now.v[u].e[i] > kLargest<DT>);
    }
#pragma unroll
    for (int hh = 0; hh < NH; hh++) {
      wave_fence();
#pragma unroll
      for (int u = 0; u < 2; u++) {
        const unsigned e = now.v[u].e[hh];
        const bool bad = e > kLargest<DT>;
        const float by = mx_scale(bad ? 0u : e);
#pragma unroll
        for (int s = 0; s < NS / NH; s++)
          *reinterpret_cast<uint4*>(vt + (16 * u + c) * kVRow<DP> + channel_of<DP>(s, g)) = mx_widen<DT>(bad ? 0u : now.v[u].w[NS / NH * hh + s], by);
      }
      wave_fence();
#pragma unroll
      for (int n = 0; n < ND / NH; n++) {
        const uint16_t* at = vt + (4 * g + (c >> 2)) * kVRow<DP> + 16 * n + 4 * (c & 3);
        const uint2 lo = read_transposed(at), hi = read_transposed(at + 16 * kVRow<DP>);
        o[ND / NH * hh + n] = mfma16<DT>(uint4{lo.x, lo.y, hi.x, hi.y}, p, o[ND / NH * hh + n]);
      }
    }
    // blocks without numbers: NaN for the rows that see them
    unsigned long long some = 0;
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int i = 0; i < NE; i++) some |= odd[u][i];
    if (!some) continue;
#pragma unroll
    for (int n = 0; n < ND; n++) settle(o[n]);
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int i = 0; i < NE; i++)
        for (unsigned long long left = odd[u][i]; left; left &= left - 1) {
          const int who = (int)__builtin_ctzll(left);
          const int block = DP == 64 ? (who >> 4) >> 1 : 4 * i + (who >> 4);
          if (strip * STRIP + 16 * u + (who & 15) <= sees) {
#pragma unroll
            for (int n = 0; n < ND; n++)
              if (n / 2 == block) o[n] = floatx4_t{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
          }
        }
  }
  l = column_sum(l);
#pragma unroll
  for (int n = 0; n < ND; n++) settle(o[n]);

  // the waves' results
  if (g == 0) {
    stat[0][wave][c] = m;
    stat[1][wave][c] = l;
  }
  constexpr int ROW = kHalf<DP> + 4;  // numbers from row to row in LDS: the four lanes of a column and their neighbours in different banks
  static_assert(ROWS * ROW * 4 <= STRIP * kVRow<DP> * 2, "a wave's sums fit where its values were");
  const float* sums = reinterpret_cast<const float*>(lds);
  float* mine = reinterpret_cast<float*>(vt);
  float* part = a.partial + ((long long)(tile * a.Hkv + head) * a.pieces + piece) * kPartial<DP>;
#pragma unroll
  for (int hh = 0; hh < NH; hh++) {
    __syncthreads();
#pragma unroll
    for (int n = 0; n < ND / NH; n++) *reinterpret_cast<floatx4_t*>(mine + c * ROW + 16 * n + 4 * g) = o[ND / NH * hh + n];
    __syncthreads();
    for (int at = (int)threadIdx.x * 4; at < ROWS * kHalf<DP>; at += 64 * WAVES * 4) {
      const int r = at / kHalf<DP>, in = at % kHalf<DP>, ch = hh * kHalf<DP> + in;
      float top = -__builtin_inff();
#pragma unroll
      for (int w = 0; w < WAVES; w++) top = fmaxf(top, stat[0][w][r]);
      const float base = top == -__builtin_inff() ? 0.f : top;
      floatx4_t sum = {0.f, 0.f, 0.f, 0.f};
      float all = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; w++) {
        const float f = __builtin_amdgcn_exp2f((stat[0][w][r] - base) * a.c);
        const floatx4_t v = *reinterpret_cast<const floatx4_t*>(sums + w * (STRIP * kVRow<DP> / 2) + r * ROW + in);
#pragma unroll
        for (int j = 0; j < 4; j++) sum[j] += v[j] * f;
        all += stat[1][w][r] * f;
      }
      const int of = t.first + r, qi = of / a.group;
      if (qi >= t.queries) continue;
      if (pieces > 1) {
        *reinterpret_cast<floatx4_t*>(part + r * DP + ch) = sum;
        if (ch == 0) {
          part[ROWS * DP + r] = top;
          part[ROWS * DP + ROWS + r] = all;
        }
      } else {
        const long long place = (t.start + qi) * ((long long)a.Hkv * a.group) + head * a.group + of % a.group;
        const Sums of_row = sums_of<DT>(a, all, top);
#pragma unroll
        for (int j = 0; j < 4; j++)
          if (ch + j < a.D) a.out[place * a.D + ch + j] = esp_from_float<DT>(sum[j] * of_row.by);
        if (a.lse && ch == 0) a.lse[place] = of_row.lse;
        if (no_number(a, all, table, t.end, t.length - t.queries + qi)) {
          for (int j = 0; j < 4; j++)
            if (ch + j < a.D) a.out[place * a.D + ch + j] = NAN16;
          if (a.lse && ch == 0) a.lse[place] = __builtin_nanf("");
        }
      }
    }
  }
}

// The pieces of a row, joined: a workgroup for each row of a tile; its groups of DP / 4 threads (four channels each) take pieces in turn and their sums are added in order
template <int DT, int DP>
__global__ void __launch_bounds__(256) k_attend_join(const AttendArgs a) {
  constexpr int QUADS = DP / 4, GROUPS = 256 / QUADS;
  __shared__ float factor[MOST_PIECES], sums[MOST_PIECES], waves[4];
  __shared__ floatx4_t of_group[GROUPS][QUADS];
  const unsigned rows = (unsigned)a.rows;
  const int r = (int)(blockIdx.x % rows), head = (int)(blockIdx.x / rows % (unsigned)a.Hkv), tile = (int)(blockIdx.x / rows / (unsigned)a.Hkv);
  const Tile t = find_tile(a, tile, ROWS);
  const int of = t.first + r, qi = of / a.group;
  if (qi >= t.queries) return;
  const int pieces = pieces_of(t.end, a.pieces);
  if (pieces == 1) return;
  const float* part = a.partial + (long long)(tile * a.Hkv + head) * a.pieces * kPartial<DP>;
  const int quad = (int)threadIdx.x % QUADS, group = (int)threadIdx.x / QUADS;
  float top = -__builtin_inff();
  for (int i = (int)threadIdx.x; i < pieces; i += 256) {
    const float v = part[(long long)i * kPartial<DP> + ROWS * DP + r];
    factor[i] = v;
    sums[i] = part[(long long)i * kPartial<DP> + ROWS * DP + ROWS + r];
    top = fmaxf(top, v);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if ((threadIdx.x & 63u) == 0) waves[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(waves[0], waves[1]), fmaxf(waves[2], waves[3]));
  const float base = top == -__builtin_inff() ? 0.f : top;
  floatx4_t sum = {0.f, 0.f, 0.f, 0.f};
  float all = 0.f;
#pragma unroll 4
  for (int i = group; i < pieces; i += GROUPS) {
    const floatx4_t v = *reinterpret_cast<const floatx4_t*>(part + (long long)i * kPartial<DP> + r * DP + 4 * quad);
    const float f = __builtin_amdgcn_exp2f((factor[i] - base) * a.c);
#pragma unroll
    for (int j = 0; j < 4; j++) sum[j] += v[j] * f;
    all += sums[i] * f;
  }
  of_group[group][quad] = sum;
  __syncthreads();
  if (quad == 0) factor[group] = all;  // (all have read the factors)
  __syncthreads();
  if (group) return;
  all = 0.f;
  sum = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < GROUPS; i++) {
    const floatx4_t v = of_group[i][quad];
#pragma unroll
    for (int j = 0; j < 4; j++) sum[j] += v[j];
    all += factor[i];
  }
  const Sums of_row = sums_of<DT>(a, all, top);
  const long long place = (t.start + qi) * ((long long)a.Hkv * a.group) + head * a.group + of % a.group;
#pragma unroll
  for (int j = 0; j < 4; j++)
    if (4 * quad + j < a.D) a.out[place * a.D + 4 * quad + j] = esp_from_float<DT>(sum[j] * of_row.by);
  if (a.lse && quad == 0) a.lse[place] = of_row.lse;
  if (no_number(a, all, a.table + (long long)t.b * a.width, t.end, t.length - t.queries + qi)) {
    for (int j = 0; j < 4; j++)
      if (4 * quad + j < a.D) a.out[place * a.D + 4 * quad + j] = NAN16;
    if (a.lse && quad == 0) a.lse[place] = __builtin_nanf("");
  }
}

// ---- prompts: many rows of a sequence ----------------------------------------------------------------
// A workgroup of W waves takes 32 W rows, 32 a wave as the columns of the 32 x 32 instruction (lane 32 h + c: operands hold k = 8 h .. 8 h + 7 of row / column c, results rows
// 8 (j / 4) + 4 h + j % 4 of column c).  The tokens come in tiles that all waves share, brought to 16 bits once, in two buffers: while one is multiplied the
// codes of the tile after the next are on their way and the next is written to the other buffer.
// Measured: 8192 tokens, 64 heads on 8 of 128 channels 1360 us (810 TFLOP/s, where a large library product of the type reaches 1560; the matrix pipe is busy 30 %, the vector unit 50 %,
// mostly with exponentials): two waves a SIMD do not cover each other's waits.  The keys a tile ahead of the values, so that their products stand beside the exponentials, a higher priority of the waves
// in the products, and 32 tokens a tile were built and were slower (1490, 1500, 1520).  256 channels, 16 heads on 4: 855 us (640 TFLOP/s), with 16 of 256 registers spilled (8 waves; 29 with 4); 192
// channels 844, 80 (64 heads on 8) 1335, 64 830: rows of 192 and 80 channels take the time of 256 and 128.
template <int DP>
constexpr int kTile = DP == 256 ? 32 : 64;  // tokens of a tile
template <int DP>
constexpr int kKRow = DP + 8;   // 16-bit numbers from token to token: sixteen rows of 16 bytes lie in different banks
template <int DP>
constexpr int kWideV = DP + 32;  // four rows of 64 bytes do
template <int DP>
constexpr int kBuffer = kTile<DP> * (kKRow<DP> + kWideV<DP>);

template <int DT>
__device__ __forceinline__ floatx16_t mfma32(uint4 a, uint4 b, floatx16_t c) {
  if (DT == ESPARSE_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

template <int DT, int DP, int W>
__global__ void __launch_bounds__(64 * W, 2) k_attend_many(const AttendArgs a) {
  constexpr int TT = kTile<DP>, TB = TT / 32 /* 1 or 2 */, NS = DP / 16, ND = DP / 32, THREADS = 64 * W;
  constexpr int CH = TT * DP / 32;                       // pieces of 16 bytes (a block) of the keys of a tile, and of the values
  constexpr int ITEMS = (2 * CH + THREADS - 1) / THREADS;  // of a thread
  static_assert(CH % 64 == 0, "whole waves");
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ unsigned long long odd[2][2 * CH / 64];  // keys whose page is none, values without number
  uint16_t* buffers = reinterpret_cast<uint16_t*>(lds);
  const int wave = wave_uniform((int)(threadIdx.x >> 6)), lane = (int)(threadIdx.x & 63u), c = lane & 31, h = lane >> 5;
  // the tiles that see most first; neighbouring workgroups (which go to different L2s) take different heads
  const int head = (int)(blockIdx.x % (unsigned)a.Hkv), tile = a.tiles - 1 - (int)(blockIdx.x / (unsigned)a.Hkv);
  const Tile t = find_tile(a, tile, 32 * W);
  if (t.first >= (long long)t.queries * a.group) return;
  const int tiles = (t.end + TT - 1) / TT;
  const int32_t* table = a.table + (long long)t.b * a.width;

  const int row = t.first + 32 * wave + c, query = row / a.group;
  const bool live = query < t.queries;
  const int sees = live ? t.length - t.queries + query : -1;
  uint4 q[NS];
#pragma unroll
  for (int s = 0; s < NS; s++) {
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    const int ch = 16 * s + 8 * h;
    if (live) load_8(a.q + (t.start + query) * a.ldq + (long long)(head * a.group + row % a.group) * a.D + ch, a.D - ch, v);
    q[s] = uint4{oriented(a, v[0]), oriented(a, v[1]), oriented(a, v[2]), oriented(a, v[3])};
  }
  // the wave's rows see all tokens up to `all` and none from `most` on
  const int first_row = t.first + 32 * wave, last_row = min(first_row + 31, t.queries * a.group - 1);
  const bool any = first_row <= last_row;
  const int all = any ? t.length - t.queries + first_row / a.group : 0, most = any ? t.length - t.queries + last_row / a.group + 1 : 0;

  floatx16_t o[ND];
#pragma unroll
  for (int n = 0; n < ND; n++)
#pragma unroll
    for (int j = 0; j < 16; j++) o[n][j] = 0.f;
  float m = -__builtin_inff(), l = 0.f;
  bool beyond = false;  // (of some row of the wave)

  uint4 code[ITEMS];
  unsigned scl[ITEMS];
  bool there[ITEMS];
  auto fetch = [&](int i) {
#pragma unroll
    for (int it = 0; it < ITEMS; it++) {
      const int item = it * THREADS + (int)threadIdx.x, piece = item % CH, token = i * TT + piece / (DP / 32), block = piece % (DP / 32);
      const bool keys = item < CH;
      there[it] = false;
      code[it] = uint4{0u, 0u, 0u, 0u};
      scl[it] = 0;
      if (item < 2 * CH && token < t.end) {
        const int page = table[token >> a.page_bits];
        there[it] = page >= 0 && page < a.pages;
        if (there[it]) {
          const long long r = (((long long)page * a.Hkv + head) << a.page_bits) + (token & ((1 << a.page_bits) - 1));
          code[it] = *reinterpret_cast<const uint4*>((keys ? a.k_data : a.v_data) + r * (DP / 2) + 16 * block);
          scl[it] = (keys ? a.k_scales : a.v_scales)[r * (DP / 32) + block];
        }
      }
    }
  };
  auto put = [&](int buffer) {
    uint16_t* kb = buffers + buffer * kBuffer<DP>;
    uint16_t* vb = kb + TT * kKRow<DP>;
#pragma unroll
    for (int it = 0; it < ITEMS; it++) {
      const int item = it * THREADS + (int)threadIdx.x, piece = item % CH, token = piece / (DP / 32), block = piece % (DP / 32);
      if (item >= 2 * CH) break;
      const bool keys = item < CH, bad = keys ? !there[it] : scl[it] > kLargest<DT>;
      const unsigned long long marks = __ballot(bad);
      if (lane == 0) odd[buffer][item / 64] = marks;
      uint16_t* to = (keys ? kb + token * kKRow<DP> : vb + token * kWideV<DP>) + 32 * block;
      const float by = mx_scale(!keys && bad ? 0u : scl[it]);
      const uint32_t w[4] = {code[it].x, code[it].y, code[it].z, code[it].w};
#pragma unroll
      for (int j = 0; j < 4; j++) *reinterpret_cast<uint4*>(to + 8 * j) = mx_widen<DT>(!keys && bad ? 0u : w[j], by);
    }
  };
  if (tiles > 0) {
    fetch(0);
    put(0);
    fetch(1);
  }
  for (int i = 0; i < tiles; i++) {
    __syncthreads();
    if (i + 1 < tiles) {
      put((i + 1) & 1);
      fetch(i + 2);
    }
    const int begin = i * TT;
    if (begin >= most) continue;
    const uint16_t* kb = buffers + (i & 1) * kBuffer<DP>;
    const uint16_t* vb = kb + TT * kKRow<DP>;
    floatx16_t x[TB];
#pragma unroll
    for (int b = 0; b < TB; b++) {
#pragma unroll
      for (int j = 0; j < 16; j++) x[b][j] = 0.f;
#pragma unroll
      for (int s = 0; s < NS; s++) x[b] = mfma32<DT>(*reinterpret_cast<const uint4*>(kb + (32 * b + c) * kKRow<DP> + 16 * s + 8 * h), q[s], x[b]);
    }
    if constexpr (TB == 2) settle(x[0], x[1]);
    else settle(x[0]);
    unsigned long long gone = 0, none = 0;
#pragma unroll
    for (int w = 0; w < CH / 64; w++) gone |= odd[i & 1][w], none |= odd[i & 1][CH / 64 + w];
    if (begin + TT - 1 > all || wave_uniform((int)(gone != 0))) {
#pragma unroll
      for (int b = 0; b < TB; b++)
#pragma unroll
        for (int j = 0; j < 16; j++) {
          const int at = 32 * b + 8 * (j / 4) + 4 * h + j % 4, piece = at * (DP / 32);
          if (begin + at > sees || (odd[i & 1][piece / 64] >> (piece % 64) & 1ull)) x[b][j] = -__builtin_inff();
        }
    }
    float top = m;
#pragma unroll
    for (int b = 0; b < TB; b++)
#pragma unroll
      for (int j = 0; j < 16; j++) top = fmaxf(top, x[b][j]);
    top = half_max(top);
    const float base = top == -__builtin_inff() ? 0.f : top;
    float scaled = base * a.c;
    if (__ballot(top > m) || beyond) {
      const float shrink = __builtin_amdgcn_exp2f((m - base) * a.c);
      l *= shrink;
#pragma unroll
      for (int n = 0; n < ND; n++)
#pragma unroll
        for (int j = 0; j < 16; j++) o[n][j] *= shrink;
      m = top;
      const bool row_beyond = !(fabsf(scaled) < NEAR);
      beyond = __ballot(row_beyond) != 0;
      if (__builtin_expect(beyond, 0)) {
        const float off = row_beyond ? base : 0.f;
#pragma unroll
        for (int b = 0; b < TB; b++)
#pragma unroll
          for (int j = 0; j < 16; j++) x[b][j] -= off;
        scaled = row_beyond ? 0.f : scaled;
      }
    }
    uint4 p[2 * TB];
#pragma unroll
    for (int b = 0; b < TB; b++) {
#pragma unroll
      for (int j = 0; j < 16; j++) {
        x[b][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][j], a.c, kOffset<DT> - scaled));
        l += x[b][j];
      }
#pragma unroll
      for (int s = 0; s < 2; s++)
        p[2 * b + s] = uint4{pack_2<DT>(x[b][8 * s], x[b][8 * s + 1]), pack_2<DT>(x[b][8 * s + 2], x[b][8 * s + 3]), pack_2<DT>(x[b][8 * s + 4], x[b][8 * s + 5]),
                             pack_2<DT>(x[b][8 * s + 6], x[b][8 * s + 7])};
    }
#pragma unroll
    for (int n = 0; n < ND; n++)
#pragma unroll
      for (int s = 0; s < 2 * TB; s++) {
        const uint16_t* at = vb + (16 * s + 4 * h + ((lane & 15) >> 2)) * kWideV<DP> + 32 * n + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        const uint2 lo = read_transposed(at), hi = read_transposed(at + 8 * kWideV<DP>);
        o[n] = mfma32<DT>(uint4{lo.x, lo.y, hi.x, hi.y}, p[s], o[n]);
      }
    if (wave_uniform((int)(none != 0))) {  // blocks without number: NaN for the rows that see them
#pragma unroll
      for (int n = 0; n < ND; n++) settle(o[n]);
      for (int w = 0; w < CH / 64; w++)
        for (unsigned long long left = odd[i & 1][CH / 64 + w]; left; left &= left - 1) {
          const int piece = 64 * w + (int)__builtin_ctzll(left);
          if (begin + piece / (DP / 32) <= sees) {
#pragma unroll
            for (int n = 0; n < ND; n++)
              if (n == piece % (DP / 32))
#pragma unroll
                for (int j = 0; j < 16; j++) o[n][j] = __builtin_nanf("");
          }
        }
    }
  }
#pragma unroll
  for (int n = 0; n < ND; n++) settle(o[n]);
  l = half_sum(l);
  if (!live) return;
  const Sums of_row = sums_of<DT>(a, l, m);
  const long long place = (t.start + query) * ((long long)a.Hkv * a.group) + head * a.group + row % a.group;
#pragma unroll
  for (int n = 0; n < ND; n++)
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
      const int ch = 32 * n + 8 * (j / 4) + 4 * h;
      uint16_t* to = a.out + place * a.D + ch;
      const uint32_t v[2] = {pack_2<DT>(o[n][j] * of_row.by, o[n][j + 1] * of_row.by), pack_2<DT>(o[n][j + 2] * of_row.by, o[n][j + 3] * of_row.by)};
      if (ch + 4 <= a.D) {
        store_8(to, v);
      } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
          if (ch + e < a.D) to[e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
      }
    }
  if (a.lse && h == 0) a.lse[place] = of_row.lse;
  if (no_number(a, l, table, t.end, sees)) {
    for (int ch = 4 * h; ch < a.D; ch += 8)  // (those that this lane has written)
      for (int e = 0; e < 4; e++)
        if (ch + e < a.D) a.out[place * a.D + ch + e] = NAN16;
    if (a.lse && h == 0) a.lse[place] = __builtin_nanf("");
  }
}

long long tiles_of(long long T, int B, int group, bool ragged, int rows) {
  return ragged ? T * group / rows + B : (long long)B * ((group + rows - 1) / rows);
}
// pieces that a sequence is cut into at most: until the workgroups fill the chip, for the longest that the table has room for
int most_pieces(long long items, long long tokens) {
  const long long strips = (tokens + STRIP - 1) / STRIP, longest = (strips + LEAST - 1) / LEAST, want = items >= 256 ? (4096 + items - 1) / items : (1024 + items - 1) / items;
  return (int)std::max<long long>(1, std::min({longest, want, (long long)MOST_PIECES}));
}

}  // namespace

// Waves of a workgroup of the kernel for many rows (128 or 256 rows), 0: the kernel for few rows.  Both take a time that grows with the lengths, which are not known here.  The kernel for few rows
// spreads any number of rows over the chip by cutting the tokens into pieces, the other needs workgroups: one sequence of 8192 tokens, 64 heads on 8 of 128 channels, with 16, 64,
// 256, 512, 1024 queries 30, 76, 206, 363, 557 us against 296, 305, 304, 304, 327; 16 heads on 4 of 256 channels with 16, 256, 1024 queries 25, 171, 485 against 900 throughout.
// So by the number of tiles of sixteen rows; and of few rows for each sequence most of a tile of 128 would be empty.  Both this and the number of pieces go by a batch's averages: one prompt of 4096
// tokens with 47 single tokens over 2000 each takes 476 us (64 heads on 8), in two calls 372 + 39; one token over 131072 with 47 over 500 each 166 us, in two calls 40 + 21.
constexpr long long MANY_ROWS = 64, MOST_ROWS = 1024;
int waves_of_many(long long T, int B, int group, int Hkv, int row, bool ragged) {
  const long long each = ragged ? T * group / B : group, tiles = (T * group + ROWS - 1) / ROWS * Hkv;
  if (each < MANY_ROWS || tiles < (row == 256 ? 2048 : 1536)) return 0;
  return each >= MOST_ROWS && tiles_of(T, B, group, ragged, 256) * Hkv >= 256 ? 8 : 4;
}

size_t esp_cache_attention_workspace(const esparse_cache* cache, long long T, int B, int q_heads, long long width, bool ragged) {
  const int group = q_heads / cache->heads, dp = esp_cache_row(cache->head_dim);
  if (waves_of_many(T, B, group, cache->heads, dp, ragged)) return 0;
  const long long items = tiles_of(T, B, group, ragged, ROWS) * cache->heads;
  const int pieces = most_pieces(items, width * cache->page);
  return pieces == 1 ? 0 : (size_t)items * pieces * (ROWS * dp + 2 * ROWS) * sizeof(float);
}

int esp_cache_attention_device(esparse_ctx* ctx, const void* q, long long ldq, long long T, int q_heads, int dtype, const esparse_cache* cache,
                               const int32_t* table, long long width, const int32_t* lengths, const int32_t* starts, int B, double scale, void* out, float* lse,
                               void* workspace) {
  AttendArgs a = {};
  a.q = (const uint16_t*)q;
  a.k_data = (const unsigned char*)cache->k_data, a.k_scales = (const unsigned char*)cache->k_scales;
  a.v_data = (const unsigned char*)cache->v_data, a.v_scales = (const unsigned char*)cache->v_scales;
  a.table = table, a.lengths = lengths, a.starts = starts;
  a.out = (uint16_t*)out, a.lse = lse, a.partial = (float*)workspace;
  a.ldq = ldq, a.T = T, a.pages = cache->pages, a.width = width;
  a.B = B, a.Hkv = cache->heads, a.group = q_heads / cache->heads, a.D = cache->head_dim, a.page_bits = __builtin_ctz((unsigned)cache->page);
  a.c = (float)std::fabs(scale * 1.4426950408889634);
  a.natural = (float)std::fabs(scale);
  a.flip = scale < 0 ? 0x80008000u : 0u;
  a.keep = a.c == 0.f ? 0u : ~0u;
  if (a.c == 0.f) a.c = 1.f;
  const int row = esp_cache_row(a.D);
  if (const int waves = waves_of_many(T, B, a.group, a.Hkv, row, starts != nullptr)) {
    a.tiles = (int)tiles_of(T, B, a.group, starts != nullptr, 32 * waves);
    const dim3 grid((unsigned)a.tiles * (unsigned)a.Hkv);
#define GO(DT, DP, W)                                                                            \
  {                                                                                              \
    static std::atomic<unsigned long long> done{0};                                              \
    constexpr size_t bytes = (size_t)2 * kBuffer<DP> * 2;                                        \
    ESP_HIP(ctx, raise_dynamic_lds(done, ctx->device, &k_attend_many<DT, DP, W>, bytes));        \
    hipLaunchKernelGGL((k_attend_many<DT, DP, W>), grid, dim3(64 * W), bytes, ctx->stream, a);   \
  }
#define ROW(DT, W)                  \
  {                                 \
    if (row == 64) GO(DT, 64, W)    \
    else if (row == 128) GO(DT, 128, W) \
    else GO(DT, 256, W)             \
  }
    if (dtype == ESPARSE_F16) {
      if (waves == 8) ROW(ESPARSE_F16, 8)
      else ROW(ESPARSE_F16, 4)
    } else {
      if (waves == 8) ROW(ESPARSE_BF16, 8)
      else ROW(ESPARSE_BF16, 4)
    }
#undef ROW
#undef GO
    ESP_HIP(ctx, hipGetLastError());
    return ESPARSE_OK;
  }
  const long long tiles = tiles_of(T, B, a.group, starts != nullptr, ROWS);
  a.tiles = (int)tiles;
  a.pieces = most_pieces(tiles * a.Hkv, width * cache->page);
  a.rows = starts ? ROWS : std::min(ROWS, a.group);
  const dim3 grid((unsigned)(tiles * a.Hkv * a.pieces));
#define GO(DT, DP)                                                                                                                 \
  {                                                                                                                                \
    static std::atomic<unsigned long long> done{0};                                                                                \
    constexpr size_t bytes = (size_t)WAVES * STRIP * kVRow<DP> * 2;                                                                \
    ESP_HIP(ctx, raise_dynamic_lds(done, ctx->device, &k_attend_few<DT, DP>, bytes));                                              \
    hipLaunchKernelGGL((k_attend_few<DT, DP>), grid, dim3(64 * WAVES), bytes, ctx->stream, a);                                     \
    if (a.pieces > 1) hipLaunchKernelGGL((k_attend_join<DT, DP>), dim3((unsigned)(tiles * a.Hkv * a.rows)), dim3(256), 0, ctx->stream, a);  \
  }
  if (dtype == ESPARSE_F16) {
    if (row == 64) GO(ESPARSE_F16, 64)
    else if (row == 128) GO(ESPARSE_F16, 128)
    else GO(ESPARSE_F16, 256)
  } else {
    if (row == 64) GO(ESPARSE_BF16, 64)
    else if (row == 128) GO(ESPARSE_BF16, 128)
    else GO(ESPARSE_BF16, 256)
  }
#undef GO
  ESP_HIP(ctx, hipGetLastError());
  return ESPARSE_OK;
}
