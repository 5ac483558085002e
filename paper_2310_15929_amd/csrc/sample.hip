// A token drawn from each row of logits (include/esparse.h): w_i = exp((x_i - max) / temperature); top-k, top-p and min-p each keep a beginning of the order "larger
// first, equal ones by index"; the token is the first, by index, up to which more than u of the kept sum has come.
//
// Nothing is sorted.  k_pieces, a workgroup for each piece of a row, reads the row once and leaves the piece's maximum and, for 256 ranges of x (an eighth of a doubling of
// the weight wide, on a grid that all pieces share, counted down from the range of the maximum; the last one holds all the rest), how many values or how much weight lie
// in each.  k_rows, a workgroup a row, adds these up and then
//   with top_k up to MOST, or where the values above the range that the first cut falls in fit a list: puts those into a list in LDS (one more read of the row) and does the rest there,
//   else: lists the values of the range that a cut falls in alone, learns from the pieces' ranges what each piece keeps, and reads one piece to find the token.
// A cut in a list is found by counting its values in 256 parts of their span, then in the part where the cut falls, until 64 are left, which a wave compares with each other.  The
// same search over the indices draws the token.
// A token's share of a large vocabulary is small beside 2^-24: weights are exponentials in 64 bits (float64 runs at the rate of float32 here), sums are of whole
// numbers or in float64 in a fixed order: results do not depend on chance.  What is lost: 2^-47 of each exponential; half of 2^-48 of the piece's largest weight where a weight is added to a
// piece's range (V 2^-49 of the row's largest in all); half of 2^-(62 - index bits) where a range is added to the row's (of up to 2^16 ranges that hold something: V 2^-46); 2^-40 of a weight in the
// range that a cut falls in.
// Measured: 1 x 32000 f16 with top_k 50 and top_p 0.9 3 + 17 us, 64 x 131072 bf16 with top_p 0.95 17 + 52, 777 x 50021 f32 with top_k 1000 and both others 32 (4.9 TB/s) + 137.  k_rows is bound by
// the chain of its steps - loads, a search, barriers - and by the one compute unit that reads a row (64 KB in 4 us, a hundred instructions for eight values); spilled registers cost
// it more than fewer waves (1024 threads with 128 registers: 64 us instead of 52).  With 512 threads of 176 to 211 registers a compute unit holds one row at a time: 777 rows are three rounds of 256 and a
// fourth of nine.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx.h"

namespace {

constexpr int BINS = 256;
constexpr int NT = 512;        // threads of a row (8 for each of the 64 elements that are compared with each other)
constexpr int PT = 512;        // threads of a piece
constexpr int LIST = 3328;     // values that a list holds
constexpr int MOST = 2048;     // with top_k up to this the pieces count values and leave their weights to the list
constexpr int COPIES = 4;      // of a piece's ranges, for neighbouring lanes: additions to one place wait for each other (64 x 131072 equal values 586 -> 568 us; no difference where they are spread)
constexpr double STEPS = 8.;   // ranges for each doubling of the weight
constexpr double LOG2E = 1.4426950408889634;

struct SampleArgs {
  const void* logits;
  long long R, V, ld;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  long long* tokens;
  float* logprob;
  // of each piece
  unsigned long long* weight;  // [R][pieces][BINS]
  uint32_t* count;             // [R][pieces][BINS]
  float* top;                  // [R][pieces] the largest value; NaN: a value of the piece is NaN or plus infinity
  int32_t* where;              // [R][pieces] index of the first of the largest
  int pieces, per;             // pieces of a row, values of a piece
};

// eight values from place i on (left of them: the rest is minus infinity)
template <int DT>
__device__ __forceinline__ void load_values(const void* row, long long i, long long left, float (&x)[8]) {
  if constexpr (DT == ESPARSE_F32) {
    const float* p = reinterpret_cast<const float*>(row) + i;
    if (left >= 8) {
      __builtin_memcpy(x, p, 32);
    } else {
#pragma unroll
      for (int j = 0; j < 8; j++) x[j] = j < left ? p[j] : -__builtin_inff();
    }
  } else {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + i;
    uint32_t v[4];
    load_8(p, left, v);
#pragma unroll
    for (int j = 0; j < 4; j++) {
      x[2 * j] = esp_to_float<DT>((uint16_t)v[j]);
      x[2 * j + 1] = esp_to_float<DT>((uint16_t)(v[j] >> 16));
    }
    if (left < 8) {
#pragma unroll
      for (int j = 0; j < 8; j++)
        if (j >= left) x[j] = -__builtin_inff();
    }
  }
}

// 2^y for y <= 0, to 2^-47 (below 2^-1022 to the numbers there are): e^(r ln 2) by its series to the 11th power, |r| <= 1/2
__device__ __forceinline__ double exp2_of(double y) {
  if (!(y > -1100.)) return 0.;
  const double n = __builtin_rint(y), z = (y - n) * 0.6931471805599453;
  double s = 1. / 39916800.;
  s = __builtin_fma(s, z, 1. / 3628800.);
  s = __builtin_fma(s, z, 1. / 362880.);
  s = __builtin_fma(s, z, 1. / 40320.);
  s = __builtin_fma(s, z, 1. / 5040.);
  s = __builtin_fma(s, z, 1. / 720.);
  s = __builtin_fma(s, z, 1. / 120.);
  s = __builtin_fma(s, z, 1. / 24.);
  s = __builtin_fma(s, z, 1. / 6.);
  s = __builtin_fma(s, z, 0.5);
  s = __builtin_fma(s, z, 1.);
  s = __builtin_fma(s, z, 1.);
  return __builtin_ldexp(s, (int)n);
}

// the scale of the exponents; 0: the largest is taken; NaN: no temperature
__device__ __forceinline__ double per_doubling(const SampleArgs& a, long long r) {
  if (!a.temperature) return LOG2E;
  const float t = a.temperature[r];
  if (t == 0.f) return 0.;
  return t > 0.f && t < __builtin_inff() ? LOG2E / (double)t : (double)__builtin_nanf("");
}

// The range of x is floor(8 x scale), in 32 bits: it grows with x, which is all that is asked of it
__device__ __forceinline__ float range_step(double scale) { return fminf((float)(scale * STEPS), 3.4028234663852886e38f); }
__device__ __forceinline__ float range_of(float x, float step) { return __builtin_floorf(fminf(fmaxf(x * step, -0x1p100f), 0x1p100f)); }
__device__ __forceinline__ int bin_of(float x, float high, float step) {
  const float d = high - range_of(x, step);
  return d < (float)(BINS - 1) ? (int)d : BINS - 1;
}
// whether the pieces of a row count values, and whether they add weights
__device__ __forceinline__ bool counts(long long k) { return k > 0; }
__device__ __forceinline__ bool weighs(long long k) { return k <= 0 || k > MOST; }

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// V8: eights of values of a thread
template <int DT, int V8>
__global__ void __launch_bounds__(PT) k_pieces(const SampleArgs a) {
  __shared__ unsigned long long weight[COPIES][BINS + 1];
  __shared__ uint32_t count[COPIES][BINS + 1];
  __shared__ float tops[PT / 64];
  __shared__ int first, bad;
  const long long r = blockIdx.x / (unsigned)a.pieces;
  const int piece = (int)(blockIdx.x % (unsigned)a.pieces);
  const long long begin = (long long)piece * a.per, left = a.V - begin < a.per ? a.V - begin : a.per;
  const void* row = reinterpret_cast<const unsigned char*>(a.logits) + (r * a.ld + begin) * (DT == ESPARSE_F32 ? 4 : 2);
  for (int i = (int)threadIdx.x; i < COPIES * (BINS + 1); i += PT) (&weight[0][0])[i] = 0ull, (&count[0][0])[i] = 0u;
  if (threadIdx.x == 0) first = 0x7fffffff, bad = 0;
  float x[V8][8];
  float top = -__builtin_inff();
  bool none = false;
#pragma unroll
  for (int v = 0; v < V8; v++) {
    const int at = (v * PT + (int)threadIdx.x) * 8;
    load_values<DT>(row, at, left - at, x[v]);
#pragma unroll
    for (int j = 0; j < 8; j++) {
      none |= !(x[v][j] < __builtin_inff());
      top = fmaxf(top, x[v][j]);
    }
  }
  top = wave_max(top);
  if ((threadIdx.x & 63u) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  if (none) bad = 1;
#pragma unroll
  for (int w = 0; w < PT / 64; w++) top = fmaxf(top, tops[w]);
  const double scale = per_doubling(a, r);
  const long long k = a.top_k ? a.top_k[r] : 0;
  if (top > -__builtin_inff()) {
    const float step = range_step(scale), high = range_of(top, step);
    int own = 0x7fffffff;
#pragma unroll
    for (int v = V8 - 1; v >= 0; v--)
#pragma unroll
      for (int j = 7; j >= 0; j--)
        if (x[v][j] == top) own = (v * PT + (int)threadIdx.x) * 8 + j;
    if (own != 0x7fffffff) atomicMin(&first, own);
    if (scale > 0. && counts(k)) {
#pragma unroll
      for (int v = 0; v < V8; v++)
#pragma unroll
        for (int j = 0; j < 8; j++)
          if (x[v][j] > -__builtin_inff() && x[v][j] <= top) atomicAdd(&count[threadIdx.x % COPIES][bin_of(x[v][j], high, step)], 1u);
    }
    if (scale > 0. && weighs(k)) {
#pragma unroll
      for (int v = 0; v < V8; v++)
#pragma unroll
        for (int j = 0; j < 8; j++)
          if (x[v][j] > -__builtin_inff() && x[v][j] <= top) {
            const double w = exp2_of(((double)x[v][j] - (double)top) * scale);
            // w 2^48 rounded: the low bits of w + 16
            atomicAdd(&weight[threadIdx.x % COPIES][bin_of(x[v][j], high, step)], __builtin_bit_cast(unsigned long long, w + 16.) - __builtin_bit_cast(unsigned long long, 16.));
          }
    }
  }
  __syncthreads();
  const long long at = r * a.pieces + piece;
  if (threadIdx.x < BINS) {
    unsigned long long w = 0ull;
    uint32_t c = 0u;
#pragma unroll
    for (int i = 0; i < COPIES; i++) w += weight[i][threadIdx.x], c += count[i][threadIdx.x];
    if (weighs(k)) a.weight[at * BINS + threadIdx.x] = w;
    if (counts(k)) a.count[at * BINS + threadIdx.x] = c;
  }
  if (threadIdx.x == 0) {
    a.top[at] = bad ? __builtin_nanf("") : top;
    a.where[at] = (int32_t)(begin + first);
  }
}

// values in their order as whole numbers (minus 0 is 0)
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
typedef unsigned long long u64;

struct Row {
  const void* logits;
  long long V;
  float top, step, high;
  int index_bits;
  double scale;
  double unit;  // what a weight is multiplied with for the sums of the row's ranges: these stay below 2^63
};
__device__ __forceinline__ double weight_of(const Row& r, float x) { return exp2_of(((double)x - (double)r.top) * r.scale); }

// Rank of a value: its key, without the bits that are the same for all numbers of the type, and behind it its index, counted down: larger ranks come first in the order.
// (Short ranks are told apart by few of their bits: a cut is found in one or two steps)
template <int DT>
constexpr int kDropped = DT == ESPARSE_F16 ? 13 : (DT == ESPARSE_BF16 ? 16 : 0);
template <int DT>
__device__ __forceinline__ u64 rank_of(const Row& r, float x, uint32_t index) {
  return (u64)(key_of(x) >> kDropped<DT>) << r.index_bits | (((1u << r.index_bits) - 1u) - index);
}
template <int DT>
__device__ __forceinline__ uint32_t key_at(const Row& r, u64 rank) {  // (the dropped bits: 0 of positive numbers, 1 of negative ones)
  const uint32_t k = (uint32_t)(rank >> r.index_bits) << kDropped<DT>;
  return k & 0x80000000u ? k : k | ((1u << kDropped<DT>) - 1u);
}
template <int DT>
__device__ __forceinline__ float value_at(const Row& r, u64 rank) {
  return value_of(key_at<DT>(r, rank));
}
__device__ __forceinline__ uint32_t index_at(const Row& r, u64 rank) {
  const uint32_t all = (1u << r.index_bits) - 1u;
  return all - ((uint32_t)rank & all);
}
// the smallest rank that a number with this key or a larger one can have
template <int DT>
__device__ __forceinline__ u64 rank_from(const Row& r, uint32_t key) {
  const uint32_t ones = (1u << kDropped<DT>) - 1u;
  const u64 k = key & 0x80000000u ? ((u64)key + ones) >> kDropped<DT> : key >> kDropped<DT>;
  return k << r.index_bits;
}

// f(values, index of the first) for the values of a row, eight in a row for a thread (behind the end: minus infinity).  A row is read by one compute unit, which waits for memory
// most of the time: a thread's next loads, 128 bytes of them, are on their way while it looks at the last
template <int DT, class F>
__device__ __forceinline__ void each_eight(const Row& r, F f) {
  constexpr int EACH = DT == ESPARSE_F32 ? 4 : 2, AHEAD = DT == ESPARSE_F32 ? 4 : 8, WORDS = 2 * EACH;
  const unsigned char* p = reinterpret_cast<const unsigned char*>(r.logits);
  const uint32_t full = (uint32_t)(r.V / 8);
  uint32_t raw[AHEAD][WORDS];
  auto fetch = [&](uint32_t b, int h) {
    const uint32_t i = b < full ? b : full - 1u;
    __builtin_memcpy(raw[h], p + (long long)i * (8 * EACH), 8 * EACH);
  };
  if (full) {
#pragma unroll
    for (int h = 0; h < AHEAD; h++) fetch(threadIdx.x + h * NT, h);
  }
  for (uint32_t b0 = 0; b0 < full; b0 += AHEAD * NT) {
#pragma unroll
    for (int h = 0; h < AHEAD; h++) {
      const uint32_t b = b0 + h * NT + threadIdx.x;
      if (b0 + h * NT >= full) break;
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; j++) {
        if constexpr (DT == ESPARSE_F32) x[j] = __builtin_bit_cast(float, raw[h][j]);
        else x[j] = esp_to_float<DT>((uint16_t)(raw[h][j / 2] >> (16 * (j & 1))));
      }
      if (b0 + (AHEAD + h) * NT < full) fetch(b + AHEAD * NT, h);
      if (b < full) f(x, b * 8u);
    }
  }
  if (threadIdx.x == 0 && full * 8ll < r.V) {
    float x[8];
    load_values<DT>(p + full * 8ll * EACH, 0, r.V - full * 8ll, x);
    f(x, full * 8u);
  }
}
// f(value, index) for those from `from` to `to`, one after the other (little code; where it is long, a kernel that runs once waits for its instructions)
template <int DT, class F>
__device__ __forceinline__ void each_between(const Row& r, float from, float to, F f) {
  constexpr int EACH = DT == ESPARSE_F32 ? 4 : 2;
  for (long long at = (long long)threadIdx.x * 8; at < r.V; at += NT * 8) {
    float x[8];
    load_values<DT>(reinterpret_cast<const unsigned char*>(r.logits) + at * EACH, 0, r.V - at, x);
    uint32_t in = 0;
#pragma unroll
    for (int j = 0; j < 8; j++) in |= (x[j] >= from && x[j] <= to ? 1u : 0u) << j;
    for (; in; in &= in - 1u) {
      const int j = (int)__builtin_ctz(in);
      float v = x[0];
#pragma unroll
      for (int e = 1; e < 8; e++) v = j == e ? x[e] : v;
      f(v, (uint32_t)at + (uint32_t)j);
    }
  }
}

struct Shared {
  u64 rank[LIST];      // the list: values with their index
  u64 weight[LIST];    // their weights as whole numbers
  u64 part_weight[BINS];
  uint32_t part_count[BINS];
  u64 row_weight[BINS];
  uint32_t row_count[BINS];
  u64 few[64], few_weight[64];
  double share[BINS];  // of the pieces: the weight of their maxima, how far their ranges are moved
  int moved[BINS];
  double wave[NT / 64];
  u64 sum, least, cut_last, cut_kept;
  int listed, fews, token, latest;
};

__device__ __forceinline__ u64 wave_sum(u64 v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ u64 wave_min(u64 v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    const u64 w = __shfl_xor(v, o);
    v = w < v ? w : v;
  }
  return v;
}

// the values from `from` to `to` of a row into the list (s.listed: how many there are; the first LIST are kept)
template <int DT>
__device__ __forceinline__ void collect(const Row& r, Shared& s, float from, float to) {
  each_eight<DT>(r, [&](const float (&x)[8], uint32_t i) {
    uint32_t in = 0;
#pragma unroll
    for (int j = 0; j < 8; j++) in |= (x[j] >= from && x[j] <= to ? 1u : 0u) << j;
    if (!in) return;
    int at = atomicAdd(&s.listed, (int)__popc(in));
    for (; in; in &= in - 1u, at++) {
      const int j = (int)__builtin_ctz(in);
      float v = x[0];
#pragma unroll
      for (int e = 1; e < 8; e++) v = j == e ? x[e] : v;
      if (at < LIST) s.rank[at] = rank_of<DT>(r, v, i + j);
    }
  });
}

// Every wave for itself, 4 of the 256 parts a lane: the first part that holds something and up to which `need` has come (the last that holds anything where none reaches it;
// -1: all are empty), with what came before it.
template <class T, class U>
struct Pick {
  int part;
  T before;  // of what is counted
  U other;   // of the companion
};
template <class T, class U, class A, class B>
__device__ __forceinline__ Pick<T, U> pick(A value, B other, T need) {
  const int lane = (int)(threadIdx.x & 63u);
  T v[4], sum = 0;
  U o[4], osum = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    v[i] = value(4 * lane + i);
    o[i] = other(4 * lane + i);
    sum += v[i];
    osum += o[i];
  }
  T upto = sum;
  U oupto = osum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T a = __shfl_up(upto, d);
    const U b = __shfl_up(oupto, d);
    if (lane >= d) upto += a, oupto += b;
  }
  T c = upto - sum, hit_c = 0, last_c = 0;
  U w = oupto - osum, hit_w = 0, last_w = 0;
  int hit = -1, last = -1;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (v[i] > 0) {
      last = 4 * lane + i, last_c = c, last_w = w;
      if (hit < 0 && c + v[i] >= need) hit = last, hit_c = c, hit_w = w;
    }
    c += v[i];
    w += o[i];
  }
  const u64 hits = __ballot(hit >= 0), lasts = __ballot(last >= 0);
  if (hits) {
    const int from = (int)__builtin_ctzll(hits);
    return {__shfl(hit, from), __shfl(hit_c, from), __shfl(hit_w, from)};
  }
  if (lasts) {
    const int from = 63 - (int)__builtin_clzll(lasts);
    return {__shfl(last, from), __shfl(last_c, from), __shfl(last_w, from)};
  }
  return {-1, 0, 0};
}

// A cut in an order, larger keys first: what it leaves are the keys from `last` on, their weight is `kept`
struct Cut {
  u64 last, kept;
};
// Of the first n of the list those of rank `floor` or more, in the order of their ranks' bits in `mask`, which lie in [lo, hi), `inside` of them at most.  By weight: those are kept before which
// less than `need` has come, else the first `need`.
__device__ __forceinline__ Cut find_cut(Shared& s, int n, u64 floor, u64 mask, u64 lo, u64 hi, u64 inside, bool by_weight, u64 need) {
  u64 came = 0, weight = 0;  // in front of hi
#pragma unroll 1
  for (;;) {
    const bool few = inside <= 64;
    const u64 span = hi - lo;
    const int bits = 64 - (int)__builtin_clzll((span - 1) | 1ull), shift = bits > 8 ? bits - 8 : 0;
    if (threadIdx.x < BINS) s.part_weight[threadIdx.x] = 0ull, s.part_count[threadIdx.x] = 0u;
    if (threadIdx.x == 0) s.fews = 0, s.cut_last = ~0ull, s.cut_kept = 0ull;
    __syncthreads();
#pragma unroll 1
    for (int i = (int)threadIdx.x; i < n; i += NT) {
      const u64 rank = s.rank[i], key = rank & mask, w = s.weight[i];
      if (rank >= floor && key >= lo && key < hi) {
        if (few) {
          const int at = atomicAdd(&s.fews, 1);
          if (at < 64) s.few[at] = key, s.few_weight[at] = w;
        } else {
          const int at = (int)((hi - 1 - key) >> shift);
          atomicAdd(&s.part_weight[at], w);
          atomicAdd(&s.part_count[at], 1u);
        }
      }
    }
    __syncthreads();
    if (few) {
      const int m = s.fews < 64 ? s.fews : 64;
      // every element against all others: 8 lanes for one, eight of the others each
      const int one = (int)(threadIdx.x >> 3), part = (int)(threadIdx.x & 7u);
      const u64 mine = s.few[one];
      u64 before = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const int other = 8 * part + i;
        if (other < m && s.few[other] > mine) before += by_weight ? s.few_weight[other] : 1ull;
      }
#pragma unroll
      for (int o = 4; o; o >>= 1) before += __shfl_xor(before, o);
      if (part == 0 && one < m && came + before < need) {
        atomicMin(&s.cut_last, mine);
        atomicAdd(&s.cut_kept, s.few_weight[one]);
      }
      __syncthreads();
      const Cut r = {s.cut_last < hi ? s.cut_last : hi, weight + s.cut_kept};
      __syncthreads();
      return r;
    }
    const Pick<u64, u64> p = pick<u64, u64>([&](int i) { return by_weight ? s.part_weight[i] : (u64)s.part_count[i]; }, [&](int i) { return s.part_weight[i]; }, need - came);
    if (p.part < 0) {  // elements without weight: none stands before another, all are kept
      __syncthreads();
      return {lo, weight};
    }
    const u64 inner_weight = s.part_weight[p.part];
    inside = s.part_count[p.part];
    came += p.before;
    weight += p.other;
    hi -= (u64)p.part << shift;
    lo = hi - lo > (1ull << shift) ? hi - (1ull << shift) : lo;
    __syncthreads();
    if (shift == 0 || (!by_weight && came + inside == need)) return {lo, weight + inner_weight};
  }
}

// Every wave for itself: the smallest key up to `most` for which yes() holds; it holds for `most` and for all above the first.  Looked for among 64 keys around a guess, and
// where that is too far off among all
template <class F>
__device__ __forceinline__ uint32_t first_key(uint32_t most, double guess, F yes) {
  constexpr uint32_t least = 0x00800000u;  // (the least number)
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t lo = least, hi = most;
  const uint32_t near = key_of((float)fmin(fmax(guess, -3.4028234663852886e38), (double)value_of(most)));
  if (near >= least + 32u && near <= most) {
    const u64 held = __ballot(near - 32u + lane > most || yes(value_of(near - 32u + lane)));
    if (held && !(held & 1ull)) {
      const uint32_t at = near - 32u + (uint32_t)__builtin_ctzll(held);
      return at < most ? at : most;
    }
  }
#pragma unroll 1
  while (lo < hi) {
    const uint32_t step = (hi - lo) / 64u + 1u, mine = hi - lo > lane * step ? lo + lane * step : hi;
    const u64 held = __ballot(yes(value_of(mine)));
    const uint32_t at = held ? (uint32_t)__builtin_ctzll(held) : 64u;
    const uint32_t below = at ? lo + (at - 1u) * step + 1u : lo;  // (the lane before the first does not hold)
    hi = at < 64u && hi - lo > at * step ? lo + at * step : hi;
    lo = below < hi ? below : hi;
  }
  return lo;
}

// whole numbers for the weights of a range: 2^40 to 2^41 for its largest
__device__ __forceinline__ double unit_of(int bin) { return __builtin_ldexp(1., 40 + bin / (int)STEPS); }

// Rows in which more values than the list takes are alike, seldom: the range [lo, hi) of a cut narrowed until its values fit; what came before it is returned in came and weight, how
// many are left in s.listed
template <int DT>
__device__ __forceinline__ void narrow(const Row& r, Shared& s, bool by_weight, u64 need, double unit, u64* lo_hi, u64* came_weight) {
  u64 lo = lo_hi[0], hi = lo_hi[1], came = 0, weight = 0, inside = ~0ull;
  while (inside > LIST) {
    const int bits = 64 - (int)__builtin_clzll((hi - lo - 1) | 1ull), shift = bits > 8 ? bits - 8 : 0;
    __syncthreads();
    if (threadIdx.x < BINS) s.part_weight[threadIdx.x] = 0ull, s.part_count[threadIdx.x] = 0u;
    __syncthreads();
    each_between<DT>(r, value_at<DT>(r, lo), value_at<DT>(r, hi - 1), [&](float x, uint32_t i) {
      const u64 rank = rank_of<DT>(r, x, i);
      if (rank >= lo && rank < hi) {
        const int at = (int)((hi - 1 - rank) >> shift);
        atomicAdd(&s.part_weight[at], (u64)__builtin_fma(weight_of(r, x), unit, 0.5));
        atomicAdd(&s.part_count[at], 1u);
      }
    });
    __syncthreads();
    Pick<u64, u64> p = pick<u64, u64>([&](int i) { return by_weight ? s.part_weight[i] : (u64)s.part_count[i]; }, [&](int i) { return s.part_weight[i]; }, need - came);
    if (p.part < 0) {  // nothing weighs anything: the last of them is as good as any
      const Pick<u64, u64> some = pick<u64, u64>([&](int i) { return (u64)s.part_count[i]; }, [&](int) { return 0ull; }, ~0ull);
      p = {some.part < 0 ? 0 : some.part, 0, 0};
    }
    inside = s.part_count[p.part];
    came += p.before;
    weight += p.other;
    hi -= (u64)p.part << shift;
    lo = hi - lo > (1ull << shift) ? hi - (1ull << shift) : lo;
  }
  __syncthreads();
  if (threadIdx.x == 0) s.listed = 0;
  __syncthreads();
  each_between<DT>(r, value_at<DT>(r, lo), value_at<DT>(r, hi - 1), [&](float x, uint32_t i) {
    const u64 rank = rank_of<DT>(r, x, i);
    if (rank >= lo && rank < hi) {
      const int at = atomicAdd(&s.listed, 1);
      if (at < LIST) s.rank[at] = rank;
    }
  });
  __syncthreads();
  lo_hi[0] = lo, lo_hi[1] = hi, came_weight[0] = came, came_weight[1] = weight;
}
// the weights of the ranges from the row itself (top_k small, and still too many values alike for the list)
template <int DT>
__device__ __forceinline__ void weigh_row(const Row& r, Shared& s) {
  if (threadIdx.x < BINS) s.part_weight[threadIdx.x] = 0ull;
  __syncthreads();
  each_between<DT>(r, -3.4028234663852886e38f, r.top, [&](float x, uint32_t) {
    const int bin = bin_of(x, r.high, r.step);
    atomicAdd(&s.part_weight[bin], (u64)__builtin_fma(weight_of(r, x), unit_of(bin), 0.5));
  });
  __syncthreads();
  if (threadIdx.x < BINS) s.row_weight[threadIdx.x] = (u64)((double)s.part_weight[threadIdx.x] * (r.unit / unit_of((int)threadIdx.x)));
  __syncthreads();
}
// the sum of what is kept, the same way
template <int DT>
__device__ __forceinline__ double sum_row(const Row& r, Shared& s, u64 last) {
  double sum = 0.;
  each_between<DT>(r, -3.4028234663852886e38f, r.top, [&](float x, uint32_t i) {
    if (rank_of<DT>(r, x, i) >= last) sum += weight_of(r, x);
  });
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63u) == 0) s.wave[threadIdx.x >> 6] = sum;
  __syncthreads();
  double total = 0.;
  for (int i = 0; i < NT / 64; i++) total += s.wave[i];
  __syncthreads();
  return total;
}

template <int DT>
__global__ void __launch_bounds__(NT) k_rows(const SampleArgs a) {
  __shared__ Shared s;
  const long long r = blockIdx.x;
  const float* tops = a.top + r * a.pieces;
  const int lane = (int)(threadIdx.x & 63u);
  const long long k = a.top_k ? a.top_k[r] : 0;
  const u64* pw = a.weight + r * a.pieces * BINS;
  const uint32_t* pc = a.count + r * a.pieces * BINS;
  // the first of what the pieces have left, asked for before it is known what it is for
  constexpr int EARLY = 8;
  u64 early_w[EARLY];
  uint32_t early_c[EARLY];
#pragma unroll
  for (int i = 0; i < EARLY; i++) {
    const int at = (int)threadIdx.x + i * NT, of = at < a.pieces * BINS ? at : 0;
    early_w[i] = weighs(k) ? pw[of] : 0ull;
    early_c[i] = counts(k) ? pc[of] : 0u;
  }
  Row row;
  row.logits = reinterpret_cast<const unsigned char*>(a.logits) + r * a.ld * (DT == ESPARSE_F32 ? 4 : 2);
  row.V = a.V;
  row.scale = per_doubling(a, r);
  bool bad = !(row.scale >= 0.);
  float top = -__builtin_inff();
  for (int p = lane; p < a.pieces; p += 64) {
    const float t = tops[p];
    bad |= t != t;
    top = fmaxf(top, t);
  }
  top = wave_max(top);
  if (__ballot(bad) || top == -__builtin_inff()) {
    if (threadIdx.x == 0) {
      a.tokens[r] = -1;
      if (a.logprob) a.logprob[r] = __builtin_nanf("");
    }
    return;
  }
  if (row.scale == 0.) {
    if (threadIdx.x == 0) {
      int p = 0;
      while (tops[p] != top) p++;
      a.tokens[r] = a.where[r * a.pieces + p];
      if (a.logprob) a.logprob[r] = 0.f;
    }
    return;
  }
  row.top = top;
  row.step = range_step(row.scale);
  row.high = range_of(top, row.step);
  row.index_bits = 32 - __builtin_clz((uint32_t)(a.V - 1) | 1u);
  row.unit = __builtin_ldexp(1., 62 - row.index_bits);
  const float given_p = a.top_p ? a.top_p[r] : 1.f, given_min = a.min_p ? a.min_p[r] : 0.f, given_u = a.u[r];
  const bool cut_p = given_p < 1.f, cut_min = given_min > 0.f;
  const double top_p = given_p > 0.f ? (double)given_p : 0., least = given_min < 1.f ? (double)given_min : 1.;
  const double u = given_u > 0.f ? (given_u < 1.f ? (double)given_u : 0x1.fffffep-1) : 0.;

  // the row's ranges: those of the pieces, each moved by the distance of the maxima
  const bool weighed = weighs(k);
  if (threadIdx.x < BINS) s.row_weight[threadIdx.x] = 0ull, s.row_count[threadIdx.x] = 0u;
  if (threadIdx.x < (unsigned)a.pieces) {
    const float t = tops[threadIdx.x];
    s.moved[threadIdx.x] = t > -__builtin_inff() ? (int)fminf(row.high - range_of(t, row.step), (float)BINS) : BINS;
    s.share[threadIdx.x] = weight_of(row, t);
  }
  if (threadIdx.x == 0) s.listed = 0, s.sum = 0ull, s.least = ~0ull, s.token = 0x7fffffff, s.latest = -1;
  __syncthreads();
  for (int at = (int)threadIdx.x, n = 0; at < a.pieces * BINS; at += NT, n++) {
    u64 w = 0ull;
    uint32_t c = 0u;
    if (n < EARLY) {
#pragma unroll
      for (int i = 0; i < EARLY; i++)
        if (i == n) w = early_w[i], c = early_c[i];
    } else {
      if (weighed) w = pw[at];
      if (counts(k)) c = pc[at];
    }
    const int p = at / BINS, bin = min(at % BINS + s.moved[p], BINS - 1);
    if (weighed && w) atomicAdd(&s.row_weight[bin], (u64)__builtin_fma((double)w * 0x1p-48 * s.share[p], row.unit, 0.5));
    if (counts(k) && c) atomicAdd(&s.row_count[bin], c);
  }
  __syncthreads();

  // Ranks of the values of a range: [first of the range, first of the range above it)
  auto begin_of = [&](int bin) {  // (all waves get the same)
    return rank_from<DT>(row, bin == BINS - 1 ? 0x00800000u : first_key(key_of(top), (double)(row.high - (float)bin) / (double)row.step, [&](float x) { return row.high - range_of(x, row.step) <= (float)bin; }));
  };
  const u64 past_top = rank_from<DT>(row, key_of(top)) + (1ull << row.index_bits);
  auto row_weights = [&](int i) { return s.row_weight[i]; };
  auto nothing = [](int) { return 0ull; };

  // where the first cut falls by number
  Pick<u64, u64> by_number = {-1, 0, 0};
  if (counts(k)) by_number = pick<u64, u64>([&](int i) { return (u64)s.row_count[i]; }, row_weights, (u64)k);
  const u64 upto = by_number.part >= 0 ? by_number.before + s.row_count[by_number.part] : 0ull;
  const bool cut_k = counts(k) && upto >= (u64)k, all_listed = counts(k) && upto <= LIST;  // (without the first: the row has fewer values than top_k)
  double total = 0.;  // of what is kept so far
  if (!all_listed) {
    if (!weighed) weigh_row<DT>(row, s);
    const Pick<u64, u64> all = pick<u64, u64>(row_weights, nothing, ~0ull);
    total = (double)(all.before + s.row_weight[all.part]) / row.unit;
  }

  // The cuts, one after the other, and the draw where all that may be kept is in the list
  u64 last = 0, drawn = 0;  // everything of rank `last` and above is kept
  int held = -1;            // the range in the list
  u64 all_sum = 0;
  constexpr double UNIT = 0x1p50;  // less than 2^12 weights of up to 1
#pragma unroll 1
  for (int phase = 0; phase < 3; phase++) {
    int bin = -1;
    u64 lo = 0, hi = ~0ull, need = 0, came = 0, before_weight = 0;
    double above = 0., unit = UNIT;
    const bool by_weight = phase > 0;
    bool fill = false;
    if (phase == 0) {
      if (!cut_k && !all_listed) continue;
      bin = by_number.part;
      need = (u64)k;
      fill = all_listed;
    } else if (phase == 1) {
      if (!cut_p) continue;
      if (all_listed) {
        const double target = __builtin_ceil(top_p * (double)all_sum);
        need = target > 1. ? (u64)target : 1ull;
        lo = last;
        hi = past_top;
      } else {
        const double target = top_p * total;
        const Pick<u64, u64> p = pick<u64, u64>(row_weights, nothing, (u64)__builtin_ceil(target * row.unit));
        bin = p.part;
        above = (double)p.before / row.unit;
        const double rest = __builtin_ceil((target - above) * unit_of(bin));
        need = rest > 1. ? (u64)rest : 1ull;
      }
    } else {
      if (!all_listed) break;
      // min-p, and the sum of what is kept
      u64 lowest = ~0ull, sum = 0;
      const int n = s.listed;
      if (cut_min) {
#pragma unroll 1
        for (int i = (int)threadIdx.x; i < n; i += NT)
          if (s.rank[i] >= last && s.rank[i] < lowest && weight_of(row, value_at<DT>(row, s.rank[i])) >= least) lowest = s.rank[i];
        lowest = wave_min(lowest);
        if (lane == 0) atomicMin(&s.least, lowest);
        __syncthreads();
        last = s.least > last ? s.least : last;
      }
#pragma unroll 1
      for (int i = (int)threadIdx.x; i < n; i += NT) sum += s.rank[i] >= last ? s.weight[i] : 0ull;
      sum = wave_sum(sum);
      if (lane == 0) atomicAdd(&s.sum, sum);
      __syncthreads();
      all_sum = s.sum;
      total = (double)all_sum * (1. / UNIT);
      need = (u64)(u * (double)all_sum) + 1ull;
      hi = 1ull << row.index_bits;
    }
    if (!all_listed) {
      lo = begin_of(bin);
      hi = bin == 0 ? past_top : begin_of(bin - 1);
      unit = unit_of(bin);
      if (phase == 0) {
        u64 sum = by_number.other;
        if (!weighed) {  // (the weights of the ranges were not known then)
          sum = 0ull;
          for (int b = lane; b < bin; b += 64) sum += s.row_weight[b];
          sum = wave_sum(sum);
        }
        above = (double)sum / row.unit;
        if (upto == (u64)k) {
          last = lo;
          total = above + (double)s.row_weight[bin] / row.unit;
          continue;
        }
        need = (u64)k - by_number.before;
      } else if (hi <= last) {  // top-k has kept less
        continue;
      }
      fill = held != bin;
    } else if (fill) {
      lo = begin_of(bin);
      hi = past_top;
    }
    if (fill) {
      __syncthreads();
      if (threadIdx.x == 0) s.listed = 0;
      __syncthreads();
      collect<DT>(row, s, value_at<DT>(row, lo), value_at<DT>(row, hi - 1));
      __syncthreads();
      held = bin;
      if (s.listed > LIST) {
        u64 range[2] = {lo, hi}, before[2];
        narrow<DT>(row, s, by_weight, need, unit, range, before);
        lo = range[0], hi = range[1], came = before[0], before_weight = before[1];
        held = -1;
      }
      const int n = s.listed;
#pragma unroll 1
      for (int i = (int)threadIdx.x; i < n; i += NT) {
        const double w = weight_of(row, value_at<DT>(row, s.rank[i]));
        const u64 v = (u64)__builtin_fma(w, unit, 0.5);
        s.weight[i] = v ? v : (w > 0. ? 1ull : 0ull);  // (what can be drawn is never nothing: u may be 0)
      }
      __syncthreads();
    }
    const Cut c = find_cut(s, s.listed, phase == 0 || !all_listed ? 0ull : last, phase == 2 ? (1ull << row.index_bits) - 1ull : ~0ull, lo, hi, (u64)s.listed, by_weight, need > came ? need - came : 1ull);
    if (phase == 2) {
      drawn = c.last;
      break;
    }
    if (phase == 0) {
      all_sum = c.kept;
      if (!all_listed) total = above + (double)(before_weight + c.kept) / unit;
    }
    last = c.last > last ? c.last : last;
  }
  if (all_listed) {
    for (int i = (int)threadIdx.x; i < s.listed; i += NT)
      if ((s.rank[i] & ((1ull << row.index_bits) - 1ull)) == drawn) {
        a.tokens[r] = (long long)index_at(row, drawn);
        if (a.logprob) a.logprob[r] = (float)(((double)value_at<DT>(row, s.rank[i]) - (double)top) * (row.scale * 0.6931471805599453) - log(total));
      }
    return;
  }
  if (cut_min) {
    const u64 at = rank_from<DT>(row, first_key(key_of(top), (double)top + log2(least) / row.scale, [&](float x) { return weight_of(row, x) >= least; }));
    last = at > last ? at : last;
  }

  // what each piece keeps of the range that the cut is in, and of those above it
  long long begin = 0, end = a.V;
  double rest = 0.;
  if (weighed) {
    const int edge = last ? bin_of(value_at<DT>(row, last), row.high, row.step) : BINS;  // no cut: all ranges
    const double unit = unit_of(edge < BINS ? edge : 0);
    u64* part = s.part_weight;                           // [pieces]
    double* kept = reinterpret_cast<double*>(s.weight);  // [pieces]
    const int pieces = a.pieces;
    __syncthreads();
    for (int p = (int)threadIdx.x; p < pieces; p += NT) part[p] = 0ull;
    __syncthreads();
    auto add = [&](u64 rank, u64 n) { atomicAdd(&part[index_at(row, rank) / (uint32_t)a.per], n); };
    if (edge < BINS) {
      if (held == edge) {
#pragma unroll 1
        for (int i = (int)threadIdx.x; i < s.listed; i += NT)
          if (s.rank[i] >= last) add(s.rank[i], s.weight[i]);
      } else {
        const u64 hi = edge == 0 ? past_top : begin_of(edge - 1);
        each_between<DT>(row, value_at<DT>(row, last), value_at<DT>(row, hi - 1), [&](float x, uint32_t i) {
          const double w = weight_of(row, x);
          const u64 n = (u64)__builtin_fma(w, unit, 0.5);
          if (rank_of<DT>(row, x, i) >= last) add(rank_of<DT>(row, x, i), n ? n : (w > 0. ? 1ull : 0ull));
        });
      }
    }
    __syncthreads();
    for (int p = (int)(threadIdx.x >> 6); p < pieces; p += NT / 64) {
      double w = 0.;
      const int stop = edge == BINS ? BINS : edge - s.moved[p];  // ranges of the piece above the cut's
#pragma unroll
      for (int i = 0; i < BINS / 64; i++) {
        const double v = ((double)pw[p * BINS + 64 * i + lane] * 0x1p-48) * s.share[p];
        w += 64 * i + lane < stop ? v : 0.;
      }
#pragma unroll
      for (int o = 32; o; o >>= 1) w += __shfl_xor(w, o);
      if (edge < BINS) w += (double)part[p] / unit;
      if (lane == 0) kept[p] = w;
    }
    __syncthreads();
    // the piece of the token: the first up to which more than u of the sum has come (up to 256: a wave picks)
    auto kept_of = [&](int i) { return i < pieces ? kept[i] : 0.; };
    double target = __builtin_inf();
    Pick<double, double> p;
#pragma unroll 1
    for (int pass = 0; pass < 2; pass++) {  // their sum, then the piece
      p = pick<double, double>(kept_of, [](int) { return 0.; }, target);
      if (pass == 0) {
        total = p.before + kept_of(p.part);
        rest = u * total;
        target = nextafter(rest, __builtin_inf());
      }
    }
    begin = (long long)p.part * a.per;
    end = begin + a.per < a.V ? begin + a.per : a.V;
    rest -= p.before;
    __syncthreads();
  } else {
    total = sum_row<DT>(row, s, last);
    rest = u * total;
  }
  // the token: sums over threads that hold neighbouring values
  for (long long at = begin; at < end; at += NT * 8) {
    float x[8];
    double w[8], sum = 0.;
    const long long mine = at + (long long)threadIdx.x * 8;
    load_values<DT>(row.logits, mine < end ? mine : 0, mine < end ? end - mine : 0, x);
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const bool in = x[j] > -__builtin_inff() && rank_of<DT>(row, x[j], (uint32_t)(mine + j)) >= last;
      w[j] = in ? weight_of(row, x[j]) : 0.;
      sum += w[j];
    }
    double upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double v = __shfl_up(upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 63) s.wave[threadIdx.x >> 6] = upto;
    __syncthreads();
    double before = 0., all = 0.;
    for (int i = 0; i < NT / 64; i++) {
      if (i < (int)(threadIdx.x >> 6)) before += s.wave[i];
      all += s.wave[i];
    }
    before += upto - sum;
    // the first whose sum passes the rest; the last one kept where rounding leaves none
    int found = 0x7fffffff, latest = -1;
    double c = before;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      c += w[j];
      if (w[j] > 0.) {
        latest = (int)(mine + j);
        if (c > rest && found == 0x7fffffff) found = latest;
      }
    }
    if (found != 0x7fffffff) atomicMin(&s.token, found);
    if (latest >= 0) atomicMax(&s.latest, latest);
    __syncthreads();
    rest -= all;
    if (s.token != 0x7fffffff) break;
  }
  if (threadIdx.x == 0) {
    const int token = s.token != 0x7fffffff ? s.token : s.latest;
    float x[8];
    load_values<DT>(row.logits, token < 0 ? 0 : token, 1, x);
    a.tokens[r] = token;
    if (a.logprob) a.logprob[r] = token < 0 ? __builtin_nanf("") : (float)(((double)x[0] - (double)top) * (row.scale * 0.6931471805599453) - log(total));
  }
}

// values of a piece: of few rows small ones, so that there are workgroups for the chip
int piece_of(long long R, long long V) {
  const long long values = R * V;
  return values <= (1ll << 21) && V <= (1ll << 20) ? PT * 8 : PT * 8 * 2;
}

}  // namespace

size_t esp_sample_workspace(long long R, long long V) {
  const long long per = piece_of(R, V), pieces = (V + per - 1) / per;
  return (size_t)(R * pieces) * (BINS * 12 + 8);
}

int esp_sample_device(esparse_ctx* ctx, const void* logits, long long R, long long V, long long ld, int dtype, const float* temperature, const int32_t* top_k,
                      const float* top_p, const float* min_p, const float* u, long long* tokens, float* logprob, void* ws) {
  SampleArgs a = {};
  a.logits = logits, a.R = R, a.V = V, a.ld = ld;
  a.u = u, a.temperature = temperature, a.top_k = top_k, a.top_p = top_p, a.min_p = min_p, a.tokens = tokens, a.logprob = logprob;
  a.per = piece_of(R, V);
  a.pieces = (int)((V + a.per - 1) / a.per);
  const long long all = R * a.pieces;
  a.weight = (unsigned long long*)ws;
  a.count = (uint32_t*)(a.weight + all * BINS);
  a.top = (float*)(a.count + all * BINS);
  a.where = (int32_t*)(a.top + all);
#define GO(DT)                                                                                                       \
  {                                                                                                                  \
    if (a.per == PT * 8) hipLaunchKernelGGL((k_pieces<DT, 1>), dim3((unsigned)all), dim3(PT), 0, ctx->stream, a);    \
    else hipLaunchKernelGGL((k_pieces<DT, 2>), dim3((unsigned)all), dim3(PT), 0, ctx->stream, a);                    \
    hipLaunchKernelGGL((k_rows<DT>), dim3((unsigned)R), dim3(NT), 0, ctx->stream, a);                                \
  }
  if (dtype == ESPARSE_F16) GO(ESPARSE_F16)
  else if (dtype == ESPARSE_BF16) GO(ESPARSE_BF16)
  else GO(ESPARSE_F32)
#undef GO
  ESP_HIP(ctx, hipGetLastError());
  return ESPARSE_OK;
}
