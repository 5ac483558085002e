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
// numbers or in float64 in a fixed order: results do not depend on chance.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx.h"

namespace {

constexpr int BINS = 256;
constexpr int NT = 1024;       // threads of a row
constexpr int PT = 512;        // threads of a piece
constexpr int LIST = 3328;     // values that a list holds
constexpr int MOST = 2048;     // with top_k up to this the pieces count values and leave their weights to the list
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
  __shared__ unsigned long long weight[BINS];
  __shared__ uint32_t count[BINS];
  __shared__ float tops[PT / 64];
  __shared__ int first, bad;
  const long long r = blockIdx.x / (unsigned)a.pieces;
  const int piece = (int)(blockIdx.x % (unsigned)a.pieces);
  const long long begin = (long long)piece * a.per, left = a.V - begin < a.per ? a.V - begin : a.per;
  const void* row = reinterpret_cast<const unsigned char*>(a.logits) + (r * a.ld + begin) * (DT == ESPARSE_F32 ? 4 : 2);
  if (threadIdx.x < BINS) weight[threadIdx.x] = 0ull, count[threadIdx.x] = 0u;
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
          if (x[v][j] > -__builtin_inff() && x[v][j] <= top) atomicAdd(&count[bin_of(x[v][j], high, step)], 1u);
    }
    if (scale > 0. && weighs(k)) {
#pragma unroll
      for (int v = 0; v < V8; v++)
#pragma unroll
        for (int j = 0; j < 8; j++)
          if (x[v][j] > -__builtin_inff() && x[v][j] <= top) {
            const double w = exp2_of(((double)x[v][j] - (double)top) * scale);
            atomicAdd(&weight[bin_of(x[v][j], high, step)], (unsigned long long)__builtin_fma(w, 281474976710656., 0.5));
          }
    }
  }
  __syncthreads();
  const long long at = r * a.pieces + piece;
  if (threadIdx.x < BINS) {
    if (weighs(k)) a.weight[at * BINS + threadIdx.x] = weight[threadIdx.x];
    if (counts(k)) a.count[at * BINS + threadIdx.x] = count[threadIdx.x];
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
// ... and with their index: larger numbers come first in the order
__device__ __forceinline__ unsigned long long rank_of(float x, uint32_t index) { return (unsigned long long)key_of(x) << 32 | (uint32_t)~index; }

struct Row {
  const void* logits;
  long long V;
  float top, step, high;
  double scale;
};
__device__ __forceinline__ double weight_of(const Row& r, float x) { return exp2_of(((double)x - (double)r.top) * r.scale); }

// f(value, index) for the values of a row, eight in a row for a thread; the next eight are on their way meanwhile
template <int DT, class F>
__device__ __forceinline__ void each_value(const Row& r, F f) {
  constexpr int EACH = DT == ESPARSE_F32 ? 4 : 2;
  const unsigned char* p = reinterpret_cast<const unsigned char*>(r.logits);
  const long long first = (long long)threadIdx.x * 8;
  float x[2][8], y[2][8];
  auto fetch = [&](long long at, float (&to)[2][8]) {
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const long long i = at + (long long)h * NT * 8;
      load_values<DT>(p + (i < r.V ? i : 0) * EACH, 0, i < r.V ? r.V - i : 0, to[h]);
    }
  };
  fetch(first, x);
  for (long long at = first; at < r.V; at += (long long)NT * 16) {
    fetch(at + (long long)NT * 16, y);
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int j = 0; j < 8; j++) f(x[h][j], (uint32_t)(at + (long long)h * NT * 8 + j));  // (behind the end: minus infinity)
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int j = 0; j < 8; j++) x[h][j] = y[h][j];
  }
}

typedef unsigned long long u64;

struct Shared {
  u64 rank[LIST];      // the list: values with their index
  u64 weight[LIST];    // their weights as whole numbers
  u64 part_weight[BINS];
  uint32_t part_count[BINS];
  double row_weight[BINS];
  uint32_t row_count[BINS];
  u64 few[64], few_weight[64];
  double wave[NT / 64];
  u64 sum, least;
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
// The elements of `each` (each(f): f(key, weight) for those of this thread, the same ones every time) with keys in [lo, hi), `inside` of them at most.  By weight: those are kept before which less than
// `need` has come, else the first `need`.
template <class E>
__device__ Cut find_cut(Shared& s, E each, u64 lo, u64 hi, u64 inside, bool by_weight, u64 need) {
  u64 came = 0, weight = 0;  // in front of hi
  const int lane = (int)(threadIdx.x & 63u);
  for (;;) {
    if (inside <= 64) {
      if (threadIdx.x == 0) s.fews = 0;
      __syncthreads();
      each([&](u64 k, u64 w) {
        if (k >= lo && k < hi) {
          const int at = atomicAdd(&s.fews, 1);
          if (at < 64) s.few[at] = k, s.few_weight[at] = w;
        }
      });
      __syncthreads();
      const int n = s.fews < 64 ? s.fews : 64;
      const u64 mine = lane < n ? s.few[lane] : 0ull, own = lane < n ? s.few_weight[lane] : 0ull;
      u64 before = came;
      for (int i = 0; i < n; i++)
        if (s.few[i] > mine) before += by_weight ? s.few_weight[i] : 1ull;
      const bool keep = lane < n && before < need;
      const Cut r = {wave_min(keep ? mine : hi), weight + wave_sum(keep ? own : 0ull)};
      __syncthreads();
      return r;
    }
    const u64 span = hi - lo;
    const int bits = 64 - (int)__builtin_clzll((span - 1) | 1ull), shift = bits > 8 ? bits - 8 : 0;
    if (threadIdx.x < BINS) s.part_weight[threadIdx.x] = 0ull, s.part_count[threadIdx.x] = 0u;
    __syncthreads();
    each([&](u64 k, u64 w) {
      if (k >= lo && k < hi) {
        const int at = (int)((hi - 1 - k) >> shift);
        atomicAdd(&s.part_weight[at], w);
        atomicAdd(&s.part_count[at], 1u);
      }
    });
    __syncthreads();
    Pick<u64, u64> p;
    if (by_weight) p = pick<u64, u64>([&](int i) { return s.part_weight[i]; }, [&](int) { return 0ull; }, need - came);
    else p = pick<u64, u64>([&](int i) { return (u64)s.part_count[i]; }, [&](int i) { return s.part_weight[i]; }, need - came);
    if (p.part < 0) {  // elements without weight: none stands before another, all are kept
      __syncthreads();
      return {lo, weight};
    }
    const u64 inner = s.part_count[p.part], inner_weight = s.part_weight[p.part];
    came += p.before;
    weight += by_weight ? p.before : p.other;
    hi -= (u64)p.part << shift;
    lo = hi - lo > (1ull << shift) ? hi - (1ull << shift) : lo;
    inside = inner;
    __syncthreads();
    if (shift == 0 || (!by_weight && came + inner == need)) return {lo, weight + inner_weight};
  }
}

// Every wave for itself: the smallest key up to `most` for which yes() holds; it holds for `most` and for all above the first
template <class F>
__device__ __forceinline__ uint32_t first_key(uint32_t most, F yes) {
  uint32_t lo = 0x00800000u, hi = most;  // (from the least number)
  const uint32_t lane = threadIdx.x & 63u;
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

template <int DT>
__global__ void __launch_bounds__(NT) k_rows(const SampleArgs a) {
  __shared__ Shared s;
  const long long r = blockIdx.x;
  const float* tops = a.top + r * a.pieces;
  const int lane = (int)(threadIdx.x & 63u);
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
  const long long k = a.top_k ? a.top_k[r] : 0;
  const float given_p = a.top_p ? a.top_p[r] : 1.f, given_min = a.min_p ? a.min_p[r] : 0.f, given_u = a.u[r];
  const bool cut_p = given_p < 1.f, cut_min = given_min > 0.f;
  const double top_p = given_p > 0.f ? (double)given_p : 0., least = given_min < 1.f ? (double)given_min : 1.;
  const double u = given_u > 0.f ? (given_u < 1.f ? (double)given_u : 0x1.fffffep-1) : 0.;

  // the row's ranges: those of the pieces, each moved by the distance of the maxima
  const u64* pw = a.weight + r * a.pieces * BINS;
  const uint32_t* pc = a.count + r * a.pieces * BINS;
  auto moved = [&](int p) { return tops[p] > -__builtin_inff() ? (int)fminf(row.high - range_of(tops[p], row.step), (float)BINS) : BINS; };
  auto share = [&](int p) { return weight_of(row, tops[p]); };
  const bool weighed = weighs(k);
  if (threadIdx.x < BINS - 1) {
    double w = 0.;
    uint32_t c = 0;
    for (int p = 0; p < a.pieces; p++) {
      const int b = (int)threadIdx.x - moved(p);
      if (b >= 0) {
        if (weighed) w += ((double)pw[p * BINS + b] * 0x1p-48) * share(p);
        if (counts(k)) c += pc[p * BINS + b];
      }
    }
    s.row_weight[threadIdx.x] = w;
    s.row_count[threadIdx.x] = c;
  } else if (threadIdx.x >= NT - 64) {
    double w = 0.;
    uint32_t c = 0;
    for (int p = 0; p < a.pieces; p++) {
      if (!(tops[p] > -__builtin_inff())) continue;
      const int m = moved(p), from = m > BINS - 1 ? 0 : BINS - 1 - m;
      for (int b = from + lane; b < BINS; b += 64) {
        if (weighed) w += ((double)pw[p * BINS + b] * 0x1p-48) * share(p);
        if (counts(k)) c += pc[p * BINS + b];
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) w += __shfl_xor(w, o), c += __shfl_xor(c, o);
    if (lane == 0) s.row_weight[BINS - 1] = w, s.row_count[BINS - 1] = c;
  }
  if (threadIdx.x == 0) s.listed = 0, s.sum = 0ull, s.least = ~0ull, s.token = 0x7fffffff, s.latest = -1;
  __syncthreads();

  // Ranks of the values of a range: [first of the range, first of the range above it)
  auto begin_of = [&](int bin) {  // (all waves get the same)
    return (u64)(bin == BINS - 1 ? 0x00800000u : first_key(key_of(top), [&](float x) { return row.high - range_of(x, row.step) <= (float)bin; })) << 32;
  };
  auto end_of = [&](int bin) { return bin == 0 ? (u64)(key_of(top) + 1u) << 32 : begin_of(bin - 1); };

  // where the first cut falls by number
  Pick<u64, u64> by_number = {-1, 0, 0};
  if (counts(k)) by_number = pick<u64, u64>([&](int i) { return (u64)s.row_count[i]; }, [&](int) { return 0ull; }, (u64)k);
  const bool cut_k = by_number.part >= 0 && by_number.before + s.row_count[by_number.part] >= (u64)k;

  u64 last = 0;  // everything of this rank and above is kept
  const u64 listable = cut_k ? by_number.before + s.row_count[by_number.part] : ~0ull;
  if (listable <= LIST) {
    // everything down to the end of that range
    constexpr double UNIT = 0x1p50;  // less than 2^12 weights of up to 1
    const u64 from = begin_of(by_number.part);
    const float lowest = value_of((uint32_t)(from >> 32));
    each_value<DT>(row, [&](float x, uint32_t i) {
      if (x >= lowest) {
        const int at = atomicAdd(&s.listed, 1);
        if (at < LIST) s.rank[at] = rank_of(x, i);
      }
    });
    __syncthreads();
    const int n = s.listed < LIST ? s.listed : LIST;
    for (int i = (int)threadIdx.x; i < n; i += NT) {
      const double w = weight_of(row, value_of((uint32_t)(s.rank[i] >> 32)));
      const u64 v = (u64)__builtin_fma(w, UNIT, 0.5);
      s.weight[i] = v ? v : (w > 0. ? 1ull : 0ull);  // (what can be drawn is never nothing: u may be 0)
    }
    auto each = [&](auto f) {
      for (int i = (int)threadIdx.x; i < n; i += NT) f(s.rank[i], s.weight[i]);
    };
    __syncthreads();
    const Cut by_k = find_cut(s, each, 0ull, ~0ull, (u64)n, false, (u64)k);
    last = by_k.last;
    if (cut_p) {
      const double target = __builtin_ceil(top_p * (double)by_k.kept);
      const Cut by_p = find_cut(s, each, last, ~0ull, (u64)k, true, target > 1. ? (u64)target : 1ull);
      last = by_p.last > last ? by_p.last : last;
    }
    u64 lowest_kept = ~0ull, sum = 0;
    if (cut_min) {
      each([&](u64 rank, u64) {
        if (rank >= last && rank < lowest_kept && weight_of(row, value_of((uint32_t)(rank >> 32))) >= least) lowest_kept = rank;
      });
      lowest_kept = wave_min(lowest_kept);
      if (lane == 0) atomicMin(&s.least, lowest_kept);
      __syncthreads();
      last = s.least > last ? s.least : last;
    }
    each([&](u64 rank, u64 w) { sum += rank >= last ? w : 0ull; });
    sum = wave_sum(sum);
    if (lane == 0) atomicAdd(&s.sum, sum);
    __syncthreads();
    const u64 total = s.sum;
    // ~index: the first by index are the largest
    const u64 drawn = find_cut(
                          s,
                          [&](auto f) {
                            each([&](u64 rank, u64 w) {
                              if (rank >= last && w) f(rank & 0xffffffffull, w);
                            });
                          },
                          0ull, 1ull << 32, (u64)n, true, (u64)(u * (double)total) + 1ull)
                          .last;
    each([&](u64 rank, u64) {
      if ((rank & 0xffffffffull) == drawn) {
        a.tokens[r] = (long long)(uint32_t)~drawn;
        if (a.logprob)
          a.logprob[r] = (float)(((double)value_of((uint32_t)(rank >> 32)) - (double)top) * (row.scale * 0.6931471805599453) - log((double)total * (1. / UNIT)));
      }
    });
    return;
  }

  // Too many for the list.  The weights of the ranges, where the pieces have not added them
  auto unit_of = [&](int bin) { return __builtin_ldexp(1., 40 + bin / (int)STEPS); };  // 2^40 to 2^41 for the largest weight of a range
  if (!weighed) {
    if (threadIdx.x < BINS) s.part_weight[threadIdx.x] = 0ull;
    __syncthreads();
    each_value<DT>(row, [&](float x, uint32_t) {
      if (x > -__builtin_inff()) {
        const int bin = bin_of(x, row.high, row.step);
        atomicAdd(&s.part_weight[bin], (u64)__builtin_fma(weight_of(row, x), unit_of(bin), 0.5));
      }
    });
    __syncthreads();
    if (threadIdx.x < BINS) s.row_weight[threadIdx.x] = (double)s.part_weight[threadIdx.x] / unit_of((int)threadIdx.x);
    __syncthreads();
  }
  auto row_weights = [&](int i) { return s.row_weight[i]; };
  int held = -1;  // the range in the list (all of it)
  u64 held_from = 0, held_to = 0;
  // a cut in a range, from the list, or from the row where the range does not fit it
  auto cut_in = [&](int bin, bool by_weight, u64 need) {
    const u64 lo = begin_of(bin), hi = end_of(bin);
    const double unit = unit_of(bin);
    if (held != bin) {
      __syncthreads();
      if (threadIdx.x == 0) s.listed = 0;
      __syncthreads();
      const float from = value_of((uint32_t)(lo >> 32)), to = value_of((uint32_t)(hi >> 32) - 1u);
      each_value<DT>(row, [&](float x, uint32_t i) {
        if (x >= from && x <= to) {
          const int at = atomicAdd(&s.listed, 1);
          if (at < LIST) s.rank[at] = rank_of(x, i);
        }
      });
      __syncthreads();
      held = s.listed <= LIST ? bin : -1;
      held_from = lo, held_to = hi;
      if (held >= 0) {
        for (int i = (int)threadIdx.x; i < s.listed; i += NT)
          s.weight[i] = (u64)__builtin_fma(weight_of(row, value_of((uint32_t)(s.rank[i] >> 32))), unit, 0.5);
      }
      __syncthreads();
    }
    const u64 inside = (u64)s.listed;
    if (held >= 0)
      return find_cut(
          s,
          [&](auto f) {
            for (int i = (int)threadIdx.x; i < (int)inside; i += NT) f(s.rank[i], s.weight[i]);
          },
          lo, hi, inside, by_weight, need);
    return find_cut(
        s,
        [&](auto f) {
          each_value<DT>(row, [&](float x, uint32_t i) {
            const u64 rank = rank_of(x, i);
            if (rank >= lo && rank < hi && x > -__builtin_inff()) f(rank, (u64)__builtin_fma(weight_of(row, x), unit, 0.5));
          });
        },
        lo, hi, inside, by_weight, need);
  };
  double total;  // of what is kept so far
  {
    const Pick<double, double> all = pick<double, double>(row_weights, [](int) { return 0.; }, __builtin_inf());
    total = all.before + s.row_weight[all.part];
  }
  if (cut_k) {
    const int bin = by_number.part;
    double above = 0.;
    for (int b = lane; b < bin; b += 64) above += s.row_weight[b];
#pragma unroll
    for (int o = 32; o; o >>= 1) above += __shfl_xor(above, o);
    if (listable == (u64)k) {
      last = begin_of(bin);
      total = above + s.row_weight[bin];
    } else {
      const Cut c = cut_in(bin, false, (u64)k - by_number.before);
      last = c.last;
      total = above + (double)c.kept / unit_of(bin);
    }
  }
  if (cut_p) {
    const double target = top_p * total;
    const Pick<double, double> p = pick<double, double>(row_weights, [](int) { return 0.; }, target);
    if (end_of(p.part) > last) {  // (else top-k has kept less)
      const double rest = __builtin_ceil((target - p.before) * unit_of(p.part));
      const Cut c = cut_in(p.part, true, rest > 1. ? (u64)rest : 1ull);
      last = c.last > last ? c.last : last;
    }
  }
  if (cut_min) {
    const u64 at = (u64)first_key(key_of(top), [&](float x) { return weight_of(row, x) >= least; }) << 32;
    last = at > last ? at : last;
  }

  // what each piece keeps of the range that the cut is in, and of those above it
  long long begin = 0, end = a.V;
  double rest = 0.;
  const int edge = last ? bin_of(value_of((uint32_t)(last >> 32)), row.high, row.step) : BINS;  // no cut: all ranges
  const double unit = unit_of(edge < BINS ? edge : 0);
  if (weighed) {
    // (the list may be in use: the parts are free)
    u64* part = s.part_weight;                          // [pieces]
    double* kept = reinterpret_cast<double*>(s.weight);  // [pieces], once the list is read
    const int pieces = a.pieces;
    __syncthreads();
    for (int p = (int)threadIdx.x; p < pieces; p += NT) part[p] = 0ull;
    __syncthreads();
    auto add = [&](u64 rank, double w) {
      const u64 n = (u64)__builtin_fma(w, unit, 0.5);
      atomicAdd(&part[(uint32_t)~rank / (uint32_t)a.per], n ? n : (w > 0. ? 1ull : 0ull));
    };
    if (edge < BINS) {
      if (held == edge) {
        for (int i = (int)threadIdx.x; i < s.listed; i += NT)
          if (s.rank[i] >= last) add(s.rank[i], weight_of(row, value_of((uint32_t)(s.rank[i] >> 32))));
      } else {
        const u64 hi = end_of(edge);
        const float from = value_of((uint32_t)(last >> 32)), to = value_of((uint32_t)(hi >> 32) - 1u);
        each_value<DT>(row, [&](float x, uint32_t i) {
          if (x >= from && x <= to && rank_of(x, i) >= last) add(rank_of(x, i), weight_of(row, x));
        });
      }
    }
    __syncthreads();
    for (int p = (int)(threadIdx.x >> 6); p < pieces; p += NT / 64) {
      double w = 0.;
      const int stop = edge == BINS ? BINS : edge - moved(p);  // ranges of the piece above the cut's
      if (tops[p] > -__builtin_inff()) {
        const double by = share(p);
        for (int b = lane; b < stop; b += 64) w += ((double)pw[p * BINS + b] * 0x1p-48) * by;
      }
#pragma unroll
      for (int o = 32; o; o >>= 1) w += __shfl_xor(w, o);
      if (edge < BINS) w += (double)part[p] / unit;
      if (lane == 0) kept[p] = w;
    }
    __syncthreads();
    // the piece of the token: the first up to which more than u of the sum has come (up to 256: a wave picks)
    auto kept_of = [&](int i) { return i < pieces ? kept[i] : 0.; };
    const Pick<double, double> all = pick<double, double>(kept_of, [](int) { return 0.; }, __builtin_inf());
    total = all.before + kept_of(all.part);
    const double target = u * total;
    const Pick<double, double> p = pick<double, double>(kept_of, [](int) { return 0.; }, nextafter(target, __builtin_inf()));
    begin = (long long)p.part * a.per;
    end = begin + a.per < a.V ? begin + a.per : a.V;
    rest = target - p.before;
    __syncthreads();
  } else {
    double sum = 0.;
    each_value<DT>(row, [&](float x, uint32_t i) {
      if (x > -__builtin_inff() && rank_of(x, i) >= last) sum += weight_of(row, x);
    });
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) s.wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    total = 0.;
    for (int i = 0; i < NT / 64; i++) total += s.wave[i];
    rest = u * total;
    __syncthreads();
  }
  // the token: sums over threads that hold neighbouring values
  for (long long at = begin; at < end; at += NT * 8) {
    float x[8];
    double w[8], sum = 0.;
    const long long mine = at + (long long)threadIdx.x * 8;
    load_values<DT>(row.logits, mine < end ? mine : 0, mine < end ? end - mine : 0, x);
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const bool in = x[j] > -__builtin_inff() && rank_of(x[j], (uint32_t)(mine + j)) >= last;
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
  return values <= (1ll << 21) && V <= (1ll << 20) ? PT * 8 : PT * 8 * 4;
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
    else hipLaunchKernelGGL((k_pieces<DT, 4>), dim3((unsigned)all), dim3(PT), 0, ctx->stream, a);                    \
    hipLaunchKernelGGL((k_rows<DT>), dim3((unsigned)R), dim3(NT), 0, ctx->stream, a);                                \
  }
  if (dtype == ESPARSE_F16) GO(ESPARSE_F16)
  else if (dtype == ESPARSE_BF16) GO(ESPARSE_BF16)
  else GO(ESPARSE_F32)
#undef GO
  ESP_HIP(ctx, hipGetLastError());
  return ESPARSE_OK;
}
