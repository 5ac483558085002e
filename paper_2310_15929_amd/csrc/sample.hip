// A token drawn from each row of logits (include/esparse.h): w_i = exp((x_i - max) / temperature); top-k, top-p and min-p each keep a beginning of the order "larger
// first, equal ones by index"; the token is the first, by index, up to which more than u of the kept sum has come.
//
// Nothing is sorted.  k_pieces, a workgroup for each piece of a row, reads the row once and leaves the piece's maximum and, for 256 ranges of x (an eighth of a doubling of
// the weight wide, on a grid that all pieces share, counted down from the range of the maximum; the last one holds all the rest), how many values
// and how much weight lie in each.  k_rows, a workgroup a row, adds these up, knows the range in which a cut falls, and reads the row again for that range's values only:
// they fit a list in LDS (or are split further first), of which the value and the index of the last one kept are found by splitting the list's span in 256 again and
// again.  What each piece keeps then follows from its ranges, and one piece is read to find the token.
// A token's share of a large vocabulary is small beside 2^-24: weights are exponentials in 64 bits (float64 runs at the rate of float32 here), sums are of whole
// numbers (2^48 for a piece's largest weight) or in float64 in a fixed order: results do not depend on chance.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx.h"

namespace {

constexpr int BINS = 256;
constexpr int NT = 1024;       // threads of a row
constexpr int PT = 512;        // threads of a piece
constexpr int LIST = 4096;     // values that a list holds
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

// 2^y for y <= 0, to 2^-50 (below 2^-1022 to the numbers there are): e^(r ln 2) by its series to the 12th power, |r| <= 1/2
__device__ __forceinline__ double exp2_of(double y) {
  if (!(y > -1100.)) return 0.;
  const double n = __builtin_rint(y), z = (y - n) * 0.6931471805599453;
  double s = 1. / 479001600.;
  s = __builtin_fma(s, z, 1. / 39916800.);
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

// ranges are those of floor(8 x scale)
__device__ __forceinline__ double range_of(float x, double scale) { return __builtin_floor((double)x * (scale * STEPS)); }

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
  if (top > -__builtin_inff()) {
    int own = 0x7fffffff;
    const double high = range_of(top, scale);
#pragma unroll
    for (int v = 0; v < V8; v++) {
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float f = x[v][j];
        if (f == top) own = min(own, (v * PT + (int)threadIdx.x) * 8 + j);
        if (scale > 0. && f > -__builtin_inff() && f <= top) {
          const double d = high - range_of(f, scale);
          const int bin = d < (double)(BINS - 1) ? (int)d : BINS - 1;
          const double w = exp2_of(((double)f - (double)top) * scale);
          atomicAdd(&weight[bin], (unsigned long long)__builtin_fma(w, 281474976710656., 0.5));
          atomicAdd(&count[bin], 1u);
        }
      }
    }
    if (own != 0x7fffffff) atomicMin(&first, own);
  }
  __syncthreads();
  const long long at = r * a.pieces + piece;
  if (threadIdx.x < BINS) {
    a.weight[at * BINS + threadIdx.x] = weight[threadIdx.x];
    a.count[at * BINS + threadIdx.x] = count[threadIdx.x];
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
  float top;
  double scale;
};
__device__ __forceinline__ double weight_of(const Row& r, float x) { return exp2_of(((double)x - (double)r.top) * r.scale); }

// f(value, index) for the values first .. end - 1 of a row, eight in a row for a thread
template <int DT, class F>
__device__ __forceinline__ void each_value(const Row& r, long long first, long long end, F f) {
  for (long long at = first + (long long)threadIdx.x * 8; at < end; at += (long long)NT * 8) {
    float x[8];
    load_values<DT>(reinterpret_cast<const unsigned char*>(r.logits) + at * (DT == ESPARSE_F32 ? 4 : 2), 0, end - at, x);
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (at + j < end) f(x[j], (uint32_t)(at + j));
  }
}

struct Shared {
  unsigned long long list[LIST];
  unsigned long long weight[BINS];
  uint32_t count[BINS];
  double row_weight[BINS];  // of the row's ranges
  uint32_t row_count[BINS];
  double wave[NT / 64];
  unsigned long long lo, hi, before_weight;
  unsigned long long before_count, inside;
  int listed, chosen, bin;
  double before, total;
};

// the smallest key from that of the least number to `most` for which yes() holds; it holds for `most` and for all above the first
template <class F>
__device__ __forceinline__ uint32_t first_key(uint32_t most, F yes) {
  uint32_t lo = 0x00800000u, hi = most;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (yes(value_of(mid))) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}
// the smallest of the values that lie in one of the ranges 0 .. bin, counted down from `high`, that of the maximum
__device__ __forceinline__ uint32_t range_begin(double high, int bin, float top, double scale) {
  return first_key(key_of(top), [&](float x) { return high - range_of(x, scale) <= bin; });
}

// How a cut is found: the values whose rank lies in [lo, hi) are looked through, those above are kept.  By number: `need` more of them are kept.  By weight: those are
// kept before which less than `target` (a whole number) has come.  Returns the rank of the last one kept, and the weight of [that, hi).
// unit: what a weight is multiplied with to be a whole number.
template <int DT>
__device__ unsigned long long cut(const Row& r, Shared& s, unsigned long long lo, unsigned long long hi, unsigned long long inside, bool by_weight,
                                  unsigned long long need, double unit, unsigned long long* kept) {
  unsigned long long came = 0;  // number or weight that came before hi
  unsigned long long weight_before = 0;
  bool listed = false;
  for (;;) {
    if (!listed && inside <= LIST) {
      if (threadIdx.x == 0) s.listed = 0;
      __syncthreads();
      each_value<DT>(r, 0, r.V, [&](float x, uint32_t i) {
        const unsigned long long k = rank_of(x, i);
        if (k >= lo && k < hi && x > -__builtin_inff()) {
          const int at = atomicAdd(&s.listed, 1);
          if (at < LIST) s.list[at] = k;
        }
      });
      __syncthreads();
      listed = true;
    }
    const unsigned long long span = hi - lo;
    const int bits = 64 - __builtin_clzll(span - 1 | 1ull), shift = bits > 8 ? bits - 8 : 0;
    if (threadIdx.x < BINS) s.weight[threadIdx.x] = 0ull, s.count[threadIdx.x] = 0u;
    __syncthreads();
    auto put = [&](unsigned long long k) {
      if (k >= lo && k < hi) {
        const int bin = (int)((hi - 1 - k) >> shift);
        const float x = value_of((uint32_t)(k >> 32));
        atomicAdd(&s.weight[bin], (unsigned long long)__builtin_fma(weight_of(r, x), unit, 0.5));
        atomicAdd(&s.count[bin], 1u);
      }
    };
    if (listed) {
      const int n = s.listed < LIST ? s.listed : LIST;
      for (int i = (int)threadIdx.x; i < n; i += NT) put(s.list[i]);
    } else {
      each_value<DT>(r, 0, r.V, [&](float x, uint32_t i) {
        if (x > -__builtin_inff()) put(rank_of(x, i));
      });
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      unsigned long long c = came, w = weight_before;
      int at = -1;
      unsigned long long c_at = 0, w_at = 0;
      for (int b = 0; b < BINS; b++) {
        if (!s.count[b]) continue;
        if (by_weight && at >= 0 && c >= need) break;
        at = b, c_at = c, w_at = w;
        c += by_weight ? s.weight[b] : s.count[b];
        w += s.weight[b];
        if (c >= need) break;
      }
      s.chosen = at;
      s.before_count = c_at;
      s.before_weight = w_at;
      s.inside = at >= 0 ? s.count[at] : 0;
    }
    __syncthreads();
    const int at = s.chosen;
    came = s.before_count;
    weight_before = s.before_weight;
    inside = s.inside;
    if (at < 0) {  // nothing in it
      *kept = weight_before;
      __syncthreads();
      return hi;
    }
    hi = hi - ((unsigned long long)at << shift);
    lo = hi - lo > (1ull << shift) ? hi - (1ull << shift) : lo;
    const unsigned long long last = s.weight[at];
    __syncthreads();
    if (shift == 0) {
      *kept = weight_before + last;
      return lo;
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(NT) k_rows(const SampleArgs a) {
  __shared__ Shared s;
  const long long r = blockIdx.x;
  const float* tops = a.top + r * a.pieces;
  Row row;
  row.logits = reinterpret_cast<const unsigned char*>(a.logits) + r * a.ld * (DT == ESPARSE_F32 ? 4 : 2);
  row.V = a.V;
  row.scale = per_doubling(a, r);
  float top = -__builtin_inff();
  bool bad = !(row.scale >= 0.);
  int where = 0;
  for (int p = 0; p < a.pieces; p++) {
    const float t = tops[p];
    bad |= t != t;
    if (t > top) top = t, where = p;
  }
  row.top = top;
  if (bad || top == -__builtin_inff()) {
    if (threadIdx.x == 0) {
      a.tokens[r] = -1;
      if (a.logprob) a.logprob[r] = __builtin_nanf("");
    }
    return;
  }
  if (row.scale == 0.) {
    if (threadIdx.x == 0) {
      a.tokens[r] = a.where[r * a.pieces + where];
      if (a.logprob) a.logprob[r] = 0.f;
    }
    return;
  }
  // the row's ranges: those of the pieces, each moved by the distance of the maxima
  const unsigned long long* pw = a.weight + r * a.pieces * BINS;
  const uint32_t* pc = a.count + r * a.pieces * BINS;
  const double high = range_of(top, row.scale);
  auto moved = [&](int p) {  // how far (BINS: all of the piece is in the last range)
    const double d = high - range_of(tops[p], row.scale);
    return d < (double)BINS ? (int)d : BINS;
  };
  auto share = [&](int p) { return exp2_of(((double)tops[p] - (double)top) * row.scale); };
  if (threadIdx.x < BINS - 1) {
    double w = 0.;
    uint32_t c = 0;
    for (int p = 0; p < a.pieces; p++) {
      const int b = (int)threadIdx.x - (tops[p] > -__builtin_inff() ? moved(p) : BINS);
      if (b >= 0) {
        w += ((double)pw[p * BINS + b] * 0x1p-48) * share(p);
        c += pc[p * BINS + b];
      }
    }
    s.row_weight[threadIdx.x] = w;
    s.row_count[threadIdx.x] = c;
  } else if (threadIdx.x >= NT - 64) {
    const int lane = (int)threadIdx.x - (NT - 64);
    double w = 0.;
    uint32_t c = 0;
    for (int p = 0; p < a.pieces; p++) {
      if (!(tops[p] > -__builtin_inff())) continue;
      const int m = moved(p), from = m > BINS - 1 ? 0 : BINS - 1 - m;
      for (int b = from + lane; b < BINS; b += 64) {
        w += ((double)pw[p * BINS + b] * 0x1p-48) * share(p);
        c += pc[p * BINS + b];
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) w += __shfl_xor(w, o), c += __shfl_xor(c, o);
    if (lane == 0) s.row_weight[BINS - 1] = w, s.row_count[BINS - 1] = c;
  }
  __syncthreads();

  // the cuts: everything of rank `last` and above is kept
  unsigned long long last = 0;
  auto bounds = [&](int bin, unsigned long long& lo, unsigned long long& hi) {
    lo = (unsigned long long)(bin == BINS - 1 ? 0x00800000u : range_begin(high, bin, top, row.scale)) << 32;
    hi = (unsigned long long)(bin == 0 ? key_of(top) + 1u : range_begin(high, bin - 1, top, row.scale)) << 32;
  };
  // whole numbers for the weights of a range: 2^40 to 2^41 for its largest
  auto unit_of = [&](int bin) { return __builtin_ldexp(1., 40 + bin / (int)STEPS); };
  const long long k = a.top_k ? a.top_k[r] : 0;
  double total = 0.;  // of what is kept so far
  for (int b = 0; b < BINS; b++) total += s.row_weight[b];
  if (k > 0) {
    unsigned long long n = 0;
    double above = 0.;
    int b = 0;
    for (; b < BINS; b++) {
      if (n + s.row_count[b] >= (unsigned long long)k) break;
      n += s.row_count[b];
      above += s.row_weight[b];
    }
    if (b < BINS) {
      unsigned long long lo, hi, kept;
      bounds(b, lo, hi);
      if (n + s.row_count[b] == (unsigned long long)k) {
        last = lo;
        total = above + s.row_weight[b];
      } else {
        last = cut<DT>(row, s, lo, hi, s.row_count[b], false, k - n, unit_of(b), &kept);
        total = above + (double)kept / unit_of(b);
      }
    }
  }
  const float top_p = a.top_p ? a.top_p[r] : 1.f;
  if (top_p < 1.f) {
    const double target = (top_p > 0.f ? (double)top_p : 0.) * total;
    double above = 0., upto = 0.;
    int full = 0;
    for (int b = 0; b < BINS; b++) {  // the first range that reaches the target (the last one that holds any, where rounding leaves none)
      if (!s.row_count[b]) continue;
      full = b;
      above = upto;
      upto += s.row_weight[b];
      if (upto >= target) break;
    }
    unsigned long long lo, hi, kept;
    bounds(full, lo, hi);
    if (hi > last) {  // (else top-k has kept less)
      const double rest = (target - above) * unit_of(full);
      const unsigned long long need = rest > 1. ? (unsigned long long)__builtin_ceil(rest) : 1ull;
      const unsigned long long at = cut<DT>(row, s, lo, hi, s.row_count[full], true, need, unit_of(full), &kept);
      last = at > last ? at : last;
    }
  }
  const float min_p = a.min_p ? a.min_p[r] : 0.f;
  if (min_p > 0.f) {
    const double least = min_p < 1.f ? (double)min_p : 1.;
    const uint32_t key = first_key(key_of(top), [&](float x) { return weight_of(row, x) >= least; });
    const unsigned long long at = (unsigned long long)key << 32;
    last = at > last ? at : last;
  }

  // what each piece keeps of the range that the cut is in, and of those above it
  int edge = BINS;  // no cut: all ranges
  if (last) {
    const double d = high - range_of(value_of((uint32_t)(last >> 32)), row.scale);
    edge = d < (double)(BINS - 1) ? (int)d : BINS - 1;
  }
  unsigned long long lo = 0, hi = 0;
  double* kept = reinterpret_cast<double*>(s.list);                       // [pieces]
  unsigned long long* part = s.list + LIST / 2;                           // [pieces]
  const int pieces = a.pieces;
  __syncthreads();
  for (int p = (int)threadIdx.x; p < pieces; p += NT) part[p] = 0ull;
  __syncthreads();
  if (last) {
    bounds(edge, lo, hi);
    each_value<DT>(row, 0, row.V, [&](float x, uint32_t i) {
      const unsigned long long rank = rank_of(x, i);
      if (rank >= last && rank < hi && x > -__builtin_inff()) {
        const double w = weight_of(row, x);
        const unsigned long long n = (unsigned long long)__builtin_fma(w, unit_of(edge), 0.5);
        atomicAdd(&part[i / (uint32_t)a.per], n ? n : (w > 0. ? 1ull : 0ull));  // (what can be drawn is never nothing: u may be 0)
      }
    });
  }
  __syncthreads();
  for (int p = (int)(threadIdx.x >> 6); p < pieces; p += NT / 64) {
    double w = 0.;
    if (tops[p] > -__builtin_inff()) {
      const int m = moved(p), lane = (int)(threadIdx.x & 63u);
      const int stop = edge == BINS ? BINS : edge - m;  // ranges of the piece above the cut's
      const double by = share(p);
      for (int b = lane; b < stop; b += 64) w += ((double)pw[p * BINS + b] * 0x1p-48) * by;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) w += __shfl_xor(w, o);
    if (last) w += (double)part[p] / unit_of(edge);
    if ((threadIdx.x & 63u) == 0) kept[p] = w;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double all = 0.;
    for (int p = 0; p < pieces; p++) all += kept[p];
    const float given = a.u[r];
    const double u = given > 0.f ? (given < 1.f ? (double)given : 0x1.fffffep-1) : 0.;
    double rest = u * all;
    int at = -1;
    for (int p = 0; p < pieces; p++) {
      if (!(kept[p] > 0.)) continue;
      if (at >= 0 && rest < 0.) break;
      at = p;
      if (rest < kept[p]) break;
      bool more = false;
      for (int q = p + 1; q < pieces; q++) more |= kept[q] > 0.;
      if (!more) break;
      rest -= kept[p];
    }
    s.chosen = at < 0 ? 0 : at;
    s.before = rest;
    s.total = all;
    s.bin = -1;
  }
  __syncthreads();
  // the token in its piece: sums over threads that hold neighbouring values
  const long long begin = (long long)s.chosen * a.per, end = begin + a.per < a.V ? begin + a.per : a.V;
  double rest = s.before;
  for (long long at = begin; at < end; at += NT * 8) {
    float x[8];
    double w[8], sum = 0.;
    const long long mine = at + (long long)threadIdx.x * 8;
    load_values<DT>(row.logits, mine < end ? mine : 0, mine < end ? end - mine : 0, x);
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const bool in = mine + j < end && x[j] > -__builtin_inff() && rank_of(x[j], (uint32_t)(mine + j)) >= last;
      w[j] = in ? weight_of(row, x[j]) : 0.;
      sum += w[j];
    }
    double upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double v = __shfl_up(upto, o);
      if ((int)(threadIdx.x & 63u) >= o) upto += v;
    }
    if ((threadIdx.x & 63u) == 63u) s.wave[threadIdx.x >> 6] = upto;
    __syncthreads();
    double before = 0., all = 0.;
    for (int i = 0; i < NT / 64; i++) {
      if (i < (int)(threadIdx.x >> 6)) before += s.wave[i];
      all += s.wave[i];
    }
    before += upto - sum;
    // candidates: the first whose sum passes the rest; the last one kept where rounding leaves none
    int found = 0x7fffffff, latest = -1;
    double c = before;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      c += w[j];
      if (w[j] > 0.) {
        latest = (int)(mine + j);
        if (c > rest && found == 0x7fffffff) found = (int)(mine + j);
      }
    }
    if (threadIdx.x == 0) s.chosen = 0x7fffffff;
    __syncthreads();
    if (found != 0x7fffffff) atomicMin(&s.chosen, found);
    if (latest >= 0) atomicMax(&s.bin, latest);
    __syncthreads();
    const int got = s.chosen;
    rest -= all;
    if (got != 0x7fffffff) {
      if (threadIdx.x == 0) s.bin = got;
      break;
    }
    __syncthreads();
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const int token = s.bin;
    a.tokens[r] = token;
    if (a.logprob) {
      float x[8];
      load_values<DT>(row.logits, token < 0 ? 0 : token, 1, x);
      a.logprob[r] = token < 0 ? __builtin_nanf("") : (float)(((double)x[0] - (double)top) * (row.scale * 0.6931471805599453) - log(s.total));
    }
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
