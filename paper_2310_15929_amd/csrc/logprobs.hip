// Log probabilities of given tokens, the entropy and the most probable alternatives of rows of logits.
//   with m the row's largest logit, s = sum exp(x - m), t = sum (x - m) exp(x - m):
//   log p(token) = x_token - m - ln s,   entropy = ln s - t / s,   all in fp32 (x - m is taken before it is scaled to base 2).
// Bound by memory, at 16 bits nearly by the vector unit too (about 11 issue slots a value: conversion, maximum, difference, exponential, two sums).
// A row is read once: each thread keeps a running maximum with s and t relative to it, and brings them to a new maximum where four 16-byte pieces
// hold one.  Where there are few rows a row is cut into pieces, a workgroup each; a second launch joins them.
//   Alternatives: T = the k-th largest of the threads' own maxima is a lower bound of the k-th largest value, so only threads whose
// maximum reaches T (about k of them) read their values a second time, and only values of at least T are looked at: little more than k, unless many
// are equal, as where a mask leaves fewer values than alternatives.  There the list overflows: the values above T are listed, then the first ones that are T
// itself, in order (8 x 131072 with 20 alternatives where a mask leaves 5 values: 25 us, 2048 rows of them 261; with k rounds of a search for the next in order
// 82 and 2250).  If a few threads hold so many values above T that this list overflows too, those rounds take its place.  Order: larger value first, then lower index.
//   Measured, cold, captured: 2048 x 131072 16-bit 103 us (5.2 TB/s; 20 alternatives 143: the second read), 2048 x 32000 31 us (4.2 TB/s), 555 x 50021 32-bit 27.6 us (4.0 TB/s:
// two pieces a row, 4.3 workgroups a compute unit; 5 alternatives 32.4), 8 x 131072 5.8 us (20 alternatives 10.7), 1 x 32000 5.7 us (20 alternatives 9.9).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "intrinsics.h"

namespace {

constexpr int LIST = 1024;  // candidates for the alternatives that a workgroup can hold

struct LpPartial {  // of a piece
  float m, s, t, pad;
};

// the order of floats as unsigned numbers; 0 is below them all.  (-0 and +0 are one value: added to +0 first)
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// larger for what comes first: value, then the lower index
__device__ __forceinline__ unsigned long long rank_key(float f, uint32_t index) { return (unsigned long long)order_key(f) << 32 | (uint32_t)~index; }

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = __builtin_fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

__device__ __forceinline__ float natural_exp(float d) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_exp2f(d * 1.44269504088896340736f);
#else
  return d;
#endif
}

// what a row is answered with, from its m, s, t
struct LpOut {
  const void* logits;
  const long long* tokens;
  float* logprob;
  float* entropy;
  int32_t* top_ids;
  float* top_logprobs;
  long long V, ld;
  int dtype, top;
};
__device__ __forceinline__ float logit_at(const LpOut& o, long long row, long long i) {
  if (o.dtype == ESPARSE_F32) return reinterpret_cast<const float*>(o.logits)[row * o.ld + i];
  const uint16_t u = reinterpret_cast<const uint16_t*>(o.logits)[row * o.ld + i];
  return o.dtype == ESPARSE_F16 ? esp_to_float<ESPARSE_F16>(u) : esp_to_float<ESPARSE_BF16>(u);
}
__device__ __forceinline__ float minus_infinity() { return -__builtin_inff(); }
// ln p of a value; a row without any probability gives minus infinity, one with a NaN or an infinite logit NaN
__device__ __forceinline__ float log_prob(float x, float m, float s) {
  if (s == 0.f) return minus_infinity();
  return (x - m) - __builtin_logf(s);
}
// the row's token (asked for early: its logit is another trip to memory) and that logit
__device__ __forceinline__ long long token_of(const LpOut& o, long long row) { return o.tokens && o.logprob ? o.tokens[row] : -1; }
__device__ __forceinline__ float token_logit(const LpOut& o, long long row, long long id) { return id >= 0 && id < o.V ? logit_at(o, row, id) : 0.f; }
__device__ __forceinline__ void answer_row(const LpOut& o, long long row, long long id, float x, float m, float s, float t) {
  if (o.tokens && o.logprob) o.logprob[row] = id < 0 ? 0.f : (id >= o.V ? __builtin_nanf("") : log_prob(x, m, s));
  if (o.entropy) o.entropy[row] = s == 0.f ? 0.f : __builtin_logf(s) - t / s;
}

constexpr int NT = 256, NW = NT / 64;

// The first `top` of n candidates (all different, at most 64 C) to put(place, candidate): a candidate's place is the number of those before it.  Every wave
// holds all of them and counts for each NW-th (each thread in a loop over the list in shared memory: 1 x 32000 with 20 alternatives 13.2 instead of 10.6 us;
// more than 128 candidates are rare, and registers for them would cost the kernels an eighth of their waves)
template <int C, class Put>
__device__ __forceinline__ void place_from(const unsigned long long* list, int n, int top, const Put& put) {
  const int lane = threadIdx.x & 63, wave = wave_uniform((int)(threadIdx.x >> 6));
  unsigned long long own[C];
  int place[C];
#pragma unroll
  for (int c = 0; c < C; c++) {
    own[c] = c * 64 + lane < n ? list[c * 64 + lane] : 0ull;
    place[c] = top;
  }
#pragma unroll
  for (int c = 0; c < C; c++)
    for (int l = wave; l < 64 && c * 64 + l < n; l += NW) {
      const unsigned long long k = (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(own[c] >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)own[c], l);
      int before = 0;
#pragma unroll
      for (int d = 0; d < C; d++) before += __builtin_popcountll(__ballot(own[d] > k));
      place[c] = lane == l ? before : place[c];
    }
#pragma unroll
  for (int c = 0; c < C; c++)
    if (place[c] < top) put(place[c], own[c]);
}
template <class Put>
__device__ __forceinline__ void place_candidates(const unsigned long long* list, int n, int top, const Put& put) {
  if (n <= 64) {
    place_from<1>(list, n, top, put);
  } else if (n <= 128) {
    place_from<2>(list, n, top, put);
  } else {
    for (int i = threadIdx.x; i < n; i += NT) {
      const unsigned long long k = list[i];
      int place = 0;
      for (int j = 0; j < n; j++) place += list[j] > k;
      if (place < top) put(place, k);
    }
  }
}
__device__ __forceinline__ void answer_place(const LpOut& o, long long row, int place, unsigned long long k, float m, float s) {
  o.top_ids[row * o.top + place] = (int32_t)~(uint32_t)k;
  o.top_logprobs[row * o.top + place] = log_prob(key_value((uint32_t)(k >> 32)), m, s);
}
// a row with a NaN or an infinite logit: none of its values is looked at (a NaN has no place in the order: one with its sign set is below minus infinity)
__device__ __forceinline__ void answer_no_places(const LpOut& o, long long row) {
  for (int i = threadIdx.x; i < o.top; i += NT) {
    o.top_ids[row * o.top + i] = -1;
    o.top_logprobs[row * o.top + i] = __builtin_nanf("");
  }
}

// One wave with C keys a lane: the largest 32-bit pattern that at least `top` of the keys reach, or one below it that at most half as many again and SLACK more do
constexpr int SLACK = 8;  // fewer rounds of the search for a few values more to look at
template <int C>
__device__ __forceinline__ uint32_t key_bound(const uint32_t (&key)[C], int top) {
  uint32_t bound = 0;
  for (int bit = 31; bit >= 0; bit--) {
    const uint32_t trial = bound | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < C; i++) n += __builtin_popcountll(__ballot(key[i] >= trial));
    if (n >= top) {
      bound = trial;
      if (n <= top + top / 2 + SLACK) break;
    }
  }
  return bound;
}

constexpr int AT_ONCE = 4;  // pieces of 16 bytes a thread reads at a time

// values of a 16-byte unit; behind the row's end minus infinity
template <int DT>
struct LpUnit {
  static constexpr int E = DT == ESPARSE_F32 ? 4 : 8;
  uint32_t raw[4];
  __device__ __forceinline__ void load(const void* row, long long at, long long V) {
    const long long left = V - at;
    if constexpr (DT == ESPARSE_F32) {
      const float* p = reinterpret_cast<const float*>(row) + at;
      if (left >= E) {
        __builtin_memcpy(raw, p, 16);
      } else {
#pragma unroll
        for (int i = 0; i < 4; i++) raw[i] = 0xff800000u;
        if (left > 0) {
#pragma unroll
          for (int i = 0; i < 4; i++) raw[i] = __builtin_bit_cast(uint32_t, p[i < left ? i : left - 1]);
        }
#pragma unroll
        for (int i = 0; i < 4; i++) raw[i] = i < left ? raw[i] : 0xff800000u;
      }
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + at;
      constexpr uint32_t low = DT == ESPARSE_F16 ? 0xfc00u : 0xff80u;
      if (left >= E) {
        __builtin_memcpy(raw, p, 16);
      } else {
        uint32_t t[8];
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] = low;
        if (left > 0) {  // all loads under way at once: places behind the last repeat it
#pragma unroll
          for (int i = 0; i < 8; i++) t[i] = p[i < left ? i : left - 1];
        }
#pragma unroll
        for (int i = 0; i < 4; i++) raw[i] = (2 * i < left ? t[2 * i] : low) | (2 * i + 1 < left ? t[2 * i + 1] : low) << 16;
      }
    }
  }
  __device__ __forceinline__ float value(int i) const {
    if constexpr (DT == ESPARSE_F32) return __builtin_bit_cast(float, raw[i]);
    else return esp_to_float<DT>((uint16_t)(raw[i / 2] >> (16 * (i & 1))));
  }
};

// One workgroup: `units` units of the row from unit `piece * units` on (PARTS: results to the workspace; otherwise the whole row).
template <int DT, bool PARTS>
__global__ void __launch_bounds__(NT) k_lp_row(const LpOut o, unsigned pieces, unsigned units, LpPartial* __restrict__ part, unsigned long long* __restrict__ part_top) {
  using Unit = LpUnit<DT>;
  constexpr int E = Unit::E;
  __shared__ float s_m[NW], s_s[NW], s_t[NW];
  __shared__ uint32_t s_key[NT];
  __shared__ unsigned long long s_list[LIST];
  __shared__ unsigned long long s_next[NW];
  __shared__ uint32_t s_from;
  __shared__ int s_n, s_threads;
  const long long row = PARTS ? blockIdx.x / pieces : blockIdx.x, V = o.V;
  const unsigned piece = PARTS ? blockIdx.x - (unsigned)row * pieces : 0, tid = threadIdx.x, wave = tid >> 6;
  const unsigned all = (unsigned)((V + E - 1) / E), first = piece * units, end = first + units < all ? first + units : all;
  const void* x = reinterpret_cast<const unsigned char*>(o.logits) + row * o.ld * (DT == ESPARSE_F32 ? 4 : 2);
  const long long id = !PARTS && tid == 0 ? token_of(o, row) : -1;
  float m = minus_infinity(), from = 0.f, s = 0.f, t = 0.f;  // from: m, 0 while there is none
  auto take = [&](const Unit* v, auto count) {
    constexpr int N = decltype(count)::value;
    float top = m;
#pragma unroll
    for (int j = 0; j < N; j++)
#pragma unroll
      for (int i = 0; i < E; i++) top = __builtin_fmaxf(top, v[j].value(i));
    if (top > m) {
      const float d = from - top, f = natural_exp(d);
      t = s == 0.f ? 0.f : f * __builtin_fmaf(s, __builtin_fmaxf(d, -128.f), t);
      s = s == 0.f ? 0.f : s * f;  // (the first maximum may be so low that f is infinite)
      m = from = top;
    }
#pragma unroll
    for (int j = 0; j < N; j++)
#pragma unroll
      for (int i = 0; i < E; i++) {
        const float d = v[j].value(i) - from, p = natural_exp(d);
        s += p;
        t = __builtin_fmaf(p, __builtin_fmaxf(d, -128.f), t);  // (p is 0 far above that; minus infinity times 0 is none)
      }
  };
  // (a second set of registers for the next values: no faster, 32 instead of 31 us for 2048 x 32000; eight workgroups a compute unit take turns as it is)
  unsigned u = first + tid, of_wave = first + (unsigned)wave_uniform((int)(tid & ~63u));
  for (; of_wave + (AT_ONCE - 1) * NT + 63 < end; u += AT_ONCE * NT, of_wave += AT_ONCE * NT) {
    Unit v[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; j++) v[j].load(x, (long long)(u + j * NT) * E, V);
    take(v, std::integral_constant<int, AT_ONCE>{});
  }
  // the last ones, as many as there are: a place without a value costs the vector unit as much as one with (100 x 131072: 13.7 us in whole turns, 12.1 so)
  if (of_wave < end) {
    Unit v[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; j++)
      if (of_wave + j * NT < end) v[j].load(x, u + j * NT < end ? (long long)(u + j * NT) * E : V, V);
#pragma unroll
    for (int j = 0; j < AT_ONCE; j++)
      if (of_wave + j * NT < end) take(v + j, std::integral_constant<int, 1>{});
  }
  const float x_id = !PARTS && tid == 0 ? token_logit(o, row, id) : 0.f;
  const float wm = wave_max(m);
  if ((tid & 63u) == 0) s_m[wave] = wm;
  const bool any = first + tid < end;  // (a thread without values is below all others)
  if (o.top) s_key[tid] = any ? order_key(m) : 0u;
  if (tid == 0) s_n = s_threads = 0;
  __syncthreads();
  float row_m = s_m[0];
#pragma unroll
  for (int i = 1; i < NW; i++) row_m = __builtin_fmaxf(row_m, s_m[i]);
  {
    const float to = row_m == minus_infinity() ? 0.f : row_m, d = from - to, f = natural_exp(d);
    t = s == 0.f ? 0.f : f * __builtin_fmaf(s, __builtin_fmaxf(d, -128.f), t);
    s = s == 0.f ? 0.f : s * f;
  }
  s = wave_sum(s);
  t = wave_sum(t);
  if ((tid & 63u) == 0) {
    s_s[wave] = s;
    s_t[wave] = t;
  }
  if (o.top && wave == 0) {
    uint32_t key[NW];
#pragma unroll
    for (int i = 0; i < NW; i++) key[i] = s_key[i * 64 + tid];
    const uint32_t bound = key_bound(key, o.top);
    if (tid == 0) s_from = bound;
  }
  __syncthreads();
  s = s_s[0];
  t = s_t[0];
#pragma unroll
  for (int i = 1; i < NW; i++) {
    s += s_s[i];
    t += s_t[i];
  }
  if (tid == 0) {
    if (PARTS) part[row * pieces + piece] = LpPartial{row_m, s, t, 0.f};
    else answer_row(o, row, id, x_id, row_m, s, t);
  }
  if (!o.top) return;
  if (s != s) {  // (the same for all threads)
    if constexpr (PARTS) {
      for (int i = tid; i < o.top; i += NT) part_top[(row * pieces + piece) * o.top + i] = 0;
    } else {
      answer_no_places(o, row);
    }
    return;
  }
  const uint32_t from_key = s_from;
  // the threads that reach T, in any order; all threads look at those threads' units
  if (any && order_key(m) >= from_key) s_key[atomicAdd(&s_threads, 1)] = tid;
  __syncthreads();
  const unsigned turns = (end - first + NT - 1) / NT, looks = (unsigned)s_threads * turns;
  // the values of at least `least` of those threads; where there are too many for the list, a second time those above `tie`
  uint32_t least = from_key, tie = 0;
  int n = 0;
  for (bool again = false;; again = true) {
    int slot = 0;
    for (unsigned q = tid; q < looks && slot < LIST; q += NT) {
      const unsigned w = first + (q % turns) * NT + s_key[q / turns];
      if (w >= end) continue;
      Unit r;
      r.load(x, (long long)w * E, V);
#pragma unroll
      for (int i = 0; i < E; i++) {
        const long long at = (long long)w * E + i;
        const float y = r.value(i);
        if (at < V && order_key(y) >= least) {
          slot = atomicAdd(&s_n, 1);
          if (slot < LIST) s_list[slot] = rank_key(y, (uint32_t)at);
        }
      }
    }
    __syncthreads();
    n = s_n;
    if (__builtin_expect(n <= LIST || again, 1)) break;
    // the lowest of the maxima that reach T.  At least `top` threads have it or more, so the values above it and the first equal ones are enough
    tie = any && order_key(m) >= from_key ? order_key(m) : ~0u;
#pragma unroll
    for (int w = 32; w; w >>= 1) {
      const uint32_t other = __shfl_xor(tie, w);
      tie = other < tie ? other : tie;
    }
    if ((tid & 63u) == 0) s_next[wave] = tie;
    __syncthreads();
    tie = (uint32_t)s_next[0];
#pragma unroll
    for (int i = 1; i < NW; i++) tie = (uint32_t)s_next[i] < tie ? (uint32_t)s_next[i] : tie;
    least = tie + 1u;  // (no maximum is NaN: there is a key above it)
    if (tid == 0) s_n = 0;
    __syncthreads();
  }
  if (__builtin_expect(tie != 0u && n < o.top, 0)) {  // the first values that are `tie`, NT units at a time: a thread's are behind those of the threads before it
    for (unsigned w0 = first; n < o.top && w0 < end; w0 += NT) {
      Unit r;
      unsigned equal = 0;
      const unsigned w = w0 + tid;
      if (w < end) {
        r.load(x, (long long)w * E, V);
#pragma unroll
        for (int i = 0; i < E; i++) equal |= (unsigned)((long long)w * E + i < V && order_key(r.value(i)) == tie) << i;
      }
      int place = __builtin_popcount(equal);
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int lower = __shfl_up(place, d);
        place += (int)(tid & 63u) >= d ? lower : 0;
      }
      if ((tid & 63u) == 63u) s_next[wave] = (unsigned long long)place;
      place += n - __builtin_popcount(equal);
      __syncthreads();
#pragma unroll
      for (unsigned i = 0; i < NW; i++) {
        const int count = (int)s_next[i];
        place += i < wave ? count : 0;
        n += count;
      }
      for (; equal && place < o.top; equal &= equal - 1u) s_list[place++] = (unsigned long long)tie << 32 | (uint32_t)~(w * E + (unsigned)__builtin_ctz(equal));
      __syncthreads();
    }
    n = n < o.top ? n : o.top;
  }
  if (__builtin_expect(n > LIST, 0)) {  // the next in order, again and again
    __syncthreads();
    unsigned long long before = ~0ull;
    for (int k = 0; k < o.top; k++) {
      unsigned long long best = 0;
      for (unsigned w = first + tid; w < end; w += NT) {
        Unit r;
        r.load(x, (long long)w * E, V);
#pragma unroll
        for (int i = 0; i < E; i++) {
          const long long at = (long long)w * E + i;
          if (at < V) {
            const unsigned long long key = rank_key(r.value(i), (uint32_t)at);
            if (key < before && key > best) best = key;
          }
        }
      }
#pragma unroll
      for (int w = 32; w; w >>= 1) {
        const unsigned long long other = __shfl_xor(best, w);
        best = other > best ? other : best;
      }
      if ((tid & 63u) == 0) s_next[wave] = best;
      __syncthreads();
      best = s_next[0];
#pragma unroll
      for (int i = 1; i < NW; i++) best = s_next[i] > best ? s_next[i] : best;
      if (tid == 0) s_list[k] = best;
      before = best;
      __syncthreads();
    }
    n = o.top;
  }
  if (PARTS) {
    // this piece's first `top`, in order; a piece with fewer values ends in zeros
    unsigned long long* to = part_top + (row * pieces + piece) * o.top;
    place_candidates(s_list, n, o.top, [&](int place, unsigned long long k) { to[place] = k; });
    for (int i = n + tid; i < o.top; i += NT) to[i] = 0;
  } else {
    place_candidates(s_list, n, o.top, [&](int place, unsigned long long k) { answer_place(o, row, place, k, row_m, s); });
  }
}

constexpr int MAX_PIECES = LIST / ESPARSE_MAX_TOP;
static_assert(MAX_PIECES <= 64 && LIST % NT == 0, "a lane for every piece");

// Joins the pieces of a row: one workgroup a row.  Bound by its trips to memory one after the other, so all that does not depend on another answer is read at
// the start and each wave joins the sums for itself (8 rows of 131072 with 20 alternatives, both launches, captured: 10.7 us; with the pieces, the lists and the
// token read one after the other and a search for the bound bit by bit 13.3)
__global__ void __launch_bounds__(NT) k_lp_join(const LpOut o, unsigned pieces, const LpPartial* __restrict__ part, const unsigned long long* __restrict__ part_top) {
  __shared__ unsigned long long s_list[LIST];
  __shared__ int s_n;
  const long long row = blockIdx.x;
  const unsigned tid = threadIdx.x, lane = tid & 63u;
  const LpPartial p = lane < pieces ? part[row * pieces + lane] : LpPartial{minus_infinity(), 0.f, 0.f, 0.f};
  const unsigned long long* lists = part_top + row * pieces * o.top;
  const unsigned count = pieces * o.top;
  unsigned long long mine[LIST / NT];
#pragma unroll
  for (int i = 0; i < LIST / NT; i++) mine[i] = i * NT + tid < count ? lists[i * NT + tid] : 0ull;
  const unsigned jth = o.top ? (o.top + pieces - 1) / pieces : 1;
  const uint32_t share = o.top && lane < pieces ? (uint32_t)(lists[lane * o.top + jth - 1] >> 32) : 0u;
  const long long id = tid == 0 ? token_of(o, row) : -1;
  const float x_id = tid == 0 ? token_logit(o, row, id) : 0.f;
  if (tid == 0) s_n = 0;
  const float m = wave_max(p.m), from = m == minus_infinity() ? 0.f : m, d = (p.m == minus_infinity() ? 0.f : p.m) - from, f = natural_exp(d);
  const bool some = p.s != 0.f;  // (its sums are taken from another maximum)
  const float s = wave_sum(some ? p.s * f : 0.f), t = wave_sum(some ? f * __builtin_fmaf(p.s, __builtin_fmaxf(d, -128.f), p.t) : 0.f);
  if (tid == 0) answer_row(o, row, id, x_id, m, s, t);
  if (!o.top) return;
  if (s != s) {
    answer_no_places(o, row);
    return;
  }
  // A key that at least `top` alternatives reach: the lists are in order, and of their j-th (j pieces >= top) the q-th largest (q j >= top) is reached by j of q
  // lists each (0: no value)
  const unsigned qth = (o.top + jth - 1) / jth;
  unsigned before = 0;
  for (unsigned l = 0; l < pieces; l++) {
    const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)share, (int)l);
    before += k > share || (k == share && l < lane);
  }
  const unsigned long long who = __ballot(lane < pieces && before == qth - 1);
  const uint32_t bound = (uint32_t)__builtin_amdgcn_readlane((int)share, (int)__builtin_ctzll(who));
  __syncthreads();
#pragma unroll
  for (int i = 0; i < LIST / NT; i++)
    if (mine[i] && (uint32_t)(mine[i] >> 32) >= bound) s_list[atomicAdd(&s_n, 1)] = mine[i];
  __syncthreads();
  place_candidates(s_list, s_n, o.top, [&](int place, unsigned long long k) { answer_place(o, row, place, k, m, s); });
}

// Workgroups of a row: one where the rows fill the chip (1024 of them are four a compute unit; 1024 x 50048 16-bit: 25.2 us, cut in two 27.9), otherwise as many as
// bring it there, of 512 units at least (two for each thread) or, with alternatives, whose lists have to be joined, 1024 (with 512: 8 x 131072 10.7 instead of
// 10.0 us, 1 x 16000 8.6 instead of 6.8, though 1 x 32000 9.0 instead of 9.7)
struct LpPlan {
  unsigned pieces, units;
};

LpPlan plan(long long R, long long V, int dtype, int top) {
  const int e = dtype == ESPARSE_F32 ? 4 : 8;
  const long long units = (V + e - 1) / e;
  long long pieces = (1024 + R - 1) / R;
  if (pieces > units / (top ? 1024 : 512)) pieces = units / (top ? 1024 : 512);
  if (pieces > MAX_PIECES) pieces = MAX_PIECES;
  if (pieces < 1) pieces = 1;
  const long long per = (units + pieces - 1) / pieces;
  return {(unsigned)((units + per - 1) / per), (unsigned)per};
}

template <int DT>
hipError_t launch(const LpOut& o, long long R, const LpPlan& p, void* ws, hipStream_t st) {
  LpPartial* part = reinterpret_cast<LpPartial*>(ws);
  unsigned long long* tops = reinterpret_cast<unsigned long long*>(part + R * p.pieces);
  if (p.pieces == 1) {
    hipLaunchKernelGGL((k_lp_row<DT, false>), dim3((unsigned)R), dim3(NT), 0, st, o, 1u, p.units, part, tops);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((k_lp_row<DT, true>), dim3((unsigned)(R * p.pieces)), dim3(NT), 0, st, o, p.pieces, p.units, part, tops);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_lp_join, dim3((unsigned)R), dim3(256), 0, st, o, p.pieces, part, tops);
  return hipGetLastError();
}

}  // namespace

size_t esp_token_logprobs_workspace(long long R, long long V, int dtype, int top) {
  const LpPlan p = plan(R, V, dtype, top);
  return p.pieces == 1 ? 0 : (size_t)R * p.pieces * (sizeof(LpPartial) + 8u * (size_t)top);
}

int esp_token_logprobs_device(esparse_ctx* ctx, const void* logits, long long R, long long V, long long ld, int dtype, const long long* tokens, int top,
                              float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs, void* ws) {
  const LpOut o = {logits, tokens, logprob, entropy, top_ids, top_logprobs, V, ld, dtype, top};
  const LpPlan p = plan(R, V, dtype, top);
  if (dtype == ESPARSE_F16) ESP_HIP(ctx, launch<ESPARSE_F16>(o, R, p, ws, ctx->stream));
  else if (dtype == ESPARSE_BF16) ESP_HIP(ctx, launch<ESPARSE_BF16>(o, R, p, ws, ctx->stream));
  else ESP_HIP(ctx, launch<ESPARSE_F32>(o, R, p, ws, ctx->stream));
  return ESPARSE_OK;
}
