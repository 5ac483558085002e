// Log probabilities of given tokens, the entropy and the most probable alternatives of rows of logits.
//   with m the row's largest logit, s = sum exp(x - m), t = sum (x - m) exp(x - m):
//   log p(token) = x_token - m - ln s,   entropy = ln s - t / s,   all in fp32 (x - m is taken before it is scaled to base 2).
// Bound by memory at many rows: a row, or one of the pieces that it is cut into where there are few rows, is read once into
// registers; maximum, sums and the alternatives are taken there.  A second launch joins the pieces of a row.
//   Alternatives: T = the k-th largest of the threads' own maxima is a lower bound of the k-th largest value, so only values
// of at least T are looked at again - little more than k of them, unless many are equal: where their list overflows, k
// rounds of a search for the next in order take its place.  Order: larger value first, then lower index.
#include <hip/hip_runtime.h>

#include "common.h"

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
__device__ __forceinline__ void answer_row(const LpOut& o, long long row, float m, float s, float t) {
  if (o.tokens && o.logprob) {
    const long long id = o.tokens[row];
    o.logprob[row] = id < 0 ? 0.f : (id >= o.V ? __builtin_nanf("") : log_prob(logit_at(o, row, id), m, s));
  }
  if (o.entropy) o.entropy[row] = s == 0.f ? 0.f : __builtin_logf(s) - t / s;
}

// The first `top` of n candidates (n >= top, all different) to their places: a candidate's place is the number of those before it.
__device__ __forceinline__ void place_candidates(const unsigned long long* list, int n, int top, int nt, int32_t* ids, float* lps, float m, float s) {
  for (int i = threadIdx.x; i < n; i += nt) {
    const unsigned long long k = list[i];
    int place = 0;
    for (int j = 0; j < n; j++) place += list[j] > k;
    if (place < top) {
      ids[place] = s != s ? -1 : (int32_t)~(uint32_t)k;
      lps[place] = s != s ? s : log_prob(key_value((uint32_t)(k >> 32)), m, s);
    }
  }
}

// A workgroup of NT threads holds `C` pieces of 16 bytes a thread.  PARTS: the row is cut, the results go to the workspace.
template <int DT, int NT, int C, bool PARTS>
__global__ void __launch_bounds__(NT) k_lp_row(const LpOut o, long long R, unsigned pieces, LpPartial* __restrict__ part, unsigned long long* __restrict__ part_top) {
  constexpr int E = DT == ESPARSE_F32 ? 4 : 8, NW = NT / 64;
  __shared__ float s_a[NW], s_b[NW];
  __shared__ uint32_t s_key[NT];
  __shared__ unsigned long long s_list[LIST];
  __shared__ unsigned long long s_next[NW];
  __shared__ uint32_t s_from;
  __shared__ int s_n;
  const long long row = PARTS ? blockIdx.x / pieces : blockIdx.x;
  const unsigned piece = PARTS ? blockIdx.x % pieces : 0, tid = threadIdx.x, wave = tid >> 6;
  const long long base = (long long)piece * (NT * C * E);
  const long long V = o.V;
  uint32_t raw[C][4];
  // value i of this thread's piece j stands at base + (j NT + tid) E + i; behind the row's end there are minus infinities
#pragma unroll
  for (int j = 0; j < C; j++) {
    const long long at = base + (long long)(j * NT + tid) * E, left = V - at;
    if (DT == ESPARSE_F32) {
      const float* p = reinterpret_cast<const float*>(o.logits) + row * o.ld + at;
      if (left >= E) {
        __builtin_memcpy(raw[j], p, 16);
      } else {
#pragma unroll
        for (int i = 0; i < 4; i++) raw[j][i] = i < left ? __builtin_bit_cast(uint32_t, p[i]) : 0xff800000u;
      }
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(o.logits) + row * o.ld + at;
      constexpr uint32_t low = DT == ESPARSE_F16 ? 0xfc00u : 0xff80u;
      if (left >= E) {
        __builtin_memcpy(raw[j], p, 16);
      } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
          uint32_t a = low, b = low;
          if (2 * i < left) a = p[2 * i];
          if (2 * i + 1 < left) b = p[2 * i + 1];
          raw[j][i] = a | b << 16;
        }
      }
    }
  }
  auto value = [&](int j, int i) -> float {
    if constexpr (DT == ESPARSE_F32) return __builtin_bit_cast(float, raw[j][i]);
    else return esp_to_float<DT>((uint16_t)(raw[j][i / 2] >> (16 * (i & 1))));
  };
  float mine = minus_infinity();
#pragma unroll
  for (int j = 0; j < C; j++)
#pragma unroll
    for (int i = 0; i < E; i++) mine = __builtin_fmaxf(mine, value(j, i));
  const float wm = wave_max(mine);
  if ((tid & 63u) == 0) s_a[wave] = wm;
  const bool any = base + (long long)tid * E < V;  // (a thread without values is below all others)
  if (o.top) s_key[tid] = any ? order_key(mine) : 0u;
  if (tid == 0) s_n = 0;
  __syncthreads();
  float m = s_a[0];
#pragma unroll
  for (int i = 1; i < NW; i++) m = __builtin_fmaxf(m, s_a[i]);
  __syncthreads();
  // (a row of minus infinities: taken from 0, so that its sum is 0; plus infinities and NaN make the sums NaN)
  const float from = m == minus_infinity() ? 0.f : m;
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int j = 0; j < C; j++)
#pragma unroll
    for (int i = 0; i < E; i++) {
      const float d = value(j, i) - from, p = natural_exp(d);
      s += p;
      t = __builtin_fmaf(p, __builtin_fmaxf(d, -128.f), t);  // (p is 0 far above that; minus infinity times 0 is none)
    }
  s = wave_sum(s);
  t = wave_sum(t);
  if ((tid & 63u) == 0) {
    s_a[wave] = s;
    s_b[wave] = t;
  }
  // T: the largest 32-bit pattern that at least `top` of the threads' maxima reach, to within twice as many (one wave)
  if (o.top && wave == 0) {
    uint32_t from_key = 0;
    for (int bit = 31; bit >= 0; bit--) {
      const uint32_t trial = from_key | 1u << bit;
      int n = 0;
#pragma unroll
      for (int i = 0; i < NW; i++) n += __builtin_popcountll(__ballot(s_key[i * 64 + tid] >= trial));
      if (n >= o.top) {
        from_key = trial;
        if (n <= o.top + o.top / 2) break;
      }
    }
    if (tid == 0) s_from = from_key;
  }
  __syncthreads();
  s = s_a[0];
  t = s_b[0];
#pragma unroll
  for (int i = 1; i < NW; i++) {
    s += s_a[i];
    t += s_b[i];
  }
  if (tid == 0) {
    if (PARTS) part[row * pieces + piece] = LpPartial{m, s, t, 0.f};
    else answer_row(o, row, m, s, t);
  }
  if (!o.top) return;
  const uint32_t from_key = s_from;
  if (any && order_key(mine) >= from_key) {
#pragma unroll
    for (int j = 0; j < C; j++)
#pragma unroll
      for (int i = 0; i < E; i++) {
        const long long at = base + (long long)(j * NT + tid) * E + i;
        const float x = value(j, i);
        if (at < V && order_key(x) >= from_key) {
          const int slot = atomicAdd(&s_n, 1);
          if (slot < LIST) s_list[slot] = rank_key(x, (uint32_t)at);
        }
      }
  }
  __syncthreads();
  int n = s_n;
  if (n > LIST) {  // many equal values: the next in order, again and again
    __syncthreads();
    unsigned long long before = ~0ull;
    for (int k = 0; k < o.top; k++) {
      unsigned long long best = 0;
#pragma unroll
      for (int j = 0; j < C; j++)
#pragma unroll
        for (int i = 0; i < E; i++) {
          const long long at = base + (long long)(j * NT + tid) * E + i;
          if (at < V) {
            const unsigned long long key = rank_key(value(j, i), (uint32_t)at);
            if (key < before && key > best) best = key;
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
    for (int i = tid; i < n; i += NT) {
      const unsigned long long k = s_list[i];
      int place = 0;
      for (int j = 0; j < n; j++) place += s_list[j] > k;
      if (place < o.top) to[place] = k;
    }
    for (int i = n + tid; i < o.top; i += NT) to[i] = 0;
  } else {
    place_candidates(s_list, n, o.top, NT, o.top_ids + row * o.top, o.top_logprobs + row * o.top, m, s);
  }
}

// joins the pieces of a row: one workgroup a row
__global__ void __launch_bounds__(256) k_lp_join(const LpOut o, unsigned pieces, const LpPartial* __restrict__ part, const unsigned long long* __restrict__ part_top) {
  __shared__ float s_a[4], s_b[4];
  __shared__ unsigned long long s_list[LIST];
  __shared__ unsigned long long s_low[4];
  __shared__ int s_n;
  const long long row = blockIdx.x;
  const unsigned tid = threadIdx.x, wave = tid >> 6;
  const LpPartial* p = part + row * pieces;
  float m = minus_infinity();
  unsigned long long low = 0;  // the largest of the pieces' last alternatives: nothing below it is among the row's
  for (unsigned i = tid; i < pieces; i += 256) {
    m = __builtin_fmaxf(m, p[i].m);
    if (o.top) {
      const unsigned long long k = part_top[(row * pieces + i + 1) * o.top - 1];
      low = k > low ? k : low;
    }
  }
  m = wave_max(m);
#pragma unroll
  for (int w = 32; w; w >>= 1) {
    const unsigned long long other = __shfl_xor(low, w);
    low = other > low ? other : low;
  }
  if ((tid & 63u) == 0) {
    s_a[wave] = m;
    s_low[wave] = low;
  }
  if (tid == 0) s_n = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; i++) {
    m = __builtin_fmaxf(m, s_a[i]);
    low = s_low[i] > low ? s_low[i] : low;
  }
  __syncthreads();
  const float from = m == minus_infinity() ? 0.f : m;
  float s = 0.f, t = 0.f;
  for (unsigned i = tid; i < pieces; i += 256) {
    const float pm = p[i].m == minus_infinity() ? 0.f : p[i].m, d = pm - from;
    if (p[i].s != 0.f) {  // (its sums are taken from another maximum)
      const float f = natural_exp(d);
      s += p[i].s * f;
      t += f * __builtin_fmaf(p[i].s, __builtin_fmaxf(d, -128.f), p[i].t);
    }
  }
  s = wave_sum(s);
  t = wave_sum(t);
  if ((tid & 63u) == 0) {
    s_a[wave] = s;
    s_b[wave] = t;
  }
  __syncthreads();
  s = s_a[0] + s_a[1] + s_a[2] + s_a[3];
  t = s_b[0] + s_b[1] + s_b[2] + s_b[3];
  if (tid == 0) answer_row(o, row, m, s, t);
  if (!o.top) return;
  const unsigned long long* lists = part_top + row * pieces * o.top;
  for (unsigned i = tid; i < pieces * o.top; i += 256) {
    const unsigned long long k = lists[i];
    if (k >= low && k) {
      const int slot = atomicAdd(&s_n, 1);
      if (slot < LIST) s_list[slot] = k;
    }
  }
  __syncthreads();
  // (pieces * top <= LIST: the list holds them all)
  place_candidates(s_list, s_n, o.top, 256, o.top_ids + row * o.top, o.top_logprobs + row * o.top, m, s);
}

// How a row is cut: into pieces of 16 KiB of registers a workgroup of 256 threads where the rows alone leave compute units idle
struct LpPlan {
  int nt, c;         // threads of a workgroup, pieces of 16 bytes a thread
  unsigned pieces;   // workgroups of a row
};
constexpr int MAX_PIECES = LIST / ESPARSE_MAX_TOP;

LpPlan plan(long long R, long long V, int dtype) {
  const int e = dtype == ESPARSE_F32 ? 4 : 8;
  const long long units = (V + e - 1) / e;
  (void)R;
  static const int shapes[][2] = {{256, 1}, {256, 2}, {256, 4}, {256, 8}, {512, 8}, {1024, 8}, {1024, 16}};
  for (auto& s : shapes)
    if (units <= (long long)s[0] * s[1]) return {s[0], s[1], 1u};
  return {1024, 16, (unsigned)((units + 16383) / 16384)};
}

template <int DT>
hipError_t launch(const LpOut& o, long long R, const LpPlan& p, void* ws, hipStream_t st) {
  LpPartial* part = reinterpret_cast<LpPartial*>(ws);
  unsigned long long* tops = reinterpret_cast<unsigned long long*>(part + R * p.pieces);
#define GO(NT, C)                                                                                                                        \
  if (p.nt == NT && p.c == C) {                                                                                                          \
    if (p.pieces == 1) hipLaunchKernelGGL((k_lp_row<DT, NT, C, false>), dim3((unsigned)R), dim3(NT), 0, st, o, R, 1u, part, tops);       \
    else hipLaunchKernelGGL((k_lp_row<DT, NT, C, true>), dim3((unsigned)(R * p.pieces)), dim3(NT), 0, st, o, R, p.pieces, part, tops);   \
  }
  GO(256, 1) GO(256, 2) GO(256, 4) GO(256, 8) GO(512, 8) GO(1024, 8) GO(1024, 16)
#undef GO
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.pieces == 1) return e;
  hipLaunchKernelGGL(k_lp_join, dim3((unsigned)R), dim3(256), 0, st, o, p.pieces, part, tops);
  return hipGetLastError();
}

}  // namespace

size_t esp_token_logprobs_workspace(long long R, long long V, int dtype, int top) {
  const LpPlan p = plan(R, V, dtype);
  return p.pieces == 1 ? 0 : (size_t)R * p.pieces * (sizeof(LpPartial) + 8u * (size_t)top);
}
long long esp_token_logprobs_most(int dtype) { return (long long)MAX_PIECES * 16384 * (dtype == ESPARSE_F32 ? 4 : 8); }

int esp_token_logprobs_device(esparse_ctx* ctx, const void* logits, long long R, long long V, long long ld, int dtype, const long long* tokens, int top,
                              float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs, void* ws) {
  const LpOut o = {logits, tokens, logprob, entropy, top_ids, top_logprobs, V, ld, dtype, top};
  const LpPlan p = plan(R, V, dtype);
  if (dtype == ESPARSE_F16) ESP_HIP(ctx, launch<ESPARSE_F16>(o, R, p, ws, ctx->stream));
  else if (dtype == ESPARSE_BF16) ESP_HIP(ctx, launch<ESPARSE_BF16>(o, R, p, ws, ctx->stream));
  else ESP_HIP(ctx, launch<ESPARSE_F32>(o, R, p, ws, ctx->stream));
  return ESPARSE_OK;
}
