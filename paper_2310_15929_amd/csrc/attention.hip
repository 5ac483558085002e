// Attention over a cache held in microscaled 4 bits (include/esparse.h, csrc/heads.hip): o = sum_j p_j v_j, p = softmax(scale q.k_j), one pass over the tokens
// with the running maximum m and sum l of the softmax:  m' = max(m, x_j), l' = l 2^(c (m - m')) + sum 2^(c (x_j - m')), o' likewise, c = scale log2(e).
//
// The rows of a tile are the queries of one head of the cache, (token, query head of the group) in order: 16 of them are the columns of the 16-bit matrix
// instruction (lane l = 16 g + c: operands hold k = 8 g .. 8 g + 7 of row / column c, results rows 4 g + j of column c).
//   scores  X^T[token, row] = K Q^T.  Lane (c, g) loads 16 bytes of token c: channels 32 g .. 32 g + 31, one block with one scale, brought to 16 bits by the
//           conversion that takes the scale; its j-th word is the operand of step j (which k a channel takes does not matter as long as Q's agrees).
//   output  O^T[channel, row] += V^T P^T.  The lane holds the probabilities of tokens 4 g + j of two groups of 16 for its row: with the tokens of a step numbered that
//           way P^T is an operand as it stands.  V needs token and channel exchanged: it goes through LDS in 16 bits and comes back by the transposing read, which
//           hands a lane four tokens of one channel.  P is rounded to the 16 bits of the output's type, as V is held: the matrix instruction takes both so; sums
//           and statistics are in 32 bits.
// The statistics of a row are those of a column of X^T: they stay in the lane but for two exchanges (lanes 16 and 32 apart) a strip of 32 tokens.
// A block without number (scale 255) of V is left out of the product and put into the rows that see its token afterwards, so that masked tokens cannot reach a row.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "intrinsics.h"
#include "mx.h"

namespace {

constexpr int STRIP = 32;      // tokens of a step
constexpr int ROWS = 16;       // rows of a tile
constexpr int WAVES = 4;
constexpr int LEAST = 8;       // strips of a piece, where a long sequence is cut

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
  float c;  // scale log2(e)
};

// where a tile is: the sequence, its first row, and what its rows see
struct Tile {
  int b, first, queries;  // sequence, first row of the tile among the sequence's, queries of the sequence
  long long start;        // first query of the sequence
  int length, end;        // tokens of the sequence; those that the tile's last row sees
};

__device__ __forceinline__ long long clamp_to(long long v, long long lo, long long hi) { return v < lo ? lo : (v > hi ? hi : v); }

// Tiles of sequence b begin at floor(starts[b] group / rows) + b: enough for all of its rows, found by counting the sequences that begin no later (64 at a time)
__device__ __forceinline__ Tile find_tile(const AttendArgs& a, int tile, int rows) {
  Tile t;
  if (!a.starts) {
    const int each = (a.group + rows - 1) / rows;
    t.b = tile / each;
    t.first = (tile % each) * rows;
    t.start = t.b;
    t.queries = 1;
  } else {
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      const int b = b0 + (int)(threadIdx.x & 63u);
      const bool yes = b < a.B && clamp_to(a.starts[b < a.B ? b : 0], 0, a.T) * a.group / rows + b <= tile;
      const int found = (int)__popcll(__ballot(yes));
      before += found;
      if (found < 64) break;
    }
    t.b = wave_uniform(before > 0 ? before - 1 : 0);
    t.start = clamp_to(a.starts[t.b], 0, a.T);
    const long long stop = clamp_to(a.starts[t.b + 1], t.start, a.T);
    t.queries = (int)(stop - t.start);
    t.first = (int)(tile - (t.start * a.group / rows + t.b)) * rows;
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

// maximum over the four lanes of a column
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

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

template <int DT>
__device__ __forceinline__ uint32_t pack_2(float a, float b) {
  return esp_from_float<DT>(a) | (uint32_t)esp_from_float<DT>(b) << 16;
}

template <int DP>
constexpr int kVRow = DP + 16;  // 16-bit numbers from token to token in LDS: eight tokens' columns lie in different banks
template <int DP>
constexpr int kPartial = ROWS * DP + 2 * ROWS;

// One tile of 16 rows and a piece of its tokens: the waves take strips in turn, their results are joined in LDS
template <int DT, int DP>
__global__ void __launch_bounds__(64 * WAVES) k_attend_few(const AttendArgs a) {
  constexpr int NS = DP / 32, ND = DP / 16;
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
  floatx4_t o[ND];
#pragma unroll
  for (int n = 0; n < ND; n++) o[n] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;
  const int32_t* table = a.table + (long long)t.b * a.width;

  for (int strip = from + wave; strip < to; strip += WAVES) {
    Codes<DP> kc[2], vc[2];
    bool there[2];
    int page[2];
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const int at = strip * STRIP + 16 * u;
      page[u] = at < t.end ? wave_uniform(table[at >> a.page_bits]) : -1;
      there[u] = page[u] >= 0 && page[u] < a.pages;
    }
#pragma unroll
    for (int u = 0; u < 2; u++) {
      if (there[u]) {
        const int at = strip * STRIP + 16 * u;
        const long long r = (((long long)page[u] * a.Hkv + head) << a.page_bits) + (at & ((1 << a.page_bits) - 1)) + c;
        load_codes<DP>(a.k_data, a.k_scales, r, g, kc[u]);
        load_codes<DP>(a.v_data, a.v_scales, r, g, vc[u]);
      }
      if (!there[u] || strip * STRIP + 16 * u + c >= t.end) {  // tokens that no row sees: no numbers of theirs take part
        if (!there[u]) kc[u] = Codes<DP>{};
        vc[u] = Codes<DP>{};
      }
    }
    // V into LDS
    unsigned long long odd[2][DP == 256 ? 2 : 1];
    wave_fence();
#pragma unroll
    for (int u = 0; u < 2; u++) {
#pragma unroll
      for (int i = 0; i < (DP == 256 ? 2 : 1); i++) odd[u][i] = __ballot(vc[u].e[i] == 255u);
#pragma unroll
      for (int s = 0; s < NS; s++) {
        const unsigned e = vc[u].e[DP == 256 ? s / 4 : 0];
        *reinterpret_cast<uint4*>(vt + (16 * u + c) * kVRow<DP> + channel_of<DP>(s, g)) = mx_widen<DT>(e == 255u ? 0u : vc[u].w[s], mx_scale(e == 255u ? 0u : e));
      }
    }
    wave_fence();
    // scores
    float x[2][4];
#pragma unroll
    for (int u = 0; u < 2; u++) {
      floatx4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; s++) acc = mfma16<DT>(mx_widen<DT>(kc[u].w[s], mx_scale(kc[u].e[DP == 256 ? s / 4 : 0])), qv[s], acc);
#pragma unroll
      for (int j = 0; j < 4; j++) x[u][j] = there[u] && strip * STRIP + 16 * u + 4 * g + j <= sees ? acc[j] * a.c : -__builtin_inff();
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int j = 0; j < 4; j++) top = fmaxf(top, x[u][j]);
    top = column_max(top);
    const float base = top == -__builtin_inff() ? 0.f : top, shrink = __builtin_amdgcn_exp2f(m - base);
    m = top;
    l *= shrink;
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        x[u][j] = __builtin_amdgcn_exp2f(x[u][j] - base);
        l += x[u][j];
      }
    const uint4 p = {pack_2<DT>(x[0][0], x[0][1]), pack_2<DT>(x[0][2], x[0][3]), pack_2<DT>(x[1][0], x[1][1]), pack_2<DT>(x[1][2], x[1][3])};
#pragma unroll
    for (int n = 0; n < ND; n++) {
      const uint16_t* at = vt + (4 * g + (c >> 2)) * kVRow<DP> + 16 * n + 4 * (c & 3);
      const uint2 lo = read_transposed(at), hi = read_transposed(at + 16 * kVRow<DP>);
#pragma unroll
      for (int j = 0; j < 4; j++) o[n][j] *= shrink;
      o[n] = mfma16<DT>(uint4{lo.x, lo.y, hi.x, hi.y}, p, o[n]);
    }
    // blocks without numbers: NaN for the rows that see them
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int i = 0; i < (DP == 256 ? 2 : 1); i++)
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

  // the waves' results
  __syncthreads();
  float* mine = reinterpret_cast<float*>(lds) + wave * (ROWS * DP);
  if (g == 0) {
    stat[0][wave][c] = m;
    stat[1][wave][c] = l;
  }
#pragma unroll
  for (int n = 0; n < ND; n++) *reinterpret_cast<floatx4_t*>(mine + c * DP + 16 * n + 4 * g) = o[n];
  __syncthreads();
  float* part = a.partial + ((long long)(tile * a.Hkv + head) * a.pieces + piece) * kPartial<DP>;
  for (int at = (int)threadIdx.x * 4; at < ROWS * DP; at += 64 * WAVES * 4) {
    const int r = at / DP, ch = at % DP;
    float top = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < WAVES; w++) top = fmaxf(top, stat[0][w][r]);
    const float base = top == -__builtin_inff() ? 0.f : top;
    floatx4_t sum = {0.f, 0.f, 0.f, 0.f};
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; w++) {
      const float f = __builtin_amdgcn_exp2f(stat[0][w][r] - base);
      const floatx4_t v = *reinterpret_cast<const floatx4_t*>(reinterpret_cast<const float*>(lds) + w * (ROWS * DP) + at);
#pragma unroll
      for (int j = 0; j < 4; j++) sum[j] += v[j] * f;
      all += stat[1][w][r] * f;
    }
    if (pieces > 1) {
      *reinterpret_cast<floatx4_t*>(part + at) = sum;
      if (ch == 0) {
        part[ROWS * DP + r] = top;
        part[ROWS * DP + ROWS + r] = all;
      }
    } else {
      const int of = t.first + r, qi = of / a.group;
      if (qi < t.queries) {
        const long long place = (t.start + qi) * ((long long)a.Hkv * a.group) + head * a.group + of % a.group;
        const float by = all == 0.f ? 0.f : 1.f / all;
#pragma unroll
        for (int j = 0; j < 4; j++)
          if (ch + j < a.D) a.out[place * a.D + ch + j] = esp_from_float<DT>(all == 0.f ? 0.f : sum[j] * by);
        if (a.lse && ch == 0) a.lse[place] = all == 0.f ? -__builtin_inff() : (base + log2f(all)) * 0.6931471805599453f;
      }
    }
  }
}

// pieces of a tile, joined in order
template <int DT, int DP>
__global__ void __launch_bounds__(256) k_attend_join(const AttendArgs a) {
  const int head = (int)(blockIdx.x % (unsigned)a.Hkv), tile = (int)(blockIdx.x / (unsigned)a.Hkv);
  const Tile t = find_tile(a, tile, ROWS);
  if (t.first >= (long long)t.queries * a.group) return;
  const int pieces = pieces_of(t.end, a.pieces);
  if (pieces == 1) return;
  const float* part = a.partial + (long long)(tile * a.Hkv + head) * a.pieces * kPartial<DP>;
  for (int at = (int)threadIdx.x * 4; at < ROWS * DP; at += 1024) {
    const int r = at / DP, ch = at % DP, of = t.first + r, qi = of / a.group;
    if (qi >= t.queries) continue;
    float top = -__builtin_inff();
    for (int i = 0; i < pieces; i++) top = fmaxf(top, part[(long long)i * kPartial<DP> + ROWS * DP + r]);
    const float base = top == -__builtin_inff() ? 0.f : top;
    floatx4_t sum = {0.f, 0.f, 0.f, 0.f};
    float all = 0.f;
    for (int i = 0; i < pieces; i++) {
      const float* p = part + (long long)i * kPartial<DP>;
      const float f = __builtin_amdgcn_exp2f(p[ROWS * DP + r] - base);
      const floatx4_t v = *reinterpret_cast<const floatx4_t*>(p + at);
#pragma unroll
      for (int j = 0; j < 4; j++) sum[j] += v[j] * f;
      all += p[ROWS * DP + ROWS + r] * f;
    }
    const long long place = (t.start + qi) * ((long long)a.Hkv * a.group) + head * a.group + of % a.group;
    const float by = all == 0.f ? 0.f : 1.f / all;
#pragma unroll
    for (int j = 0; j < 4; j++)
      if (ch + j < a.D) a.out[place * a.D + ch + j] = esp_from_float<DT>(all == 0.f ? 0.f : sum[j] * by);
    if (a.lse && ch == 0) a.lse[place] = all == 0.f ? -__builtin_inff() : (base + log2f(all)) * 0.6931471805599453f;
  }
}

long long tiles_of(long long T, int B, int group, bool ragged, int rows) {
  return ragged ? T * group / rows + B : (long long)B * ((group + rows - 1) / rows);
}
// pieces that a sequence is cut into at most: until the workgroups fill the chip, for the longest that the table has room for
int most_pieces(long long items, long long tokens) {
  const long long strips = (tokens + STRIP - 1) / STRIP, longest = (strips + LEAST - 1) / LEAST, want = (1024 + items - 1) / items;
  return (int)std::max<long long>(1, std::min(longest, want));
}

}  // namespace

size_t esp_cache_attention_workspace(const esparse_cache* cache, long long T, int B, int q_heads, long long width, bool ragged) {
  const int group = q_heads / cache->heads, dp = esp_cache_row(cache->head_dim);
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
  a.c = (float)(scale * 1.4426950408889634);
  const long long tiles = tiles_of(T, B, a.group, starts != nullptr, ROWS);
  a.tiles = (int)tiles;
  a.pieces = most_pieces(tiles * a.Hkv, width * cache->page);
  const int row = esp_cache_row(a.D);
  const dim3 grid((unsigned)(tiles * a.Hkv * a.pieces));
#define GO(DT, DP)                                                                                                                 \
  {                                                                                                                                \
    static std::atomic<unsigned long long> done{0};                                                                                \
    constexpr size_t bytes = (size_t)WAVES * STRIP * kVRow<DP> * 2;                                                                \
    static_assert(bytes >= (size_t)WAVES * ROWS * DP * 4, "the joined sums fit");                                                  \
    ESP_HIP(ctx, raise_dynamic_lds(done, ctx->device, &k_attend_few<DT, DP>, bytes));                                              \
    hipLaunchKernelGGL((k_attend_few<DT, DP>), grid, dim3(64 * WAVES), bytes, ctx->stream, a);                                     \
    if (a.pieces > 1) hipLaunchKernelGGL((k_attend_join<DT, DP>), dim3((unsigned)(tiles * a.Hkv)), dim3(256), 0, ctx->stream, a);  \
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
