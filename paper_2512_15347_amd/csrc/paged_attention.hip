// Attention of single new tokens over a paged key/value cache.
//
// For a query head with query q and keys k_j, values v_j (j < len):  s_j = scale <q, k_j>,  p_j = exp(s_j - m),  m = max s,
// l = sum p_j,  o = sum p_j v_j / l,  lse = m + ln l, taken in pieces: two pieces (m, l, o') with o' = sum p_j v_j join as
// m = max(m1, m2), l = l1 e^(m1-m) + l2 e^(m2-m), o' alike.  m begins at the lowest finite number and the maximum passes NaN over, so m is
// never -inf or NaN: a score of -inf has the weight 0 whatever came before it, and a NaN is in l and o' and stays there through every join.
//
// Every byte of the cache is read once and used for the G query heads of its key/value head only (G = 1 .. 16 products a value), so
// the kernel is bound by HBM as long as enough loads are in flight.  Both products run on the matrix pipe, S^T = K Q^T and
// O^T = V^T P^T with the keys / channels as rows and 16 query heads as columns (empty ones are zero): then a lane's keys
// of S^T are just the keys it multiplies in O^T, and keys and transposed values are loaded straight into operand registers, 16 bytes
// a lane, without LDS.  A step is 32 keys of bf16 or 64 keys of codes; the next step's keys are asked for when this step's have been
// multiplied, its values likewise.  Codes are converted to bf16, which holds them exactly; the scales go into the logits and the output.
//
// Work is split in one of two ways.  Short rows, and very many rows, are one workgroup each per key/value head (WHOLE): no second launch.
// Otherwise (EVEN) the units of 4 steps of all rows and heads, one after another, are cut into as many equal ranges as the device
// holds workgroups, wherever a row begins or ends: rows of any lengths end together, and a workgroup streams through its range with one
// start only.  A range has at most two rows that it does not cover whole, its first and its last; their pieces go to the
// workspace and a second launch joins them.
//
// Measured: 384 rows of 1 to 4096 tokens, 32 / 8 heads of 128, codes (1.6 GB): 293 us, 5.5 TB/s, where a plain read of 4 GiB reaches 5.3
// to 6.3; three rows of 65 to 131 thousand tokens in bf16 (0.65 GB): 126 us, of which the join takes 10; 48 rows of up to 1178 tokens with
// heads of 64 (65 MB with the shared prompt counted once a row): 14 us; one row of 77 tokens: 4 us, and 8 with the call.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>
#include "paged_cache.hpp"
#include "operands.hpp"

namespace pg {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

constexpr int PA_THREADS = 256, PA_WAVES = 4;
constexpr int PA_HEADS = 16;                         // query heads of a tile: the columns of a 16 x 16 MFMA

constexpr int PA_PAGES = 512;                        // page numbers in LDS at a time
constexpr int PA_EVEN_QUERIES = 2048;                // whose prefix sums are held in LDS
constexpr int PA_RANGES = 512;                       // of an EVEN call, at most: two workgroups a compute unit, what the registers of wide heads leave
                                                     // room for (384 rows of up to 4096 tokens in codes: 296 us, 335 with 768 and 305 with 1024)

struct PagedArgs {
  CacheView c;
  const uint8_t *k, *v;                              // of the layer
  const float *k_scale, *v_scale;
  const uint16_t* q;
  int64_t q_stride, out_stride;
  const int32_t *table, *row_of, *lens;
  int n_q, n_rows, heads_q, group, q_tiles;
  float scale_log2;
  uint16_t* out;
  float* lse;
  int ranges, log2_ranges;                           // EVEN: workgroups
  int64_t* total;                                    // EVEN: units of all rows, heads and tiles, for the second launch
  int4* opened;                                      // EVEN: query, head tile, unit and units of the row that each range begins in
  float* parts;                                      // EVEN: [range][first, last][query head of the tile][HD + 4]: m, l, -, -, o'
};

// tokens of a query, and whether its row and length are what the table holds
__device__ __forceinline__ int query_length(const PagedArgs& a, int query, int& row) {
  row = a.row_of ? a.row_of[query] : query;
  const int len = a.lens[query];
  if ((unsigned)row < (unsigned)a.n_rows && len >= 0 && (int64_t)len <= (int64_t)a.c.width << a.c.page_shift) return len;
  atomicOr(a.c.status, CACHE_RANGE);
  row = 0;
  return 0;
}
// first unit of a range
__device__ __forceinline__ int64_t range_start(int64_t total, int log2_ranges, int r) { return total * r >> log2_ranges; }

__device__ __forceinline__ bf16x8 as_bf16(uint4 w) { return __builtin_bit_cast(bf16x8, w); }
// a and b cut to bf16
__device__ __forceinline__ uint32_t upper_halves(float a, float b) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
}
// eight codes -> eight bf16 (exact: e4m3 has three bits of fraction)
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t a, uint32_t b) {
  const auto x0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)a, false), x1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)a, true);
  const auto x2 = __builtin_amdgcn_cvt_pk_f32_fp8((int)b, false), x3 = __builtin_amdgcn_cvt_pk_f32_fp8((int)b, true);
  return as_bf16(uint4{pack_bf16x2(x0[0], x0[1]), pack_bf16x2(x1[0], x1[1]), pack_bf16x2(x2[0], x2[1]), pack_bf16x2(x3[0], x3[1])});
}

template <int HD, bool F8>
struct Step {
  static constexpr int KEYS = F8 ? 64 : 32;          // of a step
  static constexpr int U = KEYS / 32;                // groups of 32 keys: one MFMA of O^T each
  static constexpr int ELT = F8 ? 1 : 2;
  static constexpr int PIECE = HD * ELT / 4 < 16 ? HD * ELT / 4 : 16;   // bytes of a key row that a lane loads at once
  static constexpr int PIECES = HD * ELT / 4 / PIECE;
  static constexpr int OCTETS = HD / 32;             // MFMAs along a key row
};

// The query's operand registers: octet j of lane (n, c) holds the eight channels that the key operand has there.
template <int HD, bool F8>
__device__ __forceinline__ int channel_of(int j, int c) {
  using S = Step<HD, F8>;
  if (!F8 || S::PIECE == 8) return j * 32 + c * 8;
  return (j >> 1) * 64 + c * 16 + (j & 1) * 8;
}

struct Piece { float m, l; };
// what the sum of a softmax gives: nothing to divide by where no score has a weight, NaN where one was NaN
__device__ __forceinline__ float over(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f; }

template <int HD, bool F8, bool EVEN>
__global__ __launch_bounds__(PA_THREADS, 2) void paged_attention_kernel(PagedArgs a) {
  using S = Step<HD, F8>;
  constexpr int DT = HD / 16, U = S::U;              // tiles of channels, groups of 32 keys
  constexpr int UNIT = PA_WAVES * S::KEYS;           // tokens: a step of each wave
  __shared__ __align__(16) float lds_o[PA_WAVES][PA_HEADS][HD + 4];
  __shared__ Piece lds_ml[PA_WAVES][PA_HEADS];
  __shared__ int lds_page[PA_PAGES + 4];
  __shared__ int lds_cum[EVEN ? PA_EVEN_QUERIES : 1];
  const int lane = threadIdx.x & 63, n = lane & 15, c = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int shift = a.c.page_shift, page_tokens = 1 << shift;
  const uint32_t head_bytes = (uint32_t)(HD * S::ELT) << shift, page_bytes = head_bytes * (uint32_t)a.c.heads;

  // EVEN: consecutive ranges on one XCD, so that rows of one head that share pages find them in its L2
  const int range = EVEN ? (int)(blockIdx.x % 8) * (a.ranges / 8) + (int)(blockIdx.x / 8) : 0;
  int units = 0;                                     // of all queries, one head and tile
  int64_t at = 0, stop = 1;                          // EVEN: units, of all heads and tiles
  if constexpr (EVEN) {
    int mine[PA_EVEN_QUERIES / PA_THREADS];
    const int per = (a.n_q + PA_THREADS - 1) / PA_THREADS, first = threadIdx.x * per;
#pragma unroll
    for (int i = 0; i < PA_EVEN_QUERIES / PA_THREADS; ++i) {
      int row;
      mine[i] = i < per && first + i < a.n_q ? (query_length(a, first + i, row) + UNIT - 1) / UNIT : 0;
    }
    int sum = 0;
#pragma unroll
    for (int i = 0; i < PA_EVEN_QUERIES / PA_THREADS; ++i) sum += mine[i];
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 63) lds_page[wave] = incl;
    __syncthreads();
    int before = incl - sum;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) {
      before += w < wave ? lds_page[w] : 0;
      units += lds_page[w];
    }
#pragma unroll
    for (int i = 0; i < PA_EVEN_QUERIES / PA_THREADS; ++i)
      if (i < per && first + i < a.n_q) {
        lds_cum[first + i] = before += mine[i];
        if (mine[i] == 0 && (first + i) % a.ranges == range)     // no tokens: nobody else comes by
          for (int e = 0; e < a.heads_q; ++e) {
            for (int ch = 0; ch < HD; ch += 8) *(uint4*)(a.out + (first + i) * a.out_stride + (int64_t)e * HD + ch) = uint4{0, 0, 0, 0};
            if (a.lse) a.lse[(int64_t)(first + i) * a.heads_q + e] = -INFINITY;
          }
      }
    __syncthreads();
    const int64_t total = (int64_t)units * a.c.heads * a.q_tiles;
    at = range_start(total, a.log2_ranges, range);
    stop = range_start(total, a.log2_ranges, range + 1);
    if (threadIdx.x == 0) {
      if (range == 0) *a.total = total;
      if (at >= stop) a.opened[range] = int4{0, 0, 0, 0};
    }
  }
  int query = EVEN ? -1 : (int)blockIdx.z, ht = EVEN ? 0 : (int)blockIdx.y;
  for (bool opening = true; at < stop; opening = false) {
  int begin = 0, row, len, whole_units = 0, first_unit = 0, last_unit = 0;
  if constexpr (EVEN) {
    ht = (int)(at / units);
    const int rest = (int)(at % units);
    if (query < 0 || rest == 0) {                    // the range, or a head, begins: first query with cum > rest
      int lo = 0, hi = a.n_q - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (lds_cum[mid] > rest) hi = mid; else lo = mid + 1;
      }
      query = lo;
    } else {
      do ++query;                                    // rest < units, which is the last one's cum
      while (lds_cum[query] <= rest);
    }
    query = __builtin_amdgcn_readfirstlane(query);
    const int base = query ? lds_cum[query - 1] : 0;
    whole_units = lds_cum[query] - base;
    first_unit = rest - base;
    last_unit = (int)min((int64_t)whole_units, first_unit + (stop - at));
    at += last_unit - first_unit;
    begin = first_unit * UNIT;
    if (opening && threadIdx.x == 0) a.opened[range] = int4{query, ht, first_unit, whole_units};
  }
  len = query_length(a, query, row);
  const int finish = EVEN ? min(len, last_unit * UNIT) : len;
  if constexpr (!EVEN) at = stop;
  const int h = ht / a.q_tiles, tile = ht % a.q_tiles;
  const int heads = min(PA_HEADS, a.group - tile * PA_HEADS);           // of this tile
  const int head0 = h * a.group + tile * PA_HEADS;

  bf16x8 q[S::OCTETS];
#pragma unroll
  for (int j = 0; j < S::OCTETS; ++j) {
    uint4 w = {0, 0, 0, 0};
    if (n < heads) w = *(const uint4*)(a.q + query * a.q_stride + (int64_t)(head0 + n) * HD + channel_of<HD, F8>(j, c));
    q[j] = as_bf16(w);
  }
  const float scale = a.scale_log2 * (a.k_scale ? a.k_scale[h] : 1.0f);

  f32x4v o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x4v{0.f, 0.f, 0.f, 0.f};
  float m = -FLT_MAX, l = 0.0f;
  const uint8_t* k_head = a.k + (int64_t)h * head_bytes;
  const uint8_t* v_head = a.v + (int64_t)h * head_bytes;
  // lane (r = n, c): key row r of tile t is key 8 U (r / 4) + 4 t + r % 4 of the step; it multiplies keys 8 U c ... 8 U c + 8 U - 1
  const int key_lane = 8 * U * (n >> 2) + (n & 3), key_values = 8 * U * c;

  for (; begin < finish; begin += PA_PAGES << shift) {
    const int end = (int)min((int64_t)finish, begin + ((int64_t)PA_PAGES << shift));
    const int pages = (end - begin + (begin & (page_tokens - 1)) + page_tokens - 1) >> shift;
    const int32_t* table = a.table + (int64_t)row * a.c.width + (begin >> shift);
    __syncthreads();                                 // what was there has been read
    // page numbers; steps that reach past the last page find it again
    for (int i = threadIdx.x; i < pages + 4; i += PA_THREADS) {
      int p = table[min(i, pages - 1)];
      if ((unsigned)p >= (unsigned)a.c.n_pages) {
        atomicOr(a.c.status, CACHE_RANGE);
        p = 0;
      }
      lds_page[i] = p;
    }
    __syncthreads();
    uint4 kr[2 * U][S::PIECES], vr[DT];
    auto load_keys = [&](int key0) {                 // key0: of the step, from the chunk's begin
#pragma unroll
      for (int t = 0; t < 2 * U; ++t) {
        const int key = key0 + key_lane + 4 * t;
        const uint8_t* p = k_head + (uint64_t)(uint32_t)lds_page[key >> shift] * page_bytes +
                           (uint32_t)((key & (page_tokens - 1)) * (HD * S::ELT) + c * S::PIECE);
#pragma unroll
        for (int j = 0; j < S::PIECES; ++j) {
          if constexpr (S::PIECE == 16) kr[t][j] = *(const uint4*)(p + j * 64);
          else *(uint2*)&kr[t][j] = *(const uint2*)p;
        }
      }
    };
    auto load_values = [&](int key0) {
      const int key = key0 + key_values;
      const uint8_t* p = v_head + (uint64_t)(uint32_t)lds_page[key >> shift] * page_bytes +
                         (uint32_t)(((n << shift) + (key & (page_tokens - 1))) * S::ELT);
#pragma unroll
      for (int d = 0; d < DT; ++d) vr[d] = *(const uint4*)(p + (((uint32_t)d * 16 * S::ELT) << shift));
    };
    const int tokens = end - begin;
    int key0 = wave * S::KEYS;
    if (key0 < tokens) {
      load_keys(key0);
      load_values(key0);
    }
    // MORE: a step follows, whose keys and values are asked for.  Under a branch inside the loop they made every wait for values wait for
    // the keys of the next step, too: the compiler has to assume that nothing was asked for after the values.
    auto work = [&](auto more) {
      constexpr bool MORE = decltype(more)::value;
      const int next = key0 + PA_WAVES * S::KEYS;
      f32x4v s[2 * U];
#pragma unroll
      for (int t = 0; t < 2 * U; ++t) {
        s[t] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < S::PIECES; ++j) {
          const uint4 w = kr[t][j];
          if constexpr (!F8) {
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(w), q[j], s[t], 0, 0, 0);
          } else if constexpr (S::PIECE == 8) {
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(w.x, w.y), q[j], s[t], 0, 0, 0);
          } else {
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(w.x, w.y), q[2 * j], s[t], 0, 0, 0);
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(w.z, w.w), q[2 * j + 1], s[t], 0, 0, 0);
          }
        }
      }
      if constexpr (MORE) load_keys(next);
      const int there = tokens - key0;               // keys of the step that exist, if fewer than KEYS
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2 * U; ++t) {
        s[t] *= scale;
        // without a branch around it: where scores are first read behind one, this compiler has left out the wait states that a product's
        // result needs, and read some of them too early
        if constexpr (!MORE) {
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][i] = key_values + 4 * t + i < there ? s[t][i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
      }
      top = across_rows(top, [](float x, float y) { return fmaxf(x, y); });
      if (__ballot(top > m)) {                       // seldom after a row's first steps
        const float m_new = fmaxf(m, top);
        const float shrink = __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= shrink;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= shrink;
      }
      // a probability is kept as the sum of two bf16: the matrix pipe has time for both, and 8 bits alone would make the output's error
      // 1.4 times as large.  Where values may be infinite (codes are not), both parts have to be positive, or infinity would meet a 0 or its
      // opposite: the first is the probability cut to 8 bits, not rounded, and the second at least the smallest normal number
      bf16x8 hi[U], lo[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float p[8], rest[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(s[2 * u + (e >> 2)][e & 3] - m);
          l += p[e];
        }
        if constexpr (F8) {
          hi[u] = as_bf16(uint4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])});
#pragma unroll
          for (int e = 0; e < 8; ++e) rest[e] = p[e] - (float)hi[u][e];
        } else {
          hi[u] = as_bf16(uint4{upper_halves(p[0], p[1]), upper_halves(p[2], p[3]), upper_halves(p[4], p[5]), upper_halves(p[6], p[7])});
#pragma unroll
          for (int e = 0; e < 8; ++e) rest[e] = fmaxf(p[e] - (float)hi[u][e], FLT_MIN);
        }
        lo[u] = as_bf16(uint4{pack_bf16x2(rest[0], rest[1]), pack_bf16x2(rest[2], rest[3]), pack_bf16x2(rest[4], rest[5]), pack_bf16x2(rest[6], rest[7])});
      }
      if (!MORE && there < S::KEYS) {                // what lies behind the last token may be anything, NaN too
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          uint32_t w[4] = {vr[d].x, vr[d].y, vr[d].z, vr[d].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            constexpr int PER = 4 / S::ELT;          // keys of a word
            const int left = there - key_values - e * PER;
            w[e] = left >= PER ? w[e] : left <= 0 ? 0u : w[e] & ((1u << (8 * S::ELT * left)) - 1);
          }
          vr[d] = uint4{w[0], w[1], w[2], w[3]};
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const uint4 w = vr[d];
        if constexpr (!F8) {
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(w), hi[0], o[d], 0, 0, 0);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(w), lo[0], o[d], 0, 0, 0);
        } else {
          const bf16x8 v0 = codes_to_bf16(w.x, w.y), v1 = codes_to_bf16(w.z, w.w);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, hi[0], o[d], 0, 0, 0);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, lo[0], o[d], 0, 0, 0);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, hi[1], o[d], 0, 0, 0);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, lo[1], o[d], 0, 0, 0);
        }
      }
      if constexpr (MORE) load_values(next);
      key0 = next;
    };
    while (key0 + PA_WAVES * S::KEYS < tokens) work(std::true_type{});
    if (key0 < tokens) work(std::false_type{});
  }
  l = across_rows(l, [](float x, float y) { return x + y; });
#pragma unroll
  for (int d = 0; d < DT; ++d) *(f32x4v*)&lds_o[wave][n][d * 16 + c * 4] = o[d];
  if (c == 0) lds_ml[wave][n] = Piece{m, l};
  __syncthreads();
  // the four waves' pieces; thread: head i / (HD / 4), four channels
  const float v_scale = a.v_scale ? a.v_scale[h] : 1.0f;
  for (int i = threadIdx.x; i < heads * (HD / 4); i += PA_THREADS) {
    const int head = i / (HD / 4), ch = i % (HD / 4) * 4;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) top = fmaxf(top, lds_ml[w][head].m);
    float sum = 0.0f;
    f32x4v acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) {
      const Piece p = lds_ml[w][head];
      const float f = __builtin_amdgcn_exp2f(p.m - top);
      sum += p.l * f;
      acc += *(const f32x4v*)&lds_o[w][head][ch] * f;
    }
    acc *= v_scale;
    const int64_t item = (int64_t)query * a.heads_q + head0 + head;
    if (!EVEN || last_unit - first_unit == whole_units) {
      acc *= over(sum);
      *(uint2*)(a.out + query * a.out_stride + (int64_t)(head0 + head) * HD + ch) = pack_bf16x4(float4{acc[0], acc[1], acc[2], acc[3]});
      if (a.lse && ch == 0) a.lse[item] = lse_of(top, sum);
    } else {
      float* part = a.parts + (((int64_t)range * 2 + !opening) * PA_HEADS + head) * (HD + 4);
      *(f32x4v*)(part + 4 + ch) = acc;
      if (ch == 0) *(float2*)part = float2{top, sum};
    }
  }
  }
}

// Joins the pieces of the row that range r begins in, if r is the first to begin inside of it: one query head, every HD / 4 threads go
// through a part of the pieces, four channels each.
template <int HD>
__global__ __launch_bounds__(PA_THREADS) void paged_join_kernel(PagedArgs a) {
  constexpr int LANES = HD / 4, PARTS = PA_THREADS / LANES;
  __shared__ __align__(16) float lds_o[PARTS][HD];
  __shared__ Piece lds_ml[PARTS];
  const int r0 = blockIdx.x, column = blockIdx.y, part = threadIdx.x / LANES, ch = threadIdx.x % LANES * 4;
  const int4 row = a.opened[r0];
  const int64_t total = *a.total;
  if (row.z == 0) return;
  const auto start = [&](int r) { return range_start(total, a.log2_ranges, r); };
  const auto last_before = [&](int64_t unit) { return (int)((((uint64_t)unit << a.log2_ranges) - 1) / (uint64_t)total); };   // range, unit >= 1
  const int64_t start0 = start(r0), begin = start0 - row.z, end = begin + row.w;
  const int tile = row.y % a.q_tiles, head = row.y / a.q_tiles * a.group + tile * PA_HEADS + column;
  const int before = last_before(start0);            // the range that ends here; there are empty ones where units are few
  if (start(before) > begin || column >= a.group - tile * PA_HEADS) return;
  const int last = last_before(end);
  Piece x = {-INFINITY, 0.0f};
  f32x4v acc = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](Piece y, f32x4v o) {
    if (y.m == -INFINITY) return;                    // no piece
    const float m = fmaxf(x.m, y.m), f = __builtin_amdgcn_exp2f(x.m - m), g = __builtin_amdgcn_exp2f(y.m - m);
    x = Piece{m, x.l * f + y.l * g};
    acc = acc * f + o * g;
  };
  // a range's piece of this row is its first, but for a range that begins before the row: there it is the last
  constexpr int AHEAD = 4;
  for (int i = before + part; i <= last; i += AHEAD * PARTS) {
    Piece y[AHEAD];
    f32x4v o[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int at = i + k * PARTS, r = at <= last ? at : before;
      const float* p = a.parts + ((int64_t)(2 * r + (start(r) < begin)) * PA_HEADS + column) * (HD + 4);
      const float2 ml = *(const float2*)p;
      y[k] = Piece{at <= last && start(at) < start(at + 1) ? ml.x : -INFINITY, ml.y};
      o[k] = *(const f32x4v*)(p + 4 + ch);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) add(y[k], o[k]);
  }
  *(f32x4v*)&lds_o[part][ch] = acc;
  if (ch == 0) lds_ml[part] = x;
  __syncthreads();
  if (part) return;
#pragma unroll
  for (int i = 1; i < PARTS; ++i) add(lds_ml[i], *(const f32x4v*)&lds_o[i][ch]);
  acc *= over(x.l);
  *(uint2*)(a.out + row.x * a.out_stride + (int64_t)head * HD + ch) = pack_bf16x4(float4{acc[0], acc[1], acc[2], acc[3]});
  if (a.lse && ch == 0) a.lse[(int64_t)row.x * a.heads_q + head] = lse_of(x.m, x.l);
}

// Ranges of an EVEN call, 0 for WHOLE.  `span` is the longest row in units of heads of 128 channels, each of which takes a workgroup
// alone 1.3 us; heads of 64 and 32 take 0.6 and 0.3, with codes 0.8 and 0.6 (a part of their steps does not depend on the width).
// EVEN costs 7 us more (prefix sums, second launch), and an item's span some 1/200 of that of a workgroup alone once all items share the
// device's bandwidth; longer rows are left waiting for at the end of a WHOLE call in any number, sooner where there
// are more items than compute units.  WHOLE and EVEN in us, rows of 1 token up to the span, by items x span:  8 x 8: 13.7, 11.6;
// 8 x 32: 45, 12.2;  32 x 8: 13.7, 11.8;  128 x 8: 14.1, 19.2;  128 x 16: 25.1, 25.0;  256 x 16: 27.8, 33.3;  384 x 8: 25.5, 28.4;
// 384 x 14: 40, 37;  576 x 16: 77, 55;  768 x 14: 67, 69;  768 x 32: 178, 161;  1024 x 128: 822, 748;  3072 x 8: 157, 166;  3072 x 32: 575, 566;
// and rows that are all of one length: 1024 x 13: 144, 155.
struct PagedSplit {
  int64_t item, unit, units, span;                   // items of a query; tokens of a unit, units of the longest row; span in 128ths
  PagedSplit(const pg_cache* c, int heads_q, int max_len) {
    item = c->heads * ((heads_q / c->heads + PA_HEADS - 1) / PA_HEADS);
    unit = c->dtype == PG_CACHE_E4M3 ? 256 : 128;
    units = (max_len + unit - 1) / unit;
    span = units * (c->dtype == PG_CACHE_E4M3 ? (c->head_dim + 64) * 2 / 3 : c->head_dim);
  }
  bool long_rows(int64_t n_q) const { return span > (n_q * item > 256 ? 12 : 16) * 128; }
  bool few_rows(int64_t n_q) const { return span > 6 * 128 + n_q * item * span / 200; }
  int ranges(int64_t n_q) const {
    int64_t r = 8;                                   // no more than there are units: empty ones cost the join its time
    while (r < PA_RANGES && r < n_q * item * units) r *= 2;
    return (int)r;
  }
};
static int ranges_of(const pg_cache* c, int64_t n_q, int heads_q, int max_len) {
  const PagedSplit s(c, heads_q, max_len);
  if (n_q > PA_EVEN_QUERIES || !(s.long_rows(n_q) || s.few_rows(n_q))) return 0;
  if (n_q * ((int64_t)c->width * c->page / s.unit + 1) > 1 << 30) return 0;    // units are counted in 32 bits
  return s.ranges(n_q);
}
static size_t paged_bytes(const pg_cache* c, int ranges) {
  return ranges ? 16 + (size_t)ranges * (sizeof(int4) + 2 * PA_HEADS * (c->head_dim + 4) * sizeof(float)) : 0;
}

static pg_status paged_sizes(const pg_cache* c, int32_t n_q, int32_t heads_q, int32_t max_len, const char* who) {
  PG_TRY(check_cache(c, true, who));
  if (n_q < 0 || heads_q < 1 || max_len < 0) return fail(PG_EINVAL, "%s: %d queries of %d heads, lengths up to %d", who, n_q, heads_q, max_len);
  if (heads_q % c->heads) return fail(PG_ESHAPE, "%s: %d query heads for %d key/value heads", who, heads_q, c->heads);
  const int64_t tiles = (heads_q / c->heads + PA_HEADS - 1) / PA_HEADS;
  if (n_q > 65535 || c->heads * tiles > 65535 || n_q * c->heads * tiles >= 1 << 24)
    return fail(PG_ESHAPE, "%s: %d queries of %d heads pass a launch's 65535 rows or 2^24 workgroups", who, n_q, heads_q);
  return PG_OK;
}

}  // namespace pg

using namespace pg;

extern "C" size_t pg_paged_attention_workspace(const pg_cache* c, int32_t n_q, int32_t heads_q, int32_t max_len) {
  if (paged_sizes(c, n_q, heads_q, max_len, "pg_paged_attention_workspace") != PG_OK) return 0;
  // What any call of no more and no longer queries needs.  Some of them is cut into ranges if the one of most queries is, which has
  // the lower bound on long rows, or one query alone, which are the fewest; it has the most ranges with as many queries as ranges are for.
  const PagedSplit s(c, heads_q, max_len);
  const int64_t most = std::min(n_q, PA_EVEN_QUERIES);
  return n_q && (s.long_rows(most) || s.few_rows(1)) ? paged_bytes(c, s.ranges(most)) : 0;
}

extern "C" pg_status pg_paged_attention(const pg_cache* c, int32_t layer, const uint16_t* q, int64_t q_stride, const int32_t* table,
                                        int32_t n_rows, const int32_t* row_of, const int32_t* lens, int32_t n_q, int32_t heads_q,
                                        double scale, int32_t max_len, uint16_t* out, int64_t out_stride, float* lse, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  const char* who = "pg_paged_attention";
  PG_TRY(paged_sizes(c, n_q, heads_q, max_len, who));
  if (layer < 0 || layer >= c->layers) return fail(PG_EINVAL, "%s: layer %d of %d", who, layer, c->layers);
  const float scale_log2 = (float)((scale == 0.0 ? 1.0 / std::sqrt((double)c->head_dim) : scale) * 1.4426950408889634);
  if (!std::isfinite(scale_log2)) return fail(PG_EINVAL, "%s: scale is not finite in 32 bits", who);
  if (n_q == 0) return PG_OK;
  if (!q || !table || !lens || !out) return fail(PG_EINVAL, "%s: null pointer", who);
  if (n_rows < 1 || (!row_of && n_rows < n_q)) return fail(PG_EINVAL, "%s: a table of %d rows for %d queries", who, n_rows, n_q);
  PagedArgs a{};
  const int64_t row = (int64_t)heads_q * c->head_dim;
  if (q_stride < row || out_stride < row || q_stride % 8 || out_stride % 8 || (((uintptr_t)q | (uintptr_t)out) & 15))
    return fail(PG_ESHAPE, "%s: queries and outputs must be 16-byte aligned, their strides (%lld, %lld) multiples of 8", who,
                (long long)q_stride, (long long)out_stride);
  a.ranges = ranges_of(c, n_q, heads_q, max_len);
  const size_t need = paged_bytes(c, a.ranges);
  if (need && (!workspace || workspace_bytes < need))
    return fail(PG_EWORKSPACE, "%s: %zu bytes of workspace, %zu given", who, need, workspace ? workspace_bytes : 0);
  if ((uintptr_t)workspace & 15) return fail(PG_ESHAPE, "%s: the workspace must be 16-byte aligned", who);
  a.c = view_of(c);
  const size_t layer_bytes = page_bytes(c) * c->n_pages;
  a.k = (const uint8_t*)c->k + layer * layer_bytes;
  a.v = (const uint8_t*)c->v + layer * layer_bytes;
  a.k_scale = c->k_scale ? c->k_scale + (int64_t)layer * c->heads : nullptr;
  a.v_scale = c->v_scale ? c->v_scale + (int64_t)layer * c->heads : nullptr;
  a.q = q; a.q_stride = q_stride; a.out = out; a.out_stride = out_stride;
  a.table = table; a.row_of = row_of; a.lens = lens; a.n_rows = n_rows;
  a.heads_q = heads_q; a.group = heads_q / c->heads; a.q_tiles = (a.group + PA_HEADS - 1) / PA_HEADS;
  a.n_q = n_q;
  a.scale_log2 = scale_log2;
  a.lse = lse;
  a.opened = (int4*)workspace; a.parts = (float*)(a.opened + a.ranges);
  a.total = (int64_t*)(a.parts + (size_t)a.ranges * 2 * PA_HEADS * (c->head_dim + 4));
  while (1 << a.log2_ranges < a.ranges) ++a.log2_ranges;
  const dim3 block(PA_THREADS), join((unsigned)a.ranges, (unsigned)std::min(a.group, PA_HEADS));
  const dim3 grid = a.ranges ? dim3((unsigned)a.ranges) : dim3(1, (unsigned)(c->heads * a.q_tiles), (unsigned)n_q);
  hipStream_t s = (hipStream_t)stream;
  const bool f8 = c->dtype == PG_CACHE_E4M3;
#define PG_PAGED(HD)                                                                                                       \
  do {                                                                                                                     \
    if (!a.ranges) {                                                                                                       \
      f8 ? paged_attention_kernel<HD, true, false><<<grid, block, 0, s>>>(a) : paged_attention_kernel<HD, false, false><<<grid, block, 0, s>>>(a); \
    } else {                                                                                                               \
      f8 ? paged_attention_kernel<HD, true, true><<<grid, block, 0, s>>>(a) : paged_attention_kernel<HD, false, true><<<grid, block, 0, s>>>(a);   \
      PG_LAUNCH_CHECK("paged_attention_kernel");                                                                           \
      paged_join_kernel<HD><<<join, block, 0, s>>>(a);                                                                     \
    }                                                                                                                      \
  } while (0)
  if (c->head_dim == 32) PG_PAGED(32);
  else if (c->head_dim == 64) PG_PAGED(64);
  else PG_PAGED(128);
#undef PG_PAGED
  PG_LAUNCH_CHECK(a.ranges ? "paged_join_kernel" : "paged_attention_kernel");
  return PG_OK;
}
