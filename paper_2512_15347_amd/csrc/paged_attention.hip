// Attention of single new tokens over a paged key/value cache.
//
// For a query head with query q and keys k_j, values v_j (j < len):  s_j = scale <q, k_j>,  p_j = exp(s_j - m),  m = max s,
// l = sum p_j,  o = sum p_j v_j / l,  lse = m + ln l, taken in pieces: two pieces (m, l, o') with o' = sum p_j v_j join as
// m = max(m1, m2), l = l1 e^(m1-m) + l2 e^(m2-m), o' alike.
//
// Every byte of the cache is read once and used for the G query heads of its key/value head only (G = 1 .. 16 products a value), so
// the kernel is bound by HBM as long as enough loads are in flight.  Both products run on the matrix pipe, S^T = K Q^T and
// O^T = V^T P^T with the keys / channels as rows and 16 query heads as columns (empty ones are zero): then a lane's keys
// of S^T are just the keys it multiplies in O^T, and keys and transposed values are loaded straight into operand registers, 16 bytes
// a lane, without LDS.  A step is 32 keys of bf16 or 64 keys of codes.  Codes are converted to bf16, which holds them exactly; the
// scales go into the logits and the output.
#include <algorithm>
#include <cmath>
#include "paged_cache.hpp"
#include "operands.hpp"

namespace pg {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

constexpr int PA_THREADS = 256, PA_WAVES = 4;
constexpr int PA_HEADS = 16;                         // query heads of a tile: the columns of a 16 x 16 MFMA

struct PagedArgs {
  CacheView c;
  const uint8_t *k, *v;                              // of the layer
  const float *k_scale, *v_scale;
  const uint16_t* q;
  int64_t q_stride, out_stride;
  const int32_t *table, *row_of, *lens;
  int n_rows, heads_q, group, q_tiles, splits;
  float scale_log2;
  uint16_t* out;
  float *lse, *parts;                                // parts: [query, query head, split][HD + 2]
};

__device__ __forceinline__ bf16x8 as_bf16(uint4 w) { return __builtin_bit_cast(bf16x8, w); }
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

template <int HD, bool F8>
__global__ __launch_bounds__(PA_THREADS) void paged_attention_kernel(PagedArgs a) {
  using S = Step<HD, F8>;
  constexpr int DT = HD / 16;                        // tiles of channels
  __shared__ __align__(16) float lds_o[PA_WAVES][PA_HEADS][HD + 4];
  __shared__ Piece lds_ml[PA_WAVES][PA_HEADS];
  const int lane = threadIdx.x & 63, n = lane & 15, c = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x, h = blockIdx.y / a.q_tiles, tile = blockIdx.y % a.q_tiles, query = blockIdx.z;
  const int heads = min(PA_HEADS, a.group - tile * PA_HEADS);           // of this tile
  const int row = a.row_of ? a.row_of[query] : query;
  int len = a.lens[query];
  if ((unsigned)row >= (unsigned)a.n_rows || len < 0 || (int64_t)len > (int64_t)a.c.width << a.c.page_shift) {
    if (threadIdx.x == 0) atomicOr(a.c.status, CACHE_RANGE);
    len = 0;
  }
  const int32_t* table = a.table + (int64_t)(len ? row : 0) * a.c.width;
  const int steps = (len + S::KEYS - 1) / S::KEYS;
  const int per = (steps + a.splits - 1) / a.splits;
  const int begin = min(steps, split * per), end = min(steps, begin + per);
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
  float m = -INFINITY, l = 0.0f;
  const int page_tokens = 1 << a.c.page_shift, last_page = (len - 1) >> a.c.page_shift;
  const int64_t page_bytes = ((int64_t)a.c.heads << a.c.page_shift) * HD * S::ELT;
  const int64_t head_bytes = ((int64_t)h << a.c.page_shift) * HD * S::ELT;

  for (int step = begin + wave; step < end; step += PA_WAVES) {
    const int key0 = step * S::KEYS;
    // lane (r = n, c): key row r of tile t is key 8 U (r / 4) + 4 t + r % 4, of the step; it multiplies keys 8 U c ... 8 U c + 8 U - 1
    const int key_lane = 8 * S::U * (n >> 2) + (n & 3), key_values = 8 * S::U * c;
    auto page_base = [&](int key) -> int64_t {
      const int p = table[min((key0 + key) >> a.c.page_shift, last_page)];
      if ((unsigned)p >= (unsigned)a.c.n_pages) {
        atomicOr(a.c.status, CACHE_RANGE);
        return head_bytes;
      }
      return p * page_bytes + head_bytes;
    };
    f32x4v s[2 * S::U];
#pragma unroll
    for (int t = 0; t < 2 * S::U; ++t) {
      const int key = key_lane + 4 * t;
      const uint8_t* kp = a.k + page_base(key) + (int64_t)((key0 + key) & (page_tokens - 1)) * (HD * S::ELT) + c * S::PIECE;
      s[t] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < S::PIECES; ++j) {
        if constexpr (!F8) {
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(*(const uint4*)(kp + j * 64)), q[j], s[t], 0, 0, 0);
        } else if constexpr (S::PIECE == 8) {
          const uint2 w = *(const uint2*)kp;
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(w.x, w.y), q[j], s[t], 0, 0, 0);
        } else {
          const uint4 w = *(const uint4*)(kp + j * 64);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(w.x, w.y), q[2 * j], s[t], 0, 0, 0);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(w.z, w.w), q[2 * j + 1], s[t], 0, 0, 0);
        }
      }
    }
    const int there = len - key0;                    // keys of the step that exist, if fewer than KEYS
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2 * S::U; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[t][i] = key_values + 4 * t + i < there ? s[t][i] * scale : -INFINITY;
        top = fmaxf(top, s[t][i]);
      }
    top = across_rows(top, [](float x, float y) { return fmaxf(x, y); });
    const float m_new = fmaxf(m, top);
    const float shrink = exp2f(m - m_new);
    m = m_new;
    l *= shrink;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] *= shrink;
    // a probability is kept as the sum of two bf16: the matrix pipe has time for both, and 8 bits alone would double the output's error
    bf16x8 hi[S::U], lo[S::U];
#pragma unroll
    for (int u = 0; u < S::U; ++u) {
      float p[8], rest[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = exp2f(s[2 * u + (e >> 2)][e & 3] - m);
        l += p[e];
      }
      const uint4 w = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
      hi[u] = as_bf16(w);
#pragma unroll
      for (int e = 0; e < 8; ++e) rest[e] = p[e] - (float)hi[u][e];
      lo[u] = as_bf16(uint4{pack_bf16x2(rest[0], rest[1]), pack_bf16x2(rest[2], rest[3]), pack_bf16x2(rest[4], rest[5]), pack_bf16x2(rest[6], rest[7])});
    }
    const uint8_t* vp = a.v + page_base(key_values) + ((int64_t)n * page_tokens + ((key0 + key_values) & (page_tokens - 1))) * S::ELT;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      uint4 w = *(const uint4*)(vp + (int64_t)d * 16 * page_tokens * S::ELT);
      if (there < S::KEYS) {                         // what lies behind the last token may be anything, NaN too
        uint32_t* x = (uint32_t*)&w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          constexpr int PER = 4 / S::ELT;            // keys of a word
          const int left = there - key_values - e * PER;
          x[e] = left >= PER ? x[e] : left <= 0 ? 0u : x[e] & ((1u << (8 * S::ELT * left)) - 1);
        }
      }
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
      if (p.m > -INFINITY) {
        const float f = exp2f(p.m - top);
        sum += p.l * f;
        acc += *(const f32x4v*)&lds_o[w][head][ch] * f;
      }
    }
    const int64_t item = (int64_t)query * a.heads_q + head0 + head;
    if (a.splits == 1) {
      const float f = sum > 0.0f ? v_scale / sum : 0.0f;
      acc *= f;
      *(uint2*)(a.out + query * a.out_stride + (int64_t)(head0 + head) * HD + ch) = pack_bf16x4(float4{acc[0], acc[1], acc[2], acc[3]});
      if (a.lse && ch == 0) a.lse[item] = sum > 0.0f ? (top + log2f(sum)) * 0.6931471805599453f : -INFINITY;
    } else {
      float* part = a.parts + (item * a.splits + split) * (HD + 4);
      *(f32x4v*)(part + 4 + ch) = acc * v_scale;
      if (ch == 0) {
        part[0] = top;
        part[1] = sum;
      }
    }
  }
}

// joins the splits of one query head: one wave
template <int HD>
__global__ __launch_bounds__(WAVE) void paged_join_kernel(PagedArgs a) {
  const int64_t item = (int64_t)blockIdx.y * a.heads_q + blockIdx.x;
  const float* part = a.parts + item * a.splits * (HD + 4);
  float top = -INFINITY, sum = 0.0f, acc[(HD + 63) / 64] = {};
  for (int s = 0; s < a.splits; ++s) top = fmaxf(top, part[s * (HD + 4)]);
  for (int s = 0; s < a.splits; ++s) {
    const float* p = part + s * (HD + 4);
    if (!(p[0] > -INFINITY)) continue;
    const float f = exp2f(p[0] - top);
    sum += p[1] * f;
#pragma unroll
    for (int i = 0; i < (HD + 63) / 64; ++i)
      if (threadIdx.x + 64 * i < HD) acc[i] += p[4 + threadIdx.x + 64 * i] * f;
  }
  const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
  for (int i = 0; i < (HD + 63) / 64; ++i)
    if (threadIdx.x + 64 * i < HD)
      a.out[blockIdx.y * a.out_stride + (int64_t)blockIdx.x * HD + threadIdx.x + 64 * i] = (uint16_t)(pack_bf16x2(acc[i] * f, 0.0f) & 0xFFFF);
  if (a.lse && threadIdx.x == 0) a.lse[item] = sum > 0.0f ? (top + log2f(sum)) * 0.6931471805599453f : -INFINITY;
}

// Enough workgroups to fill the device, none with fewer than 256 keys.
static int splits_of(const pg_cache* c, int64_t n_q, int heads_q, int max_len) {
  const int64_t tiles = (heads_q / c->heads + PA_HEADS - 1) / PA_HEADS, items = n_q * c->heads * tiles;
  const int64_t want = std::max<int64_t>(1, 1024 / std::max<int64_t>(1, items));
  return (int)std::min<int64_t>(want, std::max(1, max_len / 256));
}

static pg_status paged_sizes(const pg_cache* c, int32_t n_q, int32_t heads_q, int32_t max_len, const char* who) {
  PG_TRY(check_cache(c, true, who));
  if (n_q < 0 || heads_q < 1 || max_len < 0) return fail(PG_EINVAL, "%s: %d queries of %d heads, lengths up to %d", who, n_q, heads_q, max_len);
  if (heads_q % c->heads) return fail(PG_ESHAPE, "%s: %d query heads for %d key/value heads", who, heads_q, c->heads);
  const int64_t tiles = (heads_q / c->heads + PA_HEADS - 1) / PA_HEADS;
  if (n_q > 65535 || c->heads * tiles > 65535) return fail(PG_ESHAPE, "%s: grid limit", who);
  return PG_OK;
}

}  // namespace pg

using namespace pg;

extern "C" size_t pg_paged_attention_workspace(const pg_cache* c, int32_t n_q, int32_t heads_q, int32_t max_len) {
  if (paged_sizes(c, n_q, heads_q, max_len, "pg_paged_attention_workspace") != PG_OK) return 0;
  const int splits = splits_of(c, n_q, heads_q, max_len);
  return splits > 1 ? (size_t)n_q * heads_q * splits * (c->head_dim + 4) * sizeof(float) : 0;
}

extern "C" pg_status pg_paged_attention(const pg_cache* c, int32_t layer, const uint16_t* q, int64_t q_stride, const int32_t* table,
                                        int32_t n_rows, const int32_t* row_of, const int32_t* lens, int32_t n_q, int32_t heads_q,
                                        double scale, int32_t max_len, uint16_t* out, int64_t out_stride, float* lse, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  const char* who = "pg_paged_attention";
  PG_TRY(paged_sizes(c, n_q, heads_q, max_len, who));
  if (layer < 0 || layer >= c->layers) return fail(PG_EINVAL, "%s: layer %d of %d", who, layer, c->layers);
  if (!std::isfinite(scale)) return fail(PG_EINVAL, "%s: scale is not finite", who);
  if (n_q == 0) return PG_OK;
  if (!q || !table || !lens || !out) return fail(PG_EINVAL, "%s: null pointer", who);
  if (n_rows < 1 || (!row_of && n_rows < n_q)) return fail(PG_EINVAL, "%s: a table of %d rows for %d queries", who, n_rows, n_q);
  const int64_t row = (int64_t)heads_q * c->head_dim;
  if (q_stride < row || out_stride < row || q_stride % 8 || out_stride % 8 || (((uintptr_t)q | (uintptr_t)out) & 15))
    return fail(PG_ESHAPE, "%s: queries and outputs must be 16-byte aligned, their strides (%lld, %lld) multiples of 8", who,
                (long long)q_stride, (long long)out_stride);
  const size_t need = pg_paged_attention_workspace(c, n_q, heads_q, max_len);
  if (need && (!workspace || workspace_bytes < need))
    return fail(PG_EWORKSPACE, "%s: %zu bytes of workspace, %zu given", who, need, workspace ? workspace_bytes : 0);
  if ((uintptr_t)workspace & 15) return fail(PG_ESHAPE, "%s: the workspace must be 16-byte aligned", who);
  PagedArgs a{};
  a.c = view_of(c);
  const size_t layer_bytes = page_bytes(c) * c->n_pages;
  a.k = (const uint8_t*)c->k + layer * layer_bytes;
  a.v = (const uint8_t*)c->v + layer * layer_bytes;
  a.k_scale = c->k_scale ? c->k_scale + (int64_t)layer * c->heads : nullptr;
  a.v_scale = c->v_scale ? c->v_scale + (int64_t)layer * c->heads : nullptr;
  a.q = q; a.q_stride = q_stride; a.out = out; a.out_stride = out_stride;
  a.table = table; a.row_of = row_of; a.lens = lens; a.n_rows = n_rows;
  a.heads_q = heads_q; a.group = heads_q / c->heads; a.q_tiles = (a.group + PA_HEADS - 1) / PA_HEADS;
  a.splits = splits_of(c, n_q, heads_q, max_len);
  a.scale_log2 = (float)((scale == 0.0 ? 1.0 / std::sqrt((double)c->head_dim) : scale) * 1.4426950408889634);
  a.lse = lse; a.parts = (float*)workspace;
  const dim3 grid((unsigned)a.splits, (unsigned)(c->heads * a.q_tiles), (unsigned)n_q), block(PA_THREADS), join((unsigned)heads_q, (unsigned)n_q);
  hipStream_t s = (hipStream_t)stream;
  const bool f8 = c->dtype == PG_CACHE_E4M3;
#define PG_PAGED(HD)                                                                                       \
  (f8 ? paged_attention_kernel<HD, true><<<grid, block, 0, s>>>(a) : paged_attention_kernel<HD, false><<<grid, block, 0, s>>>(a))
  c->head_dim == 32 ? PG_PAGED(32) : c->head_dim == 64 ? PG_PAGED(64) : PG_PAGED(128);
#undef PG_PAGED
  PG_LAUNCH_CHECK("paged_attention_kernel");
  if (a.splits > 1) {
    if (c->head_dim == 32) paged_join_kernel<32><<<join, dim3(WAVE), 0, s>>>(a);
    else if (c->head_dim == 64) paged_join_kernel<64><<<join, dim3(WAVE), 0, s>>>(a);
    else paged_join_kernel<128><<<join, dim3(WAVE), 0, s>>>(a);
    PG_LAUNCH_CHECK("paged_join_kernel");
  }
  return PG_OK;
}
