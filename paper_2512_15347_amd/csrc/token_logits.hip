// Logits of a token policy: penalties, biases and grammar masks, and the draw of a token with its log-prob.
//
// A workgroup takes chunks of one row's vocabulary.  How often each of a chunk's tokens occurs is counted in LDS from the row's
// history (32 bits a token: integer sums, so their order does not matter), so no counts are kept between calls and nothing but the
// history has to follow a member through a prune.  The logits are read once, asked for before the counting starts; groups of eight tokens
// without a count or a bias skip the rules.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include "common.hpp"
#include "operands.hpp"
#include "philox.hpp"

namespace pg {

constexpr int LOGIT_THREADS = 256;
constexpr int LOGIT_WAVES = LOGIT_THREADS / WAVE;
constexpr int LANE_TOKENS = 8;                       // a group: 16 or 32 bytes, two Philox blocks, one byte of a mask
constexpr int PASS_TOKENS = LOGIT_THREADS * LANE_TOKENS;
constexpr uint32_t STREAM_TOKEN = 2u;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// LDS word of a token: how often it is in the output, and whether it is in the prompt or has a bias
constexpr uint32_t IN_PROMPT = 1u << 31, HAS_BIAS = 1u << 30, COUNT = HAS_BIAS - 1;

struct LogitArgs {
  pg_logits d;
  int words;                                         // of a mask
  int per;                                           // chunks of a workgroup
  bool count;                                        // there is a history or a bias list
};

// What one row needs.
struct RowRules {
  float rep, freq, pres;
  const uint8_t* allow;                              // NULL: everything; bit v % 8 of byte v / 8
  int bias_lo, bias_hi, made, prompt;
};

__device__ __forceinline__ RowRules row_rules(const LogitArgs& a, int r) {
  const pg_logits& d = a.d;
  RowRules q;
  q.rep = d.repetition ? d.repetition[r] : 1.0f;
  q.freq = d.frequency ? d.frequency[r] : 0.0f;
  q.pres = d.presence ? d.presence[r] : 0.0f;
  q.allow = nullptr;
  if (d.allow) {
    const int m = d.allow_row ? d.allow_row[r] : r;
    if (m >= 0 && m < d.n_masks) q.allow = (const uint8_t*)(d.allow + (int64_t)m * a.words);
  }
  q.bias_lo = q.bias_hi = q.made = q.prompt = 0;
  if (d.bias_offsets) {
    q.bias_lo = max(0, d.bias_offsets[r]);
    q.bias_hi = min(d.n_bias, d.bias_offsets[r + 1]);
  }
  if (d.tokens) {
    q.made = min(max(d.n_tokens[r], 0), d.tokens_stride);
    q.prompt = d.n_prompt ? min(max(d.n_prompt[r], 0), q.made) : 0;
  }
  return q;
}

// A lane's groups of one chunk: logits from any address that is a multiple of their size (the hardware takes unaligned 16-byte
// loads) and mask bytes.  Group g of the workgroup starts at token g * PASS_TOKENS of the chunk.
template <bool BF16, int G>
struct Groups {
  uint32_t raw[G][BF16 ? 4 : 8];
  uint32_t allowed[G];

  __device__ __forceinline__ void load(const LogitArgs& a, const RowRules& q, int64_t row, int v0, int n) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int i = g * PASS_TOKENS + (int)threadIdx.x * LANE_TOKENS, left = n - i;
      allowed[g] = 0;
      if (left <= 0) continue;
      const char* p = (const char*)a.d.logits + (row + v0 + i) * (BF16 ? 2 : 4);
      if (left >= LANE_TOKENS) {
        __builtin_memcpy(raw[g], p, BF16 ? 16 : 32);
      } else {
#pragma unroll
        for (int e = 0; e < LANE_TOKENS; ++e) {
          const uint32_t x = e >= left ? 0u : BF16 ? ((const uint16_t*)p)[e] : ((const uint32_t*)p)[e];
          if (!BF16) raw[g][e] = x;
          else raw[g][e >> 1] = e & 1 ? raw[g][e >> 1] | x << 16 : x;
        }
      }
      allowed[g] = (q.allow ? q.allow[(v0 + i) >> 3] : 0xFFu) & (left >= LANE_TOKENS ? 0xFFu : (1u << left) - 1);
    }
  }
  __device__ __forceinline__ float logit(int g, int e) const {
    return __builtin_bit_cast(float, !BF16 ? raw[g][e] : e & 1 ? raw[g][e >> 1] & 0xFFFF0000u : raw[g][e >> 1] << 16);
  }
};

// The chunk's LDS words from the history and the bias list.
template <int G>
__device__ __forceinline__ void count_tokens(const LogitArgs& a, const RowRules& q, int r, int v0, int n, uint32_t* lds) {
  const pg_logits& d = a.d;
  __syncthreads();                                   // the words of the chunk before have been read
#pragma unroll
  for (int g = 0; g < 2 * G; ++g) ((uint4*)lds)[g * LOGIT_THREADS + threadIdx.x] = uint4{0, 0, 0, 0};
  __syncthreads();
  const int32_t* t = d.tokens + (int64_t)r * d.tokens_stride;
#pragma unroll 4
  for (int i = threadIdx.x; i < q.made; i += LOGIT_THREADS) {
    const uint32_t at = (uint32_t)t[i] - (uint32_t)v0;
    if (at < (uint32_t)n) {
      if (i < q.prompt) atomicOr(&lds[at], IN_PROMPT);
      else atomicAdd(&lds[at], 1u);
    }
  }
  for (int i = q.bias_lo + threadIdx.x; i < q.bias_hi; i += LOGIT_THREADS) {
    const uint32_t at = (uint32_t)d.bias_ids[i] - (uint32_t)v0;
    if (at < (uint32_t)n) atomicOr(&lds[at], HAS_BIAS);
  }
  __syncthreads();
}

// z of one token that has a count or a bias; the order and the rounding of the operations are the interface's.
__device__ __forceinline__ float adjusted(const LogitArgs& a, const RowRules& q, float x, uint32_t word, int v) {
  if (word & (IN_PROMPT | COUNT)) {
    x = x > 0.0f ? x / q.rep : x * q.rep;
    x = x - q.freq * (float)(word & COUNT);
    if (word & COUNT) x = x - q.pres;
  }
  if (word & HAS_BIAS) {
    int lo = q.bias_lo, hi = q.bias_hi - 1;          // the first entry that is not below v
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.d.bias_ids[mid] < v) lo = mid + 1; else hi = mid;
    }
    if (a.d.bias_ids[lo] == v) x = x + a.d.bias_values[lo];
  }
  return x;
}

// z of group g; tokens that are not allowed, or past the row, get -inf
template <bool BF16, int G>
__device__ __forceinline__ void group_logits(const LogitArgs& a, const RowRules& q, const Groups<BF16, G>& x, int g, int v0, const uint32_t* lds,
                                             float* z) {
#pragma unroll
  for (int e = 0; e < LANE_TOKENS; ++e) z[e] = x.logit(g, e);
  if (a.count) {
    const int i = g * PASS_TOKENS + (int)threadIdx.x * LANE_TOKENS;
    const uint4 w0 = *(const uint4*)(lds + i), w1 = *(const uint4*)(lds + i + 4);
    const uint32_t w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
    if ((w[0] | w[1] | w[2] | w[3]) | (w[4] | w[5] | w[6] | w[7])) {
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e)
        if (w[e]) z[e] = adjusted(a, q, z[e], w[e], v0 + i + e);
    }
  }
#pragma unroll
  for (int e = 0; e < LANE_TOKENS; ++e) z[e] = x.allowed[g] >> e & 1 ? z[e] : -INFINITY;
}

template <bool BF16, int G>
__global__ __launch_bounds__(LOGIT_THREADS) void logits_adjust_kernel(LogitArgs a, float* out, int64_t out_stride) {
  extern __shared__ uint32_t lds[];
  constexpr int CHUNK = G * PASS_TOKENS;
  const int r = blockIdx.y, v0 = blockIdx.x * CHUNK;
  const int n = min(CHUNK, a.d.vocab - v0);
  const RowRules q = row_rules(a, r);
  Groups<BF16, G> x;
  x.load(a, q, (int64_t)r * a.d.stride, v0, n);
  if (a.count) count_tokens<G>(a, q, r, v0, n, lds);
  float* to = out + (int64_t)r * out_stride + v0;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int i = g * PASS_TOKENS + (int)threadIdx.x * LANE_TOKENS, left = n - i;
    if (left <= 0) continue;
    float z[8];
    group_logits<BF16, G>(a, q, x, g, v0, lds, z);
    if (left >= LANE_TOKENS) {
      __builtin_memcpy(to + i, z, 32);
    } else {
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e)
        if (e < left) to[i + e] = z[e];
    }
  }
}

// ---------------------------------------------------------------- the draw
// What a chunk, a wave or a lane knows of a row: the largest y and the sum of exp(y - top) (NaN once a y was NaN or +inf), the best
// score with its token and that token's y.
struct Draw {
  float top, sum, score, y;
  int token;                                         // INT_MAX: none
};
__device__ __forceinline__ Draw no_draw() { return Draw{-FLT_MAX, 0.0f, -INFINITY, -INFINITY, INT32_MAX}; }
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }
__device__ __forceinline__ void join(Draw& a, const Draw& b) {
  const float top = fmaxf(a.top, b.top);
  a.sum = a.sum * exp_of(a.top - top) + b.sum * exp_of(b.top - top);
  a.top = top;
  if (b.score > a.score || (b.score == a.score && b.token < a.token)) {
    a.score = b.score;
    a.token = b.token;
    a.y = b.y;
  }
}
template <int CTRL>
__device__ __forceinline__ int permuted(int w) { return __builtin_amdgcn_update_dpp(w, w, CTRL, 0xF, 0xF, false); }
__device__ __forceinline__ float wave_max(float v) {
  auto f = [](int w) { return __builtin_bit_cast(float, w); };
  v = fmaxf(v, f(permuted<0xB1>(__builtin_bit_cast(int, v))));
  v = fmaxf(v, f(permuted<0x4E>(__builtin_bit_cast(int, v))));
  v = fmaxf(v, f(permuted<0x141>(__builtin_bit_cast(int, v))));
  v = fmaxf(v, f(permuted<0x140>(__builtin_bit_cast(int, v))));
  return across_rows(v, [](float x, float y) { return fmaxf(x, y); });
}
__device__ __forceinline__ Draw wave_join(Draw a) {
  const float top = wave_max(a.top);
  a.sum = wave_allsum(a.sum * exp_of(a.top - top));
  a.top = top;
  const float best = wave_max(a.score);
  int token = a.score == best ? a.token : INT32_MAX;
#pragma unroll
  for (int d = 32; d; d >>= 1) token = min(token, __shfl_xor(token, d));
  const uint64_t holder = __ballot(a.score == best && a.token == token);
  a.y = holder ? __shfl(a.y, (int)__builtin_ctzll(holder)) : -INFINITY;
  a.score = best;
  a.token = token;
  return a;
}

// Few tokens can win: with E >= w (w the uniform variate of E = -log1p(-w)) a token's score y - ln E reaches a bound b only if
// w <= exp(y - b) = p exp(top - b), where p = exp(y - top) is what the softmax's sum needs anyway.  So a token costs its
// Philox word, one exponential and one multiply-add; b is the best lower bound y - ln w - w (ln E <= ln w + w for w <= 1/2) of
// a token that the workgroup has seen, and only tokens that reach it get their score, from the C library's logarithms.
template <bool BF16, int G>
__global__ __launch_bounds__(LOGIT_THREADS) void sample_chunk_kernel(LogitArgs a, const float* temperature, uint32_t k0, uint32_t k1,
                                                                     uint32_t step, const int32_t* ids, Draw* parts) {
  extern __shared__ uint32_t lds[];
  __shared__ Draw waves[LOGIT_WAVES];
  __shared__ int shared_bound;                       // the bits of a float, ordered as integers
  constexpr int CHUNK = G * PASS_TOKENS;
  const int r = blockIdx.y;
  const RowRules q = row_rules(a, r);
  const float t = temperature ? temperature[r] : 1.0f;
  const bool greedy = t == 0.0f;
  const float inv = 1.0f / (greedy ? 1.0f : t);
  const uint32_t id = ids ? (uint32_t)ids[r] : (uint32_t)r;
  auto ordered = [](int b) { return b ^ (b >> 31 & 0x7FFFFFFF); };       // its own inverse
  if (threadIdx.x == 0) shared_bound = ordered(__builtin_bit_cast(int, -INFINITY));
  if (!a.count) __syncthreads();
  Draw mine = no_draw();
  for (int c = 0; c < a.per; ++c) {
    const int64_t first = ((int64_t)blockIdx.x * a.per + c) * CHUNK;
    if (first >= a.d.vocab) break;
    const int v0 = (int)first, n = min(CHUNK, a.d.vocab - v0);
    Groups<BF16, G> x;
    x.load(a, q, (int64_t)r * a.d.stride, v0, n);
    if (a.count) count_tokens<G>(a, q, r, v0, n, lds);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int i = g * PASS_TOKENS + (int)threadIdx.x * LANE_TOKENS, v = v0 + i;
      if (n - (g * PASS_TOKENS + (int)(threadIdx.x & ~63u) * LANE_TOKENS) <= 0) continue;      // nothing of the wave's
      float y[8];
      group_logits<BF16, G>(a, q, x, g, v0, lds, y);
      if (greedy) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (y[e] > mine.score) {                   // tokens ascend within a lane
            mine.score = mine.y = y[e];
            mine.token = v + e;
          }
      }
      float top = mine.top;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] *= inv;
        top = fmaxf(top, y[e]);
      }
      float sum = mine.sum * exp_of(mine.top - top);
      mine.top = top;
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = exp_of(y[e] - top);
        sum += p[e];
      }
      mine.sum = sum;
      if (greedy) continue;
      const u32x4 b0 = philox4x32_10(u32x4{(uint32_t)v >> 2, step, id, STREAM_TOKEN}, k0, k1);
      const u32x4 b1 = philox4x32_10(u32x4{((uint32_t)v >> 2) + 1, step, id, STREAM_TOKEN}, k0, k1);
      const float w[8] = {(float)b0.x, (float)b0.y, (float)b0.z, (float)b0.w, (float)b1.x, (float)b1.y, (float)b1.z, (float)b1.w};
      float bound = __builtin_bit_cast(float, ordered(*(volatile int*)&shared_bound));
      // 2^32, and 1e-3 for the rounding of the exponentials
      const float reach = exp_of(top - bound) * 4.2992672e9f;
      float far = -1.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) far = fmaxf(far, __builtin_fmaf(p[e], reach, -w[e]));
      if (!__ballot(far >= 0.0f)) continue;
      float up[8], low = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = (w[e] + 0.5f) * 2.3283064365386963e-10f;
        up[e] = y[e] - LN2 * __builtin_amdgcn_logf(u);
        if (u < 0.5f) low = fmaxf(low, up[e] - u);
      }
      low = wave_max(low);
      low -= 1e-4f + 1e-6f * fabsf(low);             // what the logarithms above may be off
      if (low > bound) {
        bound = low;
        atomicMax(&shared_bound, ordered(__builtin_bit_cast(int, bound)));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (up[e] >= bound && y[e] > -INFINITY) {
          const float u = fminf((w[e] + 0.5f) * 2.3283064365386963e-10f, 0.99999994f);
          const float score = y[e] - logf(-log1pf(-u));
          if (score > mine.score) {
            mine.score = score;
            mine.token = v + e;
            mine.y = y[e];
          }
        }
    }
  }
  if (!(t >= 0.0f && t < INFINITY)) mine.sum = __builtin_nanf("");
  mine = wave_join(mine);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < LOGIT_WAVES; ++w) join(mine, waves[w]);
    parts[(int64_t)r * gridDim.x + blockIdx.x] = mine;
  }
}

__global__ __launch_bounds__(WAVE) void sample_finish_kernel(const Draw* parts, int chunks, int32_t* token, float* logp) {
  const int r = blockIdx.x;
  Draw mine = no_draw();
  for (int i = threadIdx.x; i < chunks; i += WAVE) join(mine, parts[(int64_t)r * chunks + i]);
  mine = wave_join(mine);
  if (threadIdx.x == 0) {
    const bool bad = mine.sum != mine.sum, none = mine.token == INT32_MAX;
    token[r] = none || bad ? -1 : mine.token;
    logp[r] = bad ? __builtin_nanf("") : none ? -INFINITY : mine.y - mine.top - logf(mine.sum);
  }
}

// ---------------------------------------------------------------- host side

// Groups of a lane in a chunk (1, 2 or 4).  The history is read once a chunk and LDS holds 4 bytes a token, so chunks are long (8192
// tokens: 32 KB, five workgroups a compute unit) unless there are too few rows to fill the device with such.
static int groups_of(int64_t rows, int64_t vocab) {
  int g = 4;
  while (g > 1 && rows * ((vocab + g * PASS_TOKENS - 1) / (g * PASS_TOKENS)) < 1024) g /= 2;
  return g;
}
// Chunks of a workgroup in a draw: the bound that the tokens have to reach is found anew by each workgroup, so it takes several chunks
// where that leaves enough workgroups.
struct DrawGrid { int groups, per, workgroups; };
static DrawGrid draw_grid(int64_t rows, int64_t vocab) {
  const int g = groups_of(rows, vocab);
  const int64_t chunks = (vocab + g * PASS_TOKENS - 1) / (g * PASS_TOKENS);
  const int64_t per = std::min<int64_t>(chunks, std::max<int64_t>(1, rows * chunks / 2048));
  return DrawGrid{g, (int)per, (int)((chunks + per - 1) / per)};
}

static pg_status logit_args(const pg_logits* d, const char* who, LogitArgs& a) {
  if (!d) return fail(PG_EINVAL, "%s: desc is NULL", who);
  if (d->rows < 0 || d->vocab < 1 || (d->dtype != PG_LOGITS_F32 && d->dtype != PG_LOGITS_BF16))
    return fail(PG_EINVAL, "%s: %d rows of %d tokens, dtype %d", who, d->rows, d->vocab, d->dtype);
  if (d->rows > 65535) return fail(PG_ESHAPE, "%s: %d rows (at most 65535)", who, d->rows);
  if (d->vocab > 1 << 30) return fail(PG_ESHAPE, "%s: %d tokens", who, d->vocab);
  if (d->rows && !d->logits) return fail(PG_EINVAL, "%s: logits is NULL", who);
  if (d->stride < d->vocab) return fail(PG_EINVAL, "%s: rows %lld elements apart hold no %d tokens", who, (long long)d->stride, d->vocab);
  if ((uintptr_t)d->logits & (d->dtype == PG_LOGITS_BF16 ? 1 : 3)) return fail(PG_ESHAPE, "%s: logits are not aligned to their size", who);
  if (d->tokens && (!d->n_tokens || d->tokens_stride < 0)) return fail(PG_EINVAL, "%s: tokens without n_tokens", who);
  if (!d->tokens && (d->repetition || d->frequency || d->presence)) return fail(PG_EINVAL, "%s: penalties without tokens", who);
  if (d->bias_offsets && (d->n_bias < 0 || (d->n_bias && (!d->bias_ids || !d->bias_values))))
    return fail(PG_EINVAL, "%s: bias_offsets without a list", who);
  if (d->allow && d->n_masks < 1) return fail(PG_EINVAL, "%s: %d masks", who, d->n_masks);
  if (d->allow && !d->allow_row && d->n_masks < d->rows) return fail(PG_EINVAL, "%s: %d masks for %d rows", who, d->n_masks, d->rows);
  a.d = *d;
  if (!(d->repetition || d->frequency || d->presence)) a.d.tokens = nullptr;
  if (d->n_bias == 0) a.d.bias_offsets = nullptr;
  a.words = (d->vocab + 31) / 32;
  a.count = a.d.tokens || a.d.bias_offsets;
  return PG_OK;
}

// launches F<bf16, groups>
#define PG_LOGIT_KERNEL(F, groups, ...)                                                   \
  do {                                                                                    \
    const bool b = a.d.dtype == PG_LOGITS_BF16;                                           \
    const size_t lds = a.count ? (size_t)(groups) * PASS_TOKENS * 4 : 0;                  \
    switch (groups) {                                                                     \
      case 1: b ? F<true, 1><<<grid, block, lds, s>>>(__VA_ARGS__) : F<false, 1><<<grid, block, lds, s>>>(__VA_ARGS__); break; \
      case 2: b ? F<true, 2><<<grid, block, lds, s>>>(__VA_ARGS__) : F<false, 2><<<grid, block, lds, s>>>(__VA_ARGS__); break; \
      default: b ? F<true, 4><<<grid, block, lds, s>>>(__VA_ARGS__) : F<false, 4><<<grid, block, lds, s>>>(__VA_ARGS__);      \
    }                                                                                     \
  } while (0)

}  // namespace pg

using namespace pg;

extern "C" pg_status pg_logits_adjust(const pg_logits* desc, float* out, int64_t out_stride, void* stream) {
  LogitArgs a{};
  PG_TRY(logit_args(desc, "pg_logits_adjust", a));
  if (a.d.rows == 0) return PG_OK;
  if (!out) return fail(PG_EINVAL, "pg_logits_adjust: out is NULL");
  if ((uintptr_t)out & 3 || out_stride < a.d.vocab) return fail(PG_ESHAPE, "pg_logits_adjust: out rows %lld floats apart", (long long)out_stride);
  if ((const void*)out == a.d.logits && (a.d.dtype != PG_LOGITS_F32 || out_stride != a.d.stride))
    return fail(PG_EINVAL, "pg_logits_adjust: in place needs fp32 logits of the same stride");
  const int groups = groups_of(a.d.rows, a.d.vocab);
  const dim3 grid((unsigned)((a.d.vocab + groups * PASS_TOKENS - 1) / (groups * PASS_TOKENS)), (unsigned)a.d.rows), block(LOGIT_THREADS);
  hipStream_t s = (hipStream_t)stream;
  PG_LOGIT_KERNEL(logits_adjust_kernel, groups, a, out, out_stride);
  PG_LAUNCH_CHECK("logits_adjust_kernel");
  return PG_OK;
}

extern "C" int64_t pg_sample_scratch_floats(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1) return 0;
  return (int64_t)rows * draw_grid(rows, vocab).workgroups * (int64_t)(sizeof(Draw) / sizeof(float));
}

extern "C" pg_status pg_sample_tokens(const pg_logits* desc, const float* temperature, uint64_t seed, uint32_t step, const int32_t* ids,
                                      int32_t* token, float* logp, float* scratch, void* stream) {
  LogitArgs a{};
  PG_TRY(logit_args(desc, "pg_sample_tokens", a));
  if (a.d.rows == 0) return PG_OK;
  if (!token || !logp || !scratch) return fail(PG_EINVAL, "pg_sample_tokens: null pointer");
  hipStream_t s = (hipStream_t)stream;
  const DrawGrid g = draw_grid(a.d.rows, a.d.vocab);
  a.per = g.per;
  const dim3 grid((unsigned)g.workgroups, (unsigned)a.d.rows), block(LOGIT_THREADS);
  PG_LOGIT_KERNEL(sample_chunk_kernel, g.groups, a, temperature, (uint32_t)seed, (uint32_t)(seed >> 32), step, ids, (Draw*)scratch);
  PG_LAUNCH_CHECK("sample_chunk_kernel");
  sample_finish_kernel<<<dim3((unsigned)a.d.rows), dim3(WAVE), 0, s>>>((const Draw*)scratch, (int)grid.x, token, logp);
  PG_LAUNCH_CHECK("sample_finish_kernel");
  return PG_OK;
}
