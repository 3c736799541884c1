// Logits of a token policy: penalties, biases and grammar masks, and the draw of a token with its log-prob.
//
// A workgroup takes a chunk of one row's vocabulary.  How often each of its tokens occurs is counted in LDS from the row's
// history (32 bits a token: integer sums, so their order does not matter), so no counts are kept between calls and nothing but the
// history has to follow a member through a prune.  The logits are then read once.
#include <cmath>
#include "common.hpp"
#include "operands.hpp"
#include "philox.hpp"

namespace pg {

constexpr int LOGIT_THREADS = 256;
constexpr int LOGIT_WAVES = LOGIT_THREADS / WAVE;
constexpr int LANE_TOKENS = 8;                       // per lane and pass: 16 or 32 bytes, two Philox blocks
constexpr int PASS_TOKENS = LOGIT_THREADS * LANE_TOKENS;
constexpr uint32_t STREAM_TOKEN = 2u;
// LDS word of a token: how often it is in the output, and whether it is in the prompt or has a bias
constexpr uint32_t IN_PROMPT = 1u << 31, HAS_BIAS = 1u << 30, COUNT = HAS_BIAS - 1;

struct LogitArgs {
  pg_logits d;
  int words;                                         // of a mask
  int chunk;                                         // tokens of a workgroup
  bool count;                                        // LDS words are needed
};

// 8 logits from any address that is a multiple of their size: the hardware takes unaligned 16-byte loads
template <bool BF16>
__device__ __forceinline__ void load_logits(const void* row, int v, int n, float* x) {
  if (BF16) {
    const uint16_t* p = (const uint16_t*)row + v;
    if (n >= LANE_TOKENS) {
      uint32_t w[4];
      __builtin_memcpy(w, p, 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __builtin_bit_cast(float, e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < n ? bf16_to_f32(p[e]) : -INFINITY;
    }
  } else {
    const float* p = (const float*)row + v;
    if (n >= LANE_TOKENS) {
      __builtin_memcpy(x, p, 32);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < n ? p[e] : -INFINITY;
    }
  }
}

// What one row needs.
struct RowRules {
  float rep, freq, pres;
  const uint32_t* allow;                             // NULL: everything
  int bias_lo, bias_hi;
  bool penalised;
};

__device__ __forceinline__ RowRules row_rules(const LogitArgs& a, int r) {
  const pg_logits& d = a.d;
  RowRules q;
  q.penalised = d.tokens != nullptr;
  q.rep = d.repetition ? d.repetition[r] : 1.0f;
  q.freq = d.frequency ? d.frequency[r] : 0.0f;
  q.pres = d.presence ? d.presence[r] : 0.0f;
  q.allow = nullptr;
  if (d.allow) {
    const int m = d.allow_row ? d.allow_row[r] : r;
    if (m >= 0 && m < d.n_masks) q.allow = d.allow + (int64_t)m * a.words;
  }
  q.bias_lo = q.bias_hi = 0;
  if (d.bias_offsets) {
    q.bias_lo = max(0, d.bias_offsets[r]);
    q.bias_hi = min(d.n_bias, d.bias_offsets[r + 1]);
  }
  return q;
}

// The chunk's LDS words from the history and the bias list.
__device__ __forceinline__ void count_tokens(const LogitArgs& a, const RowRules& q, int r, int v0, int n, uint32_t* lds) {
  const pg_logits& d = a.d;
  for (int i = threadIdx.x; i < n; i += LOGIT_THREADS) lds[i] = 0;
  __syncthreads();
  if (d.tokens) {
    const int made = min(max(d.n_tokens[r], 0), d.tokens_stride);
    const int prompt = d.n_prompt ? min(max(d.n_prompt[r], 0), made) : 0;
    const int32_t* t = d.tokens + (int64_t)r * d.tokens_stride;
    for (int i = threadIdx.x; i < made; i += LOGIT_THREADS) {
      const uint32_t at = (uint32_t)t[i] - (uint32_t)v0;
      if (at < (uint32_t)n) {
        if (i < prompt) atomicOr(&lds[at], IN_PROMPT);
        else atomicAdd(&lds[at], 1u);
      }
    }
  }
  for (int i = q.bias_lo + threadIdx.x; i < q.bias_hi; i += LOGIT_THREADS) {
    const int id = d.bias_ids[i];
    if (id >= v0 && id < v0 + n) atomicOr(&lds[id - v0], HAS_BIAS);
  }
  __syncthreads();
}

// z of one token; the order and the rounding of the operations are the interface's.
__device__ __forceinline__ float adjusted(const LogitArgs& a, const RowRules& q, float x, uint32_t word, int v) {
  if (q.penalised) {
    const uint32_t c = word & COUNT;
    if (word & (IN_PROMPT | COUNT)) {
      x = x > 0.0f ? x / q.rep : x * q.rep;
      x = x - q.freq * (float)c;
      if (c) x = x - q.pres;
    }
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

__global__ __launch_bounds__(LOGIT_THREADS) void logits_adjust_kernel(LogitArgs a, float* out, int64_t out_stride) {
  extern __shared__ uint32_t lds[];
  const int r = blockIdx.y, v0 = blockIdx.x * a.chunk;
  const int n = min(a.chunk, a.d.vocab - v0);
  const RowRules q = row_rules(a, r);
  if (a.count) count_tokens(a, q, r, v0, n, lds);
  const void* row = (const char*)a.d.logits + (int64_t)r * a.d.stride * (a.d.dtype == PG_LOGITS_BF16 ? 2 : 4);
  float* to = out + (int64_t)r * out_stride;
  for (int base = 0; base < n; base += PASS_TOKENS) {
    const int i = base + (int)threadIdx.x * LANE_TOKENS, left = n - i;
    if (left <= 0) continue;
    const int v = v0 + i;
    float x[8];
    if (a.d.dtype == PG_LOGITS_BF16) load_logits<true>(row, v, left, x);
    else load_logits<false>(row, v, left, x);
    const uint32_t bits = q.allow ? q.allow[v >> 5] >> (v & 31) : 0xFFu;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e < left) {
        if (a.count) x[e] = adjusted(a, q, x[e], lds[i + e], v + e);
        if (!(bits >> e & 1)) x[e] = -INFINITY;
      }
    }
    if (left >= LANE_TOKENS) {
      __builtin_memcpy(to + v, x, 32);
    } else {
      for (int e = 0; e < left; ++e) to[v + e] = x[e];
    }
  }
}

// ---------------------------------------------------------------- the draw
// What a chunk, a wave or a lane knows of a row: the largest y and the sum of exp(y - top), the best score with its token and that
// token's y, and whether something cannot be sampled.
struct Draw {
  float top, sum, score, y;
  int token;                                         // INT_MAX: none
  uint32_t bad;
};
__device__ __forceinline__ Draw no_draw() { return Draw{-INFINITY, 0.0f, -INFINITY, -INFINITY, INT32_MAX, 0}; }
__device__ __forceinline__ void join(Draw& a, const Draw& b) {
  const float top = fmaxf(a.top, b.top);
  if (top > -INFINITY) a.sum = a.sum * expf(a.top - top) + b.sum * expf(b.top - top);
  a.top = top;
  if (b.score > a.score || (b.score == a.score && b.token < a.token)) {
    a.score = b.score;
    a.token = b.token;
    a.y = b.y;
  }
  a.bad |= b.bad;
}
__device__ __forceinline__ Draw wave_join(Draw a) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    Draw b;
    b.top = __shfl_xor(a.top, d);
    b.sum = __shfl_xor(a.sum, d);
    b.score = __shfl_xor(a.score, d);
    b.y = __shfl_xor(a.y, d);
    b.token = __shfl_xor(a.token, d);
    b.bad = __shfl_xor(a.bad, d);
    join(a, b);
  }
  return a;
}

__global__ __launch_bounds__(LOGIT_THREADS) void sample_chunk_kernel(LogitArgs a, const float* temperature, uint32_t k0, uint32_t k1,
                                                                     uint32_t step, const int32_t* ids, Draw* parts) {
  extern __shared__ uint32_t lds[];
  __shared__ Draw waves[LOGIT_WAVES];
  const int r = blockIdx.y, v0 = blockIdx.x * a.chunk;
  const int n = min(a.chunk, a.d.vocab - v0);
  const RowRules q = row_rules(a, r);
  if (a.count) count_tokens(a, q, r, v0, n, lds);
  const float t = temperature ? temperature[r] : 1.0f;
  const bool greedy = t == 0.0f;
  const float inv = 1.0f / (greedy ? 1.0f : t);
  const uint32_t id = ids ? (uint32_t)ids[r] : (uint32_t)r;
  const void* row = (const char*)a.d.logits + (int64_t)r * a.d.stride * (a.d.dtype == PG_LOGITS_BF16 ? 2 : 4);
  Draw mine = no_draw();
  mine.bad = !(t >= 0.0f && t < INFINITY);
  for (int base = 0; base < n; base += PASS_TOKENS) {
    const int i = base + (int)threadIdx.x * LANE_TOKENS, left = n - i;
    if (left <= 0) continue;
    const int v = v0 + i;
    float x[8];
    if (a.d.dtype == PG_LOGITS_BF16) load_logits<true>(row, v, left, x);
    else load_logits<false>(row, v, left, x);
    const uint32_t bits = q.allow ? q.allow[v >> 5] >> (v & 31) : 0xFFu;
    float top = mine.top;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float z = -INFINITY;
      if (e < left && (bits >> e & 1)) z = a.count ? adjusted(a, q, x[e], lds[i + e], v + e) : x[e];
      mine.bad |= !(z < INFINITY);
      x[e] = z;
      top = fmaxf(top, z * inv);
    }
    if (top == -INFINITY) continue;
    float sum = mine.sum * expf(mine.top - top);
    mine.top = top;
    u32x4 w[2];
    if (!greedy) {
      w[0] = philox4x32_10(u32x4{(uint32_t)(v >> 2), step, id, STREAM_TOKEN}, k0, k1);
      w[1] = philox4x32_10(u32x4{(uint32_t)(v >> 2) + 1, step, id, STREAM_TOKEN}, k0, k1);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = x[e] * inv;
      sum += expf(y - top);
      float score = x[e];
      if (!greedy) {
        const u32x4& b = w[e >> 2];
        const uint32_t m = (e & 3) == 0 ? b.x : (e & 3) == 1 ? b.y : (e & 3) == 2 ? b.z : b.w;
        const float u = fminf(((float)m + 0.5f) * 2.3283064365386963e-10f, 0.99999994f);
        score = y - logf(-log1pf(-u));
      }
      if (score > mine.score) {                      // tokens ascend within a lane
        mine.score = score;
        mine.token = v + e;
        mine.y = y;
      }
    }
    mine.sum = sum;
  }
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
    const bool none = mine.token == INT32_MAX || mine.bad;
    token[r] = none ? -1 : mine.token;
    logp[r] = mine.bad ? __builtin_nanf("") : none ? -INFINITY : mine.y - mine.top - logf(mine.sum);
  }
}

// ---------------------------------------------------------------- host side

// Tokens of a workgroup: the history is read once a chunk and LDS holds 4 bytes a token, so chunks are long (8192: 32 KB, four workgroups
// a compute unit) unless there are too few rows to fill the device with such.
static int chunk_of(int64_t rows, int64_t vocab) {
  int chunk = 8192;
  while (chunk > PASS_TOKENS && rows * ((vocab + chunk - 1) / chunk) < 1024) chunk /= 2;
  return chunk;
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
  a.chunk = chunk_of(d->rows, d->vocab);
  a.count = a.d.tokens || a.d.bias_offsets;
  return PG_OK;
}

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
  const dim3 grid((unsigned)((a.d.vocab + a.chunk - 1) / a.chunk), (unsigned)a.d.rows);
  logits_adjust_kernel<<<grid, dim3(LOGIT_THREADS), a.count ? (size_t)a.chunk * 4 : 0, (hipStream_t)stream>>>(a, out, out_stride);
  PG_LAUNCH_CHECK("logits_adjust_kernel");
  return PG_OK;
}

extern "C" int64_t pg_sample_scratch_floats(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1) return 0;
  const int chunk = chunk_of(rows, vocab);
  return (int64_t)rows * (((int64_t)vocab + chunk - 1) / chunk) * (int64_t)(sizeof(Draw) / sizeof(float));
}

extern "C" pg_status pg_sample_tokens(const pg_logits* desc, const float* temperature, uint64_t seed, uint32_t step, const int32_t* ids,
                                      int32_t* token, float* logp, float* scratch, void* stream) {
  LogitArgs a{};
  PG_TRY(logit_args(desc, "pg_sample_tokens", a));
  if (a.d.rows == 0) return PG_OK;
  if (!token || !logp || !scratch) return fail(PG_EINVAL, "pg_sample_tokens: null pointer");
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)((a.d.vocab + a.chunk - 1) / a.chunk), (unsigned)a.d.rows);
  sample_chunk_kernel<<<grid, dim3(LOGIT_THREADS), a.count ? (size_t)a.chunk * 4 : 0, s>>>(a, temperature, (uint32_t)seed, (uint32_t)(seed >> 32), step,
                                                                                        ids, (Draw*)scratch);
  PG_LAUNCH_CHECK("sample_chunk_kernel");
  sample_finish_kernel<<<dim3((unsigned)a.d.rows), dim3(WAVE), 0, s>>>((const Draw*)scratch, (int)grid.x, token, logp);
  PG_LAUNCH_CHECK("sample_finish_kernel");
  return PG_OK;
}
