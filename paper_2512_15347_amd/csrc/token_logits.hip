// Logits of a token policy: penalties, biases and grammar masks, and the draw of a token with its log-prob.
//
// A workgroup takes a range of one row's vocabulary and goes through it in groups of eight tokens a lane.  Few tokens have a penalty or a
// bias: for every 2048 or 4096 tokens the row's history is counted in LDS (32 bits a token: integer sums, so their order does not matter), the
// tokens that occur are worked out once each and left in LDS, and the groups pick them up by a bit.  So no counts are kept
// between calls, and nothing but the history has to follow a member through a prune.  The logits are read once.
//
// Adjusting is bound by HBM, and by the barriers around the counts where there is a history: 384 x 65537 in bf16 takes 35 us with nothing to adjust
// (4.4 TB/s), 49 with up to 2048 tokens of history a row, masks and lists.  Draws are bound by the vector ALU, of which 1024 SIMDs at
// four cycles an instruction issue some 600 a nanosecond: 384 x 131073 takes 67 us without history, lists and masks, 97 with all of them (the
// logits alone would be read in 20).
#include <algorithm>
#include <cfloat>
#include <cmath>
#include "common.hpp"
#include "operands.hpp"
#include "philox.hpp"
#include "token_logits.hpp"

namespace pg {

constexpr int LOGIT_THREADS = 256;
constexpr int LOGIT_WAVES = LOGIT_THREADS / WAVE;
constexpr int PASS_TOKENS = LOGIT_THREADS * LANE_TOKENS;
constexpr uint32_t STREAM_TOKEN = 2u;
// LDS word of a token: how often it is in the output, and whether it is in the prompt or has a bias; then its z
constexpr uint32_t IN_PROMPT = 1u << 31, HAS_BIAS = 1u << 30, COUNT = HAS_BIAS - 1;

// What one row needs.
struct RowRules {
  float rep, freq, pres;
  const uint8_t* allow;                              // bit v % 8 of byte v / 8; NULL: `unmasked` for all of them
  uint32_t unmasked;
  int bias_lo, bias_hi, made, prompt;
};

// What is left out is read from here: then all loads of a row's rules are under way at once instead of behind a branch each.
static __device__ const uint32_t NOTHING[2] = {0, 0};

__device__ __forceinline__ RowRules row_rules(const LogitArgs& a, int r) {
  const pg_logits& d = a.d;
  auto entry = [&](const auto* p, int i) { return p ? p + i : (decltype(p))NOTHING; };
  const float rep = *entry(d.repetition, r), freq = *entry(d.frequency, r), pres = *entry(d.presence, r);
  const int m = *entry(d.allow_row, r), lo = *entry(d.bias_offsets, r), hi = *entry(d.bias_offsets, r + 1);
  const int made = *entry(d.n_tokens, r), prompt = *entry(d.n_prompt, r);
  RowRules q;
  q.rep = d.repetition ? rep : 1.0f;
  q.freq = freq;
  q.pres = pres;
  const int mask = d.allow_row ? m : r;
  q.allow = d.allow && mask >= 0 && mask < d.n_masks ? (const uint8_t*)(d.allow + (int64_t)mask * a.words) : nullptr;
  q.unmasked = d.allow && mask != -1 ? 0u : 0xFFu;   // an index that no mask has allows nothing
  q.bias_lo = max(0, lo);
  q.bias_hi = d.bias_offsets ? min(d.n_bias, hi) : 0;
  q.made = d.tokens ? min(max(made, 0), d.tokens_stride) : 0;
  q.prompt = min(max(prompt, 0), q.made);
  return q;
}

// A lane's group: eight logits from any address that is a multiple of their size (the hardware takes unaligned 16-byte loads) and
// their bits of the mask; tokens past the end of the row are not allowed.
template <bool BF16>
struct Group {
  uint32_t raw[BF16 ? 4 : 8];
  uint32_t allowed;

  __device__ __forceinline__ void load(const LogitArgs& a, const RowRules& q, int64_t row, int64_t v) {
    const int64_t left = a.d.vocab - v;
    allowed = 0;
    if (left <= 0) return;
    const char* p = (const char*)a.d.logits + (row + v) * (BF16 ? 2 : 4);
    if (left >= LANE_TOKENS) {
      __builtin_memcpy(raw, p, BF16 ? 16 : 32);
    } else {
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e) {
        const uint32_t x = e >= left ? 0u : BF16 ? ((const uint16_t*)p)[e] : ((const uint32_t*)p)[e];
        if (!BF16) raw[e] = x;
        else raw[e >> 1] = e & 1 ? raw[e >> 1] | x << 16 : x;
      }
    }
    allowed = (q.allow ? q.allow[v >> 3] : q.unmasked) & (left >= LANE_TOKENS ? 0xFFu : (1u << left) - 1);
  }
  __device__ __forceinline__ float logit(int e) const {
    return __builtin_bit_cast(float, !BF16 ? raw[e] : e & 1 ? raw[e >> 1] & 0xFFFF0000u : raw[e >> 1] << 16);
  }
};

// LDS of a counted stretch of G * PASS_TOKENS tokens: all zero between stretches (a group clears what it picks up).
template <int G>
struct Stretch {
  static constexpr int TOKENS = G * PASS_TOKENS;
  uint32_t word[TOKENS];
  uint32_t ready[TOKENS / 32];                       // bit: word holds z
  static constexpr int LISTED = 1024;
  uint16_t seen[LISTED];                             // tokens that occur in the history, in no particular order; of more all words are looked at
  int n_seen;
};

// A lane's part of the row's history and bias list: the first entries stay in registers from stretch to stretch.
struct RowLists {
  static constexpr int KEPT = 4;                     // 1024 tokens of the workgroup's
  int32_t token[KEPT];
  int32_t bias_id, bias_before;
  float bias;
};
constexpr int32_t NO_TOKEN = -1;                     // is in no stretch

__device__ __forceinline__ RowLists row_lists(const LogitArgs& a, const RowRules& q, int r) {
  RowLists l;
  const int32_t* t = a.d.tokens + (int64_t)r * a.d.tokens_stride;
#pragma unroll
  for (int k = 0; k < RowLists::KEPT; ++k) {
    const int i = threadIdx.x + k * LOGIT_THREADS;
    l.token[k] = a.d.tokens && i < a.d.tokens_stride ? t[i] : NO_TOKEN;      // asked for beside the count itself
  }
#pragma unroll
  for (int k = 0; k < RowLists::KEPT; ++k)
    if ((int)threadIdx.x + k * LOGIT_THREADS >= q.made) l.token[k] = NO_TOKEN;
  const int i = q.bias_lo + threadIdx.x;
  const bool there = i < q.bias_hi;
  l.bias_id = there ? a.d.bias_ids[i] : NO_TOKEN;
  l.bias_before = there && i > q.bias_lo ? a.d.bias_ids[i - 1] : NO_TOKEN;
  l.bias = there ? a.d.bias_values[i] : 0.0f;
  return l;
}

// z from the history alone; the order and the rounding of the operations are the interface's.
__device__ __forceinline__ float penalised(const RowRules& q, float x, uint32_t word) {
  if (word & (IN_PROMPT | COUNT)) {
    x = x > 0.0f ? x / q.rep : x * q.rep;
    x = x - q.freq * (float)(word & COUNT);
    if (word & COUNT) x = x - q.pres;
  }
  return x;
}

// z of the tokens of v0 .. v0 + n - 1 that have a count or a bias.  Each word has one owner, who turns it into z: the first of its
// bias entries, or else the place of the token among the seen.
template <bool BF16, int G>
__device__ __forceinline__ void prepare_stretch(const LogitArgs& a, const RowRules& q, const RowLists& l, int r, int v0, int n, Stretch<G>& s) {
  const pg_logits& d = a.d;
  const int64_t row = (int64_t)r * d.stride + v0;
  auto logit = [&](uint32_t at) { return BF16 ? bf16_to_f32(((const uint16_t*)d.logits)[row + at]) : ((const float*)d.logits)[row + at]; };
  auto count = [&](uint32_t at, int i) {
    const uint32_t old = i < q.prompt ? atomicOr(&s.word[at], IN_PROMPT) : atomicAdd(&s.word[at], 1u);
    if ((old & ~HAS_BIAS) == 0) {
      const int k = atomicAdd(&s.n_seen, 1);
      if (k < Stretch<G>::LISTED) s.seen[k] = (uint16_t)at;
    }
  };
  auto finish = [&](uint32_t at, float z) {
    s.word[at] = __builtin_bit_cast(uint32_t, z);
    atomicOr(&s.ready[at >> 5], 1u << (at & 31));
  };
  __syncthreads();                                   // the stretch before has been read, and its n_seen
  float bias_x = 0.0f;
  const uint32_t bias_at = (uint32_t)l.bias_id - (uint32_t)v0;
  if (bias_at < (uint32_t)n) {
    bias_x = logit(bias_at);
    atomicOr(&s.word[bias_at], HAS_BIAS);
  }
#pragma unroll
  for (int k = 0; k < RowLists::KEPT; ++k) {
    const uint32_t at = (uint32_t)l.token[k] - (uint32_t)v0;
    if (at < (uint32_t)n) count(at, threadIdx.x + k * LOGIT_THREADS);
  }
  const int32_t* t = d.tokens + (int64_t)r * d.tokens_stride;
#pragma unroll 4
  for (int i = RowLists::KEPT * LOGIT_THREADS + threadIdx.x; i < q.made; i += LOGIT_THREADS) {
    const uint32_t at = (uint32_t)t[i] - (uint32_t)v0;
    if (at < (uint32_t)n) count(at, i);
  }
  for (int i = q.bias_lo + LOGIT_THREADS + threadIdx.x; i < q.bias_hi; i += LOGIT_THREADS) {
    const uint32_t at = (uint32_t)d.bias_ids[i] - (uint32_t)v0;
    if (at < (uint32_t)n) atomicOr(&s.word[at], HAS_BIAS);
  }
  __syncthreads();
  const bool listed = s.n_seen <= Stretch<G>::LISTED;
  for (int k = threadIdx.x; k < (listed ? s.n_seen : n); k += LOGIT_THREADS) {
    const uint32_t at = listed ? s.seen[k] : k, word = s.word[at];
    if (word && !(word & HAS_BIAS)) finish(at, penalised(q, logit(at), word));
  }
  if (q.bias_lo < q.bias_hi) __syncthreads();        // the history's owners have looked for HAS_BIAS in words that become z here
  if (bias_at < (uint32_t)n && l.bias_before != l.bias_id) finish(bias_at, penalised(q, bias_x, s.word[bias_at]) + l.bias);
  for (int i = q.bias_lo + LOGIT_THREADS + threadIdx.x; i < q.bias_hi; i += LOGIT_THREADS) {
    const uint32_t at = (uint32_t)d.bias_ids[i] - (uint32_t)v0;
    if (at < (uint32_t)n && d.bias_ids[i - 1] != d.bias_ids[i]) finish(at, penalised(q, logit(at), s.word[at]) + d.bias_values[i]);
  }
  __syncthreads();
  if (threadIdx.x == 0) s.n_seen = 0;
}

template <int G>
__device__ __forceinline__ void clear_group(int at, Stretch<G>& s) {
  *(uint4*)(s.word + at) = *(uint4*)(s.word + at + 4) = uint4{0, 0, 0, 0};
  ((uint8_t*)s.ready)[at >> 3] = 0;
}

// z of a group whose first token is number `at` of its stretch; tokens that are not allowed get -inf.  SKIP: waves whose tokens are all
// allowed pass the masks over (draws, which the vector ALU bounds: 79 -> 75 us for 384 x 131073; adjusting gets slower with it, 35 -> 48 us
// for 384 x 65537).
template <bool BF16, int G, bool SKIP>
__device__ __forceinline__ void group_logits(bool count, const Group<BF16>& x, int at, Stretch<G>& s, float* z) {
#pragma unroll
  for (int e = 0; e < LANE_TOKENS; ++e) z[e] = x.logit(e);
  if (count) {
    const uint32_t ready = ((const uint8_t*)s.ready)[at >> 3];
    if (ready) {
      const float4 w0 = *(const float4*)(s.word + at), w1 = *(const float4*)(s.word + at + 4);
      clear_group(at, s);
      const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e) z[e] = ready >> e & 1 ? w[e] : z[e];
    }
  }
  if (SKIP && !__ballot(x.allowed != 0xFFu)) return;
#pragma unroll
  for (int e = 0; e < LANE_TOKENS; ++e) z[e] = x.allowed >> e & 1 ? z[e] : -INFINITY;
}

// Goes through the workgroup's range, one group a lane and call of each(group, first token, place in the stretch); the next group is
// asked for before a group is worked on.
template <bool BF16, int G, class Each>
__device__ __forceinline__ void through_range(const LogitArgs& a, const RowRules& q, int r, Stretch<G>& s, Each each) {
  const int64_t row = (int64_t)r * a.d.stride, first = (int64_t)blockIdx.x * a.range;
  const int64_t end = min(first + a.range, (int64_t)a.d.vocab);
  RowLists lists;
  if (a.count) {
    lists = row_lists(a, q, r);
#pragma unroll
    for (int g = 0; g < 2 * G; ++g) ((uint4*)s.word)[g * LOGIT_THREADS + threadIdx.x] = uint4{0, 0, 0, 0};
    if (threadIdx.x < Stretch<G>::TOKENS / 32) s.ready[threadIdx.x] = 0;
    if (threadIdx.x == 0) s.n_seen = 0;
  }
  Group<BF16> x;
  x.load(a, q, row, first + threadIdx.x * LANE_TOKENS);
#pragma unroll 1
  for (int64_t base = first; base < end; base += PASS_TOKENS) {
    const int at = (int)((base - first) % Stretch<G>::TOKENS);
    if (a.count && at == 0) prepare_stretch<BF16, G>(a, q, lists, r, (int)base, (int)min((int64_t)Stretch<G>::TOKENS, end - base), s);
    const int64_t v = base + threadIdx.x * LANE_TOKENS;
    Group<BF16> next;
    next.load(a, q, row, base + PASS_TOKENS < end ? v + PASS_TOKENS : (int64_t)a.d.vocab);
    each(x, v, at + (int)threadIdx.x * LANE_TOKENS);
    x = next;
  }
}

template <bool BF16, int G>
__global__ __launch_bounds__(LOGIT_THREADS) void logits_adjust_kernel(LogitArgs a, float* out, int64_t out_stride) {
  extern __shared__ __align__(16) char lds[];
  Stretch<G>& s = *(Stretch<G>*)lds;
  const int r = blockIdx.y;
  const RowRules q = row_rules(a, r);
  float* to = out + (int64_t)r * out_stride;
  through_range<BF16, G>(a, q, r, s, [&](const Group<BF16>& x, int64_t v, int at) {
    const int64_t left = a.d.vocab - v;
    if (left <= 0) return;
    float z[8];
    group_logits<BF16, G, false>(a.count, x, at, s, z);
    if (left >= LANE_TOKENS) {
      __builtin_memcpy(to + v, z, 32);
    } else {
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e)
        if (e < left) to[v + e] = z[e];
    }
  });
}

// ---------------------------------------------------------------- the draw
// What a workgroup, a wave or a lane knows of a row: the largest y and the sum of exp(y - top) (NaN once a y was NaN or +inf), the best
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
__device__ __forceinline__ Draw wave_join(Draw a) {
  const float top = wave_max(a.top);
  a.sum = wave_allsum(a.sum * exp_of(a.top - top));
  a.top = top;
  const float best = wave_max(a.score);
  int token = INT32_MAX;
  float y = -INFINITY;
  for (uint64_t holders = __ballot(a.score == best && a.token != INT32_MAX); holders; holders &= holders - 1) {      // one, as a rule
    const int lane = (int)__builtin_ctzll(holders), t = __builtin_amdgcn_readlane(a.token, lane);
    if (t < token) {
      token = t;
      y = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, a.y), lane));
    }
  }
  a.y = y;
  a.score = best;
  a.token = token;
  return a;
}

__device__ __forceinline__ void finish_draw(const Draw& a, int r, int32_t* token, float* logp) {
  const bool bad = a.sum != a.sum, none = a.token == INT32_MAX;
  token[r] = none || bad ? -1 : a.token;
  logp[r] = bad ? __builtin_nanf("") : none ? -INFINITY : a.y - a.top - logf(a.sum);
}

// Few tokens can win: with E >= w (w the uniform variate of E = -log1p(-w)) a token's score y - ln E reaches a bound b only if
// w <= exp(y - b) = p exp(top - b), where p = exp(y - top) is what the softmax's sum needs anyway.  So a token costs its
// Philox word, one exponential and one multiply-add; b is the best lower bound y - ln w - w (ln E <= ln w + w for w <= 1/2) of
// a token that the workgroup has seen, and only tokens that reach it get their score.
// Five waves a SIMD: six leave 80 registers, so that some of the history's are spilled (384 x 131073 in fp32: 100 us, 92 with five).
template <bool BF16, int G>
__global__ __launch_bounds__(LOGIT_THREADS, 5) void sample_range_kernel(LogitArgs a, const float* temperature, uint32_t k0, uint32_t k1,
                                                                     uint32_t step, const int32_t* ids, Draw* parts, int32_t* token,
                                                                        float* logp) {
  extern __shared__ __align__(16) char lds[];
  Stretch<G>& s = *(Stretch<G>*)lds;
  __shared__ Draw waves[LOGIT_WAVES];
  __shared__ int shared_bound;                       // the bits of a float, ordered as integers
  const int r = blockIdx.y;
  const RowRules q = row_rules(a, r);
  const float t = temperature ? temperature[r] : 1.0f;
  const bool greedy = t == 0.0f;
  const float inv = 1.0f / (greedy ? 1.0f : t);
  const uint32_t id = ids ? (uint32_t)ids[r] : (uint32_t)r;
  auto ordered = [](int b) { return b ^ (b >> 31 & 0x7FFFFFFF); };       // its own inverse
  if (threadIdx.x == 0) shared_bound = ordered(__builtin_bit_cast(int, -INFINITY));
  __syncthreads();
  Draw mine = no_draw();
  through_range<BF16, G>(a, q, r, s, [&](const Group<BF16>& x, int64_t v, int at) {
    if (!__ballot(x.allowed)) {                      // past the row's end, or in one of the long runs that a grammar leaves out
      if (a.count) clear_group(at, s);
      return;
    }
    float y[8];
    group_logits<BF16, G, true>(a.count, x, at, s, y);
    if (greedy) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (y[e] > mine.score) {                     // tokens ascend within a lane
          mine.score = mine.y = y[e];
          mine.token = (int)v + e;
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
    if (greedy) return;
    const uint32_t block = (uint32_t)v >> 2;
    const u32x4 b0 = philox4x32_10<true>(u32x4{block, step, id, STREAM_TOKEN}, k0, k1);
    const u32x4 b1 = philox4x32_10<true>(u32x4{block + 1, step, id, STREAM_TOKEN}, k0, k1);
    const float w[8] = {(float)b0.x, (float)b0.y, (float)b0.z, (float)b0.w, (float)b1.x, (float)b1.y, (float)b1.z, (float)b1.w};
    float bound = __builtin_bit_cast(float, ordered(__hip_atomic_load(&shared_bound, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)));
    // 2^32, and 1e-3 for the rounding of the exponentials
    const float reach = exp_of(top - bound) * 4.2992672e9f;
    float far = -1.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) far = fmaxf(far, __builtin_fmaf(p[e], reach, -w[e]));
    if (!__ballot(far >= 0.0f)) return;
    float up[8], low = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = (w[e] + 0.5f) * 2.3283064365386963e-10f;
      up[e] = y[e] - LN2 * __builtin_amdgcn_logf(u);
      if (u < 0.5f) low = fmaxf(low, up[e] - u);
    }
    low = wave_max(low);
    low -= 1e-4f + 1e-6f * fabsf(low);               // what the logarithms above may be off
    if (low > bound) {
      bound = low;
      atomicMax(&shared_bound, ordered(__builtin_bit_cast(int, bound)));
    }
    uint32_t reached = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) reached |= (uint32_t)(up[e] >= bound && y[e] > -INFINITY) << e;
    while (reached) {                                // a token or two of the wave's
      const int e = __builtin_ctz(reached);
      reached &= reached - 1;
      float ye = y[0], we = w[0];
#pragma unroll
      for (int k = 1; k < 8; ++k) {
        ye = e == k ? y[k] : ye;
        we = e == k ? w[k] : we;
      }
      const float u = fminf((we + 0.5f) * 2.3283064365386963e-10f, 0.99999994f);
      // -log1p(-u): below 1/8 the series up to u^8 (the next term is 7e-9 of it), above the logarithm of 1 - u, whose rounding is 2e-7 of it
      float series = 1.0f / 8;
#pragma unroll
      for (int k = 7; k; --k) series = series * u + 1.0f / k;
      const float score = ye - LN2 * __builtin_amdgcn_logf(u < 0.125f ? series * u : -LN2 * __builtin_amdgcn_logf(1.0f - u));
      if (score > mine.score) {
        mine.score = score;
        mine.token = (int)v + e;
        mine.y = ye;
      }
    }
  });
  if (!(t >= 0.0f && t < INFINITY)) mine.sum = __builtin_nanf("");
  mine = wave_join(mine);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < LOGIT_WAVES; ++w) join(mine, waves[w]);
    if (gridDim.x == 1) finish_draw(mine, r, token, logp);
    else parts[(int64_t)r * gridDim.x + blockIdx.x] = mine;
  }
}

__global__ __launch_bounds__(WAVE) void sample_finish_kernel(const Draw* parts, int ranges, int32_t* token, float* logp) {
  const int r = blockIdx.x;
  Draw mine = no_draw();
  for (int i = threadIdx.x; i < ranges; i += WAVE) join(mine, parts[(int64_t)r * ranges + i]);
  mine = wave_join(mine);
  if (threadIdx.x == 0) finish_draw(mine, r, token, logp);
}

// ---------------------------------------------------------------- host side

// How a call is laid out: tokens of a counted stretch (2048 or 4096: a shorter one where there are few rows, so that more workgroups
// share them) and of a workgroup, and workgroups a row.  A draw's workgroup finds the bound that the tokens have to reach anew and looks
// through the history once, so it takes as many stretches as let all workgroups be resident at once, five on each compute unit (this rule and
// some 4096 workgroups, us, without a history in brackets: 384 x 65537: 60 and 70 (43 and 57); 384 x 131073: 93 and 93 (66 and 74);
// 128 x 131073: 47 and 50 (34 and 39); 640 x 65537: 87 and 97 (53 and 71); 1000 x 65537: 111 and 125 (69 and 85)).  More rows than that
// get some 4096 workgroups.  Adjusting keeps nothing but the history between stretches and gains nothing from longer ranges
// (384 x 65537 in bf16, nothing to adjust: 35 us by this rule, a stretch each, and 44 with 2048 workgroups).  (Whole rows of more than 2048 tokens in one workgroup, without
// the second launch: 10.3 us for one row of 8192, 9.9 with it; 22.8 and 21.8 for 384 rows of 12288.)
constexpr int64_t RESIDENT_DRAWS = 1280;                  // of 256 lanes, five waves a SIMD
struct LogitGrid { int groups, range, workgroups; };
static LogitGrid logit_grid(int64_t rows, int64_t vocab, bool draw) {
  // stretches of 2048 and 4096 in us: draws of 48 x 32001 (384 long stretches): 16.9, 16.6; 128 x 16384 (512): 18.1, 18.1; 48 x 65537 (816): 23.3,
  // 20.2; adjusting 128 x 16384: 7.0, 7.7; 48 x 65537: 8.9, 9.7; 384 x 16384 (1536): 14.1, 12.3
  const int g = rows * ((vocab + 2 * PASS_TOKENS - 1) / (2 * PASS_TOKENS)) < (draw ? 512 : 1024) ? 1 : 2;
  const int64_t stretches = (vocab + g * PASS_TOKENS - 1) / (g * PASS_TOKENS);
  const int64_t each = draw && rows ? RESIDENT_DRAWS / rows : 0;
  const int64_t per = each ? (stretches + each - 1) / each
                           : std::min<int64_t>(stretches, std::max<int64_t>(1, rows * stretches / (draw ? 4096 : 8192)));
  return LogitGrid{g, (int)(per * g * PASS_TOKENS), (int)((stretches + per - 1) / per)};
}
pg_status logit_args(const pg_logits* d, const char* who, LogitArgs& a, int32_t max_rows) {
  if (!d) return fail(PG_EINVAL, "%s: desc is NULL", who);
  if (d->rows < 0 || d->vocab < 1 || (d->dtype != PG_LOGITS_F32 && d->dtype != PG_LOGITS_BF16))
    return fail(PG_EINVAL, "%s: %d rows of %d tokens, dtype %d", who, d->rows, d->vocab, d->dtype);
  if (d->rows > max_rows) return fail(PG_ESHAPE, "%s: %d rows (at most %d)", who, d->rows, max_rows);
  if (d->vocab > 1 << 30 || d->rows * ((d->vocab + PASS_TOKENS - 1ll) / PASS_TOKENS) >= 1 << 24)
    return fail(PG_ESHAPE, "%s: %d rows of %d tokens pass 2^24 workgroups", who, d->rows, d->vocab);
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

bool rows_overlap(uintptr_t p, int64_t p_step, int64_t a, uintptr_t q, int64_t q_step, int64_t b, int64_t rows) {
  if (p + (rows - 1) * p_step + a <= q || q + (rows - 1) * q_step + b <= p) return false;
  for (int64_t r = 0; r < rows; ++r) {
    const int64_t lo = (int64_t)(q - p) + r * q_step;
    const int64_t i = lo >= 0 ? lo / p_step : -1;    // the last that begins at or before it
    if (i >= 0 && i < rows && lo < i * p_step + a) return true;
    if (i + 1 < rows && (i + 1) * p_step < lo + b) return true;
  }
  return false;
}

// launches F<bf16, groups>
#define PG_LOGIT_KERNEL(F, groups, ...)                                                                                          \
  do {                                                                                                                           \
    const bool b = a.d.dtype == PG_LOGITS_BF16;                                                                                  \
    const size_t lds = !a.count ? 0 : (groups) == 1 ? sizeof(Stretch<1>) : sizeof(Stretch<2>);                                   \
    if ((groups) == 1) b ? F<true, 1><<<grid, block, lds, s>>>(__VA_ARGS__) : F<false, 1><<<grid, block, lds, s>>>(__VA_ARGS__); \
    else b ? F<true, 2><<<grid, block, lds, s>>>(__VA_ARGS__) : F<false, 2><<<grid, block, lds, s>>>(__VA_ARGS__);               \
  } while (0)

}  // namespace pg

using namespace pg;

extern "C" pg_status pg_logits_adjust(const pg_logits* desc, float* out, int64_t out_stride, void* stream) {
  LogitArgs a{};
  PG_TRY(logit_args(desc, "pg_logits_adjust", a, 65535));
  if (a.d.rows == 0) return PG_OK;
  if (!out) return fail(PG_EINVAL, "pg_logits_adjust: out is NULL");
  if ((uintptr_t)out & 3 || out_stride < a.d.vocab) return fail(PG_ESHAPE, "pg_logits_adjust: out rows %lld floats apart", (long long)out_stride);
  if ((const void*)out == a.d.logits && (a.d.dtype != PG_LOGITS_F32 || out_stride != a.d.stride))
    return fail(PG_EINVAL, "pg_logits_adjust: in place needs fp32 logits of the same stride");
  const int64_t elt = a.d.dtype == PG_LOGITS_BF16 ? 2 : 4;
  if ((const void*)out != a.d.logits && rows_overlap((uintptr_t)a.d.logits, a.d.stride * elt, a.d.vocab * elt, (uintptr_t)out, out_stride * 4,
                                                     a.d.vocab * 4ll, a.d.rows))
    return fail(PG_EINVAL, "pg_logits_adjust: out overlaps the logits");
  const LogitGrid g = logit_grid(a.d.rows, a.d.vocab, false);
  a.range = g.range;
  const dim3 grid((unsigned)g.workgroups, (unsigned)a.d.rows), block(LOGIT_THREADS);
  hipStream_t s = (hipStream_t)stream;
  PG_LOGIT_KERNEL(logits_adjust_kernel, g.groups, a, out, out_stride);
  PG_LAUNCH_CHECK("logits_adjust_kernel");
  return PG_OK;
}

// No less than any call of at most so many rows and tokens writes, though a call of fewer rows may have more workgroups: up to
// RESIDENT_DRAWS rows have no more workgroups than that in all; above, where a row has `per` of its stretches a workgroup, they are fewer than
// 8192 with per = 1, and with per >= 2 at most 4096 * 3/2 + rows (per is rounded down, the workgroups of a row up).
extern "C" int64_t pg_sample_scratch_floats(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1) return 0;
  const int64_t stretches = ((int64_t)vocab + PASS_TOKENS - 1) / PASS_TOKENS;
  return std::min(rows * stretches, rows <= RESIDENT_DRAWS ? RESIDENT_DRAWS : 8192 + (int64_t)rows) * (int64_t)(sizeof(Draw) / sizeof(float));
}

extern "C" pg_status pg_sample_tokens(const pg_logits* desc, const float* temperature, uint64_t seed, uint32_t step, const int32_t* ids,
                                      int32_t* token, float* logp, float* scratch, void* stream) {
  LogitArgs a{};
  PG_TRY(logit_args(desc, "pg_sample_tokens", a, 65535));
  if (a.d.rows == 0) return PG_OK;
  if (!token || !logp || !scratch) return fail(PG_EINVAL, "pg_sample_tokens: null pointer");
  hipStream_t s = (hipStream_t)stream;
  const LogitGrid g = logit_grid(a.d.rows, a.d.vocab, true);
  a.range = g.range;
  const dim3 grid((unsigned)g.workgroups, (unsigned)a.d.rows), block(LOGIT_THREADS);
  PG_LOGIT_KERNEL(sample_range_kernel, g.groups, a, temperature, (uint32_t)seed, (uint32_t)(seed >> 32), step, ids, (Draw*)scratch, token, logp);
  PG_LAUNCH_CHECK("sample_range_kernel");
  if (g.workgroups == 1) return PG_OK;
  sample_finish_kernel<<<dim3((unsigned)a.d.rows), dim3(WAVE), 0, s>>>((const Draw*)scratch, (int)grid.x, token, logp);
  PG_LAUNCH_CHECK("sample_finish_kernel");
  return PG_OK;
}
