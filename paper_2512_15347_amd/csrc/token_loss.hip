// What a token policy learns from: log-probs of given tokens with entropy and alternatives, the divergence from a teacher's most likely
// tokens, the clipped objective of sequences, and their gradients.
//
// Of a row only three sums are needed, all relative to its largest logit m: S = sum exp((z - m) / T), U = sum exp((z - m) / T) (z - m) and, where a
// teacher's list is compared, S over the tokens that are not on it.  Then ln p = (z - m) / T - ln S and the entropy is ln S - U / (S T), a
// sum of terms of one sign.  Differences to m are exact where it matters, so that a row may be shifted by any amount; m and ln S are kept apart
// for the backward pass for the same reason.
#include <cfloat>
#include <cmath>
#include "common.hpp"
#include "operands.hpp"
#include "token_logits.hpp"

namespace pg {

constexpr int LOSS_THREADS = 256;
constexpr int LOSS_WAVES = LOSS_THREADS / WAVE;
constexpr float FAR = 200.0f;                        // exp(-FAR) is 0 in fp32

struct LossArgs {
  LogitArgs l;
  const float* temperature;
};

// What one row needs.
struct LossRow {
  int64_t at;                                        // its first logit
  const uint8_t* allow;                              // bit v % 8 of byte v / 8; NULL: `unmasked` for all of them
  uint32_t unmasked;
  float inv;                                         // 1 / temperature, NaN for one that is no temperature
  float c;                                           // the same in base 2
  float lim;                                         // z - m below which p is 0
};
__device__ __forceinline__ LossRow loss_row(const LossArgs& a, int r) {
  const pg_logits& d = a.l.d;
  LossRow q;
  q.at = (int64_t)r * d.stride;
  const int mask = d.allow_row ? d.allow_row[r] : r;
  q.allow = d.allow && mask >= 0 && mask < d.n_masks ? (const uint8_t*)(d.allow + (int64_t)mask * a.l.words) : nullptr;
  q.unmasked = d.allow && mask != -1 ? 0u : 0xFFu;   // an index that no mask has allows nothing
  const float t = a.temperature ? a.temperature[r] : 1.0f;
  q.inv = !(t >= 0.0f && t < INFINITY) ? __builtin_nanf("") : t == 0.0f ? 1.0f : 1.0f / t;
  q.c = q.inv * LOG2E;
  q.lim = -FAR * (t > 0.0f && t < INFINITY ? t : 1.0f);
  return q;
}
__device__ __forceinline__ bool allowed(const LossRow& q, int64_t v) { return (q.allow ? (uint32_t)q.allow[v >> 3] : q.unmasked) >> (v & 7) & 1; }
template <bool BF16>
__device__ __forceinline__ float logit_at(const LossArgs& a, const LossRow& q, int64_t v) {
  return BF16 ? bf16_to_f32(((const uint16_t*)a.l.d.logits)[q.at + v]) : ((const float*)a.l.d.logits)[q.at + v];
}
// -inf where a token is not allowed
template <bool BF16>
__device__ __forceinline__ float open_logit(const LossArgs& a, const LossRow& q, int64_t v) {
  return allowed(q, v) ? logit_at<BF16>(a, q, v) : -INFINITY;
}

// Sums of a lane, a wave or a range; NaN in s once a logit was NaN or +inf.
struct Sums {
  float m, s, u;
};
__device__ __forceinline__ Sums no_sums() { return Sums{-FLT_MAX, 0.0f, 0.0f}; }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ void move_to(Sums& a, float m, const LossRow& q) {
  const float t = a.m - m, f = exp2_of(t * q.c);
  a.u = f * (a.u + fmaxf(t, q.lim) * a.s);
  a.s = f * a.s;
  a.m = m;
}
__device__ __forceinline__ void join(Sums& a, Sums b, const LossRow& q) {
  const float m = fmaxf(a.m, b.m);
  move_to(a, m, q);
  move_to(b, m, q);
  a.s += b.s;
  a.u += b.u;
}
__device__ __forceinline__ void take(Sums& a, float z, const LossRow& q) {
  if (z > a.m) move_to(a, z, q);
  const float t = z - a.m, e = exp2_of(t * q.c);
  a.s += e;
  a.u += e * fmaxf(t, q.lim);
}

__device__ __forceinline__ Sums block_sums(Sums a, const LossRow& q, Sums* waves) {
  for (int o = 32; o; o >>= 1) {
    const Sums b{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.u, o)};
    join(a, b, q);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = a;
  __syncthreads();
  a = waves[0];
  for (int w = 1; w < LOSS_WAVES; ++w) join(a, waves[w], q);
  return a;
}

// Whether (z, v) comes before (y, w) among alternatives.
__device__ __forceinline__ bool before(float z, int v, float y, int w) { return z > y || (z == y && v < w); }

struct LogprobOut {
  const int32_t* target;
  float *logp, *entropy, *stats;
  int n_top;
  int32_t* top_ids;
  float* top_logp;
};

template <bool BF16>
__global__ __launch_bounds__(LOSS_THREADS) void logprob_kernel(LossArgs a, LogprobOut o) {
  __shared__ Sums waves[LOSS_WAVES];
  __shared__ float best_z[LOSS_WAVES];
  __shared__ int best_v[LOSS_WAVES];
  const int r = blockIdx.x, vocab = a.l.d.vocab;
  const LossRow q = loss_row(a, r);
  const int target = o.target ? o.target[r] : 0;
  const bool gone = target == -1;
  Sums mine = no_sums();
  if (!gone)
    for (int v = threadIdx.x; v < vocab; v += LOSS_THREADS) take(mine, open_logit<BF16>(a, q, v), q);
  mine = block_sums(mine, q, waves);
  const bool bad = mine.s != mine.s, none = mine.s == 0.0f;
  const float ln_s = none ? 0.0f : logf(mine.s);
  if (threadIdx.x == 0) {
    const float h = gone || none ? 0.0f : ln_s - q.inv * (mine.u / mine.s);
    if (o.entropy) o.entropy[r] = h;
    if (o.logp) {
      float l = __builtin_nanf("");
      if (gone) l = 0.0f;
      else if (target >= 0 && target < vocab && !bad) l = none ? -INFINITY : (open_logit<BF16>(a, q, target) - mine.m) * q.inv - ln_s;
      o.logp[r] = l;
    }
    if (o.stats) *(float4*)(o.stats + 4ll * r) = float4{none ? -INFINITY : mine.m * q.inv, ln_s, h, mine.m};
  }
  float last_z = INFINITY;
  int last_v = -1;
  for (int i = 0; i < o.n_top; ++i) {
    float z = -INFINITY;
    int at = INT32_MAX;
    if (!gone && !bad)
      for (int v = threadIdx.x; v < vocab; v += LOSS_THREADS) {
        const float x = open_logit<BF16>(a, q, v);
        if (before(last_z, last_v, x, v) && before(x, v, z, at)) {
          z = x;
          at = v;
        }
      }
    for (int k = 32; k; k >>= 1) {
      const float y = __shfl_xor(z, k);
      const int w = __shfl_xor(at, k);
      if (before(y, w, z, at)) {
        z = y;
        at = w;
      }
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      best_z[threadIdx.x >> 6] = z;
      best_v[threadIdx.x >> 6] = at;
    }
    __syncthreads();
    for (int w = 0; w < LOSS_WAVES; ++w)
      if (before(best_z[w], best_v[w], z, at)) {
        z = best_z[w];
        at = best_v[w];
      }
    const bool there = z > -INFINITY;
    last_z = z;
    last_v = at;
    if (threadIdx.x == 0) {
      if (o.top_ids) o.top_ids[(int64_t)r * o.n_top + i] = there ? at : -1;
      if (o.top_logp) o.top_logp[(int64_t)r * o.n_top + i] = bad ? __builtin_nanf("") : there ? (z - mine.m) * q.inv - ln_s : -INFINITY;
    }
  }
}

template <bool BF16>
__device__ __forceinline__ void put(void* to, int64_t at, float v) {
  if (BF16) ((uint16_t*)to)[at] = (uint16_t)pack_bf16x2(v, 0.0f);
  else ((float*)to)[at] = v;
}

template <bool BF16>
__global__ __launch_bounds__(LOSS_THREADS) void logprob_backward_kernel(LossArgs a, const int32_t* target, const float* stats, const float* g_logp,
                                                                        const float* g_entropy, void* out, int64_t out_stride) {
  const int r = blockIdx.x, vocab = a.l.d.vocab;
  const LossRow q = loss_row(a, r);
  const int t = target ? target[r] : 0;
  float g = g_logp ? g_logp[r] : 0.0f;
  const float ge = g_entropy ? g_entropy[r] : 0.0f;
  const bool still = t == -1 || (g == 0.0f && ge == 0.0f);
  if (g_logp && (t < 0 || t >= vocab)) g = __builtin_nanf("");
  const float ln_s = stats[4ll * r + 1], h = stats[4ll * r + 2], m = stats[4ll * r + 3];
  const float c0 = q.inv * (-g - ge * (h - ln_s)), c1 = -q.inv * ge * q.inv, at_target = q.inv * g;
  for (int v = threadIdx.x; v < vocab; v += LOSS_THREADS) {
    float d = 0.0f;
    if (!still) {
      const float z = open_logit<BF16>(a, q, v), x = fmaxf(z - m, q.lim);
      if (z != -INFINITY) d = exp2_of(x * q.c - ln_s * LOG2E) * (c1 * x + c0) + (v == t ? at_target : 0.0f);
    }
    put<BF16>(out, (int64_t)r * out_stride + v, d);
  }
}

// ---------------------------------------------------------------- distillation

// Entry i of a row's list counts: its token exists, and no entry before it has the same.
__device__ __forceinline__ bool first_of(const int32_t* ids, int i, int vocab) {
  const int id = ids[i];
  if (id < 0 || id >= vocab) return false;
  for (int j = 0; j < i; ++j)
    if (ids[j] == id) return false;
  return true;
}
__device__ __forceinline__ bool is_listed(const int32_t* ids, int k, int v) {
  for (int j = 0; j < k; ++j)
    if (ids[j] == v) return true;
  return false;
}

template <bool BF16>
__global__ __launch_bounds__(LOSS_THREADS) void distill_kernel(LossArgs a, int mode, const int32_t* teacher_ids, const float* teacher_logp, int k,
                                                               float* loss, float* stats) {
  __shared__ Sums waves[LOSS_WAVES];
  const int r = blockIdx.x, vocab = a.l.d.vocab;
  const LossRow q = loss_row(a, r);
  const int32_t* ids = teacher_ids + (int64_t)r * k;
  const float* t = teacher_logp + (int64_t)r * k;
  Sums mine = no_sums();
  for (int v = threadIdx.x; v < vocab; v += LOSS_THREADS)
    if (!is_listed(ids, k, v)) take(mine, open_logit<BF16>(a, q, v), q);
  const Sums rest = block_sums(mine, q, waves);
  if (threadIdx.x) return;
  double m = rest.m, most = -INFINITY;
  int n = 0;
  for (int i = 0; i < k; ++i)
    if (first_of(ids, i, vocab)) {
      ++n;
      m = fmax(m, (double)open_logit<BF16>(a, q, ids[i]));
      most = fmax(most, (double)t[i]);
    }
  double s = rest.s * exp((rest.m - m) * q.inv), sum_q = 0.0, bad = 0.0;
  for (int i = 0; i < k; ++i)
    if (first_of(ids, i, vocab)) {
      s += exp((open_logit<BF16>(a, q, ids[i]) - m) * q.inv);
      if (!(t[i] < INFINITY)) bad = __builtin_nan("");
      sum_q += exp(mode == PG_DISTILL_TOP ? t[i] - most : (double)t[i]);
    }
  const bool active = n && s != 0.0 && !(mode == PG_DISTILL_TOP && most == -INFINITY && bad == 0.0);
  double total = 0.0, q_rest = 0.0, all = 0.0, t0 = 0.0, p_rest = 0.0;
  if (active) {
    t0 = mode == PG_DISTILL_TOP ? most + log(sum_q) : 0.0;
    const double ln_rest = (rest.m - m) * q.inv + log((double)rest.s) - log(s);
    if (rest.s != 0.0f) p_rest = exp(ln_rest);
    if (mode == PG_DISTILL_TAIL && rest.s != 0.0f) q_rest = fmax(0.0, 1.0 - sum_q);
    total = bad;
    for (int i = 0; i < k; ++i)
      if (first_of(ids, i, vocab)) {
        const double lq = t[i] - t0, w = exp(lq);
        if (w > 0.0) total += w * (lq - ((open_logit<BF16>(a, q, ids[i]) - m) * q.inv - log(s)));
        all += w;
      }
    if (q_rest > 0.0) total += q_rest * (log(q_rest) - ln_rest);
    all += q_rest + bad;
  }
  loss[r] = (float)total;
  if (stats) {
    float* x = stats + (int64_t)r * PG_DISTILL_STATS;
    x[0] = (float)m;
    x[1] = (float)log(s);
    x[2] = rest.m;
    x[3] = rest.s == 0.0f ? 0.0f : logf(rest.s);
    x[4] = (float)(all * p_rest - q_rest);
    x[5] = (float)t0;
    x[6] = (float)all;
    x[7] = active ? 1.0f : 0.0f;
  }
}

template <bool BF16>
__global__ __launch_bounds__(LOSS_THREADS) void distill_backward_kernel(LossArgs a, const int32_t* teacher_ids, const float* teacher_logp, int k,
                                                                        const float* stats, const float* g_loss, void* out, int64_t out_stride) {
  const int r = blockIdx.x, vocab = a.l.d.vocab;
  const LossRow q = loss_row(a, r);
  const int32_t* ids = teacher_ids + (int64_t)r * k;
  const float* x = stats + (int64_t)r * PG_DISTILL_STATS;
  const float g = x[7] == 0.0f ? 0.0f : g_loss[r], scale = g * q.inv;
  for (int v = threadIdx.x; v < vocab; v += LOSS_THREADS) {
    float d = 0.0f;
    const float z = g != 0.0f ? open_logit<BF16>(a, q, v) : -INFINITY;
    if (z != -INFINITY) {
      int at = -1;
      for (int j = k - 1; j >= 0; --j) at = ids[j] == v ? j : at;
      d = at < 0 ? scale * x[4] * exp2_of(fmaxf(z - x[2], q.lim) * q.c - x[3] * LOG2E)
                 : scale * (x[6] * exp2_of(fmaxf(z - x[0], q.lim) * q.c - x[1] * LOG2E) - expf(teacher_logp[(int64_t)r * k + at] - x[5]));
    }
    put<BF16>(out, (int64_t)r * out_stride + v, d);
  }
}

// ---------------------------------------------------------------- the clipped objective

struct SurrogateArgs {
  const float *logp, *old, *ref, *adv, *weight;
  const int32_t* cu;
  int n_tokens;
  double lo, hi;                                     // of ln rho
  float at_lo, at_hi, kl_coef;
  float *objective, *kl, *g_logp;
  int32_t* clipped;
};

__global__ __launch_bounds__(LOSS_THREADS) void surrogate_tokens_kernel(SurrogateArgs a) {
  __shared__ double sums[2][LOSS_THREADS];
  __shared__ int counts[LOSS_THREADS];
  const int r = blockIdx.x;
  const int from = min(max(a.cu[r], 0), a.n_tokens), to = min(max(a.cu[r + 1], from), a.n_tokens), n = to - from;
  const float A = a.adv[r], w = a.weight ? a.weight[r] : 1.0f / (float)max(n, 1);
  double sum = 0.0, kl = 0.0;
  int cuts = 0;
  for (int i = from + threadIdx.x; i < to; i += LOSS_THREADS) {
    const float l = a.logp[i];
    const double d = (double)l - (double)a.old[i];
    const bool cut = A > 0.0f ? d > a.hi : A < 0.0f && d < a.lo;
    const float ra = A == 0.0f ? 0.0f : expf((float)d) * A;
    float g = cut ? 0.0f : ra, value = cut ? (A > 0.0f ? a.at_hi : a.at_lo) * A : ra;
    if (a.ref) {
      const float x = a.ref[i] - l;
      const double e = expm1((double)x);
      const float k = (float)(e - x);
      kl += k;
      value -= a.kl_coef * k;
      g += a.kl_coef * (float)e;
    }
    sum += value;
    cuts += cut;
    if (a.g_logp) a.g_logp[i] = w * g;
  }
  sums[0][threadIdx.x] = sum;
  sums[1][threadIdx.x] = kl;
  counts[threadIdx.x] = cuts;
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < LOSS_THREADS; ++i) {
    sum += sums[0][i];
    kl += sums[1][i];
    cuts += counts[i];
  }
  if (a.objective) a.objective[r] = (float)(w * sum);
  if (a.kl) a.kl[r] = (float)(kl / max(n, 1));
  if (a.clipped) a.clipped[r] = cuts;
}

// ---------------------------------------------------------------- host side

static pg_status loss_args(const pg_logits* desc, const float* temperature, const char* who, LossArgs& a) {
  PG_TRY(logit_args(desc, who, a.l, 1 << 23));
  if (desc->tokens || desc->bias_offsets) return fail(PG_EINVAL, "%s: logits with a history or biases (pg_logits_adjust first)", who);
  a.temperature = temperature;
  return PG_OK;
}
static pg_status check_gradient(const LossArgs& a, const void* out, int64_t out_stride, const char* who) {
  const pg_logits& d = a.l.d;
  const int64_t elt = d.dtype == PG_LOGITS_BF16 ? 2 : 4;
  if (!out) return fail(PG_EINVAL, "%s: d_logits is NULL", who);
  if ((uintptr_t)out & (elt - 1) || out_stride < d.vocab) return fail(PG_ESHAPE, "%s: d_logits' rows %lld elements apart", who, (long long)out_stride);
  if (out == d.logits ? out_stride != d.stride
                      : rows_overlap((uintptr_t)d.logits, d.stride * elt, d.vocab * elt, (uintptr_t)out, out_stride * elt, d.vocab * elt, d.rows))
    return fail(PG_EINVAL, "%s: d_logits overlaps the logits", who);
  return PG_OK;
}

// launches F<bf16>
#define PG_LOSS_KERNEL(F, grid, ...)                                                                            \
  do {                                                                                                          \
    if (a.l.d.dtype == PG_LOGITS_BF16) F<true><<<dim3(grid), dim3(LOSS_THREADS), 0, (hipStream_t)stream>>>(__VA_ARGS__); \
    else F<false><<<dim3(grid), dim3(LOSS_THREADS), 0, (hipStream_t)stream>>>(__VA_ARGS__);                     \
    PG_LAUNCH_CHECK(#F);                                                                                        \
  } while (0)

}  // namespace pg

using namespace pg;

extern "C" int64_t pg_logprob_scratch_floats(int32_t rows, int32_t vocab, int32_t n_top) {
  if (rows < 1 || vocab < 1 || n_top < 0) return 0;
  return 0;
}

extern "C" pg_status pg_token_logprobs(const pg_logits* desc, const float* temperature, const int32_t* target, float* logp, float* entropy,
                                       float* stats, int32_t n_top, int32_t* top_ids, float* top_logp, float* scratch, void* stream) {
  LossArgs a{};
  PG_TRY(loss_args(desc, temperature, "pg_token_logprobs", a));
  if (n_top < 0 || n_top > PG_TOP_MAX) return fail(n_top < 0 ? PG_EINVAL : PG_ESHAPE, "pg_token_logprobs: %d alternatives (at most %d)", n_top, PG_TOP_MAX);
  if (a.l.d.rows == 0) return PG_OK;
  if (logp && !target) return fail(PG_EINVAL, "pg_token_logprobs: logp without targets");
  if ((uintptr_t)stats & 15) return fail(PG_ESHAPE, "pg_token_logprobs: stats are not 16-byte aligned");
  const LogprobOut o{target, logp, entropy, stats, n_top, top_ids, top_logp};
  PG_LOSS_KERNEL(logprob_kernel, (unsigned)a.l.d.rows, a, o);
  return PG_OK;
}

extern "C" pg_status pg_token_logprobs_backward(const pg_logits* desc, const float* temperature, const int32_t* target, const float* stats,
                                                const float* g_logp, const float* g_entropy, void* d_logits, int64_t d_stride, void* stream) {
  LossArgs a{};
  PG_TRY(loss_args(desc, temperature, "pg_token_logprobs_backward", a));
  if (a.l.d.rows == 0) return PG_OK;
  if (!stats) return fail(PG_EINVAL, "pg_token_logprobs_backward: stats is NULL");
  if ((uintptr_t)stats & 15) return fail(PG_ESHAPE, "pg_token_logprobs_backward: stats are not 16-byte aligned");
  if (g_logp && !target) return fail(PG_EINVAL, "pg_token_logprobs_backward: a gradient of log-probs without targets");
  PG_TRY(check_gradient(a, d_logits, d_stride, "pg_token_logprobs_backward"));
  PG_LOSS_KERNEL(logprob_backward_kernel, (unsigned)a.l.d.rows, a, target, stats, g_logp, g_entropy, d_logits, d_stride);
  return PG_OK;
}

static pg_status distill_args(const LossArgs& a, const int32_t* ids, const float* logp, int32_t k, const float* stats, const char* who) {
  if (k < 1) return fail(PG_EINVAL, "%s: %d tokens of a teacher", who, k);
  if (k > PG_DISTILL_MAX) return fail(PG_ESHAPE, "%s: %d tokens of a teacher (at most %d)", who, k, PG_DISTILL_MAX);
  if (a.l.d.rows && (!ids || !logp)) return fail(PG_EINVAL, "%s: the teacher's list is NULL", who);
  if ((uintptr_t)stats & 15) return fail(PG_ESHAPE, "%s: stats are not 16-byte aligned", who);
  return PG_OK;
}

extern "C" int64_t pg_distill_scratch_floats(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1) return 0;
  return 0;
}

extern "C" pg_status pg_distill_loss(const pg_logits* desc, const float* temperature, int32_t mode, const int32_t* teacher_ids,
                                     const float* teacher_logp, int32_t k, float* loss, float* stats, float* scratch, void* stream) {
  LossArgs a{};
  PG_TRY(loss_args(desc, temperature, "pg_distill_loss", a));
  if (mode != PG_DISTILL_TOP && mode != PG_DISTILL_TAIL) return fail(PG_EINVAL, "pg_distill_loss: mode %d", mode);
  PG_TRY(distill_args(a, teacher_ids, teacher_logp, k, stats, "pg_distill_loss"));
  if (a.l.d.rows == 0) return PG_OK;
  if (!loss) return fail(PG_EINVAL, "pg_distill_loss: loss is NULL");
  PG_LOSS_KERNEL(distill_kernel, (unsigned)a.l.d.rows, a, mode, teacher_ids, teacher_logp, k, loss, stats);
  return PG_OK;
}

extern "C" pg_status pg_distill_backward(const pg_logits* desc, const float* temperature, const int32_t* teacher_ids, const float* teacher_logp,
                                         int32_t k, const float* stats, const float* g_loss, void* d_logits, int64_t d_stride, void* stream) {
  LossArgs a{};
  PG_TRY(loss_args(desc, temperature, "pg_distill_backward", a));
  PG_TRY(distill_args(a, teacher_ids, teacher_logp, k, stats, "pg_distill_backward"));
  if (a.l.d.rows == 0) return PG_OK;
  if (!stats || !g_loss) return fail(PG_EINVAL, "pg_distill_backward: null pointer");
  PG_TRY(check_gradient(a, d_logits, d_stride, "pg_distill_backward"));
  PG_LOSS_KERNEL(distill_backward_kernel, (unsigned)a.l.d.rows, a, teacher_ids, teacher_logp, k, stats, g_loss, d_logits, d_stride);
  return PG_OK;
}

extern "C" int64_t pg_surrogate_scratch_floats(int32_t n_seq, int32_t max_len) {
  if (n_seq < 1 || max_len < 1) return 0;
  return 0;
}

extern "C" pg_status pg_token_surrogate(const float* logp, const float* logp_old, const float* logp_ref, const float* adv, const float* weight,
                                        const int32_t* cu, int32_t n_seq, int32_t n_tokens, int32_t max_len, double clip_low, double clip_high,
                                        double kl_coef, float* objective, float* kl, int32_t* clipped, float* g_logp, float* scratch,
                                        void* stream) {
  if (n_seq < 0 || n_tokens < 0 || max_len < 0) return fail(PG_EINVAL, "pg_token_surrogate: %d sequences, %d tokens, length %d", n_seq, n_tokens, max_len);
  if (n_seq > 1 << 23) return fail(PG_ESHAPE, "pg_token_surrogate: %d sequences (at most %d)", n_seq, 1 << 23);
  if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0) || !std::isfinite(kl_coef))
    return fail(PG_EINVAL, "pg_token_surrogate: clip %g below and %g above, kl_coef %g", clip_low, clip_high, kl_coef);
  if (n_seq == 0) return PG_OK;
  if (!adv || !cu || (n_tokens && (!logp || !logp_old))) return fail(PG_EINVAL, "pg_token_surrogate: null pointer");
  const SurrogateArgs a{logp, logp_old, logp_ref, adv, weight, cu, n_tokens, std::log1p(-clip_low), std::log1p(clip_high), (float)(1.0 - clip_low),
                        (float)(1.0 + clip_high), (float)kl_coef, objective, kl, g_logp, clipped};
  surrogate_tokens_kernel<<<dim3((unsigned)n_seq), dim3(LOSS_THREADS), 0, (hipStream_t)stream>>>(a);
  PG_LAUNCH_CHECK("surrogate_tokens_kernel");
  return PG_OK;
}
