// What a token policy learns from: log-probs of given tokens with entropy and alternatives, the divergence from a teacher's most likely
// tokens, the clipped objective of sequences, and their gradients.
//
// Of a row only three sums are needed, all relative to a logit m of its own that is near the largest: S = sum exp((z - m) / T), U = sum exp((z - m) / T) (z - m) / T
// and, where a teacher's list is compared, S over the tokens that are not on it.  Then ln p = (z - m) / T - ln S and the entropy is ln S - U / S.  The largest
// logit's weight is at most 2^6: where it is above 1 the two are differences of numbers of up to 4.2, but m's own weight is at least 2^-6 of the
// largest then, so that -ln p and the entropy are 0.015 or more, and 5e-7 off.  Differences to m are exact where it matters, so that a row may be
// shifted by any amount; m and ln S are kept apart for the backward pass for the same reason.
//
// Logits are read once for the sums and once more for their gradient, and that is what bounds all but the smallest calls: 6.0 TB/s read, 5.6 TB/s where as much
// is written.  Times here are of kernels on an MI355X.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstddef>
#include <type_traits>
#include "common.hpp"
#include "operands.hpp"
#include "token_logits.hpp"

namespace pg {

constexpr int LOSS_THREADS = 256;
constexpr int LOSS_WAVES = LOSS_THREADS / WAVE;
constexpr int LOSS_TOKENS = LOSS_THREADS * LANE_TOKENS;                 // one group a lane
constexpr float FAR = 300.0f;                        // 2^-FAR is 0 in fp32

struct LossArgs {
  LogitArgs l;
  const float* temperature;
  int64_t span;                                      // elements from the first row's first logit to the last row's last
};

// What one row needs.
struct LossRow {
  int64_t at;                                        // its first logit
  int shift;                                         // slot t, of which eight are 16 aligned bytes, has token t - shift
  const uint8_t* allow;                              // bit v % 8 of byte v / 8; NULL: `unmasked` for all of them
  uint32_t unmasked;
  float t;                                           // the temperature, 1 for 0, NaN for one that is none
  float inv;                                         // its inverse, of 2^-126 where it is smaller: a number
  float c;                                           // the same in base 2
  float lim;                                         // z - m below which p is 0: (z - m) c < -FAR
};
template <bool BF16>
__device__ __forceinline__ LossRow loss_row(const LossArgs& a, int r) {
  const pg_logits& d = a.l.d;
  LossRow q;
  q.at = (int64_t)r * d.stride;
  q.shift = BF16 ? (int)((uintptr_t)d.logits / 2 + (uint64_t)q.at) & (LANE_TOKENS - 1) : 0;
  const int mask = d.allow_row ? d.allow_row[r] : r;
  q.allow = d.allow && mask >= 0 && mask < d.n_masks ? (const uint8_t*)(d.allow + (int64_t)mask * a.l.words) : nullptr;
  q.unmasked = d.allow && mask != -1 ? 0u : 0xFFu;   // an index that no mask has allows nothing
  const float t = a.temperature ? a.temperature[r] : 1.0f;
  q.t = !(t >= 0.0f && t < INFINITY) ? __builtin_nanf("") : t == 0.0f ? 1.0f : t;
  const float above = q.t < FLT_MIN ? FLT_MIN : q.t;
  q.inv = 1.0f / above;
  q.c = LOG2E / above;
  q.lim = -FAR * LN2 * (above == above ? above : 1.0f);
  return q;
}
// (z - m) / T, and the same in base 2; halves, as a difference of two logits may pass fp32's range where a large temperature brings it back.
__device__ __forceinline__ float over_t(float z, float m, const LossRow& q) {
  const float h = q.t > 1.0f ? 0.5f : 1.0f;
  return (h * z - h * m) / (h * q.t);
}
__device__ __forceinline__ float in_base_2(float z, float m, const LossRow& q) { return __builtin_fmaf(z, 0.5f, -0.5f * m) * (2.0f * q.c); }
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

// Sums of a lane, a wave or a range, with x = (z - m) c in base 2: s = sum 2^x, u = sum 2^x x; NaN in s once a logit was NaN or +inf.
struct Sums {
  float m, s, u;
};
__device__ __forceinline__ Sums no_sums() { return Sums{-FLT_MAX, 0.0f, 0.0f}; }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ void move_to(Sums& a, float m, const LossRow& q) {
  const float x = in_base_2(a.m, m, q), f = exp2_of(x);
  a.u = f * (a.u + fmaxf(x, -FAR) * a.s);
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
__device__ __forceinline__ Sums wave_sums(Sums a, const LossRow& q) {
  move_to(a, wave_max(a.m), q);
  a.s = wave_allsum(a.s);
  a.u = wave_allsum(a.u);
  return a;
}
// The workgroup's, from lanes that have the same m throughout a wave.
__device__ __forceinline__ Sums block_sums(Sums a, const LossRow& q, Sums* waves) {
  a.s = wave_allsum(a.s);
  a.u = wave_allsum(a.u);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = a;
  __syncthreads();
  a = waves[0];
#pragma unroll
  for (int w = 1; w < LOSS_WAVES; ++w) join(a, waves[w], q);
  return a;
}

// Keeps the compiler from unpacking all groups of a pass before it works on the first: two groups fit eight waves a SIMD then.
__device__ __forceinline__ void one_group_at_a_time() { __builtin_amdgcn_sched_barrier(0); }

// A lane's part of one pass over a range: G groups of eight slots and which of their tokens count: those that are in the row and in the range,
// allowed and not struck out.  16-byte loads may be unaligned, but in bf16, where a row may begin between two 4-byte words, they are a third
// slower then; in fp32 slots would cost (4096 x 65537 against a list: 215 us, a quarter more with them).
// Every logit is read once a pass and marked so, in us with and without: 4096 x 65537 94 and 100, 1178 x 131073 63 and 68, 4096 x 131072
// 177 and 199, 2048 x 131073 against a list 104 and 115.
typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(4)));

template <bool BF16, int G>
struct Pass {
  static constexpr int ELT = BF16 ? 2 : 4;
  uint32_t raw[G][BF16 ? 4 : 8];
  uint32_t bits[G];

  // Slots base + g LOSS_TOKENS + 8 lane .. of which all have tokens; the masks' bits alone are left out where there are none.
  template <bool MASKS>
  __device__ __forceinline__ void load_whole(const LossArgs& a, const LossRow& q, int base) {
    const char* p = (const char*)a.l.d.logits + (q.at + base - q.shift) * ELT;       // the wave's; a lane adds 32 bits
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < (BF16 ? 4 : 8); i += 4) {
        const Words x = __builtin_nontemporal_load((const Words*)(p + g * (LOSS_TOKENS * ELT) + threadIdx.x * (LANE_TOKENS * ELT) + 4 * i));
#pragma unroll
        for (int j = 0; j < 4; ++j) raw[g][i + j] = x[j];
      }
    if (!MASKS) return;
    const uint8_t* m = q.allow + ((base - q.shift) >> 3);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint8_t* at = m + g * (LOSS_TOKENS / LANE_TOKENS) + threadIdx.x;
      if (q.shift == 0) {
        bits[g] = *at;
      } else {
        uint16_t two;
        __builtin_memcpy(&two, at, 2);
        bits[g] = two >> (LANE_TOKENS - q.shift) & 0xFFu;
      }
    }
  }
  // Of slots up to `end`.  A group at an end of its row is read with what lies beside it in the logits' span; only the first row's first and the last
  // row's last may have nothing there.
  __device__ __forceinline__ void load_part(const LossArgs& a, const LossRow& q, int base, int end) {
    const int vocab = a.l.d.vocab;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int at = base + g * LOSS_TOKENS + (int)threadIdx.x * LANE_TOKENS, v = at - q.shift;
      const char* p = (const char*)a.l.d.logits + (q.at + v) * ELT;
      bits[g] = 0;
      if (at < end && v < vocab) {
        uint32_t there = v < 0 ? 0xFFu << -v & 0xFFu : 0xFFu;
        if (v > vocab - LANE_TOKENS) there &= (1u << (vocab - v)) - 1;
        if (q.at + v >= 0 && q.at + v + LANE_TOKENS <= a.span) {
          __builtin_memcpy(raw[g], __builtin_assume_aligned(p, BF16 ? 16 : 4), BF16 ? 16 : 32);
        } else {
#pragma unroll
          for (int e = 0; e < LANE_TOKENS; ++e) {
            const uint32_t x = !(there >> e & 1) ? 0u : BF16 ? ((const uint16_t*)p)[e] : ((const uint32_t*)p)[e];
            if (!BF16) raw[g][e] = x;
            else raw[g][e >> 1] = e & 1 ? raw[g][e >> 1] | x << 16 : x;
          }
        }
        if (q.allow) {
          const int byte = v >> 3;                   // the first token's, -1 before the row
          const uint32_t lo = byte >= 0 ? q.allow[byte] : 0u, hi = byte + 1 < 4 * a.l.words ? q.allow[byte + 1] : 0u;
          there &= (lo | hi << 8) >> (v & 7);
        }
        bits[g] = there;
      }
    }
  }
  __device__ __forceinline__ float raw_logit(int g, int e) const {
    return __builtin_bit_cast(float, !BF16 ? raw[g][e] : e & 1 ? raw[g][e >> 1] & 0xFFFF0000u : raw[g][e >> 1] << 16);
  }
  __device__ __forceinline__ void all_count() {
#pragma unroll
    for (int g = 0; g < G; ++g) bits[g] = 0xFFu;
  }
  // HOLES: -inf for what does not count
  template <bool HOLES>
  __device__ __forceinline__ float logit(int g, int e) const {
    return HOLES && !(bits[g] >> e & 1) ? -INFINITY : raw_logit(g, e);
  }
  template <bool HOLES>
  __device__ __forceinline__ float largest(int g) const {
    float top = logit<HOLES>(g, 0);
#pragma unroll
    for (int e = 1; e < LANE_TOKENS; ++e) top = fmaxf(top, logit<HOLES>(g, e));
    return top;
  }
  // of the wave's, the same in every lane
  __device__ __forceinline__ float largest(bool holes) const {
    float top = -INFINITY;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      top = fmaxf(top, holes ? largest<true>(g) : largest<false>(g));
      one_group_at_a_time();
    }
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, wave_max(top))));
  }
};

// Goes through slots first .. end - 1 of a row: each(pass, its first slot, whether some of the wave's tokens do not count) for passes that have a
// token that counts, none(first slot) for the others; `first` is a multiple of LOSS_TOKENS.  strike(t): bits of the group at slot t that are
// struck out, if STRIKES.
template <bool BF16, int G, bool STRIKES, class Strike, class Each, class None>
__device__ __forceinline__ void through(const LossArgs& a, const LossRow& q, int first, int end, Strike strike, Each each, None none) {
  const int whole = min(end, a.l.d.vocab + q.shift) - G * LOSS_TOKENS;         // the last pass of which all slots have tokens
#pragma unroll 1
  for (int base = first; base < end; base += G * LOSS_TOKENS) {
    Pass<BF16, G> x;
    bool holes = false;
    if (!q.allow && !q.unmasked) {
      none(base);
      continue;
    }
    if (base >= q.shift && base <= whole) {
      if (q.allow) x.template load_whole<true>(a, q, base);
      else x.template load_whole<false>(a, q, base);
    } else {
      x.load_part(a, q, base, end);
      holes = true;
    }
    if (STRIKES || holes || q.allow) {
      uint32_t all = 0xFFu, some = 0;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if (!q.allow && !holes) x.bits[g] = 0xFFu;
        if (STRIKES) x.bits[g] &= ~strike(base + g * LOSS_TOKENS + (int)threadIdx.x * LANE_TOKENS);
        all &= x.bits[g];
        some |= x.bits[g];
      }
      holes = __ballot(all != 0xFFu);
      if (holes && !__ballot(some != 0)) {
        none(base);
        continue;
      }
    }
    each(x, base, holes);
  }
}
constexpr auto no_strike = [](int) { return 0u; };

// What a wave has summed: every lane the sums of its own tokens, relative to one logit m for all of them, which is some logit of the wave's
// and at most a little less than the largest: 2^x stays within 2^6.
struct WaveSums {
  Sums sums;
  bool clamp;                                        // there are logits of -inf
  __device__ __forceinline__ WaveSums() : sums(no_sums()), clamp(false) {}
};

// What does not count has x = -FAR.
template <bool HOLES, bool CLAMP, bool ENTROPY, class P, int G>
__device__ __forceinline__ void add_near(const P& x, float r, const LossRow& q, float& s, float& u) {
#pragma unroll
  for (int g = 0; g < G; ++g) {
    float y[LANE_TOKENS], p[LANE_TOKENS];
#pragma unroll
    for (int e = 0; e < LANE_TOKENS; ++e) {
      y[e] = __builtin_fmaf(x.raw_logit(g, e), q.c, -r);
      if (HOLES) {
        const uint32_t counts = (uint32_t)__builtin_amdgcn_sbfe((int)x.bits[g], e, 1);
        y[e] = __builtin_bit_cast(float, (counts & __builtin_bit_cast(uint32_t, y[e])) | (~counts & __builtin_bit_cast(uint32_t, -FAR)));
      }
      p[e] = exp2_of(y[e]);
    }
#pragma unroll
    for (int e = 0; e < LANE_TOKENS; ++e) {
      s += p[e];
      if (ENTROPY) u = __builtin_fmaf(p[e], CLAMP ? fmaxf(y[e], -FAR) : y[e], u);
    }
    one_group_at_a_time();
  }
}

// Adds a pass to the sums; a logit costs an FMA, an exponential, an addition and (entropy) an FMA.  As a rule m stays, and x = z c - r is one operation,
// with r = m c as rounded; what r is off, d, is known and goes into the sums afterwards.  Where a lane's sum shows that m is too small (or that there is
// a NaN), or where r is so large that d is, too, the pass is gone through again: m becomes the largest logit of the wave's, and x = (z - m) c.
template <bool ENTROPY, bool BF16, int G>
__device__ __forceinline__ void take(WaveSums& a, Pass<BF16, G>& x, bool holes, const LossRow& q) {
  using P = Pass<BF16, G>;
  Sums sum = a.sums;                                 // written back once: stores to it in several branches keep it out of registers
  if (sum.m == -FLT_MAX) {                           // nothing has been summed, or the lowest number alone
    const float top = x.largest(holes);
    if (top > sum.m) move_to(sum, top, q);
  }
  const float r = sum.m * q.c;
  bool near = fabsf(r) < 16777216.0f;                // d is at most 1/2
  if (near) {
    float s = 0.0f, u = 0.0f;
    if (ENTROPY && a.clamp) {
      if (!holes) x.all_count();
      add_near<true, true, ENTROPY, P, G>(x, r, q, s, u);
    } else if (holes) {
      add_near<true, false, ENTROPY, P, G>(x, r, q, s, u);
    } else {
      add_near<false, false, ENTROPY, P, G>(x, r, q, s, u);
    }
    near = !__ballot(!(s <= 64.0f && u == u));
    if (near) {
      const float d = __builtin_fmaf(sum.m, q.c, -r), f = exp2_of(-d);
      s *= f;
      sum.s += s;
      if (ENTROPY) sum.u += u * f - d * s;
    }
  }
  if (!near) {
    if (!holes) x.all_count();
    float low = INFINITY;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e) low = fminf(low, x.raw_logit(g, e));
    a.clamp |= __ballot(low == -INFINITY) != 0;
    const float top = x.largest(holes);
    if (top > sum.m) move_to(sum, top, q);
    float s = 0.0f, u = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e) {
        const float y = in_base_2(x.template logit<true>(g, e), sum.m, q), p = exp2_of(y);
        s += p;
        if (ENTROPY) u = __builtin_fmaf(p, fmaxf(y, -FAR), u);
        if (e + 1 == LANE_TOKENS) one_group_at_a_time();
      }
    sum.s += s;
    if (ENTROPY) sum.u += u;
  }
  a.sums = sum;
}

// How a pass over the logits is laid out.  Rows are stretches of LOSS_TOKENS slots each, and a workgroup takes the next `share` of all rows'
// stretches: so that all workgroups are resident at once and end together (but for fp32 lists, where 1792 fit: even shares for as many took 241 us for
// 4096 x 65537, for 2048 of them 214).  What it sums of row r goes to part r + its own number.  Shares of
// at most 16 stretches, of which there are more than fit at once, cost 14 % more for 2048 x 131073 against a list and 10 % for 1178 masked rows of 65537, but
// 3 % less for 4096 x 131072.
struct LossGrid {
  int stretches, share, workgroups;
};
struct Part {
  int r, from, to;                                   // stretches of row r
  __device__ __forceinline__ Part(const LossGrid& g, int at, int stop) : r(at / g.stretches), from(at - r * g.stretches), to(min(g.stretches, from + stop - at)) {}
};
// The sums of row r: of a wave's lanes, from the parts; false where one workgroup has had it all.
__device__ __forceinline__ bool parts_of(const LossGrid& g, int r, const Sums* parts, const LossRow& q, Sums& sum) {
  const int first = r * g.stretches / g.share, last = ((r + 1) * g.stretches - 1) / g.share;
  sum = no_sums();
  for (int w = first + (int)(threadIdx.x & 63); w <= last; w += WAVE) join(sum, parts[r + w], q);
  sum = wave_sums(sum, q);
  return first < last;
}

// ---------------------------------------------------------------- alternatives
// The n best tokens lie in the n stretches of CHUNK slots whose largest logits come first (equal ones in the order of their tokens): each of
// these has a token that comes before all others of the stretches that come after.  So the pass over the logits leaves the largest logit of each
// stretch, the stretches are chosen from these, and their tokens are looked at again.  Lists that the lanes keep while they sum, and join, took 118 us for
// 1178 rows of 64 alternatives where this takes 19.  Stretches of 32 slots: 3 % more for the pass over 1178 x 131073.
constexpr int CHUNK_LANES = 8, CHUNK = CHUNK_LANES * LANE_TOKENS;

// Its bits in the order of the numbers; -0 and 0 are equal.
__device__ __forceinline__ uint32_t ordered(float z) {
  const int bits = __builtin_bit_cast(int, z + 0.0f);
  return (uint32_t)bits ^ ((uint32_t)(bits >> 31) | 0x80000000u);
}
// A logit and where it comes from in one number, the larger the earlier it comes among alternatives; 0 for -inf.  All others are distinct.
__device__ __forceinline__ uint64_t key_of(float z, int at) {
  if (!(z > -INFINITY)) return 0;
  return (uint64_t)ordered(z) << 32 | (uint32_t)~at;
}
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t bits = (uint32_t)(key >> 32);
  return __builtin_bit_cast(float, bits & 0x80000000u ? bits ^ 0x80000000u : ~bits);
}
__device__ __forceinline__ int place_of(uint64_t key) { return (int)~(uint32_t)key; }

struct TopLds {
  static constexpr int CANDIDATES = 4 * LOSS_THREADS;
  static constexpr int AT_ONCE = 16;                 // the list is compared so many at a time, zeros behind it
  uint64_t lane[LOSS_THREADS], candidate[CANDIDATES + AT_ONCE], best[PG_TOP_MAX], least;
  alignas(sizeof(float4)) float top[LOSS_THREADS / 2];
  uint32_t bound;
  int count;
};
static_assert(offsetof(TopLds, top) % sizeof(float4) == 0 && alignof(TopLds) % sizeof(float4) == 0, "four of `top` are read at once");

// Before and after the collection of candidates; s.best is the n largest of them in falling order (0: there are no more).
__device__ __forceinline__ void no_candidates(TopLds& s) {
  __syncthreads();                                   // what was there has been read
  if (threadIdx.x < PG_TOP_MAX) s.best[threadIdx.x] = 0;
  if (threadIdx.x == 0) {
    s.count = 0;
    s.least = 1;
    s.bound = ~0u;
  }
}
// Of a lane's keys key(0) .. key(N - 1) those whose bits are set, with one request for their places.
template <int N, class Key>
__device__ __forceinline__ void candidates(uint32_t some, TopLds& s, Key key) {
  if (!some) return;
  int at = atomicAdd(&s.count, __popc(some));
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (some >> i & 1) {
      if (at < TopLds::CANDIDATES) s.candidate[at] = key(i);
      ++at;
    }
}
__device__ __forceinline__ bool rank_candidates(int n, TopLds& s) {
  __syncthreads();
  const int m = s.count;
  if (m > TopLds::CANDIDATES) return false;
  if (threadIdx.x < TopLds::AT_ONCE) s.candidate[m + threadIdx.x] = 0;
  __syncthreads();
  for (int k = threadIdx.x; k < m; k += LOSS_THREADS) {
    const uint64_t key = s.candidate[k];
    int rank = 0;
    for (int i = 0; i < m; i += TopLds::AT_ONCE)
#pragma unroll
      for (int j = 0; j < TopLds::AT_ONCE; ++j) rank += s.candidate[i + j] > key;
    if (rank < n) s.best[rank] = key;
  }
  __syncthreads();
  return true;
}

// A bound that n of the lanes' values, at least, reach, and hardly more: the n-th largest among the largest of two or four adjacent lanes each.
__device__ __forceinline__ float nth_of_lanes(float top, int n, TopLds& s) {
  static_assert(PG_TOP_MAX <= LOSS_THREADS / 4, "half of the pairs at most");
  const int each = n <= LOSS_THREADS / 8 ? 4 : 2;
  top = fmaxf(top, __builtin_bit_cast(float, permuted<0xB1>(__builtin_bit_cast(int, top))));
  if (each == 4) top = fmaxf(top, __builtin_bit_cast(float, permuted<0x4E>(__builtin_bit_cast(int, top))));
  if (threadIdx.x % each == 0) s.top[threadIdx.x / each] = top;
  __syncthreads();
  if ((int)threadIdx.x < LOSS_THREADS / each) {
    top = s.top[threadIdx.x];
    int rank = 0;
    for (int i = 0; i < LOSS_THREADS / each / 4; i += 16)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float4 t = ((const float4*)s.top)[i + j];
        rank += (t.x > top) + (t.y > top) + (t.z > top) + (t.w > top);
      }
    if (rank < n) atomicMin(&s.bound, ordered(top));
  }
  __syncthreads();
  return logit_of((uint64_t)s.bound << 32);
}

// The n largest of the keys item(0) .. item(N - 1) where too many reach a bound on their logits alone.  Of the largest keys of the lanes the
// n-th is a bound that takes equal logits apart; where the lanes that have the largest keys have too many of them, n rounds of a maximum.
template <class Item>
__device__ __forceinline__ void select_by_key(int N, int n, TopLds& s, Item item) {
  const int me = threadIdx.x;
  uint64_t most = 0;
  for (int i = me; i < N; i += LOSS_THREADS) most = max(most, item(i));
  no_candidates(s);
  s.lane[me] = most;
  __syncthreads();
  int rank = 0;
  for (int i = 0; i < LOSS_THREADS; ++i) rank += s.lane[i] > most;
  if (most && rank == n - 1) s.least = most;
  __syncthreads();
  const uint64_t least = s.least;
  for (int i = me; i < N; i += LOSS_THREADS) {
    const uint64_t key = item(i);
    candidates<1>(key >= least, s, [&](int) { return key; });
  }
  if (rank_candidates(n, s)) return;
  uint64_t last = ~0ull;
  for (int k = 0; k < n && last; ++k) {
    most = 0;
    for (int i = me; i < N; i += LOSS_THREADS) {
      const uint64_t key = item(i);
      if (key < last) most = max(most, key);
    }
    __syncthreads();
    s.lane[me] = most;
    __syncthreads();
    for (int i = 0; i < LOSS_THREADS; ++i) most = max(most, s.lane[i]);
    if (me == 0) s.best[k] = most;
    last = most;
  }
  __syncthreads();
}

// The first stretches' largest logits of a lane, asked for early.
struct Kept {
  static constexpr int N = 10;                       // 163840 tokens of a row
  float z[N];
  __device__ __forceinline__ void load(const float* largest, int chunks) {
#pragma unroll
    for (int k = 0; k < N; ++k) z[k] = (int)threadIdx.x + k * LOSS_THREADS < chunks ? largest[threadIdx.x + k * LOSS_THREADS] : -INFINITY;
  }
};
__device__ __forceinline__ int chunks_of(const LossArgs& a, const LossRow& q) { return (a.l.d.vocab + q.shift + CHUNK - 1) / CHUNK; }

// The n best tokens of a row, from the largest logits of its stretches, to s.best: all lanes of a workgroup.
template <bool BF16>
__device__ __forceinline__ void alternatives(const LossArgs& a, const LossRow& q, const Kept& kept, const float* largest, int n, TopLds& s) {
  constexpr int KEPT = Kept::N;
  constexpr int AGAIN = PG_TOP_MAX * CHUNK_LANES / LOSS_THREADS;
  const int me = threadIdx.x, vocab = a.l.d.vocab, N = chunks_of(a, q);
  no_candidates(s);
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < KEPT; ++k) top = fmaxf(top, kept.z[k]);
  for (int i = me + KEPT * LOSS_THREADS; i < N; i += LOSS_THREADS) top = fmaxf(top, largest[i]);
  const float bound = nth_of_lanes(top, n, s);
  uint32_t some = 0;
#pragma unroll
  for (int k = 0; k < KEPT; ++k) some |= (uint32_t)(kept.z[k] >= bound && kept.z[k] > -INFINITY) << k;
  candidates<KEPT>(some, s, [&](int k) { return key_of(kept.z[k], me + k * LOSS_THREADS); });
  for (int i = me + KEPT * LOSS_THREADS; i < N; i += LOSS_THREADS)
    candidates<1>(largest[i] >= bound && largest[i] > -INFINITY, s, [&](int) { return key_of(largest[i], i); });
  if (!rank_candidates(n, s)) select_by_key(N, n, s, [&](int i) { return key_of(largest[i], i); });
  // the lanes look at these stretches again, eight tokens each
  const float least = logit_of(s.best[n - 1]);       // NaN for 0: nothing is below it
  const int end = vocab + q.shift;
  int first[AGAIN];                                  // their first tokens
  Pass<BF16, 1> x[AGAIN];
#pragma unroll
  for (int k = 0; k < AGAIN; ++k) {
    const int i = (me + k * LOSS_THREADS) / CHUNK_LANES;
    const uint64_t chunk = i < n ? s.best[i] : 0;
    const int slot = chunk ? place_of(chunk) * CHUNK + me % CHUNK_LANES * LANE_TOKENS : end;
    x[k].load_part(a, q, slot - me * LANE_TOKENS, end);
    first[k] = slot - q.shift;
  }
  auto logit = [&](int e) { return x[e / LANE_TOKENS].template logit<true>(0, e % LANE_TOKENS); };
  auto key = [&](int e) { return key_of(logit(e), first[e / LANE_TOKENS] + e % LANE_TOKENS); };
  no_candidates(s);
  __syncthreads();
  some = 0;
#pragma unroll
  for (int e = 0; e < AGAIN * LANE_TOKENS; ++e) some |= (uint32_t)(!(logit(e) < least) && logit(e) > -INFINITY) << e;
  candidates<AGAIN * LANE_TOKENS>(some, s, key);
  if (rank_candidates(n, s)) return;
  uint64_t all[AGAIN * LANE_TOKENS];
#pragma unroll
  for (int e = 0; e < AGAIN * LANE_TOKENS; ++e) all[e] = some >> e & 1 ? key(e) : 0;
  select_by_key(LOSS_THREADS * LANE_TOKENS * AGAIN, n, s, [&](int i) { return all[i / LOSS_THREADS]; });
}

struct LogprobOut {
  const int32_t* target;
  float *logp, *entropy, *stats;
  int n_top;
  int32_t* top_ids;
  float* top_logp;
  Sums* parts;                                       // [rows + workgroups]
  float* chunks;                                     // [rows, n_chunks]: the largest logit of each
  int n_chunks;
};

// What the whole row's sums give; all lanes of a workgroup, or (s NULL: no alternatives) of a wave.
template <bool BF16>
__device__ __forceinline__ void finish_logprob(const LossArgs& a, const LogprobOut& o, const LossRow& q, int r, int target, float at_target, const Sums& sum,
                                               const Kept& kept, TopLds* s) {
  const bool gone = target == -1, bad = !gone && sum.s != sum.s, none = gone || sum.s == 0.0f;     // a temperature that is none makes even empty sums NaN
  const float ln_s = none ? 0.0f : logf(sum.s);
  if (threadIdx.x == 0) {
    // a sum of one token's weight may be rounded to just below 1
    const float sure = none ? 0.0f : ln_s - LN2 * (sum.u / sum.s), h = sure < 0.0f ? 0.0f : sure;
    if (o.entropy) o.entropy[r] = h;
    if (o.logp) {
      float l = __builtin_nanf("");
      if (gone) l = 0.0f;
      else if (target >= 0 && target < a.l.d.vocab && !bad) l = none ? -INFINITY : fminf(over_t(at_target, sum.m, q) - ln_s, 0.0f);
      o.logp[r] = l;
    }
    if (o.stats) *(float4*)(o.stats + 4ll * r) = float4{none ? -INFINITY : sum.m / q.t, ln_s, h, sum.m};
  }
  if (!s) return;
  const int n = o.n_top;
  uint64_t key = 0;
  if (!gone && !bad && !none) {
    alternatives<BF16>(a, q, kept, o.chunks + (int64_t)r * o.n_chunks, n, *s);
    key = (int)threadIdx.x < n ? s->best[threadIdx.x] : 0;
  }
  if ((int)threadIdx.x < n) {
    if (o.top_ids) o.top_ids[(int64_t)r * n + threadIdx.x] = key ? place_of(key) : -1;
    if (o.top_logp) o.top_logp[(int64_t)r * n + threadIdx.x] = bad ? __builtin_nanf("") : key ? fminf(over_t(logit_of(key), sum.m, q) - ln_s, 0.0f) : -INFINITY;
  }
}

// Bound by reading: 1178 rows of 131073 in bf16 (309 MB) take 54 us, 5.8 TB/s, and 70 with the largest of each stretch (6 of the 16 for its stores, past
// the caches 3 more); 4096 x 65537 (537 MB) 94 us, 5.7 TB/s, and 4096 x 131072 (1074 MB) 169 us, 6.4 TB/s; in fp32 4096 x 65536 (1074 MB) 187 us, 5.7 TB/s.  Without
// any arithmetic a copy of the pass was 3 to 5 % shorter.  Loads of the next pass asked for before this one is summed cost registers and gave
// nothing (3 to 7 % more).  WHOLE: every workgroup has one row, and no launch comes after this one: 48 masked rows of 16384 with five alternatives in 12.4 us.
template <bool BF16, int G, bool TOP, bool WHOLE>
__global__ __launch_bounds__(LOSS_THREADS, WHOLE ? 2 : TOP ? 6 : 8) void logprob_kernel(LossArgs a, LossGrid grid, LogprobOut o) {
  __shared__ Sums waves[LOSS_WAVES];
  __shared__ std::conditional_t<WHOLE && TOP, TopLds, char> lists;
  const int stop = min((int)(blockIdx.x + 1) * grid.share, a.l.d.rows * grid.stretches), lane = threadIdx.x & 63;
  for (int at = blockIdx.x * grid.share; at < stop;) {
    const Part part(grid, at, stop);
    const int r = part.r;
    const LossRow q = loss_row<BF16>(a, r);
    const int target = o.target ? o.target[r] : 0;
    WaveSums mine;
    if (target != -1) {
      float* chunks = o.chunks + (int64_t)r * o.n_chunks;
      const int end = min(part.to * LOSS_TOKENS, a.l.d.vocab + q.shift);
      auto leave = [&](int base, int g, float top) { // a pass may reach past the part's end
        const int c = base / CHUNK + g * (LOSS_TOKENS / CHUNK) + (int)threadIdx.x / CHUNK_LANES;
        if (lane % CHUNK_LANES == g && c * CHUNK < end) chunks[c] = top;
      };
      through<BF16, G, false>(a, q, part.from * LOSS_TOKENS, end, no_strike, [&](Pass<BF16, G>& x, int base, bool holes) {
        if (TOP) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float top = holes ? x.template largest<true>(g) : x.template largest<false>(g);
            top = fmaxf(top, __builtin_bit_cast(float, permuted<0xB1>(__builtin_bit_cast(int, top))));
            top = fmaxf(top, __builtin_bit_cast(float, permuted<0x4E>(__builtin_bit_cast(int, top))));
            top = fmaxf(top, __builtin_bit_cast(float, permuted<0x141>(__builtin_bit_cast(int, top))));
            leave(base, g, top);
          }
        }
        take<true>(mine, x, holes, q);
      }, [&](int base) {
        if (TOP)
          for (int g = 0; g < G; ++g) leave(base, g, -INFINITY);
      });
    }
    const Sums sum = block_sums(mine.sums, q, waves);
    if (WHOLE || (!TOP && part.from == 0 && part.to == grid.stretches)) {
      const float at_target = target >= 0 && target < a.l.d.vocab ? open_logit<BF16>(a, q, target) : 0.0f;
      Kept kept;
      if constexpr (WHOLE && TOP) {
        kept.load(o.chunks + (int64_t)r * o.n_chunks, chunks_of(a, q));
        finish_logprob<BF16>(a, o, q, r, target, at_target, sum, kept, &lists);
      } else {
        finish_logprob<BF16>(a, o, q, r, target, at_target, sum, kept, nullptr);
      }
    } else if (threadIdx.x == 0) {
      o.parts[r + blockIdx.x] = sum;
    }
    if (WHOLE) return;
    at += part.to - part.from;
    if (at < stop) __syncthreads();                  // the waves' sums have been read
  }
}

template <bool BF16, bool TOP>
__global__ __launch_bounds__(LOSS_THREADS) void logprob_finish_kernel(LossArgs a, LossGrid grid, LogprobOut o) {
  __shared__ TopLds lists;
  const int r = blockIdx.x;
  const LossRow q = loss_row<BF16>(a, r);
  const int target = o.target ? o.target[r] : 0;
  const float at_target = target >= 0 && target < a.l.d.vocab ? open_logit<BF16>(a, q, target) : 0.0f;
  Kept kept;
  if (TOP && target != -1) kept.load(o.chunks + (int64_t)r * o.n_chunks, chunks_of(a, q));
  Sums sum;
  if (parts_of(grid, r, o.parts, q, sum) || TOP) finish_logprob<BF16>(a, o, q, r, target, at_target, sum, kept, TOP ? &lists : nullptr);
}

// Writes the gradient of the tokens v .. v + 7 that are in the row, but for those of `others`, in the logits' type.  PAST: not to be kept in the
// caches.
template <bool BF16, bool PAST>
__device__ __forceinline__ void put(char* row, int v, int vocab, const float* d, uint32_t others = 0) {
  char* to = row + (int64_t)v * (BF16 ? 2 : 4);
  if (v >= 0 && v + LANE_TOKENS <= vocab && !others) {
    if (BF16) {
      const uint32_t w[4] = {pack_bf16x2(d[0], d[1]), pack_bf16x2(d[2], d[3]), pack_bf16x2(d[4], d[5]), pack_bf16x2(d[6], d[7])};
      typedef uint32_t Unaligned __attribute__((ext_vector_type(4), aligned(2)));
      const Unaligned x{w[0], w[1], w[2], w[3]};
      if (PAST) __builtin_nontemporal_store(x, (Unaligned*)to);
      else *(Unaligned*)to = x;
    } else {
      __builtin_memcpy(to, d, 32);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < LANE_TOKENS; ++e)
    if (v + e >= 0 && v + e < vocab && !(others >> e & 1)) {
      if (BF16) ((uint16_t*)to)[e] = (uint16_t)pack_bf16x2(d[e], 0.0f);
      else ((float*)to)[e] = d[e];
    }
}
template <bool BF16, bool PAST, int G>
__device__ __forceinline__ void put_zeros(char* row, int v, int vocab) {
  const float nothing[LANE_TOKENS] = {};
#pragma unroll
  for (int i = 0; i < G; ++i) put<BF16, PAST>(row, v + i * LOSS_TOKENS, vocab, nothing);
}

// The gradient is p (c0 + c1 log2 p) with two numbers of the row, and g / T more at the target; where such a number, or the bound on z - m, passes fp32's
// range, at temperatures near an end of it, a token's is worked out before it is divided by T.  Bound by reading the logits again and writing as much:
// 4096 x 131072 in bf16 in 361 us, 5.9 TB/s both ways.
template <bool BF16, int G, bool PAST>
__global__ __launch_bounds__(LOSS_THREADS) void logprob_backward_kernel(LossArgs a, int pieces, const int32_t* target, const float* stats,
                                                                        const float* g_logp, const float* g_entropy, void* out, int64_t out_stride) {
  constexpr int ELT = BF16 ? 2 : 4;
  const int block = gridDim.x - 1 - blockIdx.x, r = block / pieces, piece = block - r * pieces;
  const int vocab = a.l.d.vocab, first = piece * (G * LOSS_TOKENS);
  const LossRow q = loss_row<BF16>(a, r);
  const int t = target ? target[r] : 0;
  float g = g_logp ? g_logp[r] : 0.0f;
  const float ge = g_entropy ? g_entropy[r] : 0.0f;
  char* to = (char*)out + (int64_t)r * out_stride * ELT;
  auto clear = [&](int base) { put_zeros<BF16, PAST, G>(to, base + (int)threadIdx.x * LANE_TOKENS - q.shift, vocab); };
  if (t == -1 || (g == 0.0f && ge == 0.0f)) return clear(first);
  if (g_logp && (t < 0 || t >= vocab)) g = __builtin_nanf("");
  const float4 s = *(const float4*)(stats + 4ll * r);
  const float ln_s = s.y, h = s.z, m = s.w;
  const float c0 = q.inv * (-g - ge * h), c1 = q.inv * ge * -LN2, at_target = q.inv * g, less = ln_s * LOG2E;
  // 0 times what is no number is no 0; log2 p is cut at -FAR - less; below FLT_MIN T has no inverse
  const bool odd = !(fabsf(c0) + 512.0f * fabsf(c1) + fabsf(at_target) < INFINITY && less == less && q.t >= FLT_MIN && q.lim > -INFINITY);
  auto plain = [&](float z, bool here) {             // where that is so
    if (z == -INFINITY) return 0.0f;
    const float ln_p = fmaxf(over_t(z, m, q), -FAR * LN2) - ln_s;
    return (expf(ln_p) * (-g - ge * (ln_p + h)) + (here ? g : 0.0f)) / q.t;
  };
  auto each = [&](const Pass<BF16, G>& x, int base, auto all) {
    constexpr bool HOLES = !decltype(all)::value;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int v = base + i * LOSS_TOKENS + (int)threadIdx.x * LANE_TOKENS - q.shift;
      float d[LANE_TOKENS];
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e) {
        const float z = x.template logit<HOLES>(i, e), y = __builtin_fmaf(fmaxf(z - m, q.lim), q.c, -less);
        d[e] = exp2_of(y) * __builtin_fmaf(c1, y, c0);
        if (HOLES && z == -INFINITY) d[e] = 0.0f;
      }
      const int at = t - v;
      if (at >= 0 && at < LANE_TOKENS) {
#pragma unroll
        for (int e = 0; e < LANE_TOKENS; ++e)
          if (e == at && x.template logit<HOLES>(i, e) != -INFINITY) d[e] += at_target;
      }
      put<BF16, PAST>(to, v, vocab, d);
    }
  };
  auto each_plain = [&](const Pass<BF16, G>& x, int base) {
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int v = base + i * LOSS_TOKENS + (int)threadIdx.x * LANE_TOKENS - q.shift;
      float d[LANE_TOKENS];
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e) {
        d[e] = plain(x.template logit<true>(i, e), v + e == t);
        one_group_at_a_time();
      }
      put<BF16, PAST>(to, v, vocab, d);
    }
  };
  through<BF16, G, false>(a, q, first, min(first + G * LOSS_TOKENS, vocab + q.shift), no_strike, [&](Pass<BF16, G>& x, int base, bool holes) {
    if (odd) {
      if (!holes) x.all_count();
      each_plain(x, base);
    } else if (holes) {
      each(x, base, std::false_type{});
    } else {
      each(x, base, std::true_type{});
    }
  }, clear);
}

// ---------------------------------------------------------------- distillation

constexpr int LIST_LANES = PG_DISTILL_MAX / WAVE;     // entries of a wave's lane
constexpr int LIST_SLOTS = 4 * PG_DISTILL_MAX;       // a quarter full at most
static_assert(LIST_SLOTS == 1 << 10 && PG_DISTILL_MAX == LOSS_THREADS, "ten bits of a hash, an entry a lane");
constexpr int LIST_RANGE = 1 << 17;                  // slots whose bits LDS holds at a time

// Which entries of a row's list count: the first of each token that exists.  A table of tokens in LDS with the first entry that has each.
struct ListLds {
  int token[LIST_SLOTS], first[LIST_SLOTS];
};
__device__ __forceinline__ uint32_t entries_that_count(const int* id, int k, int vocab, ListLds& s) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < LIST_SLOTS / WAVE; ++i) {
    s.token[i * WAVE + lane] = -1;
    s.first[i * WAVE + lane] = INT32_MAX;
  }
  wave_lds_sync();
  int slot[LIST_LANES];
#pragma unroll
  for (int i = 0; i < LIST_LANES; ++i) {
    slot[i] = -1;
    const int at = i * WAVE + lane;
    if (at < k && id[i] >= 0 && id[i] < vocab) {
      int h = (int)((uint32_t)id[i] * 2654435761u >> 22);
      for (int tries = 0; tries < LIST_SLOTS; ++tries, h = (h + 1) & (LIST_SLOTS - 1)) {
        const int old = atomicCAS(&s.token[h], -1, id[i]);
        if (old == -1 || old == id[i]) break;
      }
      slot[i] = h;
      atomicMin(&s.first[h], at);
    }
  }
  wave_lds_sync();
  uint32_t count = 0;
#pragma unroll
  for (int i = 0; i < LIST_LANES; ++i)
    if (slot[i] >= 0 && s.first[slot[i]] == i * WAVE + lane) count |= 1u << i;
  return count;
}

__device__ __forceinline__ double lanes_sum(double v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

struct DistillArgs {
  int mode, k;
  const int32_t* ids;
  const float* logp;
  float *loss, *stats;
  Sums* parts;                                       // [rows + workgroups]
};

// From the sums over what is not listed to the loss: the lanes of one wave.  In fp64: it is a few hundred values, and what
// is left over (1 - sum q, Q p_rest - q_rest) is a difference.  2048 lists take 12 us, bound by the way from one step to the next.
template <bool BF16>
__device__ __forceinline__ void finish_distill(const LossArgs& a, const DistillArgs& o, const LossRow& q, int r, const Sums& rest, ListLds& s) {
  const int lane = threadIdx.x & 63, vocab = a.l.d.vocab;
  int id[LIST_LANES];
  float t[LIST_LANES], z[LIST_LANES];
#pragma unroll
  for (int i = 0; i < LIST_LANES; ++i) {
    const int at = i * WAVE + lane;
    id[i] = at < o.k ? o.ids[(int64_t)r * o.k + at] : -1;
    t[i] = at < o.k ? o.logp[(int64_t)r * o.k + at] : -INFINITY;
    z[i] = id[i] >= 0 && id[i] < vocab ? open_logit<BF16>(a, q, id[i]) : -INFINITY;
  }
  const uint32_t count = entries_that_count(id, o.k, vocab, s);
  float m = rest.m, most = -INFINITY;
  bool wrong = false;
#pragma unroll
  for (int i = 0; i < LIST_LANES; ++i)
    if (count >> i & 1) {
      m = fmaxf(m, z[i]);
      most = fmaxf(most, t[i]);
      wrong |= !(t[i] < INFINITY);
    }
  m = wave_max(m);
  most = wave_max(most);
  wrong = __ballot(wrong);
  const bool top = o.mode == PG_DISTILL_TOP;
  double s_all = 0.0, sum_q = 0.0;
  const double inv = 1.0 / (double)q.t;
#pragma unroll
  for (int i = 0; i < LIST_LANES; ++i)
    if (count >> i & 1) {
      s_all += exp(((double)z[i] - m) * inv);
      sum_q += exp(top ? (double)t[i] - most : (double)t[i]);
    }
  const bool others = rest.s != 0.0f;
  s_all = lanes_sum(s_all) + (others ? rest.s * exp(((double)rest.m - m) * inv) : 0.0);
  sum_q = lanes_sum(sum_q);
  const bool active = __ballot(count != 0) && s_all != 0.0 && !(top && most == -INFINITY && !wrong);
  const double bad = wrong || s_all != s_all ? __builtin_nan("") : 0.0;      // also where no entry has a weight
  const double ln_q = top ? log(sum_q) : 0.0;
  double total = 0.0, q_rest = 0.0, p_rest = 0.0, all = 0.0;
  if (active) {
    const double ln_s = log(s_all), ln_rest = ((double)rest.m - m) * inv + log((double)rest.s) - ln_s;
    const double t0 = top ? most + ln_q : 0.0;
    if (others) p_rest = exp(ln_rest);
    if (!top && others) q_rest = fmax(0.0, 1.0 - sum_q);
#pragma unroll
    for (int i = 0; i < LIST_LANES; ++i)
      if (count >> i & 1) {
        const double lq = t[i] - t0, w = exp(lq);
        if (w > 0.0) total += w * (lq - (((double)z[i] - m) * inv - ln_s));
        all += w;
      }
    total = lanes_sum(total) + bad;
    all = lanes_sum(all) + q_rest + bad;
    if (q_rest > 0.0) total += q_rest * (log(q_rest) - ln_rest);
  }
  if (lane) return;
  o.loss[r] = (float)total;
  if (o.stats) {
    float4* x = (float4*)(o.stats + (int64_t)r * PG_DISTILL_STATS);
    x[0] = float4{m, (float)log(s_all), rest.m, others ? logf(rest.s) : 0.0f};
    // the teacher's largest value and the logarithm of their sum, apart: values shifted by 10^4 would lose 2^-11 of q to t0 as one number
    x[1] = float4{(float)(all * p_rest - q_rest), top ? most : 0.0f, active ? (float)all : -1.0f, (float)ln_q};
  }
}

// The sums over what is not listed, with a bit in LDS for each slot; bound by reading: 2048 x 131073 in bf16 (537 MB) in 93 us,
// 5.8 TB/s.  In fp32 seven waves a SIMD, for which registers suffice: 4096 x 65537 in 214 us, 5.0 TB/s, 243 with eight.
template <bool BF16, int G, bool WHOLE>
__global__ __launch_bounds__(LOSS_THREADS, WHOLE ? 2 : BF16 ? 8 : 7) void distill_kernel(LossArgs a, LossGrid grid, DistillArgs o) {
  __shared__ Sums waves[LOSS_WAVES];
  extern __shared__ uint32_t listed[];               // a bit for each slot of the row's part; WHOLE: then the table of the list
  const int stop = min((int)(blockIdx.x + 1) * grid.share, a.l.d.rows * grid.stretches);
  for (int at = blockIdx.x * grid.share; at < stop;) {
    const Part part(grid, at, stop);
    const int r = part.r;
    const int id = (int)threadIdx.x < o.k ? o.ids[(int64_t)r * o.k + threadIdx.x] : -1;
    const LossRow q = loss_row<BF16>(a, r);
    WaveSums mine;
    for (int from = part.from; from < part.to; from += LIST_RANGE / LOSS_TOKENS) {
      const int to = min(part.to, from + LIST_RANGE / LOSS_TOKENS);
      const int first = from * LOSS_TOKENS, end = min(to * LOSS_TOKENS, a.l.d.vocab + q.shift);
      for (int i = threadIdx.x; i < (to - from) * (LOSS_TOKENS / 32); i += LOSS_THREADS) listed[i] = 0;
      __syncthreads();
      const bool exists = id >= 0 && id < a.l.d.vocab;
      const int place = exists ? id + q.shift - first : -1;
      if (place >= 0 && place < end - first) atomicOr(&listed[place >> 5], 1u << (place & 31));
      __syncthreads();
      auto strike = [&](int t) { return t < end ? (uint32_t)((const uint8_t*)listed)[(t - first) >> 3] : 0u; };
      through<BF16, G, true>(a, q, first, end, strike, [&](Pass<BF16, G>& x, int, bool holes) { take<false>(mine, x, holes, q); }, [](int) {});
      __syncthreads();                               // the bits have been read
    }
    const Sums rest = block_sums(mine.sums, q, waves);
    if (WHOLE) {
      if (threadIdx.x < WAVE) finish_distill<BF16>(a, o, q, r, rest, *(ListLds*)listed);
      return;
    }
    if (threadIdx.x == 0) o.parts[r + blockIdx.x] = rest;
    at += part.to - part.from;
    if (at < stop) __syncthreads();                  // the waves' sums have been read
  }
}

template <bool BF16>
__global__ __launch_bounds__(WAVE) void distill_finish_kernel(LossArgs a, LossGrid grid, DistillArgs o) {
  __shared__ ListLds list;
  const int r = blockIdx.x;
  const LossRow q = loss_row<BF16>(a, r);
  Sums rest;
  parts_of(grid, r, o.parts, q, rest);
  finish_distill<BF16>(a, o, q, r, rest, list);
}

// What is not listed has the gradient g / T (Q p_rest - q_rest) of its share of p_rest; a listed token is written by the lane that holds its
// entry, and by no other.  Bound by reading and writing: 2048 x 131073 in bf16 in 188 us, 5.7 TB/s both ways, in fp32 4096 x 65537 in 456 us, 4.7 TB/s; in bf16 193 with the first rows
// first, of which less is still near from the pass before (log-probs': no difference).
template <bool BF16, int G, bool PAST>
__global__ __launch_bounds__(LOSS_THREADS) void distill_backward_kernel(LossArgs a, int pieces, DistillArgs o, const float* g_loss, void* out,
                                                                        int64_t out_stride) {
  constexpr int ELT = BF16 ? 2 : 4, RANGE = G * LOSS_TOKENS;
  __shared__ uint32_t listed[RANGE / 32];
  __shared__ int token[PG_DISTILL_MAX];
  __shared__ int twice;
  const int block = gridDim.x - 1 - blockIdx.x, r = block / pieces, piece = block - r * pieces;
  const LossRow q = loss_row<BF16>(a, r);
  const int vocab = a.l.d.vocab, first = piece * RANGE, end = min(first + RANGE, vocab + q.shift);
  const float4 s0 = ((const float4*)(o.stats + (int64_t)r * PG_DISTILL_STATS))[0], s1 = ((const float4*)(o.stats + (int64_t)r * PG_DISTILL_STATS))[1];
  const float g = s1.z < 0.0f ? 0.0f : g_loss[r];     // -1 for a row that nothing is learnt from
  char* to = (char*)out + (int64_t)r * out_stride * ELT;
  if (g == 0.0f) return put_zeros<BF16, PAST, G>(to, first + (int)threadIdx.x * LANE_TOKENS - q.shift, vocab);
  const bool entry = (int)threadIdx.x < o.k;
  const int id = entry ? o.ids[(int64_t)r * o.k + threadIdx.x] : -1;
  const float t = entry ? o.logp[(int64_t)r * o.k + threadIdx.x] : 0.0f;
  const int place = id >= 0 && id < vocab ? id + q.shift - first : -1;
  const bool mine = place >= 0 && place < end - first;
  if (threadIdx.x < RANGE / 32) listed[threadIdx.x] = 0;
  if (threadIdx.x == 0) twice = 0;
  token[threadIdx.x] = id;
  __syncthreads();
  if (mine) {
    const uint32_t bit = 1u << (place & 31);
    if (atomicOr(&listed[place >> 5], bit) & bit) twice = 1;
  }
  __syncthreads();
  bool writes = mine;
  if (twice && mine)
    for (int i = 0; i < (int)threadIdx.x; ++i) writes &= token[i] != id;       // the first of equal ids counts
  if (writes) {
    const float z = open_logit<BF16>(a, q, id);
    const float p = expf(fmaxf(over_t(z, s0.x, q), -FAR * LN2) - s0.y);
    const float d = z == -INFINITY ? 0.0f : g * (s1.z * p - expf((t - s1.y) - s1.w)) / q.t;
    if (BF16) ((uint16_t*)to)[id] = (uint16_t)pack_bf16x2(d, 0.0f);
    else ((float*)to)[id] = d;
  }
  const float c = g * q.inv * s1.x, less = s0.w * LOG2E;
  auto strike = [&](int t) { return t < end ? (uint32_t)((const uint8_t*)listed)[(t - first) >> 3] : 0u; };
  // as in the log-probs' gradient
  const bool odd = !(fabsf(c) < INFINITY && less == less && q.t >= FLT_MIN && q.lim > -INFINITY);
  auto plain = [&](float z) { return z == -INFINITY ? 0.0f : g * (s1.x * expf(fmaxf(over_t(z, s0.z, q), -FAR * LN2) - s0.w)) / q.t; };
  auto each = [&](const Pass<BF16, G>& x, int base, auto all, auto by_hand) {
    constexpr bool HOLES = !decltype(all)::value, PLAIN = decltype(by_hand)::value;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int v = base + i * LOSS_TOKENS + (int)threadIdx.x * LANE_TOKENS - q.shift;
      float d[LANE_TOKENS];
#pragma unroll
      for (int e = 0; e < LANE_TOKENS; ++e) {
        const float z = x.template logit<HOLES>(i, e);
        if (PLAIN) {
          d[e] = plain(z);
          one_group_at_a_time();
          continue;
        }
        d[e] = c * exp2_of(__builtin_fmaf(fmaxf(z - s0.z, q.lim), q.c, -less));
        if (HOLES && z == -INFINITY) d[e] = 0.0f;
      }
      put<BF16, PAST>(to, v, vocab, d, HOLES ? strike(v + q.shift) : 0u);
    }
  };
  // a pass without a token that counts may have listed ones among those that are not allowed
  through<BF16, G, true>(a, q, first, end, strike, [&](const Pass<BF16, G>& x, int base, bool holes) {
    if (odd) each(x, base, std::false_type{}, std::true_type{});
    else if (holes) each(x, base, std::false_type{}, std::false_type{});
    else each(x, base, std::true_type{}, std::false_type{});
  }, [&](int base) {
    Pass<BF16, G> nothing{};
    each(nothing, base, std::false_type{}, std::false_type{});
  });
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
  int pieces, piece;                                 // workgroups of a sequence, tokens of each but the last
  float* parts;                                      // [sequences, pieces, 4]
};

// What a sequence's sums give: the objective is weighted, the divergence a mean already.
__device__ __forceinline__ void finish_surrogate(const SurrogateArgs& a, int r, float objective, float kl, int cuts) {
  if (a.objective) a.objective[r] = objective;
  if (a.kl) a.kl[r] = kl;
  if (a.clipped) a.clipped[r] = cuts;
}

// Tokens for which fp32 is enough: exponentials and what they are multiplied with are of at most e^NEAR and LARGE, so that no product and no sum of a
// lane's passes 10^38.  All others, and all where a factor is larger or no number, go through fp64 until they are scaled.  Decided for all tokens that a lane
// has at once; with it 384 sequences of 16384 tokens at most take 16.1 us a call, 15.9 without.
constexpr float NEAR = 40.0f, LARGE = 1e12f;
__device__ __forceinline__ bool is_near(float l, float old, float ref, bool has_ref) {
  return fabsf(l - old) < NEAR && (!has_ref || fabsf(ref - l) < NEAR);
}

// e^x - x - 1 near 0: x^2 (1/2! + x (1/3! + x (...))), whose terms past the ninth are 2^-26 of it at x = 1/2
__device__ __forceinline__ float near_exp(float x) {
  float k = 1.0f / 3628800;
  k = __builtin_fmaf(k, x, 1.0f / 362880);
  k = __builtin_fmaf(k, x, 1.0f / 40320);
  k = __builtin_fmaf(k, x, 1.0f / 5040);
  k = __builtin_fmaf(k, x, 1.0f / 720);
  k = __builtin_fmaf(k, x, 1.0f / 120);
  k = __builtin_fmaf(k, x, 1.0f / 24);
  k = __builtin_fmaf(k, x, 1.0f / 6);
  k = __builtin_fmaf(k, x, 0.5f);
  return k * (x * x);
}
// e^x with fp32's digits and fp64's range: 2^n e^(x - n ln 2).  (The library's exp and expm1 take 96 registers: five waves a SIMD for eight.)
__device__ __forceinline__ double wide_exp(double x) {
  if (!(fabs(x) < 2000.0)) return x > 0.0 ? (double)INFINITY : x < 0.0 ? 0.0 : x;
  const double n = rint(x * 1.4426950408889634);
  return ldexp((double)expf((float)fma(n, -0.6931471805599453, x)), (int)n);
}

// One token's part of the objective, of the divergence and of the gradient; whether it was cut.
struct Token {
  float value, k, g;
  bool cut;
  __device__ __forceinline__ Token(const SurrogateArgs& a, float A, float l, float old, float ref) {
    const double d = (double)l - (double)old;
    cut = A > 0.0f ? d > a.hi : A < 0.0f && d < a.lo;
    const float ra = expf((float)d) * A;
    g = cut ? 0.0f : ra;
    value = cut ? (A > 0.0f ? a.at_hi : a.at_lo) * A : ra;
    k = 0.0f;
    if (a.ref) {
      const float x = ref - l;
      k = near_exp(x);
      float slope = k + x;
      if (!(fabsf(x) < 0.5f)) {
        const float e = expf(x);
        k = e - x - 1.0f;
        slope = e - 1.0f;
      }
      value -= a.kl_coef * k;
      g += a.kl_coef * slope;
    }
  }
};
struct FarToken {
  double value, k, g;
  bool cut;
  __device__ FarToken(const SurrogateArgs& a, float A, float l, float old, float ref) {
    const double d = (double)l - (double)old, ra = A == 0.0f ? 0.0 : wide_exp(d) * A;
    cut = A > 0.0f ? d > a.hi : A < 0.0f && d < a.lo;
    g = cut ? 0.0 : ra;
    value = cut ? (double)(A > 0.0f ? a.at_hi : a.at_lo) * A : ra;
    k = 0.0;
    if (a.ref) {
      const double x = (double)ref - (double)l;
      double e;
      if (fabs(x) < 0.5) {
        k = near_exp((float)x);
        e = k + x;
      } else {
        e = wide_exp(x) - 1.0;
        k = e == INFINITY ? e : e - x;
      }
      if (a.kl_coef != 0.0f) {                       // else the reference reaches the divergence alone
        value -= a.kl_coef * k;
        g += a.kl_coef * e;
      }
    }
  }
};

// Four numbers of a token, read or written once, and some 110 instructions bound it: 384 sequences of 16384 tokens at most, 3.1 million in all (50 MB), in
// 15.1 us (9 us of issue) and 4 for the second launch; 48 short sequences in 4.5 us.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void surrogate_tokens_kernel(SurrogateArgs a) {
  constexpr int AT_ONCE = 4;                         // tokens of a lane whose loads are under way together
  __shared__ double sums[THREADS / WAVE][2];
  __shared__ int counts[THREADS / WAVE];
  const int r = blockIdx.x / a.pieces, piece = blockIdx.x - r * a.pieces;
  const float A = a.adv[r], weight = a.weight ? a.weight[r] : 0.0f;
  const int from = min(max(a.cu[r], 0), a.n_tokens), to = min(max(a.cu[r + 1], from), a.n_tokens), n = to - from;
  const float w = a.weight ? weight : 1.0f / (float)max(n, 1);
  const int64_t first = from + (int64_t)piece * a.piece, end = piece + 1 < a.pieces ? min(first + a.piece, (int64_t)to) : to;
  if (a.pieces > 1 && first >= end) return;           // its part is not looked at
  const bool ordinary = fabsf(A) < LARGE && fabsf(a.kl_coef) < LARGE;
  float sum = 0.0f, kl = 0.0f;
  double far_sum = 0.0, far_kl = 0.0;
  int cuts = 0;
  for (int64_t i = first + threadIdx.x; i < end; i += AT_ONCE * THREADS) {
    float l[AT_ONCE], old[AT_ONCE], ref[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int64_t at = i + j * THREADS < end ? i + j * THREADS : i;       // past the end the lane's own, which no other lane writes
      l[j] = a.logp[at];
      old[j] = a.old[at];
      ref[j] = a.ref ? a.ref[at] : 0.0f;
    }
    bool near = ordinary;
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) near &= is_near(l[j], old[j], ref[j], a.ref);
    if (near) {
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
        if (i + j * THREADS < end) {
          const Token t(a, A, l[j], old[j], ref[j]);
          sum += t.value;
          kl += t.k;
          cuts += t.cut;
          if (a.g_logp) a.g_logp[i + j * THREADS] = w * t.g;
        }
    } else {                                         // read again: nothing has been written there, also where g_logp is one of the inputs
#pragma unroll 1
      for (int64_t at = i; at < min(i + AT_ONCE * THREADS, end); at += THREADS) {
        const FarToken t(a, A, a.logp[at], a.old[at], a.ref ? a.ref[at] : 0.0f);
        far_sum += t.value;
        far_kl += t.k;
        cuts += t.cut;
        if (a.g_logp) a.g_logp[at] = (float)(w * t.g);
      }
    }
  }
  sum = wave_allsum(sum);
  kl = wave_allsum(kl);
  for (int o = 32; o; o >>= 1) cuts += __shfl_xor(cuts, o);
  const bool some = __ballot(far_sum != 0.0 || far_kl != 0.0);
  if (some) {
    far_sum = lanes_sum(far_sum);
    far_kl = lanes_sum(far_kl);
  }
  if ((threadIdx.x & 63) == 0) {
    sums[threadIdx.x >> 6][0] = sum + far_sum;
    sums[threadIdx.x >> 6][1] = kl + far_kl;
    counts[threadIdx.x >> 6] = cuts;
  }
  __syncthreads();
  if (threadIdx.x) return;
  double all = 0.0, all_kl = 0.0;
  cuts = 0;
#pragma unroll
  for (int i = 0; i < THREADS / WAVE; ++i) {
    all += sums[i][0];
    all_kl += sums[i][1];
    cuts += counts[i];
  }
  const float objective = n ? (float)(w * all) : 0.0f, mean = (float)(all_kl / max(n, 1));
  if (a.pieces == 1) finish_surrogate(a, r, objective, mean, cuts);
  else *(float4*)(a.parts + 4ll * blockIdx.x) = float4{objective, mean, __builtin_bit_cast(float, cuts), 0.0f};
}

__global__ __launch_bounds__(WAVE) void surrogate_finish_kernel(SurrogateArgs a) {
  const int r = blockIdx.x;
  const int from = min(max(a.cu[r], 0), a.n_tokens), n = min(max(a.cu[r + 1], from), a.n_tokens) - from;
  double sum = 0.0, kl = 0.0;
  int cuts = 0;
  const int some = (int)min((int64_t)a.pieces, ((int64_t)n + a.piece - 1) / a.piece);
  for (int i = threadIdx.x; i < some; i += WAVE) {
    const float4 p = *(const float4*)(a.parts + 4 * ((int64_t)r * a.pieces + i));
    sum += p.x;
    kl += p.y;
    cuts += __builtin_bit_cast(int, p.z);
  }
  sum = lanes_sum(sum);
  kl = lanes_sum(kl);
  for (int o = 32; o; o >>= 1) cuts += __shfl_xor(cuts, o);
  if (threadIdx.x == 0) finish_surrogate(a, r, (float)sum, (float)kl, cuts);
}

// ---------------------------------------------------------------- host side

static pg_status loss_args(const pg_logits* desc, const float* temperature, const char* who, LossArgs& a) {
  PG_TRY(logit_args(desc, who, a.l, 1 << 23));
  if (desc->tokens || desc->bias_offsets) return fail(PG_EINVAL, "%s: logits with a history or biases (pg_logits_adjust first)", who);
  a.temperature = temperature;
  a.span = desc->rows ? (desc->rows - 1) * desc->stride + desc->vocab : 0;
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

// The most slots that a row of this call has, and that one of any call with so many tokens has.
static int64_t slots_of(const LossArgs& a) {
  const pg_logits& d = a.l.d;
  if (d.dtype != PG_LOGITS_BF16) return d.vocab;
  return d.vocab + (d.rows > 1 && d.stride % LANE_TOKENS ? LANE_TOKENS - 1 : (int64_t)((uintptr_t)d.logits / 2 % LANE_TOKENS));
}
static int64_t most_slots(int64_t vocab) { return vocab + LANE_TOKENS - 1; }
static int64_t stretches_of(int64_t slots) { return (slots + LOSS_TOKENS - 1) / LOSS_TOKENS; }

// As many workgroups as are resident at once, if there is a stretch for each; short rows are no more than 8 to a workgroup, which goes
// through them one after another.  Two groups a lane at a time with eight waves a SIMD: four with five waves cost 22 % more for 1178 x 131073, one
// 5 % more for 4096 x 65537.  With the largest of each stretch six waves fit: 8 % more with as many workgroups as eight would take.
constexpr int64_t LOSS_WORKGROUPS = 2048, TOP_WORKGROUPS = 1536, ROWS_OF_ONE = 8;
constexpr int PASS_GROUPS = 2, WHOLE_GROUPS = 4, WHOLE_STRETCHES = 8;
// Few short rows are a workgroup's each, with four groups a lane at a time, in one launch.  In us, against the two launches (and the way from one to the
// other, some 2): 48 x 16384 (8 stretches) 6.7 for 5.0 + 3.4, 256 x 16384 8.6 for 10.5 + 3.9; with alternatives 12.1 for 5.3 + 8.2, 14.7 for 8.5 + 7.8, 500 x 8192
// 13.5 for 8.4 + 8.4, but 1000 x 4096 21.4 for 8.5 + 9.5; against a list 48 x 16000 10.2 for 4.9 + 6.3, 1000 x 4000 12.0 for 9.5 + 7.0.  At 12 stretches, 48 x
// 24001 with alternatives, 15.8 for 5.9 + 8.1; at 16, 48 x 32001, 11.0 for 5.8 + 3.4, 18.5 for 6.2 + 8.4, and 14.1 for 5.7 + 6.5 against a list.
static bool whole_rows(int64_t rows, int64_t stretches) { return stretches <= WHOLE_STRETCHES && rows * stretches <= LOSS_WORKGROUPS; }
static LossGrid loss_grid(const LossArgs& a, int64_t most) {
  const int64_t rows = a.l.d.rows, stretches = stretches_of(slots_of(a)), all = rows * stretches;
  const int64_t share = whole_rows(rows, stretches) ? stretches : std::min((all + most - 1) / most, ROWS_OF_ONE * stretches);
  return LossGrid{(int)stretches, (int)share, (int)((all + share - 1) / share)};
}
// No fewer than any call of at most so many rows and tokens has: a part for each row, and one more for each workgroup.
static int64_t most_parts(int64_t rows, int64_t vocab) {
  return rows + std::min(rows * stretches_of(most_slots(vocab)), std::max(LOSS_WORKGROUPS, (rows + ROWS_OF_ONE - 1) / ROWS_OF_ONE));
}
static int n_chunks(int64_t vocab) { return (int)((most_slots(vocab) + CHUNK - 1) / CHUNK); }
static int64_t part_floats(int64_t rows, int64_t vocab) { return (most_parts(rows, vocab) * (int64_t)(sizeof(Sums) / sizeof(float)) + 3) / 4 * 4; }

// launches F<bf16, ...> with `lds` bytes; a grid has fewer than 2^32 lanes
#define PG_LOSS_LAUNCH(blocks, threads, lds, F, ...)                                                         \
  do {                                                                                                       \
    if ((int64_t)(blocks) * (threads) >> 32) return fail(PG_ESHAPE, "%lld workgroups", (long long)(blocks)); \
    F<<<dim3((unsigned)(blocks)), dim3(threads), lds, (hipStream_t)stream>>>(__VA_ARGS__);                   \
    PG_LAUNCH_CHECK(#F);                                                                                     \
  } while (0)

// f(whether the logits are bf16), as a type
template <class F>
static pg_status with_kind(const LossArgs& a, F f) {
  return a.l.d.dtype == PG_LOGITS_BF16 ? f(std::true_type{}) : f(std::false_type{});
}

}  // namespace pg

using namespace pg;

extern "C" int64_t pg_logprob_scratch_floats(int32_t rows, int32_t vocab, int32_t n_top) {
  if (rows < 1 || vocab < 1 || n_top < 0) return 0;
  return part_floats(rows, vocab) + (n_top ? (int64_t)rows * n_chunks(vocab) : 0);
}

extern "C" pg_status pg_token_logprobs(const pg_logits* desc, const float* temperature, const int32_t* target, float* logp, float* entropy,
                                       float* stats, int32_t n_top, int32_t* top_ids, float* top_logp, float* scratch, void* stream) {
  LossArgs a{};
  PG_TRY(loss_args(desc, temperature, "pg_token_logprobs", a));
  if (n_top < 0 || n_top > PG_TOP_MAX) return fail(n_top < 0 ? PG_EINVAL : PG_ESHAPE, "pg_token_logprobs: %d alternatives (at most %d)", n_top, PG_TOP_MAX);
  const int64_t rows = a.l.d.rows;
  if (rows == 0) return PG_OK;
  if (logp && !target) return fail(PG_EINVAL, "pg_token_logprobs: logp without targets");
  if ((uintptr_t)stats & 15) return fail(PG_ESHAPE, "pg_token_logprobs: stats are not 16-byte aligned");
  if (!scratch) return fail(PG_EINVAL, "pg_token_logprobs: scratch is NULL");
  if ((uintptr_t)scratch & 7) return fail(PG_ESHAPE, "pg_token_logprobs: scratch is not 8-byte aligned");
  const bool top = n_top && (top_ids || top_logp);
  const LossGrid g = loss_grid(a, top ? TOP_WORKGROUPS : LOSS_WORKGROUPS);
  const LogprobOut o{target, logp, entropy, stats, n_top, top_ids, top_logp, (Sums*)scratch, scratch + part_floats(rows, a.l.d.vocab), n_chunks(a.l.d.vocab)};
  return with_kind(a, [&](auto bf) {
    constexpr bool BF = decltype(bf)::value;
    if (whole_rows(rows, g.stretches)) {
      if (top) PG_LOSS_LAUNCH(rows, LOSS_THREADS, 0, (logprob_kernel<BF, WHOLE_GROUPS, true, true>), a, g, o);
      else PG_LOSS_LAUNCH(rows, LOSS_THREADS, 0, (logprob_kernel<BF, WHOLE_GROUPS, false, true>), a, g, o);
      return PG_OK;
    }
    if (top) PG_LOSS_LAUNCH(g.workgroups, LOSS_THREADS, 0, (logprob_kernel<BF, PASS_GROUPS, true, false>), a, g, o);
    else PG_LOSS_LAUNCH(g.workgroups, LOSS_THREADS, 0, (logprob_kernel<BF, PASS_GROUPS, false, false>), a, g, o);
    if (top) PG_LOSS_LAUNCH(rows, LOSS_THREADS, 0, (logprob_finish_kernel<BF, true>), a, g, o);
    else if (g.share % g.stretches) PG_LOSS_LAUNCH(rows, WAVE, 0, (logprob_finish_kernel<BF, false>), a, g, o);
    return PG_OK;
  });
}

// A bf16 gradient of more than 256 MiB, what the last cache holds: the next pass need not wait for what the caches write back.  Passes and gradients in turn, in
// us with and without: 1100 x 131073 (288 MB) 170 and 183, 2048 x 131073 289 and 303, 4096 x 131072 563 and 565; against a list 165 and 184, 297 and 313.
// Smaller ones are left where their reader finds them, although nothing but these two passes, again and again, is faster without: 900 x 131073 (236 MB)
// 141 and 154, 1178 x 65537 (154 MB) 102 and 102.  In fp32 the gradient takes 427 for 370.
static bool past_the_caches(const LossArgs& a) { return a.l.d.dtype == PG_LOGITS_BF16 && (int64_t)a.l.d.rows * a.l.d.vocab * 2 > 256ll << 20; }

// A gradient's workgroup goes through one pass, of four groups a lane in bf16 (4096 x 131072: two groups 2 % more, one 9 %) and of one in fp32, or where there
// are few rows, to be spread.  One, two and four groups in fp32, us: 4096 x 65537 435, 428 and 451, 4096 x 6000 40, 57 and 43; against a list, which
// each workgroup looks up anew, 456, 458 and 484, 55, 79 and 64, and 1000 x 32001 61, 62 and 69.
static bool large_passes(const LossArgs& a) { return a.l.d.dtype == PG_LOGITS_BF16 && a.l.d.rows * ((stretches_of(slots_of(a)) + 3) / 4) >= 1024; }
// f(whether the logits are bf16, groups a lane takes, whether the gradient goes past the caches), as types
template <class F>
static pg_status with_gradient(const LossArgs& a, F f) {
  const auto four = std::integral_constant<int, 4>{};
  const auto one = std::integral_constant<int, 1>{};
  if (a.l.d.dtype != PG_LOGITS_BF16) return f(std::false_type{}, one, std::false_type{});
  if (!large_passes(a)) return f(std::true_type{}, one, std::false_type{});
  return past_the_caches(a) ? f(std::true_type{}, four, std::true_type{}) : f(std::true_type{}, four, std::false_type{});
}

extern "C" pg_status pg_token_logprobs_backward(const pg_logits* desc, const float* temperature, const int32_t* target, const float* stats,
                                                const float* g_logp, const float* g_entropy, void* d_logits, int64_t d_stride, void* stream) {
  LossArgs a{};
  PG_TRY(loss_args(desc, temperature, "pg_token_logprobs_backward", a));
  const int64_t rows = a.l.d.rows;
  if (rows == 0) return PG_OK;
  if (!stats) return fail(PG_EINVAL, "pg_token_logprobs_backward: stats is NULL");
  if ((uintptr_t)stats & 15) return fail(PG_ESHAPE, "pg_token_logprobs_backward: stats are not 16-byte aligned");
  if (g_logp && !target) return fail(PG_EINVAL, "pg_token_logprobs_backward: a gradient of log-probs without targets");
  PG_TRY(check_gradient(a, d_logits, d_stride, "pg_token_logprobs_backward"));
  return with_gradient(a, [&](auto bf, auto groups, auto past) {
    constexpr int G = decltype(groups)::value;
    const int pieces = (int)((stretches_of(slots_of(a)) + G - 1) / G);
    PG_LOSS_LAUNCH(rows * pieces, LOSS_THREADS, 0, (logprob_backward_kernel<decltype(bf)::value, G, decltype(past)::value>), a, pieces, target, stats, g_logp, g_entropy, d_logits, d_stride);
    return PG_OK;
  });
}

static pg_status distill_args(const LossArgs& a, const int32_t* ids, const float* logp, int32_t k, const float* stats, const char* who) {
  if (k < 1) return fail(PG_EINVAL, "%s: %d tokens of a teacher", who, k);
  if (k > PG_DISTILL_MAX) return fail(PG_ESHAPE, "%s: %d tokens of a teacher (at most %d)", who, k, PG_DISTILL_MAX);
  if (a.l.d.rows && (!ids || !logp)) return fail(PG_EINVAL, "%s: the teacher's list is NULL", who);
  if ((uintptr_t)stats & 15) return fail(PG_ESHAPE, "%s: stats are not 16-byte aligned", who);
  return PG_OK;
}

extern "C" int64_t pg_distill_scratch_floats(int32_t rows, int32_t vocab) { return rows < 1 || vocab < 1 ? 0 : part_floats(rows, vocab); }

extern "C" pg_status pg_distill_loss(const pg_logits* desc, const float* temperature, int32_t mode, const int32_t* teacher_ids,
                                     const float* teacher_logp, int32_t k, float* loss, float* stats, float* scratch, void* stream) {
  LossArgs a{};
  PG_TRY(loss_args(desc, temperature, "pg_distill_loss", a));
  if (mode != PG_DISTILL_TOP && mode != PG_DISTILL_TAIL) return fail(PG_EINVAL, "pg_distill_loss: mode %d", mode);
  PG_TRY(distill_args(a, teacher_ids, teacher_logp, k, stats, "pg_distill_loss"));
  const int64_t rows = a.l.d.rows;
  if (rows == 0) return PG_OK;
  if (!loss || !scratch) return fail(PG_EINVAL, "pg_distill_loss: null pointer");
  if ((uintptr_t)scratch & 7) return fail(PG_ESHAPE, "pg_distill_loss: scratch is not 8-byte aligned");
  const LossGrid g = loss_grid(a, LOSS_WORKGROUPS);
  const DistillArgs o{mode, k, teacher_ids, teacher_logp, loss, stats, (Sums*)scratch};
  const size_t lds = std::min({g.stretches, g.share, LIST_RANGE / LOSS_TOKENS}) * (LOSS_TOKENS / 8);
  return with_kind(a, [&](auto bf) {
    constexpr bool BF = decltype(bf)::value;
    if (whole_rows(rows, g.stretches)) {
      PG_LOSS_LAUNCH(rows, LOSS_THREADS, std::max(lds, sizeof(ListLds)), (distill_kernel<BF, WHOLE_GROUPS, true>), a, g, o);
      return PG_OK;
    }
    PG_LOSS_LAUNCH(g.workgroups, LOSS_THREADS, lds, (distill_kernel<BF, PASS_GROUPS, false>), a, g, o);
    PG_LOSS_LAUNCH(rows, WAVE, 0, distill_finish_kernel<BF>, a, g, o);
    return PG_OK;
  });
}

extern "C" pg_status pg_distill_backward(const pg_logits* desc, const float* temperature, const int32_t* teacher_ids, const float* teacher_logp,
                                         int32_t k, const float* stats, const float* g_loss, void* d_logits, int64_t d_stride, void* stream) {
  LossArgs a{};
  PG_TRY(loss_args(desc, temperature, "pg_distill_backward", a));
  PG_TRY(distill_args(a, teacher_ids, teacher_logp, k, stats, "pg_distill_backward"));
  const int64_t rows = a.l.d.rows;
  if (rows == 0) return PG_OK;
  if (!stats || !g_loss) return fail(PG_EINVAL, "pg_distill_backward: null pointer");
  PG_TRY(check_gradient(a, d_logits, d_stride, "pg_distill_backward"));
  const DistillArgs o{0, k, teacher_ids, teacher_logp, nullptr, const_cast<float*>(stats), nullptr};
  return with_gradient(a, [&](auto bf, auto groups, auto past) {
    constexpr int G = decltype(groups)::value;
    const int pieces = (int)((stretches_of(slots_of(a)) + G - 1) / G);
    PG_LOSS_LAUNCH(rows * pieces, LOSS_THREADS, 0, (distill_backward_kernel<decltype(bf)::value, G, decltype(past)::value>), a, pieces, o, g_loss, d_logits, d_stride);
    return PG_OK;
  });
}

// Sequences of up to 8192 tokens are a workgroup's each (48 x 8192: 7.7 us, as long as in two launches); longer ones are cut into pieces of some 1024 tokens
// (from 911 on) or more, at most 4096 in all, and joined by a second launch (48 x 16384: 5.8 + 2.7 us, whole 12.5; 384 sequences of up to 16384
// 15.1 us, 5 % more with 2048 in all, 25 % with 8192).
constexpr int64_t SURROGATE_WHOLE = 8192, SURROGATE_PIECE = 1024, SURROGATE_WORKGROUPS = 4096;
static int64_t surrogate_pieces(int64_t n_seq, int64_t max_len) {
  if (max_len <= SURROGATE_WHOLE) return 1;
  return std::min((max_len + SURROGATE_PIECE - 1) / SURROGATE_PIECE, std::max<int64_t>(1, SURROGATE_WORKGROUPS / n_seq));
}

extern "C" int64_t pg_surrogate_scratch_floats(int32_t n_seq, int32_t max_len) {
  if (n_seq < 1 || max_len <= SURROGATE_WHOLE) return 0;
  return 4 * std::min<int64_t>(n_seq * ((max_len + SURROGATE_PIECE - 1) / SURROGATE_PIECE), SURROGATE_WORKGROUPS);
}

extern "C" pg_status pg_token_surrogate(const float* logp, const float* logp_old, const float* logp_ref, const float* adv, const float* weight,
                                        const int32_t* cu, int32_t n_seq, int32_t n_tokens, int32_t max_len, double clip_low, double clip_high,
                                        double kl_coef, float* objective, float* kl, int32_t* clipped, float* g_logp, float* scratch,
                                        void* stream) {
  if (n_seq < 0 || n_tokens < 0 || max_len < 0) return fail(PG_EINVAL, "pg_token_surrogate: %d sequences, %d tokens, length %d", n_seq, n_tokens, max_len);
  if (n_seq > 1 << 23) return fail(PG_ESHAPE, "pg_token_surrogate: %d sequences (at most %d)", n_seq, 1 << 23);
  if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0) || !std::isfinite((float)kl_coef))
    return fail(PG_EINVAL, "pg_token_surrogate: clip %g below and %g above, kl_coef %g", clip_low, clip_high, kl_coef);
  if (n_seq == 0) return PG_OK;
  if (!adv || !cu || (n_tokens && (!logp || !logp_old))) return fail(PG_EINVAL, "pg_token_surrogate: null pointer");
  const int pieces = (int)surrogate_pieces(n_seq, max_len);
  if (pieces > 1 && !scratch) return fail(PG_EINVAL, "pg_token_surrogate: scratch is NULL");
  if (pieces > 1 && (uintptr_t)scratch & 15) return fail(PG_ESHAPE, "pg_token_surrogate: scratch is not 16-byte aligned");
  const SurrogateArgs a{logp, logp_old, logp_ref, adv, weight, cu, n_tokens, std::log1p(-clip_low), std::log1p(clip_high), (float)(1.0 - clip_low),
                        (float)(1.0 + clip_high), (float)kl_coef, objective, kl, g_logp, clipped, pieces, (int)(((int64_t)max_len + pieces - 1) / pieces), scratch};
  // of 2^22 sequences or more 1024 lanes each are more than a grid has
  if (pieces == 1 && max_len > 1024 && n_seq < 1 << 22) PG_LOSS_LAUNCH(n_seq, 1024, 0, surrogate_tokens_kernel<1024>, a);
  else PG_LOSS_LAUNCH((int64_t)n_seq * pieces, LOSS_THREADS, 0, surrogate_tokens_kernel<LOSS_THREADS>, a);
  if (pieces > 1) PG_LOSS_LAUNCH(n_seq, WAVE, 0, surrogate_finish_kernel, a);
  return PG_OK;
}
