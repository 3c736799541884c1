// Pages of a token policy's key/value cache: taken, forked, freed, moved, and filled with new tokens.
//
// A page's state is its reference count alone (0: free), and the free page of the lowest number is taken first, so what a call
// does follows from its arguments whatever order workgroups run in.  The calls that take pages are one workgroup that scans
// the counts (4 bytes a page) and stops at the last page it needs; the pages' data, tables and counts are then gone through by
// the whole device in a second launch.
//
// Measured: a plan takes 2.8 to 7.4 us (latency: four to six dependent loads and barriers); 376 part-filled pages of twelve layers copied for
// a fork 26 us (148 MB written, the eight source pages come from the caches: the write rate of the device is 6.9 TB/s); 530 MB of pages moved
// 200 us (5.3 TB/s read and written, where a plain copy of 4 GiB reaches 4.8 to 5.6 by its grid); 135 thousand tokens of eight heads of 128 appended as codes 192 us (4.3 TB/s).
#include <cmath>
#include <type_traits>
#include "paged_cache.hpp"
#include "operands.hpp"

namespace pg {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_WAVES = PLAN_THREADS / WAVE;
constexpr int APPLY_THREADS = 256;
constexpr int MAX_COPY_BLOCKS = 8192;              // four times what the device holds (512: 71 us, 2048: 64, 8192: 62 for 248 MB)

// Exclusive prefix sum of v over the workgroup; total: the sum.  `sums` holds PLAN_WAVES + 1 values.
template <class T>
__device__ __forceinline__ T block_scan(T v, T* sums, T& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();                                 // the sums of the call before have been read
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  T before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < PLAN_WAVES; ++w) {
    const T s = sums[w];
    before += w < wave ? s : 0;
    total += s;
  }
  return before + x - v;
}

// Counts of pages p .. p + 3; those past the pool's end are no free ones.
__device__ __forceinline__ int4 counts_of(const int32_t* refs, int n_pages, int p) {
  if (p + 4 <= n_pages) return *(const int4*)(refs + p);
  return int4{p < n_pages ? refs[p] : 1, p + 1 < n_pages ? refs[p + 1] : 1, p + 2 < n_pages ? refs[p + 2] : 1, 1};
}
// The free pages in ascending order, handed out until `wanted` are found: take(rank, page).  Returns how many there were.
// `head`: the lane's counts of the first tile, which the caller has asked for before the work that precedes this.
template <class Take>
__device__ __forceinline__ int free_pages(const int32_t* refs, int n_pages, int4 head, int wanted, int* sums, Take take) {
  int found = 0;
  for (int base = 0; base < n_pages && found < wanted; base += PLAN_THREADS * 4) {
    const int p = base + (int)threadIdx.x * 4;
    const int4 r = base ? counts_of(refs, n_pages, p) : head;
    const unsigned free = (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
    int total;
    int rank = found + block_scan<int>(__popc(free), sums, total);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (free >> i & 1) {
        if (rank < wanted) take(rank, p + i);
        ++rank;
      }
    found += total;
  }
  return min(found, wanted);
}

__device__ __forceinline__ bool length_fits(int n, const CacheView& c) {
  return n >= 0 && (int64_t)n <= (int64_t)c.width << c.page_shift;
}
__device__ __forceinline__ int pages_of(int64_t n, int shift) { return (int)((n + (1 << shift) - 1) >> shift); }

__global__ __launch_bounds__(256) void cache_clear_kernel(int32_t* refs, int n_pages, int32_t* status) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n_pages) refs[i] = 0;
  if (i < 4) status[i] = 0;
}

// ---------------------------------------------------------------- reserve
// cum[r]: pages wanted by rows 0 .. r, limited to n_pages + 1; the free page of rank k is row r's with cum[r-1] <= k < cum[r].
__global__ __launch_bounds__(PLAN_THREADS) void cache_reserve_kernel(CacheView c, int32_t* refs, int32_t* table, const int32_t* lens,
                                                                     const int32_t* add, int32_t* lens_out, int n_rows) {
  extern __shared__ int cum[];
  const int4 head = counts_of(refs, c.n_pages, (int)threadIdx.x * 4);
  int* first = cum + n_rows;                         // where page number `rank` of a row goes: first[r] + rank
  __shared__ int64_t sums64[PLAN_WAVES];
  __shared__ int sums[PLAN_WAVES];
  __shared__ int bits;
  if (threadIdx.x == 0) bits = 0;
  __syncthreads();
  const int64_t room = (int64_t)c.width << c.page_shift;
  auto wants = [&](int64_t n, int64_t m, int& flag) {            // pages that a row asks for, and what is wrong with it
    flag = n < 0 || n > room || m < 0 ? CACHE_RANGE : n + m > room ? CACHE_FULL : 0;
    return flag ? 0 : pages_of(n + m, c.page_shift) - pages_of(n, c.page_shift);
  };
  int64_t carry = 0;
  int n = 0, m = 0;                                  // of the lane's row, where it has only one
  for (int base = 0; base < n_rows; base += PLAN_THREADS) {
    const int r = base + threadIdx.x;
    int flag = 0, need = 0;
    if (r < n_rows) need = wants(n = lens[r], m = add[r], flag);
    if (flag) atomicOr(&bits, flag);
    int64_t total;
    const int64_t before = carry + block_scan<int64_t>(need, sums64, total);
    if (r < n_rows) {
      cum[r] = (int)min(before + need, (int64_t)c.n_pages + 1);
      first[r] = pages_of(n, c.page_shift) - (int)min(before, (int64_t)c.n_pages + 1);
    }
    carry += total;
  }
  __syncthreads();
  const int wanted = (int)min(carry, (int64_t)c.n_pages + 1);
  const int found = free_pages(refs, c.n_pages, head, wanted, sums, [&](int rank, int page) {
    int lo = 0, hi = n_rows - 1;                     // first row with cum > rank
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (cum[mid] > rank) hi = mid; else lo = mid + 1;
    }
    table[(int64_t)lo * c.width + first[lo] + rank] = page;
    refs[page] = 1;
  });
  __syncthreads();
  for (int r = threadIdx.x; r < n_rows; r += PLAN_THREADS) {
    if (n_rows > PLAN_THREADS) n = lens[r], m = add[r];
    const int base = r ? cum[r - 1] : 0;
    int flag;
    const int need = wants(n, m, flag);
    const bool fits = !flag && (need == 0 || cum[r] <= found);
    if (!flag && !fits) {
      atomicOr(&bits, CACHE_FULL);
      for (int k = base; k < found; ++k) {           // at most one row has got a part of its pages
        int32_t* e = table + (int64_t)r * c.width + first[r] + k;
        refs[*e] = 0;
        *e = -1;
      }
    }
    lens_out[r] = n + (fits ? m : 0);
  }
  __syncthreads();
  if (threadIdx.x == 0 && bits) atomicOr(c.status, bits);
}

// ---------------------------------------------------------------- select
// scratch: [0] copies, [4 ..] of each copy in row order the page it is of and the page it goes to, then users of each source row, then
// per output row the page of its copy (-1: none)
struct SelectPlan {
  int32_t* count;
  int2* copies;
  int32_t *users, *fresh;
};
inline SelectPlan select_plan(int32_t* scratch, int n_in, int n_out) {
  return SelectPlan{scratch, (int2*)(scratch + 4), scratch + 4 + 2 * (int64_t)n_out, scratch + 4 + 2 * (int64_t)n_out + n_in};
}

__global__ __launch_bounds__(PLAN_THREADS) void cache_select_plan_kernel(CacheView c, int32_t* refs, const int32_t* table_in,
                                                                         const int32_t* lens_in, int n_in, const int32_t* src,
                                                                         int32_t* lens_out, int n_out, SelectPlan plan) {
  extern __shared__ int lds[];
  int *users = lds, *first = lds + n_in;
  const int4 head = counts_of(refs, c.n_pages, (int)threadIdx.x * 4);
  __shared__ int sums[PLAN_WAVES];
  __shared__ int bits;
  if (threadIdx.x == 0) bits = 0;
  for (int s = threadIdx.x; s < n_in; s += PLAN_THREADS) {
    users[s] = 0;
    first[s] = n_out;
  }
  __syncthreads();
  for (int r = threadIdx.x; r < n_out; r += PLAN_THREADS) {
    const int s = src[r];
    if (s >= 0 && s < n_in) {
      atomicAdd(&users[s], 1);
      atomicMin(&first[s], r);
    } else if (s != -1) {
      atomicOr(&bits, CACHE_RANGE);
    }
  }
  __syncthreads();
  const int part = (1 << c.page_shift) - 1;
  int wanted = 0;
  for (int base = 0; base < n_out; base += PLAN_THREADS) {
    const int r = base + threadIdx.x;
    int n = 0;
    bool copied = false;
    if (r < n_out) {
      const int s = src[r];
      if (s >= 0 && s < n_in) {
        n = lens_in[s];
        if (!length_fits(n, c)) {
          n = 0;
          atomicOr(&bits, CACHE_RANGE);
        }
        copied = (n & part) && first[s] != r;
      }
      lens_out[r] = n;
      plan.fresh[r] = -1;
    }
    int total;
    const int rank = wanted + block_scan<int>(copied, sums, total);
    if (copied) {
      int from = table_in[(int64_t)src[r] * c.width + (n >> c.page_shift)];
      if ((unsigned)from >= (unsigned)c.n_pages) {
        atomicOr(&bits, CACHE_RANGE);
        from = 0;
      }
      plan.copies[rank] = int2{from, r};
    }
    wanted += total;
  }
  for (int s = threadIdx.x; s < n_in; s += PLAN_THREADS) plan.users[s] = users[s];
  __syncthreads();
  const int found = free_pages(refs, c.n_pages, head, wanted, sums, [&](int rank, int page) {
    plan.fresh[plan.copies[rank].y] = page;
    plan.copies[rank].y = page;
    refs[page] = 1;
  });
  for (int k = found + threadIdx.x; k < wanted; k += PLAN_THREADS) {
    const int r = plan.copies[k].y;
    lens_out[r] = lens_out[r] & ~part;
    atomicOr(&bits, CACHE_FULL);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    plan.count[0] = found;
    if (bits) atomicOr(c.status, bits);
  }
}

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));

// page copies over all layers: item i is 16 KB (or a page's rest) of one pool's copy of one page; nothing of it is read again soon, so it
// is kept out of the way in the caches (248 MB of copies: 63 us, 75 without the hints)
struct PageCopy {
  uint8_t *k, *v;
  int64_t layer_bytes;                               // of one pool
  uint32_t page_bytes;                               // up to 2^31
  int32_t layers;
};
constexpr int COPY_PIECE = 16384;
template <bool SHARED, class Pages>
__device__ __forceinline__ void copy_pages(const PageCopy& a, int copies, int block, int blocks, Pages pages) {
  const int pieces = (int)((a.page_bytes + COPY_PIECE - 1) / COPY_PIECE);
  const int64_t items = (int64_t)copies * a.layers * 2 * pieces;
  for (int64_t i = block; i < items; i += blocks) {
    const int piece = (int)(i % pieces);
    const int64_t j = i / pieces;
    const int pool = (int)(j & 1), layer = (int)((j >> 1) % a.layers);
    int from, to;
    pages((int)((j >> 1) / a.layers), from, to);
    uint8_t* base = (pool ? a.v : a.k) + layer * a.layer_bytes;
    const uint32_t lo = (uint32_t)piece * COPY_PIECE;
    const int n = (int)min((uint32_t)COPY_PIECE, a.page_bytes - lo);
    const u32x4v* in = (const u32x4v*)(base + (int64_t)from * a.page_bytes + lo);
    u32x4v* out = (u32x4v*)(base + (int64_t)to * a.page_bytes + lo);
    constexpr int PER = COPY_PIECE / 16 / APPLY_THREADS;
    u32x4v x[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int at = threadIdx.x + e * APPLY_THREADS;
      if (at < n / 16) x[e] = SHARED ? in[at] : __builtin_nontemporal_load(in + at);
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int at = threadIdx.x + e * APPLY_THREADS;
      if (at < n / 16) __builtin_nontemporal_store(x[e], out + at);
    }
  }
}

__global__ __launch_bounds__(APPLY_THREADS) void cache_select_apply_kernel(CacheView c, PageCopy data, int32_t* refs, const int32_t* table_in,
                                                                           const int32_t* lens_in, int n_in, const int32_t* src,
                                                                           int32_t* table_out, const int32_t* lens_out, int n_out,
                                                                           SelectPlan plan) {
  int block = blockIdx.x;
  auto valid = [&](int p) {
    const bool ok = (unsigned)p < (unsigned)c.n_pages;
    if (!ok) atomicOr(c.status, CACHE_RANGE);
    return ok;
  };
  if (block < n_out) {                               // a row of the new table
    const int n = lens_out[block], s = src[block], fresh = plan.fresh[block];
    const int pages = pages_of(n, c.page_shift);
    const int32_t* in = table_in + (int64_t)s * c.width;
    int32_t* out = table_out + (int64_t)block * c.width;
    for (int j = threadIdx.x; j < c.width; j += APPLY_THREADS)
      out[j] = j >= pages ? -1 : j == pages - 1 && fresh >= 0 ? fresh : in[j];
    return;
  }
  block -= n_out;
  if (block < n_in) {                                // the reference counts of an old row's pages
    const int n = lens_in[block], change = plan.users[block] - 1;
    if (change == 0 || !length_fits(n, c)) return;
    const int whole = n >> c.page_shift, pages = pages_of(n, c.page_shift);
    const int32_t* in = table_in + (int64_t)block * c.width;
    for (int j = threadIdx.x; j < (change < 0 ? pages : whole); j += APPLY_THREADS)
      if (valid(in[j])) atomicAdd(refs + in[j], change);
    return;
  }
  block -= n_in;
  copy_pages<true>(data, plan.count[0], block, gridDim.x - n_out - n_in, [&](int i, int& from, int& to) {
    const int2 pair = plan.copies[i];
    from = pair.x;
    to = pair.y;
  });
}

// ---------------------------------------------------------------- compact
// scratch: [0] pages to move, [1] live pages, [4 ..] holes, then movers, then where a page goes
struct CompactPlan {
  int32_t *count, *holes, *movers, *goes;
};
inline CompactPlan compact_plan(int32_t* scratch, int n_pages) {
  const int half = n_pages / 2 + 1;                  // a hole and a mover are two pages
  return CompactPlan{scratch, scratch + 4, scratch + 4 + half, scratch + 4 + 2 * (int64_t)half};
}

__global__ __launch_bounds__(PLAN_THREADS) void cache_compact_plan_kernel(int32_t* refs, int n_pages, CompactPlan plan) {
  __shared__ int sums[PLAN_WAVES];
  int mine = 0, live;
  for (int p = threadIdx.x; p < n_pages; p += PLAN_THREADS) mine += refs[p] > 0;
  block_scan<int>(mine, sums, live);
  int holes = 0, movers = 0;
  for (int base = 0; base < n_pages; base += PLAN_THREADS) {
    const int p = base + threadIdx.x;
    const bool used = p < n_pages && refs[p] > 0;
    const bool hole = p < live && !used, mover = p >= live && used;
    int total;
    // as many of either kind as of the other in the end; a tile counts both in one scan
    const int rank = block_scan<int>((int)hole | (int)mover << 16, sums, total);
    if (hole) plan.holes[holes + (rank & 0xFFFF)] = p;
    if (mover) plan.movers[movers + (rank >> 16)] = p;
    holes += total & 0xFFFF;
    movers += total >> 16;
  }
  __syncthreads();
  for (int k = threadIdx.x; k < movers; k += PLAN_THREADS) {
    const int from = plan.movers[k], to = plan.holes[k];
    plan.goes[from] = to;
    refs[to] = refs[from];
    refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    plan.count[0] = movers;
    plan.count[1] = live;
  }
}

__global__ __launch_bounds__(APPLY_THREADS) void cache_compact_apply_kernel(CacheView c, PageCopy data, int32_t* table, const int32_t* lens,
                                                                            int n_rows, CompactPlan plan) {
  int block = blockIdx.x;
  if (block < n_rows) {
    const int n = lens[block], live = plan.count[1];
    if (!length_fits(n, c)) {
      if (threadIdx.x == 0) atomicOr(c.status, CACHE_RANGE);
      return;
    }
    const int pages = pages_of(n, c.page_shift);
    int32_t* row = table + (int64_t)block * c.width;
    for (int j = threadIdx.x; j < pages; j += APPLY_THREADS) {
      const int p = row[j];
      if (p >= 0 && p < live) continue;
      const int to = (unsigned)p < (unsigned)c.n_pages ? plan.goes[p] : -1;
      if ((unsigned)to < (unsigned)live) row[j] = to;
      else atomicOr(c.status, CACHE_RANGE);
    }
    return;
  }
  copy_pages<false>(data, plan.count[0], block - n_rows, gridDim.x - n_rows, [&](int i, int& from, int& to) {
    from = plan.movers[i];
    to = plan.holes[i];
  });
}

// ---------------------------------------------------------------- append
// The last r with f(r) <= u, f ascending and f(0) <= u: 64 lanes probe at a time.
template <class F>
__device__ __forceinline__ int last_not_above(int n, int64_t u, F f) {
  int lo = 0;                                        // f(lo) <= u
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + (int)(threadIdx.x & 63) * step;
    const int ok = max(1, (int)__popcll(__ballot(at < lo + n && f(at) <= u)));
    const int next = lo + (ok - 1) * step;
    n = min(step, lo + n - next);
    lo = next;
  }
  return lo;
}

__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// x / scale correctly rounded, limited to +-448 (NaN stays NaN).  With r = 1 / scale correctly rounded, q = x r and one step
// q - (q scale - x) r give the quotient's rounding (Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor",
// 1990; in this form of the step -0 stays -0).  x is limited before, to 448 scale, whose quotient rounds to 448.  The compiler's own
// division, which is longer than everything else here together, is for scales for which one of the two is not finite.
struct Quotient {
  float scale, r, most;
  __device__ explicit Quotient(float s) : scale(s), r(1.0f / s), most(448.0f * s) {}
  static __device__ __forceinline__ float within(float x, float most) {
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(x, -most), most);
  }
  __device__ __forceinline__ float operator()(uint32_t bits32) const {
    const float x = __builtin_bit_cast(float, bits32);
    if (!(r < INFINITY && most < INFINITY)) return within(x / scale, 448.0f);
    const float y = within(x, most), q = y * r;
    return __builtin_fmaf(-__builtin_fmaf(q, scale, -y), r, q);
  }
};

struct AppendArgs {
  CacheView c;
  void *k, *v;                                       // of the layer
  const float *k_scale, *v_scale;                    // of the layer, or NULL
  const uint16_t *k_new, *v_new;
  int64_t token_stride;
  const int32_t *table, *lens, *cu, *refs;
  int n_rows, n_tokens, units;
};

// One wave: 16 positions of a row (those of them that are new) of one head.  Keys are copied, values go through LDS to be
// written along the tokens: a whole block of 16 positions is 32 (bf16) or 16 contiguous bytes of each channel's row.  The four waves
// of a workgroup take consecutive blocks, so that a line of values is written from one XCD.
template <int HD, bool F8>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a) {
  using Value = typename std::conditional<F8, uint8_t, uint16_t>::type;
  constexpr int PAD = F8 ? 20 : 18;                  // tokens of a channel's row in LDS, one word of them padding
  __shared__ __align__(16) Value tile[4][HD * PAD];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const CacheView& c = a.c;
  const int head = blockIdx.x % (unsigned)c.heads, unit = (int)(blockIdx.x / (unsigned)c.heads) * 4 + wave;       // a token's heads lie together
  if (unit >= a.units) return;
  int row = unit, t0 = row, fresh = 1, part = 0;
  if (a.cu) {
    // row r owns the numbers cu[r]/16 + 2 r ..., at least as many as it has blocks of 16 positions
    row = __builtin_amdgcn_readfirstlane(last_not_above(a.n_rows, unit, [&](int r) { return (int64_t)(a.cu[r] >> 4) + 2ll * r; }));
    t0 = a.cu[row];
    fresh = a.cu[row + 1] - t0;
    part = unit - ((t0 >> 4) + 2 * row);
  }
  const int len = a.lens[row];
  if ((part < 0 && row) || t0 < 0 || fresh < 0 || t0 + (int64_t)fresh > a.n_tokens || fresh > len || !length_fits(len, c)) {
    if (lane == 0 && head == 0) atomicOr(c.status, CACHE_RANGE);
    return;
  }
  if (part < 0) return;                              // a number of the tokens before the first row's
  const int begin = len - fresh;
  const int64_t at = (begin & ~15) + (int64_t)part * 16;       // position of the block
  if (at >= len || fresh == 0) return;
  const int page = a.table[(int64_t)row * c.width + (at >> c.page_shift)];
  if ((unsigned)page >= (unsigned)c.n_pages) {
    if (lane == 0 && head == 0) atomicOr(c.status, CACHE_RANGE);
    return;
  }
  const int users = a.refs[page];
  const int slot = (int)at & ((1 << c.page_shift) - 1);
  const int64_t to = (((int64_t)page * c.heads + head) << c.page_shift) * HD;
  const Quotient ks(F8 && a.k_scale ? a.k_scale[head] : 1.0f), vs(F8 && a.v_scale ? a.v_scale[head] : 1.0f);
  Value* t = tile[wave];
  // COLS lanes read 16 bytes each of a token's channels side by side, a whole line of 128 bytes where the head has one; all loads first
  constexpr int COLS = HD / 8 < 8 ? HD / 8 : 8, TOKENS = 64 / COLS, PASSES = 16 / TOKENS, ITERS = HD / 8 / COLS;
  const int i0 = lane / COLS, col = lane % COLS * 8;
  auto there = [&](int i) { return at + i >= begin && at + i < len; };      // position i of the block is new
  u32x4v kx[PASSES][ITERS], vx[PASSES][ITERS];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    // lanes without a new token read the row's first new one again, so that no load waits for a branch
    const int i = i0 + p * TOKENS;
    const int64_t from = (there(i) ? t0 + (at + i - begin) : t0) * a.token_stride + (int64_t)head * HD + col;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
      kx[p][it] = *(const u32x4v*)(a.k_new + from + it * COLS * 8);
      vx[p][it] = *(const u32x4v*)(a.v_new + from + it * COLS * 8);
    }
  }
  if (users > 1) {                                   // whole, and others read it: the row has no place for these tokens
    if (lane == 0 && head == 0) atomicOr(c.status, CACHE_FULL);
    return;
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int i = i0 + p * TOKENS;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
      const int ch = col + it * COLS * 8;
      const int64_t kt = to + (int64_t)(slot + i) * HD + ch;
      if constexpr (F8) {
        auto codes = [](u32x4v x, const Quotient& over) {
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = over(e & 1 ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16);
          return u32x2v{to_e4m3x4(f[0], f[1], f[2], f[3]), to_e4m3x4(f[4], f[5], f[6], f[7])};
        };
        const u32x2v k = codes(kx[p][it], ks), v = codes(vx[p][it], vs);
        if (there(i)) *(u32x2v*)((uint8_t*)a.k + kt) = k;
#pragma unroll
        for (int e = 0; e < 8; ++e) t[(ch + e) * PAD + i] = (uint8_t)(v[e >> 2] >> (8 * (e & 3)));
      } else {
        if (there(i)) *(u32x4v*)((uint16_t*)a.k + kt) = kx[p][it];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[(ch + e) * PAD + i] = (uint16_t)(vx[p][it][e >> 1] >> (16 * (e & 1)));
      }
    }
  }
  wave_lds_sync();
  const int64_t vrow = to + slot;                    // channel 0 of the block
  const int width = 1 << c.page_shift;
  if (at >= begin && at + 16 <= len) {
    for (int ch = lane; ch < HD; ch += 64) {
      const uint32_t* s = (const uint32_t*)(t + ch * PAD);
      uint4* o = (uint4*)((Value*)a.v + vrow + (int64_t)ch * width);
#pragma unroll
      for (int e = 0; e < (F8 ? 1 : 2); ++e) o[e] = uint4{s[4 * e], s[4 * e + 1], s[4 * e + 2], s[4 * e + 3]};
    }
  } else {
    for (int i = (int)max((int64_t)0, begin - at); i < 16 && at + i < len; ++i)
      for (int ch = lane; ch < HD; ch += 64) ((Value*)a.v)[vrow + (int64_t)ch * width + i] = t[ch * PAD + i];
  }
}

// ---------------------------------------------------------------- host side

pg_status check_cache(const pg_cache* c, bool data, const char* who) {
  if (!c) return fail(PG_EINVAL, "%s: cache is NULL", who);
  if (c->layers < 1 || c->n_pages < 1 || c->heads < 1 || c->width < 1 || (c->dtype != PG_CACHE_BF16 && c->dtype != PG_CACHE_E4M3))
    return fail(PG_EINVAL, "%s: a cache of %d layers, %d pages, %d heads, dtype %d, tables %d wide", who, c->layers, c->n_pages, c->heads,
                c->dtype, c->width);
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128)
    return fail(PG_ESHAPE, "%s: pages of %d tokens (16, 32, 64 or 128)", who, c->page);
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128)
    return fail(PG_ESHAPE, "%s: head width %d (32, 64 or 128)", who, c->head_dim);
  if ((int64_t)c->width * c->page > 1 << 30) return fail(PG_ESHAPE, "%s: a row of %d pages passes 2^30 tokens", who, c->width);
  if (c->n_pages > INT32_MAX - 8) return fail(PG_ESHAPE, "%s: too many pages", who);
  if ((int64_t)c->heads * c->page * c->head_dim > 1 << 30) return fail(PG_ESHAPE, "%s: a page of %d heads is too large", who, c->heads);
  if (!c->refs || !c->status) return fail(PG_EINVAL, "%s: refs or status is NULL", who);
  if ((uintptr_t)c->refs & 15) return fail(PG_ESHAPE, "%s: refs must be 16-byte aligned", who);
  if (c->dtype == PG_CACHE_BF16 && (c->k_scale || c->v_scale)) return fail(PG_EINVAL, "%s: a bf16 cache has no scales", who);
  if (data && (!c->k || !c->v)) return fail(PG_EINVAL, "%s: k or v is NULL", who);
  if (data && (((uintptr_t)c->k | (uintptr_t)c->v) & 15)) return fail(PG_ESHAPE, "%s: k and v must be 16-byte aligned", who);
  return PG_OK;
}

static pg_status check_rows(int64_t n, const char* who) {
  if (n < 0) return fail(PG_EINVAL, "%s: %lld rows", who, (long long)n);
  if (n > PG_CACHE_MAX_ROWS) return fail(PG_ESHAPE, "%s: %lld rows (at most %d)", who, (long long)n, PG_CACHE_MAX_ROWS);
  return PG_OK;
}

// More than 64 KB of a workgroup's LDS have to be asked for.
static pg_status allow_lds(const void* kernel, size_t bytes) {
  if (bytes > 60000) PG_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  return PG_OK;
}

static PageCopy copy_of(const pg_cache* c) {
  const int64_t bytes = (int64_t)page_bytes(c);
  return PageCopy{(uint8_t*)c->k, (uint8_t*)c->v, bytes * c->n_pages, (uint32_t)bytes, c->layers};
}
// workgroups for the copies of at most `copies` pages
static int copy_blocks(const pg_cache* c, int64_t copies) {
  const int64_t pieces = ((int64_t)page_bytes(c) + COPY_PIECE - 1) / COPY_PIECE;
  const int64_t items = copies * c->layers * 2 * pieces;
  return (int)(items < MAX_COPY_BLOCKS ? items : MAX_COPY_BLOCKS);
}

}  // namespace pg

using namespace pg;

extern "C" pg_status pg_cache_clear(const pg_cache* c, void* stream) {
  PG_TRY(check_cache(c, false, "pg_cache_clear"));
  cache_clear_kernel<<<dim3((unsigned)((c->n_pages + 255ll) / 256)), dim3(256), 0, (hipStream_t)stream>>>(c->refs, c->n_pages, c->status);
  PG_LAUNCH_CHECK("cache_clear_kernel");
  return PG_OK;
}

extern "C" pg_status pg_cache_reserve(const pg_cache* c, int32_t* table, const int32_t* lens, const int32_t* add, int32_t* lens_out,
                                      int32_t n_rows, void* stream) {
  PG_TRY(check_cache(c, false, "pg_cache_reserve"));
  PG_TRY(check_rows(n_rows, "pg_cache_reserve"));
  if (n_rows == 0) return PG_OK;
  if (!table || !lens || !add || !lens_out) return fail(PG_EINVAL, "pg_cache_reserve: null pointer");
  PG_TRY(allow_lds((const void*)cache_reserve_kernel, (size_t)n_rows * 2 * sizeof(int)));
  cache_reserve_kernel<<<dim3(1), dim3(PLAN_THREADS), (size_t)n_rows * 2 * sizeof(int), (hipStream_t)stream>>>(view_of(c), c->refs, table, lens,
                                                                                                          add, lens_out, n_rows);
  PG_LAUNCH_CHECK("cache_reserve_kernel");
  return PG_OK;
}

extern "C" pg_status pg_cache_append(const pg_cache* c, int32_t layer, const uint16_t* k_new, const uint16_t* v_new, int64_t token_stride,
                                     const int32_t* table, const int32_t* lens, const int32_t* cu, int32_t n_rows, int32_t n_tokens,
                                     void* stream) {
  PG_TRY(check_cache(c, true, "pg_cache_append"));
  if (layer < 0 || layer >= c->layers) return fail(PG_EINVAL, "pg_cache_append: layer %d of %d", layer, c->layers);
  if (n_rows < 0 || n_tokens < 0 || (!cu && n_tokens != n_rows))
    return fail(PG_EINVAL, "pg_cache_append: %d tokens for %d rows%s", n_tokens, n_rows, cu ? "" : " of one token each");
  if (n_rows == 0 || n_tokens == 0) return PG_OK;
  if (!k_new || !v_new || !table || !lens) return fail(PG_EINVAL, "pg_cache_append: null pointer");
  if (token_stride < (int64_t)c->heads * c->head_dim || token_stride % 8 || (((uintptr_t)k_new | (uintptr_t)v_new) & 15))
    return fail(PG_ESHAPE, "pg_cache_append: tokens must be 16-byte aligned, %lld elements apart", (long long)token_stride);
  const int64_t units = cu ? n_tokens / 16 + 2ll * n_rows : n_rows;
  const int64_t blocks = (units + 3) / 4 * c->heads;
  if (blocks >= 1 << 24) return fail(PG_ESHAPE, "pg_cache_append: %lld workgroups (a launch has room for 2^24 of 256 lanes)", (long long)blocks);
  AppendArgs a{};
  a.c = view_of(c);
  const size_t layer_bytes = page_bytes(c) * c->n_pages;
  a.k = (uint8_t*)c->k + layer * layer_bytes;
  a.v = (uint8_t*)c->v + layer * layer_bytes;
  a.k_scale = c->k_scale ? c->k_scale + (int64_t)layer * c->heads : nullptr;
  a.v_scale = c->v_scale ? c->v_scale + (int64_t)layer * c->heads : nullptr;
  a.k_new = k_new; a.v_new = v_new; a.token_stride = token_stride;
  a.table = table; a.lens = lens; a.cu = cu; a.refs = c->refs; a.n_rows = n_rows; a.n_tokens = n_tokens; a.units = (int)units;
  const dim3 grid((unsigned)blocks), block(256);
  hipStream_t s = (hipStream_t)stream;
  const bool f8 = c->dtype == PG_CACHE_E4M3;
  switch (c->head_dim) {
    case 32: f8 ? cache_append_kernel<32, true><<<grid, block, 0, s>>>(a) : cache_append_kernel<32, false><<<grid, block, 0, s>>>(a); break;
    case 64: f8 ? cache_append_kernel<64, true><<<grid, block, 0, s>>>(a) : cache_append_kernel<64, false><<<grid, block, 0, s>>>(a); break;
    default: f8 ? cache_append_kernel<128, true><<<grid, block, 0, s>>>(a) : cache_append_kernel<128, false><<<grid, block, 0, s>>>(a);
  }
  PG_LAUNCH_CHECK("cache_append_kernel");
  return PG_OK;
}

extern "C" int64_t pg_cache_scratch_ints(const pg_cache* c, int32_t n_rows) {
  if (!c || n_rows < 0 || c->n_pages < 0) return 0;
  const int64_t select = 4 + 4ll * n_rows, compact = 4 + 2 * ((int64_t)c->n_pages / 2 + 1) + c->n_pages;
  return select > compact ? select : compact;
}

extern "C" pg_status pg_cache_select(const pg_cache* c, const int32_t* table_in, const int32_t* lens_in, int32_t n_in, const int32_t* src,
                                     int32_t* table_out, int32_t* lens_out, int32_t n_out, int32_t* scratch, void* stream) {
  PG_TRY(check_cache(c, true, "pg_cache_select"));
  PG_TRY(check_rows(n_in, "pg_cache_select"));
  PG_TRY(check_rows(n_out, "pg_cache_select"));
  if (n_in == 0 && n_out == 0) return PG_OK;
  if (!scratch || (n_in && (!table_in || !lens_in)) || (n_out && (!src || !table_out || !lens_out)))
    return fail(PG_EINVAL, "pg_cache_select: null pointer");
  auto overlap = [](const void* p, int64_t a, const void* q, int64_t b) {
    return (uintptr_t)p < (uintptr_t)q + b * 4 && (uintptr_t)q < (uintptr_t)p + a * 4;
  };
  if (n_in && n_out && (overlap(table_in, (int64_t)n_in * c->width, table_out, (int64_t)n_out * c->width) || overlap(lens_in, n_in, lens_out, n_out)))
    return fail(PG_EINVAL, "pg_cache_select: the new rows overlap the old ones");
  if (n_out && (overlap(src, n_out, table_out, (int64_t)n_out * c->width) || overlap(src, n_out, lens_out, n_out)))
    return fail(PG_EINVAL, "pg_cache_select: the new rows overlap src");
  if ((uintptr_t)scratch & 7) return fail(PG_ESHAPE, "pg_cache_select: scratch must be 8-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  const SelectPlan plan = select_plan(scratch, n_in, n_out);
  PG_TRY(allow_lds((const void*)cache_select_plan_kernel, (size_t)n_in * 2 * sizeof(int)));
  cache_select_plan_kernel<<<dim3(1), dim3(PLAN_THREADS), (size_t)n_in * 2 * sizeof(int), s>>>(view_of(c), c->refs, table_in, lens_in, n_in, src,
                                                                                              lens_out, n_out, plan);
  PG_LAUNCH_CHECK("cache_select_plan_kernel");
  cache_select_apply_kernel<<<dim3((unsigned)(n_out + n_in + copy_blocks(c, n_out))), dim3(APPLY_THREADS), 0, s>>>(
      view_of(c), copy_of(c), c->refs, table_in, lens_in, n_in, src, table_out, lens_out, n_out, plan);
  PG_LAUNCH_CHECK("cache_select_apply_kernel");
  return PG_OK;
}

extern "C" pg_status pg_cache_compact(const pg_cache* c, int32_t* table, const int32_t* lens, int32_t n_rows, int32_t* scratch, void* stream) {
  PG_TRY(check_cache(c, true, "pg_cache_compact"));
  if (n_rows < 0) return fail(PG_EINVAL, "pg_cache_compact: %d rows", n_rows);
  if (n_rows > 1 << 23) return fail(PG_ESHAPE, "pg_cache_compact: %d rows", n_rows);
  if (!scratch || (n_rows && (!table || !lens))) return fail(PG_EINVAL, "pg_cache_compact: null pointer");
  hipStream_t s = (hipStream_t)stream;
  const CompactPlan plan = compact_plan(scratch, c->n_pages);
  cache_compact_plan_kernel<<<dim3(1), dim3(PLAN_THREADS), 0, s>>>(c->refs, c->n_pages, plan);
  PG_LAUNCH_CHECK("cache_compact_plan_kernel");
  cache_compact_apply_kernel<<<dim3((unsigned)(n_rows + copy_blocks(c, c->n_pages / 2 + 1))), dim3(APPLY_THREADS), 0, s>>>(view_of(c), copy_of(c), table, lens, n_rows,
                                                                                                                 plan);
  PG_LAUNCH_CHECK("cache_compact_apply_kernel");
  return PG_OK;
}

extern "C" pg_status pg_cache_check(const pg_cache* c, void* stream) {
  PG_TRY(check_cache(c, false, "pg_cache_check"));
  PG_HIP(hipStreamSynchronize((hipStream_t)stream));
  int32_t st[4] = {0, 0, 0, 0};
  PG_HIP(hipMemcpy(st, c->status, sizeof(st), hipMemcpyDeviceToHost));
  if (st[0] & CACHE_RANGE) return fail(PG_EINVAL, "the cache met an index, a length or a count out of range");
  if (st[0] & CACHE_FULL) return fail(PG_EWORKSPACE, "the cache had no page for a row (pool or table width exhausted)");
  return PG_OK;
}
