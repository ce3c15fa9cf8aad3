// Distributions and tokens out of logits (unison_kv_sample).
//
// A cluster of CTAs shares a row; CTA r has a run of the vocabulary in shared
// memory, each of its warps a run of that.  Entries are read once; everything
// after that is passes over shared memory.
//
// What is kept is a beginning of the order (larger logit first, then lower
// index) less what is below min-p, so it is known by its last entry: the cut.
//   1  A bound below what may be kept.  The threads' maxima are entries, too:
//      where their running count reaches k, or their running weight the goal of
//      top-p, lies at or below the cut.  Entries of up to (tail that top-p
//      leaves out) / vocab cannot reach it either, nor those below min-p.
//   2  The entries above the bound, a few dozen mostly, go into one list, are
//      compared one by one, and give the cut, the sum of the kept weights and the
//      token: no further pass, no further barrier.
//   3  Where the list is too long: a histogram of those entries by the exponent t,
//      of counts and of weights in three digits of 14 bits (32-bit sums of those
//      are exact).  The slot in which the running count or weight reaches its goal
//      is a list then, or is counted in slots of its own first.
// The passes take few operations an entry: 2^t (one instruction), its whole
// part in 2^-40 as two halves by four operations on pairs, 32-bit sums.
//
// Rows that this does not serve (infinite or NaN logits, a vocabulary beyond
// shared memory, hundreds of entries that nothing but the index tells apart) go
// through `general`: digits of the logits' bits from the top, 256 at a time.
//
// Bound by latency: the loads of a row take 4 us, each exchange between the
// cluster's CTAs 1 to 2, and a row three to five of them, while one row's 64 KB a CTA
// leave room for three CTAs on a multiprocessor.  One row of 32,000: 9 us.  128
// rows of 128,000 in 32 bits (65 MB, 10 us at the copy rate), 57 at a time: 58 to 66 us, 13
// for a row with a short list and 38 with a histogram (6 of them).  512 rows of
// 64,000 in bf16 to distributions (131 MB, 19 us at the copy rate): 41 to 46 us.  A row
// that stays in the L2 cache instead, all rows at a time: 112 and 66 us, because
// the slowest rows are longer on their way.  CTAs of 512 threads, two on a
// multiprocessor: 98 and 86.
#include <cooperative_groups.h>

#include <type_traits>

#include "kv_tc.cuh"

namespace unison {
namespace {

namespace cg = cooperative_groups;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBins = 256;
constexpr int kSlots = 256;  // of the histogram: a thread's each
constexpr int kList = 256;   // entries that are compared one by one
static_assert(kBins <= kThreads && kSlots == kThreads && kList <= kThreads, "a thread for each");

template <typename T>
__device__ __forceinline__ float number(T x) {
  return KvType<T>::to_float(x);
}
template <>
__device__ __forceinline__ float number<float>(float x) {
  return x;
}
__device__ __forceinline__ void store_number(float *p, float x) { *p = x; }
__device__ __forceinline__ void store_number(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }
__device__ __forceinline__ void store_number(__half *p, float x) { *p = __float2half_rn(x); }
// NaN counts as -inf, -0 as 0.
__device__ __forceinline__ float logit(float x) { return x != x ? -INFINITY : __fadd_rn(x, 0.f); }
// Bits in the order of the numbers, and back.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k); }

struct Weigher {
  float top, factor;
  // floor(2^40 2^((x - m) c)).  (A product 0 * inf, of x = m or of x = -inf, is decided before.)
  __device__ __forceinline__ int64_t operator()(float x) const {
    if (x == -INFINITY) return 0;
    if (x == top) return 1ll << 40;
    return (int64_t)__fmul_rn(fmaxf(exp2f(__fmul_rn(__fsub_rn(x, top), factor)), 0.f), 1099511627776.f);  // (NaN: 0)
  }
};

// floor(P w) for P a multiple of 2^-24 and w below 2^63.
__device__ __forceinline__ int64_t times(float p, int64_t w) {
  const int64_t u = (int64_t)(p * 16777216.f);
  return u * (w >> 24) + ((u * (w & 0xFFFFFF)) >> 24);
}

// 1 / s for a whole number s, as two numbers: the first quotient, and what its
// remainder adds.  Each of the roundings is 2^-47 of it at most, so w times it is
// the quotient w / s rounded once, to 2^-24 (1 + 2^-20).
struct Inverse {
  float high, low;
  __device__ __forceinline__ explicit Inverse(int64_t s) {
    const float a = (float)s, b = (float)(s - (int64_t)a);
    high = __fdiv_rn(1.f, a);
    low = __fmul_rn(fmaf(-high, b, fmaf(-high, a, 1.f)), high);
  }
  __device__ __forceinline__ float operator()(float w) const { return fmaf(w, high, __fmul_rn(w, low)); }
};

struct Shared {
  unsigned long long pushed[2][kMaxCluster];  // one number of every CTA, in two sets by turns
  unsigned long long warp[kWarps];
  union {
    struct {
      unsigned long long sums[kBins];
      uint32_t counts[kBins];
    };
    uint4 slots[kSlots];  // entries, and the digits of their weights from the top
  };
  int64_t part[33];
  int64_t above;
  int64_t found_above;
  uint32_t found_count;
  int bin, at;
};

// A row by digits, read from global memory in every pass.  By all CTAs of a
// cluster, in step.
template <typename T>
__device__ __noinline__ void general(const unison_kv_sample_args &a, Shared &sh) {
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const int row = blockIdx.x / ctas, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int V = a.vocab;
  const T *const x = static_cast<const T *>(a.logits) + row * a.logits_row;
  const float temperature = a.temperature_row ? a.temperature_row[row] : a.temperature;
  const float top_p = a.top_p_row ? a.top_p_row[row] : a.top_p;
  const float min_p = a.min_p_row ? a.min_p_row[row] : a.min_p;
  const int top_k = a.top_k_row ? a.top_k_row[row] : a.top_k;
  const bool greedy = !(temperature > 0.f);
  cluster.sync();  // every CTA has begun: its shared memory may be written to

  // this warp's run of the vocabulary
  const int span = (V + ctas * kWarps * 32 - 1) / (ctas * kWarps * 32) * 32;
  const int64_t begin64 = (int64_t)(rank * kWarps + warp) * span;
  const int begin = (int)min(begin64, (int64_t)V), end = (int)min(begin64 + span, (int64_t)V);
  auto each = [&](auto f) {
    for (int i = begin + lane; i < end; i += 32) f(logit(number<T>(x[i])), i);
  };

  int turn = 0;
  // All CTAs' values (of thread 0), by CTA; the caller reduces them.
  auto push = [&](unsigned long long mine) -> const unsigned long long * {
    const int slot = turn++ & 1;  // a CTA that is one turn ahead writes the other one
    if (tid == 0)
      for (int c = 0; c < ctas; c++) *cluster.map_shared_rank(&sh.pushed[slot][rank], c) = mine;
    cluster.sync();
    return sh.pushed[slot];
  };
  auto sum_warps = [&](unsigned long long mine) -> unsigned long long {  // leaves the warps' sums in sh.warp
#pragma unroll
    for (int d = 16; d; d >>= 1) mine += __shfl_xor_sync(~0u, mine, d);
    __syncthreads();
    if (lane == 0) sh.warp[warp] = mine;
    __syncthreads();
    unsigned long long all = 0;
    for (int w = 0; w < kWarps; w++) all += sh.warp[w];
    return all;
  };
  auto sum_all = [&](unsigned long long mine) -> int64_t {
    const unsigned long long *p = push(sum_warps(mine));
    unsigned long long all = 0;
    for (int c = 0; c < ctas; c++) all += p[c];
    return (int64_t)all;
  };

  // ---- the largest logit and its first index, as one number
  unsigned long long best = 0;
  each([&](float y, int i) {
    const unsigned long long me = (unsigned long long)key_of(y) << 32 | (uint32_t)~i;
    best = me > best ? me : best;
  });
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const unsigned long long o = __shfl_xor_sync(~0u, best, d);
    best = o > best ? o : best;
  }
  if (lane == 0) sh.warp[warp] = best;
  __syncthreads();
  for (int w = 0; w < kWarps; w++) best = sh.warp[w] > best ? sh.warp[w] : best;
  {
    const unsigned long long *p = push(best);
    for (int c = 0; c < ctas; c++) best = p[c] > best ? p[c] : best;
  }
  const int first = (int)~(uint32_t)best;
  const uint32_t top_key = (uint32_t)(best >> 32);
  Weigher weigh;
  weigh.top = of_key(top_key);
  weigh.factor = __fdiv_rn(1.4426950408889634f, temperature);
  const bool none = weigh.top == -INFINITY;

  // ---- the cut: kept are entries above its key, and `ties` of those equal to it
  uint32_t cut = 0;
  int64_t ties = INT64_MAX, equal = INT64_MAX;
  // The entry at which the running count (or weight) reaches `goal` >= 1.
  auto select = [&](bool by_weight, int64_t goal) {
    uint32_t digits = 0;
    int64_t above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < kBins) sh.counts[tid] = 0, sh.sums[tid] = 0;
      __syncthreads();
      each([&](float y, int) {
        const uint32_t k = key_of(y);
        if (((uint64_t)(k ^ digits) >> (shift + 8)) != 0) return;
        atomicAdd(&sh.counts[k >> shift & 255], 1u);
        if (by_weight) atomicAdd(&sh.sums[k >> shift & 255], (unsigned long long)weigh(y));
      });
      cluster.sync();
      int64_t mine = 0;
      uint32_t count = 0;
      if (tid < kBins)
        for (int c = 0; c < ctas; c++) {
          const uint32_t n = *cluster.map_shared_rank(&sh.counts[255 - tid], c);
          count += n;
          mine += by_weight ? (int64_t)*cluster.map_shared_rank(&sh.sums[255 - tid], c) : (int64_t)n;
        }
      if (tid == 0) sh.bin = 0, sh.found_above = above, sh.found_count = 0;
      int64_t all;
      const int64_t before = above + block_scan(mine, sh.part, all);
      if (tid < kBins && before < goal && goal <= before + mine) {
        sh.bin = 255 - tid;
        sh.found_above = before;
        sh.found_count = count;
      }
      cluster.sync();  // every CTA has read the histograms
      digits |= (uint32_t)sh.bin << shift;
      above = sh.found_above;
      equal = sh.found_count;
    }
    cut = digits;
    const int64_t w = by_weight ? weigh(of_key(cut)) : 1;
    ties = w > 0 ? (goal - above + w - 1) / w : equal;
  };
  if (greedy || none) {
    cut = top_key;
    ties = 1;
    equal = INT64_MAX;
  } else {
    if (top_k > 0 && top_k < V) select(false, top_k);
    if (top_p < 1.f) {
      uint64_t mine = 0;
      each([&](float y, int) { mine += key_of(y) > cut ? weigh(y) : 0; });
      int64_t w = sum_all(mine);
      if (cut) w += ties * weigh(of_key(cut));  // (no logit has key 0)
      select(true, max(times(fmaxf(top_p, 0.f), w), (int64_t)1));
    }
  }
  // the last index of those equal to the cut that is kept
  int last = INT_MAX;
  if (greedy || none) {
    last = first;
  } else if (ties < equal) {
    unsigned long long mine = 0;
    each([&](float y, int) { mine += key_of(y) == cut; });
    const unsigned long long here = sum_warps(mine);
    const unsigned long long *p = push(here);
    int64_t before = 0;
    for (int c = 0; c < rank; c++) before += p[c];
    if (before < ties && ties <= before + (int64_t)here) {  // in this CTA
      int w = 0;
      while (before + (int64_t)sh.warp[w] < ties) before += sh.warp[w++];
      if (warp == w) {
        for (int i = begin; i < end; i += 32) {
          const bool is = i + lane < end && key_of(logit(number<T>(x[i + lane]))) == cut;
          const uint32_t found = __ballot_sync(~0u, is);
          if (is && before + __popc(found & ((2u << lane) - 1)) == ties)
            for (int c = 0; c < ctas; c++) *cluster.map_shared_rank(&sh.at, c) = i + lane;
          before += __popc(found);
        }
      }
    }
    cluster.sync();
    last = sh.at;
  }
  const int64_t least = (int64_t)(fminf(fmaxf(min_p, 0.f), 1.f) * 1099511627776.f);
  auto kept = [&](float y, int i) -> int64_t {  // its weight, or 0
    const uint32_t k = key_of(y);
    if (k < cut || (k == cut && i > last)) return 0;
    const int64_t w = weigh(y);
    return w >= least ? w : 0;
  };

  // ---- the kept weights' sum, the distribution, the token
  unsigned long long mine = 0;
  each([&](float y, int i) { mine += kept(y, i); });
  const unsigned long long here = sum_warps(mine);
  const unsigned long long *p = push(here);
  int64_t total = 0, before = 0;
  for (int c = 0; c < ctas; c++) {
    if (c < rank) before += p[c];
    total += p[c];
  }
  if (a.p) {
    const Inverse of_sum(max(total, (int64_t)1));
    const int64_t at = row * a.p_row;
    each([&](float y, int i) {
      const float v = of_sum((float)kept(y, i));
      if (a.p_dtype == UNISON_KV_FP32)
        static_cast<float *>(a.p)[at + i] = v;
      else if (a.p_dtype == UNISON_KV_BF16)
        static_cast<__nv_bfloat16 *>(a.p)[at + i] = __float2bfloat16_rn(v);
      else
        static_cast<__half *>(a.p)[at + i] = __float2half_rn(v);
    });
  }
  if (a.token) {
    if (total <= 0) {
      if (rank == 0 && tid == 0) a.token[row] = -1;
    } else {
      const int64_t goal = times(fminf(fmaxf(a.u[row], 0.f), 1.f - 1.f / 16777216.f), total);
      if (before <= goal && goal < before + (int64_t)here) {
        int w = 0;
        while (before + (int64_t)sh.warp[w] <= goal) before += sh.warp[w++];
        if (warp == w) {
          for (int i = begin; i < end; i += 32) {
            const int64_t one = i + lane < end ? kept(logit(number<T>(x[i + lane])), i + lane) : 0;
            int64_t sum = one;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
              const int64_t o = __shfl_up_sync(~0u, sum, d);
              if (lane >= d) sum += o;
            }
            if (before + sum - one <= goal && goal < before + sum) a.token[row] = i + lane;
            before += __shfl_sync(~0u, sum, 31);
          }
        }
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_general_kernel(const unison_kv_sample_args a) {
  follow_last_kernel();
  __shared__ Shared sh;
  general<T>(a, sh);
}

// ------------------------------------------------------- rows in shared memory --
constexpr float kLeast = -41.f;  // below 2^-40 a weight is 0

struct FastShared {
  Shared g;
  unsigned long long list[kList], weight[kList];  // entries: key, ~index; larger: earlier in the order
  unsigned long long own[kList];                  // this CTA's
  unsigned long long cut;
  int64_t cut_total, above, above_weight;
  int own_count[3], slot;
  uint32_t count;
};

__device__ __forceinline__ uint64_t fma_pair_rz(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// floor(2^40 d) of two numbers 0 <= d <= 1, each as 2^20 high + low: adding 2^23
// and rounding towards zero leaves the whole part in the low bits of a float.
// high and low get 2^23's own bits on top, kBias each.
constexpr uint32_t kBias = 0x4B000000u;
__device__ __forceinline__ void fixed_pair(uint64_t d, uint32_t (&high)[2], uint32_t (&low)[2]) {
  const uint64_t scale = pair(1048576.f, 1048576.f), whole = pair(8388608.f, 8388608.f);
  const uint64_t h = fma_pair_rz(d, scale, whole);
  const uint64_t rest = fma_pair(d, scale, fma_pair(h, pair(-1.f, -1.f), whole));  // exact, below 1
  const uint64_t l = fma_pair_rz(rest, scale, whole);
  high[0] = (uint32_t)h, high[1] = (uint32_t)(h >> 32);
  low[0] = (uint32_t)l, low[1] = (uint32_t)(l >> 32);
}
// Sum of such numbers, up to 4,095.
struct FixedSum {
  uint32_t high = 0, low = 0;
  __device__ __forceinline__ void add(uint64_t d) {
    uint32_t h[2], l[2];
    fixed_pair(d, h, l);
    high += h[0] + h[1];
    low += l[0] + l[1];
  }
  __device__ __forceinline__ int64_t sum(uint32_t n) const {  // of n numbers
    return ((int64_t)(high - n * kBias) << 20) + (low - n * kBias);
  }
};

// The larger number of each half; NaN if one of the two is.
template <typename T>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (sizeof(T) == 4)
    asm("max.NaN.f32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else if constexpr (std::is_same<T, __half>::value)
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// 16 bytes of a row as numbers.
template <typename T>
struct Piece {
  static constexpr int kN = 16 / sizeof(T);
  // -inf, once or twice
  static constexpr uint32_t kLowest = sizeof(T) == 4                       ? 0xFF800000u
                                      : std::is_same<T, __half>::value ? 0xFC00FC00u
                                                                           : 0xFF80FF80u;
  static __device__ __forceinline__ uint32_t halves(const uint4 &v) {  // the largest, for `largest`
    return larger<T>(larger<T>(v.x, v.y), larger<T>(v.z, v.w));
  }
  static __device__ __forceinline__ float largest(uint32_t h) {  // NaN if anything is
    if constexpr (sizeof(T) == 4) return __uint_as_float(h);
    const T *e = reinterpret_cast<const T *>(&h);
    return __uint_as_float(larger<float>(__float_as_uint(number<T>(e[0])), __float_as_uint(number<T>(e[1]))));
  }
  static __device__ __forceinline__ void get(const uint4 &v, float (&x)[kN]) {
    const T *e = reinterpret_cast<const T *>(&v);
#pragma unroll
    for (int i = 0; i < kN; i++) x[i] = number<T>(e[i]);
  }
};
// The cluster's barrier.  Arriving with what this thread, and those that it has
// met at the CTA's barriers, wrote before, takes until that has been seen to: so one
// warp does it for its CTA.
__device__ __forceinline__ void cluster_arrive(bool hands_on) {
  if (hands_on)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  else
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_meet(bool hands_on) {
  cluster_arrive(hands_on);
  cluster_wait();
}
__device__ __forceinline__ void cluster_sync(int warp) {
  __syncthreads();
  cluster_meet(warp == 0);
}

// An entry of a list, as one of the threads that compare it sees it.
struct Compared {
  unsigned long long entry;
  int64_t weight, weight_before;  // its own, and of those before it in the order
  int before;                     // how many those are
  int at, share, shares;          // its place, this thread's share of the comparisons
  bool real;                      // the first of its threads
  template <typename I>
  __device__ __forceinline__ I sum(I x) const {  // of its threads'
    for (int d = 1; d < shares; d <<= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
  }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 3) sample_kernel(const unison_kv_sample_args a, int span, int ahead) {
  follow_last_kernel();
  constexpr int kN = Piece<T>::kN, kStep = 32 * kN;
  constexpr int kFlight = 8;  // loads of a thread on their way
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ FastShared sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const int row = blockIdx.x / ctas, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int V = a.vocab;
  const float temperature = a.temperature_row ? a.temperature_row[row] : a.temperature;
  const float top_p = a.top_p_row ? a.top_p_row[row] : a.top_p;
  const float min_p = a.min_p_row ? a.min_p_row[row] : a.min_p;
  const int top_k = a.top_k_row ? a.top_k_row[row] : a.top_k;
  const bool greedy = !(temperature > 0.f);
  cluster_arrive(false);  // every CTA has begun: its shared memory may be written to
  sh.g.slots[tid] = make_uint4(0, 0, 0, 0);
  if (tid < 3) sh.own_count[tid] = 0;
  if (tid == 0) sh.count = 0;

  // ---- this warp's run: pieces of 16 bytes as they lie in memory, so the row
  // begins `shift` entries into its first piece; -inf before it and behind it
  const uintptr_t address = reinterpret_cast<uintptr_t>(static_cast<const T *>(a.logits) + row * a.logits_row);
  const int shift = (int)(address & 15) / (int)sizeof(T), end = V + shift;
  const T *const from = reinterpret_cast<const T *>(address & ~(uintptr_t)15);
  const int64_t begin64 = (int64_t)(rank * kWarps + warp) * span;
  const int begin = (int)min(begin64, (int64_t)INT_MAX / 2);
  T *const data = reinterpret_cast<T *>(smem) + warp * span;
  uint32_t high = Piece<T>::kLowest;  // the largest so far, NaN if anything was
  const int last = (end - 1) / kN * kN;
  const uint32_t lowest_bits = Piece<T>::kLowest;
  const T lowest = *reinterpret_cast<const T *>(&lowest_bits);
  for (int i0 = lane * kN; i0 < span; i0 += kFlight * kStep) {
    uint4 v[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; u++)
      v[u] = __ldg(reinterpret_cast<const uint4 *>(from + min(begin + i0 + u * kStep, last)));
#pragma unroll
    for (int u = 0; u < kFlight; u++) {
      const int i = i0 + u * kStep, e = begin + i;
      if (e < shift || e + kN > end) {
        T *x = reinterpret_cast<T *>(&v[u]);
#pragma unroll
        for (int j = 0; j < kN; j++)
          if (e + j < shift || e + j >= end) x[j] = lowest;
      }
      if (i < span) {
        *reinterpret_cast<uint4 *>(data + i) = v[u];
        high = larger<T>(high, Piece<T>::halves(v[u]));
      }
    }
  }
  const float mine = Piece<T>::largest(high);
  // The row that will have this place next is on its way into the L2 cache meanwhile
  // (512 rows of 64,000 in bf16: 43 us, 45 without).
  if (lane == 0 && row + ahead < a.n_rows) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(static_cast<const T *>(a.logits) + (row + ahead) * a.logits_row);
    const int64_t elements = min((int64_t)span, (int64_t)V + (int64_t)(at & 15) / (int)sizeof(T) - begin64);
    const int64_t bytes = elements * (int)sizeof(T);
    if (bytes > 0)
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"((at & ~(uintptr_t)15) + begin64 * sizeof(T)),
                   "r"((uint32_t)((bytes + 15) & ~15ll))
                   : "memory");
  }
  cluster_wait();

  int turn = 0;
  auto push = [&](unsigned long long one) -> const unsigned long long * {
    const int set = turn++ & 1;  // a CTA that is one turn ahead writes the other one
    if (tid < ctas) *cluster.map_shared_rank(&sh.g.pushed[set][rank], tid) = one;
    cluster_meet(warp == 0);
    return sh.g.pushed[set];
  };
  auto sum_warps = [&](unsigned long long one) -> unsigned long long {  // leaves the warps' sums in sh.g.warp
#pragma unroll
    for (int d = 16; d; d >>= 1) one += __shfl_xor_sync(~0u, one, d);
    __syncthreads();
    if (lane == 0) sh.g.warp[warp] = one;
    __syncthreads();
    unsigned long long all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; w++) all += sh.g.warp[w];
    return all;
  };
  auto each = [&](auto f) {  // f(pair's two logits, place of the first in the warp's run)
#pragma unroll 2
    for (int i = lane * kN; i < span; i += kStep) {
      float x[kN];
      Piece<T>::get(*reinterpret_cast<const uint4 *>(data + i), x);
#pragma unroll
      for (int j = 0; j < kN; j += 2) f(x[j], x[j + 1], i + j);
    }
  };

  // The same of pieces that have a logit of at least `from`.
  auto each_from = [&](float from, auto f) {
#pragma unroll 4
    for (int i = lane * kN; i < span; i += kStep) {
      const uint4 v = *reinterpret_cast<const uint4 *>(data + i);
      if (Piece<T>::largest(Piece<T>::halves(v)) < from) continue;
      float x[kN];
      Piece<T>::get(v, x);
#pragma unroll
      for (int j = 0; j < kN; j += 2) f(x[j], x[j + 1], i + j);
    }
  };

  // ---- the largest logit
  unsigned long long best = (unsigned long long)key_of(logit(mine)) << 1 | (mine != mine);
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const unsigned long long o = __shfl_xor_sync(~0u, best, d);
    best = max(best, o) | ((best | o) & 1);
  }
  if (lane == 0) sh.g.warp[warp] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; w++) best = max(best, sh.g.warp[w]) | ((best | sh.g.warp[w]) & 1);
  {
    const unsigned long long *p = push(best);
    for (int c = 0; c < ctas; c++) best = max(best, p[c]) | ((best | p[c]) & 1);
  }
  const float top = of_key((uint32_t)(best >> 1));
  const float factor = greedy ? 1.f : __fdiv_rn(1.4426950408889634f, temperature);
  if ((best & 1) || !isfinite(top) || (!greedy && !(factor > 0.f && factor < INFINITY))) {
    general<T>(a, sh.g);
    return;
  }
  const uint64_t tops = pair(-top, -top), factors = pair(factor, factor);
  auto exponents = [&](float x, float y) -> uint64_t { return mul_pair(add_pair(pair(x, y), tops), factors); };
  auto raise = [&](uint64_t t) -> uint64_t {
    float x, y;
    unpair(t, x, y);
    return pair(exp2_fast(x), exp2_fast(y));
  };
  auto exponent = [&](float x) -> float { return __fmul_rn(__fsub_rn(x, top), factor); };
  auto weigh = [&](float x) -> int64_t { return (int64_t)__fmul_rn(exp2_fast(exponent(x)), 1099511627776.f); };

  // f(how many CTAs, known when it is compiled), so that every CTA's words can be
  // asked for at once and none of the loads has a condition.  (With loads of c < ctas
  // and zeros else, what was loaded was right, but in 2% of the rows of one CTA with a
  // histogram the sums of some warps came out larger by their slots' counts.)
  auto by_ctas = [&](auto f) {
    static_assert(kMaxCluster == 8, "powers of two up to it");
    if (ctas == 1)
      f(std::integral_constant<int, 1>());
    else if (ctas == 2)
      f(std::integral_constant<int, 2>());
    else if (ctas == 4)
      f(std::integral_constant<int, 4>());
    else
      f(std::integral_constant<int, 8>());
  };

  // ---- lists: every CTA's own entries, read by those that want them all.  A list
  // is written again when a barrier has told that everyone has read the last one
  // (of one that was too long nobody has).
  auto enlist = [&](int which, float x, int i) {
    if (*const_cast<volatile int *>(&sh.own_count[which]) > kList) return;  // too long already
    const int to = atomicAdd(&sh.own_count[which], 1);
    if (to < kList)
      sh.own[to] = (unsigned long long)key_of(__fadd_rn(x, 0.f)) << 32 | (uint32_t)~(begin + i - shift);
  };
  int counts[kMaxCluster];
  auto gather = [&](int which) -> int {  // the length of all, and of each in `counts`
    cluster_sync(warp);
    int all = 0;
#pragma unroll
    for (int c = 0; c < kMaxCluster; c++) counts[c] = 0;
    by_ctas([&](auto n) {
      if constexpr (n.value == 1) {
        counts[0] = sh.own_count[which];
      } else {
#pragma unroll
        for (int c = 0; c < n.value; c++) counts[c] = *cluster.map_shared_rank(&sh.own_count[which], c);
      }
    });
#pragma unroll
    for (int c = 0; c < kMaxCluster; c++) all += min(counts[c], kList + 1);
    return all;
  };
  auto entry_of = [&](int count) -> unsigned long long {  // entry `tid` of all
    int c = 0, at = tid;
#pragma unroll
    for (int i = 0; i < kMaxCluster - 1; i++) {
      const bool on = c == i && at >= counts[i];
      at -= on ? counts[i] : 0;
      c += on;
    }
    if (ctas == 1) return tid < count ? sh.own[tid] : 0;
    const unsigned long long one = cluster.map_shared_rank(sh.own, min(c, ctas - 1))[min(at, kList - 1)];
    return tid < count ? one : 0;
  };

  // The list's entries, each compared with all others, by as many threads as there
  // are for one: how many are earlier in the order, and their weights.
  auto compare = [&](int count) -> Compared {
    const unsigned long long one = entry_of(count);
    if (tid < count) {
      sh.list[tid] = one;
      sh.weight[tid] = weigh(of_key((uint32_t)(one >> 32)));
    }
    __syncthreads();
    Compared c;
    c.shares = count <= kThreads / 8 ? 8 : count <= kThreads / 4 ? 4 : count <= kThreads / 2 ? 2 : 1;
    c.at = tid / c.shares;
    c.share = tid % c.shares;
    const bool there = c.at < count;
    c.real = there && c.share == 0;
    c.entry = there ? sh.list[c.at] : 0;
    c.weight = there ? (int64_t)sh.weight[c.at] : 0;
    int n = 0;
    int64_t w = 0;
#pragma unroll 4
    for (int j = c.share; j < count; j += c.shares) {
      const bool earlier = sh.list[j] > c.entry;
      n += earlier;
      w += earlier ? sh.weight[j] : 0;
    }
    c.before = c.sum(n);
    c.weight_before = c.sum(w);
    return c;
  };

  // ---- the limits
  const bool by_count = greedy || (top_k > 0 && top_k < V), by_weight = !greedy && top_p < 1.f;
  const int64_t most = greedy ? 1 : top_k;
  // (least as a number: 2^40 of it is whole)
  const float least = greedy ? 0.f : floorf(fminf(fmaxf(min_p, 0.f), 1.f) * 1099511627776.f) * (1.f / 1099511627776.f);
  const uint32_t numbers = span / 32;  // of a lane
  unsigned long long cut = 0;          // kept are entries (key, ~index) from it on upwards; 0: all
  int64_t cut_total = 0, goal = 0;     // their weights; what the running weight has to reach
  bool give_up = false;

  float low = kLeast, scale = (kSlots - 0.5f) / -kLeast, low_logit = -INFINITY;
  int level = 0, chosen = 0;
  float low2 = 0.f, scale2 = 0.f;
  auto slot_of = [&](float t) { return min((int)((t - low) * scale), kSlots - 1); };
  auto slot2_of = [&](float t) { return min(max((int)((t - low2) * scale2), 0), kSlots - 1); };
  // Entries of the histogram at this level: the slot, or -1.
  auto place = [&](float t) -> int {
    if (!(t >= low)) return -1;
    const int b = slot_of(t);
    return level == 0 ? b : b == chosen ? slot2_of(t) : -1;
  };
  auto count_in = [&](int slot, uint32_t high, uint32_t lo) {
    atomicAdd(&sh.g.slots[slot].x, 1u);
    atomicAdd(&sh.g.slots[slot].y, high >> 8);
    atomicAdd(&sh.g.slots[slot].z, (high << 6 | lo >> 14) & 0x3FFFu);
    atomicAdd(&sh.g.slots[slot].w, lo & 0x3FFFu);
  };
  // This thread's slot, from the top, in all CTAs.
  auto totals = [&](int64_t &n, int64_t &w) {
    n = w = 0;
    by_ctas([&](auto count) {
      uint4 v[count.value];
      const uint4 *const mine = &sh.g.slots[kSlots - 1 - tid];
      if constexpr (count.value == 1) {
        v[0] = *mine;
      } else {
#pragma unroll
        for (int c = 0; c < count.value; c++) v[c] = *cluster.map_shared_rank(mine, c);
      }
#pragma unroll
      for (int c = 0; c < count.value; c++) {
        n += v[c].x;
        w += ((int64_t)v[c].y << 28) + ((int64_t)v[c].z << 14) + v[c].w;
      }
    });
  };

  // ---- what is kept, and the distribution
  // 2^t of a kept entry, else 0; index: its place in the vocabulary
  auto kept = [&](float x, int index) -> float {
    const float cut_logit = cut ? of_key((uint32_t)(cut >> 32)) : -INFINITY;
    if (x < cut_logit || (cut && x == cut_logit && index > (int)~(uint32_t)cut)) return 0.f;
    const float d = exp2_fast(exponent(x));
    return d >= least ? d : 0.f;
  };
  float least_logit = -INFINITY;  // no logit below it is kept
  auto share = [&](float x, int index, const Inverse &of_sum) -> float {
    const float d = kept(x, index);
    return d > 0.f ? of_sum(truncf(__fmul_rn(d, 1099511627776.f))) : 0.f;
  };
  auto put = [&](auto *p, const Inverse &of_sum) {
    using P = typename std::remove_pointer<decltype(p)>::type;
    p += row * a.p_row - shift;  // as the row's pieces lie
    if constexpr (sizeof(P) == sizeof(T)) {
      if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll 2
        for (int i = lane * kN; i < span; i += kStep) {
          const int e = begin + i;
          if (e >= end) break;
          const uint4 all = *reinterpret_cast<const uint4 *>(data + i);
          const bool whole = e >= shift && e + kN <= end;
          if (whole && Piece<T>::largest(Piece<T>::halves(all)) < least_logit) {
            *reinterpret_cast<uint4 *>(p + e) = make_uint4(0, 0, 0, 0);
            continue;
          }
          float x[kN];
          Piece<T>::get(all, x);
#pragma unroll
          for (int j = 0; j < kN; j++) x[j] = share(x[j], e + j - shift, of_sum);
          if (whole) {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
              if constexpr (sizeof(P) == 4)
                v[j] = __float_as_uint(x[j]);
              else
                v[j] = KvType<P>::pack(x[2 * j], x[2 * j + 1]);
            }
            *reinterpret_cast<uint4 *>(p + e) = make_uint4(v[0], v[1], v[2], v[3]);
          } else {
#pragma unroll
            for (int j = 0; j < kN; j++)
              if (e + j >= shift && e + j < end) store_number(p + e + j, x[j]);
          }
        }
        return;
      }
    }
#pragma unroll 4
    for (int i = lane; i < span; i += 32) {
      const int e = begin + i;
      if (e >= shift && e < end) store_number(p + e, share(number<T>(data[i]), e - shift, of_sum));
    }
  };
  auto put_all = [&](int64_t total) {
    const Inverse of_sum(total);
    least_logit = cut ? of_key((uint32_t)(cut >> 32)) : least > 0.f ? low_logit : -INFINITY;
    if (a.p_dtype == UNISON_KV_FP32)
      put(static_cast<float *>(a.p), of_sum);
    else if (a.p_dtype == UNISON_KV_BF16)
      put(static_cast<__nv_bfloat16 *>(a.p), of_sum);
    else
      put(static_cast<__half *>(a.p), of_sum);
  };

  // ---- a bound below what may be kept
  if (greedy) {
    low = -1e-3f;  // (the largest logit is at 0, and any other may be kept out later)
  } else if (by_count || by_weight) {
    const float t = exponent(mine);
    if (t >= kLeast) {
      const int64_t w = weigh(mine);
      count_in(slot_of(t), (uint32_t)(w >> 20), (uint32_t)w & 0xFFFFFu);
    }
    int64_t weight = 0;
    if (by_count) {
      cluster_sync(warp);
    } else {
      FixedSum s;
      each([&](float x, float y, int) { s.add(raise(exponents(x, y))); });
      const unsigned long long *p = push(sum_warps(s.sum(numbers)));
      for (int c = 0; c < ctas; c++) weight += p[c];
      goal = max(times(fmaxf(top_p, 0.f), weight), (int64_t)1);
    }
    int64_t n, w;
    totals(n, w);
    const int64_t count = n;
    if (tid == 0) sh.slot = -1;
    // (2,048 threads' maxima at most: 12 bits, and their weights 52)
    static_assert(kMaxCluster * kThreads <= 2048, "one scan for both");
    unsigned long long all;
    const unsigned long long both =
        block_scan((unsigned long long)n << 52 | (unsigned long long)w,
                   reinterpret_cast<unsigned long long *>(sh.g.part), all);
    const int64_t maxima = (int64_t)(both >> 52) + count;
    const int64_t before = by_count ? (int64_t)(both >> 52) : (int64_t)(both & ((1ull << 52) - 1));
    const int64_t wanted = by_count ? most : goal;
    if (!by_count) n = w;
    if (before < wanted && wanted <= before + n) sh.slot = kSlots - 1 - tid;
    __syncthreads();
    // (less than the slot's edge by more than its rounding)
    if (sh.slot >= 0) low = fmaxf(low, kLeast + sh.slot / scale - 0.001f);
    // The cut and the entries behind it sum to more than weight - goal, so the cut's
    // weight, the largest of theirs, is above a V-th of that, and a whole number above 0.
    // (The roundings of 2^t, the quotient and the logarithm are far below the 0.01.)
    if (!by_count) low = fmaxf(low, log2f(fmaxf((float)(weight - goal) / (float)V, 1.f)) - 40.01f);
    // how many of them lie in whole slots above the bound
    if (min((int)((low - kLeast) * scale), kSlots - 1) == kSlots - 2 - tid) sh.count = (uint32_t)maxima;
  }
  if (least > 0.f && !(by_count && by_weight)) low = fmaxf(low, log2f(least) - 0.01f);
  // a logit below which no exponent reaches `low` (the difference's, quotient's and product's rounding allowed for)
  const float reach = low / factor;
  low_logit = top + reach - (fabsf(top) - reach) * 9.5e-7f;
  __syncthreads();

  // (min-p alone: the list tells the token, but the sum of what is kept is had without)
  if ((by_count || by_weight || (low > kLeast && a.token)) && sh.count <= kList && !(by_count && most > kList)) {
    // ---- the entries above it
    each_from(low_logit, [&](float x, float y, int i) {
      const float t[2] = {exponent(x), exponent(y)};
#pragma unroll
      for (int j = 0; j < 2; j++)
        if (t[j] >= low) enlist(0, j ? y : x, i + j);
    });
    const int count = gather(0);
    if (count <= kList) {
      if (a.p || rank == 0) {
        // ---- all that may be kept: compared one by one
        const Compared mine = compare(count);
        const unsigned long long me = mine.entry;
        const int64_t w = mine.weight, earlier_weight = mine.weight_before;
        const int earlier = mine.before;
        bool keep = mine.real && (!by_count || earlier < most);
        if (by_weight) {
          if (by_count) goal = max(times(fmaxf(top_p, 0.f), (int64_t)sum_warps(keep ? w : 0)), (int64_t)1);
          keep = keep && earlier_weight < goal;
        }
        if (by_count || by_weight) {  // the last entry that these limits keep
          unsigned long long last = keep ? me : ~0ull;
#pragma unroll
          for (int d = 16; d; d >>= 1) last = min(last, __shfl_xor_sync(~0u, last, d));
          __syncthreads();
          if (lane == 0) sh.g.warp[warp] = last;
          __syncthreads();
          for (int v = 0; v < kWarps; v++) last = min(last, sh.g.warp[v]);
          cut = last;
        }
        keep = keep && (earlier == 0 || w >= (int64_t)(least * 1099511627776.f));
        __syncthreads();  // the weights have been read
        if (mine.real) sh.weight[mine.at] = keep ? w : 0;
        const int64_t total = sum_warps(keep ? w : 0);
        if (rank == 0 && a.token) {
          const int64_t goal = times(fminf(fmaxf(a.u[row], 0.f), 1.f - 1.f / 16777216.f), total);
          int64_t before = 0;  // ~index: a lower one is larger
          for (int j = mine.share; j < count; j += mine.shares)
            before += (uint32_t)sh.list[j] > (uint32_t)me ? sh.weight[j] : 0;
          before = mine.sum(before);
          if (keep && before <= goal && goal < before + w) a.token[row] = (int)~(uint32_t)me;
        }
        cut_total = total;
      }
      cluster_arrive(false);  // the CTAs' lists are read until here
      if (a.p) put_all(cut_total);
      cluster_wait();
      return;
    }
    if (greedy) give_up = true;
  } else if (by_count || by_weight) {
    cluster_sync(warp);  // every CTA has read the histogram
  }

  // ---- the cut, by a histogram
  if (!give_up && (by_count || by_weight)) {
    sh.g.slots[tid] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    scale = (kSlots - 0.5f) / -low;
    auto count_all = [&]() {
      each_from(low_logit, [&](float x, float y, int) {
        const uint64_t tt = exponents(x, y);
        float t[2];
        unpair(tt, t[0], t[1]);
        if (fmaxf(t[0], t[1]) < low) return;
        uint32_t h[2], l[2];
        fixed_pair(raise(tt), h, l);
#pragma unroll
        for (int j = 0; j < 2; j++) {
          const int b = place(t[j]);
          if (b < 0) continue;
          count_in(b, h[j] - kBias, l[j] - kBias);
        }
      });
      cluster_sync(warp);
    };
    int64_t all_weight = 0;
    int lists = 0;
    // The entry at which the running count, or weight, reaches the goal.  False: there
    // is none (of a weight above 0).
    auto resolve = [&](bool by_weight, int64_t goal) -> bool {
      int64_t above = 0, above_weight = 0;
      for (;;) {
        int64_t n, w, all;
        totals(n, w);
        if (tid == 0) sh.slot = -1;
        const int64_t before = above + block_scan(n, sh.g.part, all);
        const int64_t before_weight = above_weight + block_scan(w, sh.g.part, all);
        all_weight = all;
        const int64_t at = by_weight ? before_weight : before, mine = by_weight ? w : n;
        if (at < goal && goal <= at + mine) {
          sh.slot = kSlots - 1 - tid;
          sh.count = n;
          sh.above = before;
          sh.above_weight = before_weight;
        }
        cluster_sync(warp);  // every CTA has read the histogram, and its threads the last list
        if (sh.slot < 0) return false;
        above = sh.above;
        above_weight = sh.above_weight;
        const int slot = sh.slot;
        const uint32_t count = sh.count;
        if (count <= kList) {
          lists++;
          each_from(low_logit, [&](float x, float y, int i) {
            const float t[2] = {exponent(x), exponent(y)};
#pragma unroll
            for (int j = 0; j < 2; j++)
              if (place(t[j]) == slot) enlist(lists, j ? y : x, i + j);
          });
          gather(lists);
          const Compared mine = compare(count);
          if (mine.real) {
            const int64_t weight_before = above_weight + mine.weight_before;
            const int64_t from = by_weight ? weight_before : above + mine.before, step = by_weight ? mine.weight : 1;
            if (from < goal && goal <= from + step) {
              sh.cut = mine.entry;
              sh.cut_total = weight_before + mine.weight;
            }
          }
          __syncthreads();
          cut = sh.cut;
          cut_total = sh.cut_total;
          return true;
        }
        if (level == 1) {
          give_up = true;
          return true;
        }
        // too many: a histogram of that slot alone
        low2 = low + slot / scale;
        scale2 = scale * kSlots;
        chosen = slot;
        level = 1;
        sh.g.slots[tid] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        count_all();
      }
    };
    count_all();
    if (by_count) {
      const bool limited = resolve(false, most);
      if (by_weight && !give_up) {
        goal = max(times(fmaxf(top_p, 0.f), limited ? cut_total : all_weight), (int64_t)1);
        if (level) {
          level = 0;
          cluster_sync(warp);
          sh.g.slots[tid] = make_uint4(0, 0, 0, 0);
          __syncthreads();
          count_all();
        }
        resolve(true, goal);
      }
    } else {
      resolve(true, goal);
    }
  }
  if (give_up) {
    cluster.sync();
    general<T>(a, sh.g);
    return;
  }

  // ---- the kept weights' sum, by warps where a token is drawn
  int64_t total = cut_total, before = 0, here = 0;
  if (a.token || !cut || least > 0.f) {
    int64_t sum = 0;
    if (!cut && !(least > 0.f)) {
      FixedSum s;
      each([&](float x, float y, int) { s.add(raise(exponents(x, y))); });
      sum = s.sum(numbers);
    } else {
      const float from = cut ? of_key((uint32_t)(cut >> 32)) : low_logit;
      each_from(from, [&](float x, float y, int i) {
        if (fmaxf(x, y) < from) return;
        sum += (int64_t)__fmul_rn(kept(x, begin + i - shift), 1099511627776.f);
        sum += (int64_t)__fmul_rn(kept(y, begin + i + 1 - shift), 1099511627776.f);
      });
    }
    here = sum_warps(sum);
    const unsigned long long *p = push(here);
    total = 0;
    for (int c = 0; c < ctas; c++) {
      if (c < rank) before += p[c];
      total += p[c];
    }
  }
  if (a.token) {
    const int64_t goal = times(fminf(fmaxf(a.u[row], 0.f), 1.f - 1.f / 16777216.f), total);
    if (before <= goal && goal < before + here) {
      // in a warp's run of this CTA: all threads go through that, some entries each
      int w = 0;
      while (before + (int64_t)sh.g.warp[w] <= goal) before += sh.g.warp[w++];
      const T *const run = reinterpret_cast<const T *>(smem) + w * span;
      const int each = (span + kThreads - 1) / kThreads, from = tid * each, to = min(from + each, span);
      const int first = (int)min((int64_t)(rank * kWarps + w) * span, (int64_t)INT_MAX / 2) - shift;
      auto one = [&](int i) { return (int64_t)__fmul_rn(kept(number<T>(run[i]), first + i), 1099511627776.f); };
      int64_t sum = 0, all;
      for (int i = from; i < to; i++) sum += one(i);
      before += block_scan(sum, sh.g.part, all);
      if (before <= goal && goal < before + sum) {  // one thread
        int i = from;
        while (before + one(i) <= goal) before += one(i++);
        a.token[row] = first + i;
      }
    }
  }
  cluster_arrive(false);  // the CTAs' lists are read until here
  if (a.p) put_all(total);
  cluster_wait();
}

template <typename T>
int sample_run(const unison_kv_sample_args &a, void *stream) {
  constexpr int kStep = 32 * Piece<T>::kN, kMostBytes = 160 << 10;
  const int places = 3 * kv_sm_count(), room = places / a.n_rows;
  auto span_of = [&](int ctas) {  // entries of a warp, whole steps; a row may begin 15 bytes into a piece
    return (int)(((int64_t)a.vocab + Piece<T>::kN - 1 + ctas * kWarps * kStep - 1) / (ctas * kWarps * kStep) * kStep);
  };
  auto bytes_of = [&](int ctas) { return (int64_t)span_of(ctas) * kWarps * (int)sizeof(T); };
  int ctas = 1;
  while (ctas < kMaxCluster && (bytes_of(ctas) > (64 << 10) || (ctas * 2 <= room && span_of(ctas) > 2 * kStep)))
    ctas *= 2;
  if (bytes_of(ctas) > kMostBytes)
    return kv_launch("kv_sample", dim3(a.n_rows * ctas), dim3(kThreads), 0, stream, ctas, sample_general_kernel<T>, a);
  static uint64_t done = 0;
  if (!kv_allow_smem(reinterpret_cast<const void *>(sample_kernel<T>), kMostBytes, &done)) return UNISON_ERR_CUDA;
  return kv_launch("kv_sample", dim3(a.n_rows * ctas), dim3(kThreads), (size_t)bytes_of(ctas), stream, ctas,
                   sample_kernel<T>, a, span_of(ctas), places / ctas);
}

}  // namespace
}  // namespace unison

using namespace unison;

extern "C" int unison_kv_sample(const unison_kv_sample_args *args, void *cuda_stream) {
  if (!args) return UNISON_ERR_ARG;
  const unison_kv_sample_args &a = *args;
  if (a.n_rows < 0 || a.n_rows > (1 << 27) || a.vocab < 1 || a.vocab > (1 << 22)) return UNISON_ERR_RANGE;
  if (a.dtype < 0 || a.dtype > UNISON_KV_FP32 || (a.p && (a.p_dtype < 0 || a.p_dtype > UNISON_KV_FP32)))
    return UNISON_ERR_ARG;
  if (a.n_rows == 0) return UNISON_OK;
  if (!a.logits || (!a.p && !a.token) || !a.u != !a.token) return UNISON_ERR_ARG;
  if (a.p && (a.p == a.logits || (a.n_rows > 1 && a.p_row < a.vocab))) return UNISON_ERR_ARG;  // rows are written whole
  switch (a.dtype) {
    case UNISON_KV_FP32: return sample_run<float>(a, cuda_stream);
    case UNISON_KV_BF16: return sample_run<__nv_bfloat16>(a, cuda_stream);
    default: return sample_run<__half>(a, cuda_stream);
  }
}
