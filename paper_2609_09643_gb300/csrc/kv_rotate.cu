// Norms of queries and keys for each head and their rotation by position, in
// one pass (unison_kv_rotate).
//
//   y = x w / sqrt(mean x^2 + eps), then for every pair (a, b) of y, with
//   angle = position * inv_freq:  (a cos - b sin, b cos + a sin)
//
// A warp has a token, or a share of its heads: all of a token's heads turn by the
// same angles, which the warp's lanes work out two each and leave in shared memory.
// A row belongs to a few lanes; each of them has V elements and the V others that
// they are paired with, so nothing but the sum of squares passes between lanes, and
// in place is as good as out of place.
//
// Angles in whole numbers: inv_freq / 2 pi as a 64-bit fraction of a turn, times
// the position modulo 2^64, is the fraction of a turn that is left, to 2^-33 for
// any position and frequency; in 32 bits of float a position of 10^6 would leave it
// uncertain by 0.06.  Its first 32 bits become a number of 24 (what sincospif
// takes): half a unit of half a turn, pi 2^-25, is what the angle is known to, as
// 32-bit cosines and sines are to 2^-25 themselves.
//
// Bound by memory, if the operations are few: 13,750 tokens of 32 + 8 heads of 128
// (282 MB): 52 us, 5.4 TB/s, 0.80 of the copy rate, instructions issued in 63% of
// the cycles.  A CTA a token, one element an operation: 71; rows fetched two or
// three steps ahead: 55 to 60, as fewer warps fit (eight CTAs on a multiprocessor
// leave 64 registers, and 80 bytes of a thread's are kept in local memory as it is).
// One token: 3.4 us.
#include <type_traits>

#include "kv_tc.cuh"

namespace unison {
namespace {

constexpr int kThreads = 128;
constexpr int kPairs = 128;  // of a head, at most

struct RotateParams {
  unison_kv_rotate_args a;
  const int32_t *offsets, *next_pos;  // where positions are not given
  const uint64_t *mask;
  int32_t *status;
  int n_seqs, max_tokens, n_tokens, n_heads, head_dim;
  int lanes;  // of a row: a power of two
  int shares; // warps of a token
};

// The token of an item and its position; false: there is none.
__device__ __forceinline__ bool token_of(const RotateParams &P, int64_t item, int &token, int &position) {
  if (P.a.position) {
    if (item >= P.n_tokens) return false;
    token = (int)item;
    position = P.a.position[token];
    return true;
  }
  const int b = (int)(item / P.max_tokens), node = (int)(item - (int64_t)b * P.max_tokens);
  if (b >= P.n_seqs) return false;
  const int lo = P.offsets[b], hi = P.offsets[b + 1];
  const int first = min(max(lo, 0), P.n_tokens), last = min(max(hi, first), P.n_tokens);
  const int count = min(last - first, P.max_tokens);
  if (P.status && node == 0 && (lo != first || hi != first + count)) P.status[b] = UNISON_ERR_RANGE;
  if (node >= count) return false;
  token = first + node;
  position = P.next_pos[b] + (P.mask ? __popcll(P.mask[token] & ((1ull << node) - 1)) : node);
  return true;
}

// f / (2 pi) modulo 1, as a fraction of 2^64, rounded towards zero: from 128 bits
// of 1 / (2 pi), so that what a position multiplies is off by less than a unit for
// every |f| up to 2^24.
__device__ __forceinline__ uint64_t turn_of(float f) {
  constexpr uint64_t kTurn = 0x28BE60DB9391054Aull, kRest = 0x7F09D5F47D4D3770ull;  // 2^128 / (2 pi)
  const uint32_t bits = __float_as_uint(f);
  const int e = bits >> 23 & 255;
  const uint64_t m = (bits & 0x7FFFFFu) | (e ? 0x800000u : 0u);
  const int shift = 150 - (e ? e : 1);  // f = m 2^-shift
  const uint64_t lo = m * kTurn, hi = __umul64hi(m, kTurn);
  const uint64_t w1 = lo + __umul64hi(m, kRest), w2 = hi + (w1 < lo);  // m 2^64 / (2 pi), whole numbers
  uint64_t t;
  if (shift <= 0)
    t = shift > -64 ? w1 << -shift : 0;
  else if (shift < 64)
    t = w1 >> shift | w2 << (64 - shift);
  else
    t = shift < 128 ? w2 >> (shift - 64) : 0;
  return bits >> 31 ? 0 - t : t;
}

// cos and sin of pair j at a position.
__device__ __forceinline__ float2 turned(const RotateParams &P, int j, int position) {
  const uint64_t t = turn_of(P.a.inv_freq[j]) * (uint64_t)(int64_t)position;
  float s, c;
  sincospif((float)(int32_t)(t >> 32) * (1.f / 2147483648.f), &s, &c);  // (signed, in half turns: 24 bits of it)
  return make_float2(c, s);
}
__device__ __forceinline__ float norm_factor(const RotateParams &P, float squares) {
  return rsqrtf(fmaf(squares, 1.f / (float)P.head_dim, P.a.eps));
}

// N elements, as numbers.
template <typename T, int N>
__device__ __forceinline__ void load_n(const T *p, float (&x)[N]) {
  if constexpr (N * sizeof(T) == 32) {
    const uint4 u = reinterpret_cast<const uint4 *>(p)[0], v = reinterpret_cast<const uint4 *>(p)[1];
    const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = __uint_as_float(w[i]);
  } else if constexpr (N * sizeof(T) == 16) {
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < N; i++) {
      if constexpr (sizeof(T) == 4)
        x[i] = __uint_as_float(w[i]);
      else
        x[i] = KvType<T>::to_float(reinterpret_cast<const T *>(w)[i]);
    }
  } else if constexpr (N * sizeof(T) == 8) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    const uint32_t w[2] = {u.x, u.y};
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = KvType<T>::to_float(reinterpret_cast<const T *>(w)[i]);
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_n(T *p, const float (&x)[N]) {
  if constexpr (N == 8)
    *reinterpret_cast<uint4 *>(p) = make_uint4(KvType<T>::pack(x[0], x[1]), KvType<T>::pack(x[2], x[3]),
                                               KvType<T>::pack(x[4], x[5]), KvType<T>::pack(x[6], x[7]));
  else
    *reinterpret_cast<uint2 *>(p) = make_uint2(KvType<T>::pack(x[0], x[1]), KvType<T>::pack(x[2], x[3]));
}

// V: elements of either half of a lane's unit: 4 or 8.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 8) rotate_kernel(const RotateParams P) {
  follow_last_kernel();
  __shared__ __align__(16) float cosines[kThreads / 32][kPairs], sines[kThreads / 32][kPairs];  // of every pair
  constexpr int kP = V / 2;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = P.head_dim, half = P.a.rot_dim / 2;
  const int64_t id = (int64_t)blockIdx.x * (kThreads / 32) + warp;
  const int64_t item = id / P.shares;
  const int share = (int)(id - item * P.shares);
  int token, position;
  if (!token_of(P, item, token, position)) return;

  // ---- the angles
  const int u = lane & (P.lanes - 1), mine = lane / P.lanes, at_once = 32 / P.lanes;
  for (int j = lane; j < half; j += 32) {
    const float2 t = turned(P, j, position);
    cosines[warp][j] = t.x;
    sines[warp][j] = t.y;
  }
  __syncwarp();
  // (pairs of the unit, two at a time; behind the last one whatever lies there, which is not used)
  const uint64_t *cosine = reinterpret_cast<const uint64_t *>(&cosines[warp][min(u * V, kPairs - V)]);
  const uint64_t *sine = reinterpret_cast<const uint64_t *>(&sines[warp][min(u * V, kPairs - V)]);

  // Where the two halves of a unit lie: a pair's elements R / 2 apart (or next to
  // each other, where pairs interleave); behind R one after the other.
  const bool apart = !P.a.interleaved && u * V < half, beside = P.a.interleaved && u * V < half;
  const int e0 = apart ? u * V : u * 2 * V, e1 = apart ? u * V + half : u * 2 * V + V;
  const bool real0 = e0 < D, real1 = e1 < D;
  using Words = typename std::conditional<V == 8, uint4, uint2>::type;

  // Rows `mine` + at_once * step of queries, or of keys, from step0 up to step1.
  auto turn = [&](const T *src, T *dst, int64_t from, int64_t to, int rows, int step0, int step1, const void *of) {
    if (step0 >= step1) return;
    int row = step0 * at_once + mine;
    src += row * from + e0;
    dst += row * to + e0;
    const int64_t src_step = at_once * from, dst_step = at_once * to;
    Words x0 = Words(), x1 = Words();
    auto fetch = [&] {
      if (row < rows && real0) x0 = *reinterpret_cast<const Words *>(src);
      if (row < rows && real1) x1 = *reinterpret_cast<const Words *>(src + (e1 - e0));
    };
    fetch();
    uint64_t weight[2][kP];
    if (of) {
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int e = h ? e1 : e0;
        float g[V];
#pragma unroll
        for (int j = 0; j < V; j++) g[j] = 0.f;
        if (e < D) {
          if (P.a.weight_dtype == UNISON_KV_FP32)
            load_n<float, V>(static_cast<const float *>(of) + e, g);
          else
            load_n<T, V>(static_cast<const T *>(of) + e, g);
        }
#pragma unroll
        for (int j = 0; j < kP; j++) weight[h][j] = pair(g[2 * j], g[2 * j + 1]);
      }
    }
#pragma unroll 1
    for (int step = step0; step < step1; step++) {
      uint64_t y[2][kP];
#pragma unroll
      for (int j = 0; j < kP; j++) {
        const T *a = reinterpret_cast<const T *>(&x0) + 2 * j, *b = reinterpret_cast<const T *>(&x1) + 2 * j;
        y[0][j] = pair(KvType<T>::to_float(a[0]), KvType<T>::to_float(a[1]));
        y[1][j] = pair(KvType<T>::to_float(b[0]), KvType<T>::to_float(b[1]));
      }
      const bool real = row < rows;
      row += at_once;
      src += src_step;
      if (step + 1 < step1) fetch();
      if (of) {
        uint64_t squares[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
          for (int j = 0; j < kP; j++) squares[h] = fma_pair(y[h][j], y[h][j], squares[h]);
        float s, more;
        unpair(add_pair(squares[0], squares[1]), s, more);
        s += more;
        for (int d = P.lanes >> 1; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
        s = norm_factor(P, s);
        const uint64_t factor = pair(s, s);
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
          for (int j = 0; j < kP; j++) y[h][j] = mul_pair(mul_pair(y[h][j], weight[h][j]), factor);
      }
      if (apart) {
#pragma unroll
        for (int j = 0; j < kP; j++) {
          const uint64_t a = y[0][j], b = y[1][j], c = cosine[j], s = sine[j];
          y[0][j] = fma_pair(a, c, mul_pair(b, s ^ 0x8000000080000000ull));
          y[1][j] = fma_pair(b, c, mul_pair(a, s));
        }
      } else if (beside) {
#pragma unroll
        for (int j = 0; j < V; j++) {  // pair j: two neighbours
          uint64_t &both = y[j / kP][j % kP];
          float a, b;
          unpair(both, a, b);
          const float c = reinterpret_cast<const float *>(cosine)[j], s = reinterpret_cast<const float *>(sine)[j];
          if (u * V + j < half) both = fma_pair(both, pair(c, c), mul_pair(pair(b, a), pair(-s, s)));
        }
      }
      if (real) {
        float z[V];
#pragma unroll
        for (int j = 0; j < kP; j++) unpair(y[0][j], z[2 * j], z[2 * j + 1]);
        if (real0) store_n<T, V>(dst, z);
#pragma unroll
        for (int j = 0; j < kP; j++) unpair(y[1][j], z[2 * j], z[2 * j + 1]);
        if (real1) store_n<T, V>(dst + (e1 - e0), z);
      }
      dst += dst_step;
    }
  };
  // ---- this share of the steps of queries and keys
  const int q_steps = (P.a.n_q_heads + at_once - 1) / at_once, k_steps = (P.n_heads + at_once - 1) / at_once;
  const int steps = q_steps + k_steps, step0 = steps * share / P.shares, step1 = steps * (share + 1) / P.shares;
  turn(static_cast<const T *>(P.a.q) + token * P.a.q_token, static_cast<T *>(P.a.q_out) + token * P.a.q_out_token,
       P.a.q_head, P.a.q_out_head, P.a.n_q_heads, step0, min(step1, q_steps), P.a.q_weight);
  turn(static_cast<const T *>(P.a.k) + token * P.a.k_token, static_cast<T *>(P.a.k_out) + token * P.a.k_out_token,
       P.a.k_head, P.a.k_out_head, P.n_heads, max(step0 - q_steps, 0), step1 - q_steps, P.a.k_weight);
}

// Any even number of rotated elements, one by one: for halves that are not
// whole pieces of 4.  A CTA has one token.
template <typename T>
__global__ void __launch_bounds__(kThreads) rotate_any_kernel(const RotateParams P) {
  follow_last_kernel();
  __shared__ float2 turns[128];
  __shared__ float sums[kThreads / 32];
  const int tid = threadIdx.x, D = P.head_dim, half = P.a.rot_dim / 2;
  int token, position;
  if (!token_of(P, blockIdx.x, token, position)) return;
  for (int j = tid; j < half; j += kThreads) turns[j] = turned(P, j, position);
  __syncthreads();
  for (int row = 0; row < P.a.n_q_heads + P.n_heads; row++) {
    const bool is_q = row < P.a.n_q_heads;
    const int head = is_q ? row : row - P.a.n_q_heads;
    const T *src = static_cast<const T *>(is_q ? P.a.q : P.a.k) +
                   (is_q ? token * P.a.q_token + head * P.a.q_head : token * P.a.k_token + head * P.a.k_head);
    T *dst = static_cast<T *>(is_q ? P.a.q_out : P.a.k_out) +
             (is_q ? token * P.a.q_out_token + head * P.a.q_out_head : token * P.a.k_out_token + head * P.a.k_out_head);
    const void *weight = is_q ? P.a.q_weight : P.a.k_weight;
    // units of two elements: a pair, or two neighbours behind the pairs
    float2 y = make_float2(0.f, 0.f);
    const bool real = tid < D / 2, turns_it = tid < half;
    const int a = P.a.interleaved || !turns_it ? tid * 2 : tid, b = P.a.interleaved || !turns_it ? a + 1 : tid + half;
    if (real) y = make_float2(KvType<T>::to_float(src[a]), KvType<T>::to_float(src[b]));
    float s = y.x * y.x + y.y * y.y;
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    __syncthreads();
    if ((tid & 31) == 0) sums[tid >> 5] = s;
    __syncthreads();
    if (!real) continue;
    if (weight) {
      s = 0.f;
      for (int w = 0; w < kThreads / 32; w++) s += sums[w];
      s = norm_factor(P, s);
      auto at = [&](int e) {
        return P.a.weight_dtype == UNISON_KV_FP32 ? static_cast<const float *>(weight)[e]
                                                  : KvType<T>::to_float(static_cast<const T *>(weight)[e]);
      };
      y.x *= s * at(a), y.y *= s * at(b);
    }
    if (turns_it) {
      const float2 t = turns[tid];
      y = make_float2(y.x * t.x - y.y * t.y, y.y * t.x + y.x * t.y);
    }
    const uint32_t both = KvType<T>::pack(y.x, y.y);
    reinterpret_cast<uint16_t *>(dst)[a] = (uint16_t)both;
    reinterpret_cast<uint16_t *>(dst)[b] = (uint16_t)(both >> 16);
  }
}

template <typename T>
int rotate_run(RotateParams &p, void *stream) {
  const int half = p.a.rot_dim / 2;
  const int64_t items = p.a.position ? p.n_tokens : (int64_t)p.n_seqs * p.max_tokens;
  // elements of a unit's half: as many as lie in one piece of both elements of the pairs
  const int v = p.a.interleaved || half % 8 == 0 ? 8 : half % 4 == 0 ? 4 : 1;
  if (items * 64 >= 1ll << 31) return UNISON_ERR_RANGE;
  if (v == 1) return kv_launch("kv_rotate", dim3(items), dim3(kThreads), 0, stream, 1, rotate_any_kernel<T>, p);
  const int units = (p.head_dim + 2 * v - 1) / (2 * v);
  p.lanes = 1;
  while (p.lanes < units && p.lanes < 32) p.lanes *= 2;
  // Warps of a token: a second one where the tokens leave warps' places free (16 of a
  // multiprocessor), and so on, but not for less than one step of rows.
  const int at_once = 32 / p.lanes;
  const int steps = (p.a.n_q_heads + at_once - 1) / at_once + (p.n_heads + at_once - 1) / at_once;
  p.shares = 1;
  while (p.shares < steps && p.shares < 32 && items * p.shares < kv_sm_count() * 16) p.shares *= 2;
  p.shares = min(p.shares, steps);
  const int64_t ctas = (items * p.shares * 32 + kThreads - 1) / kThreads;
  return kv_launch("kv_rotate", dim3(ctas), dim3(kThreads), 0, stream, 1,
                   v == 8 ? rotate_kernel<T, 8> : rotate_kernel<T, 4>, p);
}

bool weight_ok(const void *w, int dtype) { return kv_aligned(w, 16) && (dtype >= 0 && dtype <= UNISON_KV_FP32); }

}  // namespace
}  // namespace unison

using namespace unison;

extern "C" int unison_kv_rotate(const unison_kv_cache *cache, const unison_kv_tree *tree,
                                const unison_kv_rotate_args *args, void *cuda_stream) {
  if (!args) return UNISON_ERR_ARG;
  int rc = kv_check_cache(cache);
  if (rc != UNISON_OK) return rc;
  const unison_kv_rotate_args &a = *args;
  if (a.n_tokens < 0 || a.n_q_heads < 0 || a.rot_dim < 0 || a.rot_dim > cache->head_dim || a.rot_dim % 2)
    return UNISON_ERR_RANGE;
  if (!(a.eps >= 0.f)) return UNISON_ERR_RANGE;
  if (a.n_tokens == 0) return UNISON_OK;
  if (!a.position) {
    rc = kv_check_tree(tree, cache->n_seqs);
    if (rc != UNISON_OK) return rc;
    if (tree->n_tokens != a.n_tokens || (cache->n_seqs > 0 && !cache->next_pos)) return UNISON_ERR_ARG;
  }
  if (!a.position && cache->n_seqs == 0) return UNISON_OK;
  if (a.n_q_heads > 0 && (!kv_rows_ok(a.q, a.q_token, a.q_head) || !kv_rows_ok(a.q_out, a.q_out_token, a.q_out_head)))
    return UNISON_ERR_ARG;
  if (!kv_rows_ok(a.k, a.k_token, a.k_head) || !kv_rows_ok(a.k_out, a.k_out_token, a.k_out_head))
    return UNISON_ERR_ARG;
  if (a.rot_dim > 0 && !a.inv_freq) return UNISON_ERR_ARG;
  if (a.weight_dtype != cache->dtype && a.weight_dtype != UNISON_KV_FP32) return UNISON_ERR_ARG;
  if (!weight_ok(a.q_weight, a.weight_dtype) || !weight_ok(a.k_weight, a.weight_dtype)) return UNISON_ERR_ARG;
  RotateParams p = {};
  p.a = a;
  p.n_tokens = a.n_tokens;
  p.n_heads = cache->n_heads;
  p.head_dim = cache->head_dim;
  if (!a.position) {
    p.offsets = tree->offsets;
    p.mask = tree->mask;
    p.next_pos = cache->next_pos;
    p.status = cache->status;
    p.n_seqs = cache->n_seqs;
    p.max_tokens = tree->max_tokens;
  }
  return cache->dtype == UNISON_KV_BF16 ? rotate_run<__nv_bfloat16>(p, cuda_stream)
                                        : rotate_run<__half>(p, cuda_stream);
}
