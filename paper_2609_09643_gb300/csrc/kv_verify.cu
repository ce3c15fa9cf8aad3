// Verification of drafted tokens (unison_kv_verify).
//
// What a walk needs of the vocabulary rows is little until a draft is refused:
// p and q at the drafted tokens, which one round of loads fetches for all
// nodes at once.  Only a refusal (the sum of what is left) and the last sample
// read whole rows.  A cluster of CTAs shares the rows of one session: CTA r
// has a run of the vocabulary, each of its warps a run of that.  A pass over
// the rows is one stream of loads, one exchange of the CTAs' sums and one
// cluster barrier.
//
// Bound by the chain of passes: each refusal wants the sum that the last one
// left, and a session's next pass cannot begin before.  128 sessions' trees of 32
// nodes over 128,000 entries of 32 bits (one to four passes mostly, from the L2
// cache after the first): 63 us, while reading every row that is wanted once
// would take 19; without q 78.  One session's chain of five over 32,000 entries: 6 us.
#include <cooperative_groups.h>

#include <type_traits>

#include "kv.cuh"

namespace unison {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ float weight(float x) { return fminf(fmaxf(x, 0.f), 1.f); }  // (NaN: 0)
template <typename T>
__device__ __forceinline__ float load(const T *p, int64_t i) {
  return KvType<T>::to_float(p[i]);
}
template <>
__device__ __forceinline__ float load<float>(const float *p, int64_t i) {
  return p[i];
}
// floor(d 2^40) of 0 <= d <= 1, as 2^20 high + low.  Adding 2^23 and rounding
// towards zero leaves the whole part in the low bits of a float, so the parts
// come from five operations at the full rate; a conversion to 64 bits is served
// at a small fraction of it.  high and low get 2^23's bits on top: kBias each.
constexpr uint32_t kBias = 0x4B000000u;
__device__ __forceinline__ void fixed_parts(float d, uint32_t &high, uint32_t &low) {
  const float x = __fmul_rn(d, 1048576.f), h = __fadd_rz(x, 8388608.f);
  const float rest = __fsub_rn(x, __fsub_rn(h, 8388608.f));  // exact, below 1
  high = __float_as_uint(h);
  low = __float_as_uint(__fmaf_rz(rest, 1048576.f, 8388608.f));
}
__device__ __forceinline__ int64_t fixed(float d) {
  uint32_t high, low;
  fixed_parts(d, high, low);
  return (int64_t)(high - kBias) << 20 | (low - kBias);
}

// 16 bytes of a row as numbers.
template <typename T>
struct Quad {
  static constexpr int kN = 16 / sizeof(T);
  __device__ __forceinline__ static void get(const uint4 &v, float (&x)[kN]) {
    const T *e = reinterpret_cast<const T *>(&v);
#pragma unroll
    for (int i = 0; i < kN; i++) x[i] = load(e, i);
  }
};

// The refusals at the current node: z[i] the sum before refusal i, token[i]
// the refused token.
struct Refused {
  float z[UNISON_KV_MAX_TOKENS];
  int token[UNISON_KV_MAX_TOKENS];
};
// d at entry x, whose first weight is d and whose draft weight is y, after n
// refusals; kCount: n where it is 0 or 1, else 2.
template <bool kCertain, int kCount>
__device__ __forceinline__ float residual(const Refused &r, float d, float y, int x, int n) {
  for (int i = 0; i < (kCount < 2 ? kCount : n); i++) {
    if (kCertain)
      d = r.token[i] == x ? 0.f : d;
    else
      d = fmaxf(__fsub_rn(d, __fmul_rn(r.z[i], y)), 0.f);
  }
  return d;
}

// kCertain: without q.
template <typename T, bool kCertain>
__global__ void __launch_bounds__(kThreads) verify_kernel(const unison_kv_tree t, const unison_kv_verify_args a) {
  follow_last_kernel();
  namespace cg = cooperative_groups;
  __shared__ Refused refused;
  __shared__ int node_parent[UNISON_KV_MAX_TOKENS], node_token[UNISON_KV_MAX_TOKENS];
  __shared__ float node_u[UNISON_KV_MAX_TOKENS], node_d[UNISON_KV_MAX_TOKENS], node_y[UNISON_KV_MAX_TOKENS];
  __shared__ int64_t warp_sum[kWarps], cta_sum[2][kMaxCluster], part[33];
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const int b = blockIdx.x / ctas, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const KvRange tok = kv_tokens(t, b, nullptr);
  int32_t *path = a.path + b * a.path_stride;
  if (tok.count == 0) {  // all CTAs of the cluster
    if (rank == 0) {
      if (tid < t.max_tokens) path[tid] = -1;
      if (tid == 0) {
        a.n_path[b] = 0;
        a.next_token[b] = -1;
      }
    }
    return;
  }
  const int V = a.vocab;
  const T *const rows_p = static_cast<const T *>(a.p) + tok.first * a.p_row;
  const T *const rows_q = kCertain ? nullptr : static_cast<const T *>(a.q) + tok.first * a.q_row;
  if (tid < tok.count) {
    int parent = t.parent[tok.first + tid];
    const int token = a.token[tok.first + tid];
    if (tid == 0 || parent < 0 || parent >= tid || (unsigned)token >= (unsigned)V) parent = -1;  // never reached
    node_parent[tid] = parent;
    node_token[tid] = token;
    node_u[tid] = a.u[tok.first + tid];
    if (parent >= 0) {
      node_d[tid] = weight(load(rows_p + parent * a.p_row, token));
      node_y[tid] = kCertain ? 1.f : weight(load(rows_q + parent * a.q_row, token));
    }
  }
  cluster.sync();  // every CTA has begun: its shared memory may be written to

  // this warp's run of the vocabulary, in whole groups of 32 times 16 bytes
  constexpr int kN = Quad<T>::kN, kGroup = 32 * kN;
  constexpr int kFlight = 16 / kN;  // loads in flight of a lane, from each of the two rows
  const int span = (V + ctas * kWarps * kGroup - 1) / (ctas * kWarps * kGroup) * kGroup;
  const int64_t begin64 = (int64_t)(rank * kWarps + warp) * span;
  const int begin = (int)min(begin64, (int64_t)V), end = (int)min(begin64 + span, (int64_t)V);
  int passes = 0;
  // This lane's share of the sum over all entries of the residual at `cur`.
  auto share = [&](auto counted, int cur, int n) -> int64_t {
    constexpr int kCount = decltype(counted)::value;
    const T *p = rows_p + cur * a.p_row, *q = kCertain || kCount == 0 ? nullptr : rows_q + cur * a.q_row;
    int64_t s = 0;
    const bool whole = (((uintptr_t)p | (uintptr_t)q) & 15) == 0 && V % kN == 0;
    if (whole) {
      for (int x0 = begin + lane * kN; x0 < end; x0 += kGroup * kFlight) {
        uint4 d[kFlight], y[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; i++) {
          const int x = x0 + i * kGroup;
          d[i] = x < end ? __ldg(reinterpret_cast<const uint4 *>(p + x)) : make_uint4(0, 0, 0, 0);
          y[i] = q && x < end ? __ldg(reinterpret_cast<const uint4 *>(q + x)) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kFlight; i++) {
          float dx[kN], yx[kN];
          Quad<T>::get(d[i], dx);
          Quad<T>::get(y[i], yx);
          uint32_t high = 0, low = 0;  // of at most eight numbers
#pragma unroll
          for (int j = 0; j < kN; j++) {
            uint32_t h, l;
            const int x = x0 + i * kGroup + j;
            fixed_parts(residual<kCertain, kCount>(refused, weight(dx[j]), weight(yx[j]), x, n), h, l);
            high += h;
            low += l;
          }
          s += ((int64_t)(high - kN * kBias) << 20) + (low - kN * kBias);
        }
      }
    } else {
      for (int x0 = begin + lane; x0 < end; x0 += 32 * 2 * kFlight) {
        float d[2 * kFlight], y[2 * kFlight];
#pragma unroll
        for (int i = 0; i < 2 * kFlight; i++) {
          const int x = x0 + i * 32;
          d[i] = x < end ? load(p, x) : 0.f;
          y[i] = q && x < end ? load(q, x) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 2 * kFlight; i++)
          s += fixed(residual<kCertain, kCount>(refused, weight(d[i]), weight(y[i]), x0 + i * 32, n));
      }
    }
    return s;
  };
  // The sum over all entries of the residual after n refusals at node `cur`.
  auto total = [&](int cur, int n) -> int64_t {
    int64_t s = n == 0   ? share(std::integral_constant<int, 0>(), cur, n)
                : n == 1 ? share(std::integral_constant<int, 1>(), cur, n)
                         : share(std::integral_constant<int, 2>(), cur, n);
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    if (lane == 0) warp_sum[warp] = s;
    __syncthreads();
    const int slot = passes++ & 1;  // a CTA that is one pass ahead writes the other one
    if (tid < ctas) {
      int64_t mine = 0;
      for (int w = 0; w < kWarps; w++) mine += warp_sum[w];
      *cluster.map_shared_rank(&cta_sum[slot][rank], tid) = mine;
    }
    cluster.sync();
    int64_t all = 0;
    for (int c = 0; c < ctas; c++) all += cta_sum[slot][c];
    return all;
  };

  int cur = 0, n = 1, count = 0;  // node, accepted nodes, refusals at this node
  float z = 1.f;
  int64_t left = -1;  // sum of the residual, -1: not known
  if (rank == 0 && tid == 0) path[0] = 0;
  for (int i = 1; i < tok.count; i++) {
    if (node_parent[i] != cur) continue;
    const float y = node_y[i];
    const float d = residual<kCertain, 2>(refused, node_d[i], y, node_token[i], count);
    if (__fmul_rn(__fmul_rn(node_u[i], y), z) < d) {
      cur = i;
      count = 0;
      z = 1.f;
      left = -1;
      if (rank == 0 && tid == 0) path[n] = i;
      n++;
    } else {
      __syncthreads();
      if (tid == 0) {
        refused.z[count] = z;
        refused.token[count] = node_token[i];
      }
      __syncthreads();
      left = total(cur, ++count);
      z = __fmul_rn((float)left, 1.f / 1099511627776.f);
    }
  }
  if (left <= 0) left = total(cur, count = 0);
  if (rank == 0) {
    if (tid >= n && tid < t.max_tokens) path[tid] = -1;
    if (tid == 0) {
      a.n_path[b] = n;
      if (left <= 0) a.next_token[b] = -1;
    }
  }
  // floor(u W) with u a multiple of 2^-24 and W below 2^62
  const int64_t u = (int64_t)(fminf(fmaxf(a.u_sample[b], 0.f), 1.f - 1.f / 16777216.f) * 16777216.f);
  const int64_t goal = u * (left >> 24) + ((u * (left & 0xFFFFFF)) >> 24);
  // the CTA, the warp's run and then the entry in which the running sum passes the goal
  int64_t before = 0;
  const int slot = (passes - 1) & 1;
  for (int c = 0; c < rank; c++) before += cta_sum[slot][c];
  if (!(left > 0 && before <= goal && goal < before + cta_sum[slot][rank])) return;
  int w = 0;
  while (w < kWarps - 1 && before + warp_sum[w] <= goal) before += warp_sum[w++];
  const int lo = (rank * kWarps + w) * span, hi = min(lo + span, V);
  const int each = span / kThreads + 1;
  const T *p = rows_p + cur * a.p_row, *q = kCertain || count == 0 ? nullptr : rows_q + cur * a.q_row;
  auto entry = [&](int x) -> int64_t {
    return fixed(residual<kCertain, 2>(refused, weight(load(p, x)), q ? weight(load(q, x)) : 0.f, x, count));
  };
  const int x0 = lo + tid * each, x1 = min(x0 + each, hi);
  int64_t mine = 0, all;
  for (int x = x0; x < x1; x++) mine += entry(x);
  before += block_scan(mine, part, all);
  if (before <= goal && goal < before + mine) {  // one thread
    int x = x0;
    for (; x < x1 - 1; x++) {
      before += entry(x);
      if (before > goal) break;
    }
    a.next_token[b] = x;
  }
}

template <typename T>
int verify_run(const unison_kv_tree &t, const unison_kv_verify_args &a, void *stream) {
  // CTAs per session: as many as the sessions leave room for (two CTAs on a
  // multiprocessor, two rounds of them: a session takes one to four passes, and
  // those that end early make room; 128 sessions over 128,000 entries take 90 us in
  // one round, 67 in two and 73 in four, between events around the launch, which
  // add 4), none with less than 2,048 entries.
  const int room = 4 * kv_sm_count() / t.n_seqs, wanted = (a.vocab + 2047) / 2048;
  int ctas = 1;
  while (ctas < kMaxCluster && ctas * 2 <= max(room, 1) && ctas < wanted) ctas *= 2;
  return kv_launch("kv_verify", dim3(t.n_seqs * ctas), dim3(kThreads), 0, stream, ctas,
                   a.q ? verify_kernel<T, false> : verify_kernel<T, true>, t, a);
}

}  // namespace
}  // namespace unison

using namespace unison;

extern "C" int unison_kv_verify(const unison_kv_tree *tree, const unison_kv_verify_args *args, void *cuda_stream) {
  if (!tree || !args) return UNISON_ERR_ARG;
  const int rc = kv_check_tree(tree, tree->n_seqs);
  if (rc != UNISON_OK) return rc;
  if (args->vocab < 1 || args->vocab > (1 << 22)) return UNISON_ERR_RANGE;
  if (tree->n_seqs == 0) return UNISON_OK;
  if (!args->path || !args->n_path || !args->next_token || !args->u_sample || args->path_stride < tree->max_tokens)
    return UNISON_ERR_ARG;
  if (tree->n_tokens > 0 && (!args->p || !args->token || !args->u || !tree->parent)) return UNISON_ERR_ARG;
  switch (args->dtype) {
    case UNISON_KV_FP32: return verify_run<float>(*tree, *args, cuda_stream);
    case UNISON_KV_BF16: return verify_run<__nv_bfloat16>(*tree, *args, cuda_stream);
    case UNISON_KV_FP16: return verify_run<__half>(*tree, *args, cuda_stream);
    default: return UNISON_ERR_ARG;
  }
}
