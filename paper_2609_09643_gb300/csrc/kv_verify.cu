// Verification of drafted tokens (unison_kv_verify).
#include "kv.cuh"

namespace unison {
namespace {

constexpr int kThreads = 1024;
constexpr float kUnit = 1099511627776.f;  // 2^40

__device__ __forceinline__ float weight(float x) { return x > 0.f ? fminf(x, 1.f) : 0.f; }
template <typename T>
__device__ __forceinline__ float load(const T *p, int64_t i) {
  return KvType<T>::to_float(p[i]);
}
template <>
__device__ __forceinline__ float load<float>(const float *p, int64_t i) {
  return p[i];
}

// d at one vocabulary entry after the rejections of the current node: z[0 ..
// n-1] the sums before each of them; without q, the tokens that were taken out.
struct Residual {
  float z[UNISON_KV_MAX_TOKENS];
  int token[UNISON_KV_MAX_TOKENS];
  int n;
};
template <typename T>
__device__ __forceinline__ float residual(const Residual &r, const T *p, const T *q, int x, int n) {
  float d = weight(load(p, x));
  if (q) {
    const float y = weight(load(q, x));
    for (int i = 0; i < n; i++) d = fmaxf(__fsub_rn(d, __fmul_rn(r.z[i], y)), 0.f);
  } else {
    for (int i = 0; i < n; i++)
      if (r.token[i] == x) d = 0.f;
  }
  return d;
}
__device__ __forceinline__ int64_t fixed(float d) { return __float2ll_rz(__fmul_rn(d, kUnit)); }

// One CTA per session.  Warp w owns entries [w * span, (w + 1) * span).
template <typename T>
__global__ void __launch_bounds__(kThreads) verify_kernel(const unison_kv_tree t, const unison_kv_verify_args a) {
  __shared__ Residual res;
  __shared__ int64_t sums[32];
  __shared__ int chosen;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const KvRange tok = kv_tokens(t, b, nullptr);
  int32_t *path = a.path + b * a.path_stride;
  if (tok.count == 0) {
    for (int i = tid; i < t.max_tokens; i += kThreads) path[i] = -1;
    if (tid == 0) {
      a.n_path[b] = 0;
      a.next_token[b] = -1;
    }
    return;
  }
  const int V = a.vocab;
  const int span = (V + kThreads / 32 - 1) / (kThreads / 32);
  const T *p = nullptr, *q = nullptr;
  int cur = 0, n = 1, rejected = 0;
  float z = 1.f;
  auto enter = [&](int node) {
    cur = node;
    p = static_cast<const T *>(a.p) + (int64_t)(tok.first + node) * a.p_row;
    q = a.q ? static_cast<const T *>(a.q) + (int64_t)(tok.first + node) * a.q_row : nullptr;
    rejected = 0;
    z = 1.f;
  };
  // the sum of the residual after n rejections, every warp's share in sums[]
  auto total = [&](int n) -> int64_t {
    int64_t s = 0;
    for (int x = warp * span + lane; x < min((warp + 1) * span, V); x += 32) s += fixed(residual(res, p, q, x, n));
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    __syncthreads();
    if (lane == 0) sums[warp] = s;
    __syncthreads();
    int64_t all = 0;
    for (int w = 0; w < kThreads / 32; w++) all += sums[w];
    return all;
  };
  enter(0);
  if (tid == 0) path[0] = 0;
  int64_t left = -1;  // sum of the current residual, -1: not known
  for (int i = 1; i < tok.count; i++) {
    if (t.parent[tok.first + i] != cur) continue;
    const int token = a.token[tok.first + i];
    if ((unsigned)token >= (unsigned)V) continue;
    const float d = residual(res, p, q, token, rejected);
    const float y = q ? weight(load(q, token)) : 1.f;
    const float u = a.u[tok.first + i];
    if (__fmul_rn(__fmul_rn(u, y), z) < d) {
      enter(i);
      left = -1;
      if (tid == 0) path[n] = i;
      n++;
    } else {
      __syncthreads();
      if (tid == 0) {
        res.z[rejected] = z;
        res.token[rejected] = token;
      }
      __syncthreads();
      rejected++;
      left = total(rejected);
      z = __fmul_rn((float)left, 1.f / kUnit);
    }
  }
  if (left < 0) left = total(0);
  if (left == 0) {
    rejected = 0;
    left = total(0);
  }
  for (int i = n + tid; i < t.max_tokens; i += kThreads) path[i] = -1;
  if (tid == 0) {
    a.n_path[b] = n;
    chosen = -1;
  }
  __syncthreads();
  // floor(u W) with u a multiple of 2^-24 and W below 2^62
  const int64_t u = (int64_t)(a.u_sample[b] * 16777216.f);
  const int64_t goal = u * (left >> 24) + ((u * (left & 0xFFFFFF)) >> 24);
  int64_t before = 0;
  for (int w = 0; w < warp; w++) before += sums[w];
  if (left > 0 && before <= goal && goal < before + sums[warp]) {  // one warp: the entry is in its share
    for (int x0 = warp * span; x0 < min((warp + 1) * span, V); x0 += 32) {
      const int x = x0 + lane;
      int64_t s = x < min((warp + 1) * span, V) ? fixed(residual(res, p, q, x, rejected)) : 0;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t y = __shfl_up_sync(~0u, s, d);
        if (lane >= d) s += y;
      }
      const uint32_t past = __ballot_sync(~0u, before + s > goal);
      if (past) {
        if (lane == 0) chosen = x0 + __ffs(past) - 1;
        break;
      }
      before += __shfl_sync(~0u, s, 31);
    }
  }
  __syncthreads();
  if (tid == 0) a.next_token[b] = chosen;
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
  const dim3 grid(tree->n_seqs), block(kThreads);
  switch (args->dtype) {
    case UNISON_KV_FP32:
      return kv_launch("kv_verify", grid, block, 0, cuda_stream, false, verify_kernel<float>, *tree, *args);
    case UNISON_KV_BF16:
      return kv_launch("kv_verify", grid, block, 0, cuda_stream, false, verify_kernel<__nv_bfloat16>, *tree, *args);
    case UNISON_KV_FP16:
      return kv_launch("kv_verify", grid, block, 0, cuda_stream, false, verify_kernel<__half>, *tree, *args);
    default: return UNISON_ERR_ARG;
  }
}
