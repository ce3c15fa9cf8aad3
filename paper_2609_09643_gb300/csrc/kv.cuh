// Shared parts of the KV-cache operators (include/unison_kv.h): argument
// checks on the host, guarded look-ups and matrix fragments on the device.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/unison_kv.h"
#include "common.cuh"
#include "profile.cuh"

namespace unison {

// ------------------------------------------------------------------ host --
inline bool kv_aligned(const void *p, size_t b) { return (reinterpret_cast<uintptr_t>(p) & (b - 1)) == 0; }
inline bool kv_rows_ok(const void *p, int64_t s0, int64_t s1) {
  return p && kv_aligned(p, 16) && s0 % 8 == 0 && s1 % 8 == 0;
}

// Sizes of a cache, and the arrays that every operator reads.
inline int kv_check_cache(const unison_kv_cache *c) {
  if (!c) return UNISON_ERR_ARG;
  if (c->n_seqs < 0 || c->max_pages < 0 || c->n_pages < 0 || c->page_size < 1 || c->n_heads < 1)
    return UNISON_ERR_RANGE;
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return UNISON_ERR_RANGE;
  if (c->dtype != UNISON_KV_BF16 && c->dtype != UNISON_KV_FP16) return UNISON_ERR_ARG;
  if ((int64_t)c->max_pages * c->page_size >= (1ll << 31) - (1 << 16)) return UNISON_ERR_RANGE;  // tiles round up
  if (c->n_seqs > 0 && (!c->length || (c->max_pages > 0 && !c->page_table))) return UNISON_ERR_ARG;
  return UNISON_OK;
}

inline int kv_check_tree(const unison_kv_tree *t, int n_seqs) {
  if (!t) return UNISON_ERR_ARG;
  if (t->n_seqs < 0 || t->n_tokens < 0) return UNISON_ERR_RANGE;
  if (t->n_seqs != n_seqs) return UNISON_ERR_ARG;
  if (t->max_tokens < 1 || t->max_tokens > UNISON_KV_MAX_TOKENS) return UNISON_ERR_RANGE;
  if (t->n_seqs > 0 && !t->offsets) return UNISON_ERR_ARG;
  return UNISON_OK;
}

// A cache as the kernels take it: with slot / page_size as a multiplication
// (Granlund and Montgomery: for n < 2^31, n / d = (high(n m) + n) >> l with
// l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1).
struct KvCacheArg : unison_kv_cache {
  uint32_t page_mul, page_shift;
  KvCacheArg() = default;
  KvCacheArg(const unison_kv_cache &c) : unison_kv_cache(c), page_shift(0) {
    const uint64_t d = (uint32_t)c.page_size;
    while ((1ull << page_shift) < d) page_shift++;
    page_mul = (uint32_t)((((1ull << page_shift) - d) << 32) / d + 1);
  }
};

// Multiprocessors of the current device, asked for once per device.
int kv_sm_count();

// Raises a kernel's dynamic shared memory limit, once per device and kernel
// (`done`: a bit per device, kept by the caller beside the kernel).
bool kv_allow_smem(const void *kernel, int bytes, uint64_t *done);

// Queues a kernel of clusters of `cluster` CTAs.  It may be set up while the
// kernel before it on the stream ends: all of these kernels begin with
// follow_last_kernel().  The verdict is the launch's own, not an older error's.
template <typename... P, typename... A>
int kv_launch(const char *name, dim3 grid, dim3 block, size_t smem, void *stream, int cluster, void (*kernel)(P...),
              A &&...args) {
  cudaError_t e;
  {
    ProfSpan span(name, static_cast<cudaStream_t>(stream));
    cudaLaunchConfig_t lc = {};
    lc.gridDim = grid;
    lc.blockDim = block;
    lc.dynamicSmemBytes = smem;
    lc.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = cluster > 1 ? 2 : 1;
    e = cudaLaunchKernelEx(&lc, kernel, static_cast<P>(args)...);
  }
  count_launches(1);
  if (e == cudaSuccess) return UNISON_OK;
  cudaGetLastError();
  return UNISON_ERR_CUDA;
}

// ---------------------------------------------------------------- device --
template <typename T>
struct KvType;
template <>
struct KvType<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t pack(float a, float b) {  // a in the low half
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  static __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
  static constexpr uint32_t kExponent = 0x7F80u;  // all ones: infinity or NaN
  static constexpr int kMostWeight = 0;  // (log2)
};
template <>
struct KvType<__half> {
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  static __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
  static constexpr uint32_t kExponent = 0x7C00u;
  static constexpr int kMostWeight = 15;  // the largest number is just below 2^16
};

// A session's rows of the step's arrays, clamped to what the tree allows.
struct KvRange {
  int first, count;
};
__device__ __forceinline__ KvRange kv_tokens(const unison_kv_tree &t, int b, int32_t *status) {
  const int lo = t.offsets[b], hi = t.offsets[b + 1];
  const int first = min(max(lo, 0), t.n_tokens);
  const int last = min(max(hi, first), t.n_tokens);
  const int count = min(last - first, t.max_tokens);
  if (status && (lo != first || hi != first + count)) status[b] = UNISON_ERR_RANGE;
  return {first, count};
}
__device__ __forceinline__ int kv_length(const unison_kv_cache &c, int b) {
  const int n = c.length[b], room = c.max_pages * c.page_size;
  const int len = min(max(n, 0), room);
  if (c.status && n != len) c.status[b] = UNISON_ERR_RANGE;
  return len;
}
// Accepted nodes of a session of `tokens`, clamped, and the i-th of them, or -1
// where the path names another.
__device__ __forceinline__ int kv_path_count(const unison_kv_path &p, int b, int tokens, int32_t *status) {
  if (!p.path) return tokens;
  const int n = p.n_path[b], count = min(max(n, 0), tokens);
  if (status && n != count) status[b] = UNISON_ERR_RANGE;
  return count;
}
__device__ __forceinline__ int kv_path_node(const unison_kv_path &p, int b, int tokens, int i) {
  const int node = p.path ? p.path[(int64_t)b * p.path_stride + i] : i;
  return (unsigned)node < (unsigned)tokens ? node : -1;
}
// Page of a slot (below max_pages * page_size), as the table has it: to be
// checked by kv_page_ok when it is used, so that the load may be on its way.
constexpr int kNoSlot = INT32_MIN;
__device__ __forceinline__ int kv_page_load(const KvCacheArg &c, int b, int slot, int &off) {
  const unsigned i = (__umulhi((unsigned)slot, c.page_mul) + (unsigned)slot) >> c.page_shift;
  off = slot - (int)(i * (unsigned)c.page_size);
  return __ldg(c.page_table + (int64_t)b * c.max_pages + i);
}
__device__ __forceinline__ int kv_page_ok(const unison_kv_cache &c, int b, int page) {
  if ((unsigned)page < (unsigned)c.n_pages) return page;
  if (page != kNoSlot && c.status) c.status[b] = UNISON_ERR_RANGE;
  return -1;
}
// Page of a slot, or -1.
__device__ __forceinline__ int kv_page(const KvCacheArg &c, int b, int slot, int &off) {
  return kv_page_ok(c, b, kv_page_load(c, b, slot, off));
}

// The kernel before this one is complete and its results are seen; the next one
// may be set up from here on (it waits in the same way).
__device__ __forceinline__ void follow_last_kernel() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ uint32_t smem_u32(const void *p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// 16 bytes into shared memory, zeros where !valid (src is then not read).
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool valid) {
  const int bytes = valid ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                                        uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
               "{%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
               "{%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// What the weights 2^(score - reference) of a row are relative to, from its
// maximum: the maximum itself in bf16.  In fp16 a weight below 2^-25 would count
// in the row's sum but not in its products, so the reference lies kLower below
// the maximum, as far as weights may exceed 1.  (Scores beyond 2^20 have no use
// for it, and the difference would be rounded: a weight might not be finite.)
template <int kLower>
__device__ __forceinline__ float reference_of(float top) {
  return kLower > 0 && fabsf(top) < 1048576.f ? top - kLower : top;
}
// 2^x; results below the normal range are 0.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A row of DP elements in shared memory is DP / 8 chunks of 16 bytes; chunk c
// of row r lies at c ^ (r & 7), so that the eight rows of a matrix fragment
// are in different banks.
template <int DP>
__device__ __forceinline__ uint32_t swizzled(uint32_t base, int row, int chunk) {
  return base + row * (DP * 2) + ((chunk ^ (row & 7)) << 4);
}

// ------------------------------------------------- sharing out the tiles --
// All threads of a CTA add their values; every thread gets the exclusive
// prefix and the sum.  `part`: 33 words of shared memory.
template <typename I>
__device__ __forceinline__ I block_scan(I x, I *part, I &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (blockDim.x + 31) >> 5;
  I y = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const I z = __shfl_up_sync(~0u, y, d);
    if (lane >= d) y += z;
  }
  __syncthreads();
  if (lane == 31) part[warp] = y;
  __syncthreads();
  if (warp == 0) {
    const I mine = lane < warps ? part[lane] : 0;
    I s = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const I z = __shfl_up_sync(~0u, s, d);
      if (lane >= d) s += z;
    }
    __syncwarp();
    part[lane] = s - mine;
    if (lane == 31) part[32] = s;
  }
  __syncthreads();
  total = part[32];
  return part[warp] + y - x;
}

// The work of a call is a list of key tiles, session by session.  Every run
// (one CTA, or a few that share its keys) takes an equal stretch of the list,
// whatever the sessions' lengths are.
struct KvRun {
  int64_t total;  // tiles of the call
  int runs;       // that have work: one tile at least
  int64_t at, end;
  int b;          // the session that `at` lies in
  int64_t begin;  // index of its first tile
};
struct KvRunShared {
  int64_t part[33], begin;
  int b;
};
// By all threads of a CTA.  tiles(b): tiles of session b; most(total): how many
// runs there may be.  False: no work.
struct KvAnyRuns {
  __device__ __forceinline__ int64_t operator()(int64_t total) const { return total; }
};
template <typename F, typename M = KvAnyRuns>
__device__ __forceinline__ bool kv_find_run(KvRun &r, KvRunShared &sh, int n_seqs, int runs, int run, F tiles,
                                            M most = M()) {
  const int tid = threadIdx.x, step = blockDim.x;
  int64_t mine = tid < n_seqs ? (int64_t)tiles(tid) : 0, n;
  int64_t before = block_scan(mine, sh.part, n);
  r.total = n;
  for (int b0 = step; b0 < n_seqs; b0 += step) {
    block_scan(b0 + tid < n_seqs ? (int64_t)tiles(b0 + tid) : 0, sh.part, n);
    r.total += n;
  }
  r.runs = (int)min((int64_t)runs, most(r.total));
  if (run >= r.runs) return false;
  r.at = r.total * run / r.runs;
  r.end = r.total * (run + 1) / r.runs;
  int64_t sum = 0;
  for (int b0 = 0;; b0 += step) {
    if (n_seqs > step) {  // else the first values still stand
      mine = b0 + tid < n_seqs ? (int64_t)tiles(b0 + tid) : 0;
      before = sum + block_scan(mine, sh.part, n);
    }
    if (r.at >= before && r.at < before + mine) {
      sh.b = b0 + tid;
      sh.begin = before;
    }
    sum += n_seqs > step ? n : r.total;
    if (r.at < sum) break;
  }
  __syncthreads();
  r.b = sh.b;
  r.begin = sh.begin;
  return true;
}
// The run in whose stretch a tile lies.
__device__ __forceinline__ int kv_run_of(const KvRun &r, int64_t tile) {
  int c = (int)min((tile + 1) * r.runs / r.total, (int64_t)r.runs - 1);  // about right: the exact one is a step away
  while (c > 0 && r.total * c / r.runs > tile) c--;
  while (r.total * (c + 1) / r.runs <= tile) c++;
  return c;
}

}  // namespace unison
