// Changes of the paged cache: accepted tokens into it (unison_kv_commit), the
// least attended ones out of it (unison_kv_evict).
#include "kv.cuh"

namespace unison {
namespace {

// ---------------------------------------------------------------- commit --
struct CommitParams {
  unison_kv_cache c;
  unison_kv_tree t;
  unison_kv_step s;
  unison_kv_path path;
};

// One CTA per session; a thread moves 16 bytes at a time.
template <typename T>
__global__ void __launch_bounds__(256) commit_kernel(const CommitParams P) {
  const int b = blockIdx.x, tid = threadIdx.x;
  const int H = P.c.n_heads, chunks = P.c.head_dim / 8;
  const KvRange tok = kv_tokens(P.t, b, P.c.status);
  const int n = P.path.path ? min(max(P.path.n_path[b], 0), tok.count) : tok.count;
  const int len = kv_length(P.c, b);
  const int pos = P.c.next_pos ? P.c.next_pos[b] : len;
  bool full = len + n > P.c.max_pages * P.c.page_size;
  int off;
  if (!full && tid < n) full = kv_page(P.c, b, len + tid, off) < 0;
  // (every thread has also read what the first one will change)
  if (__syncthreads_or(full)) {
    if (tid == 0 && P.c.status) P.c.status[b] = UNISON_ERR_CAPACITY;
    return;
  }
  const int per_row = H * chunks;
  for (int i = tid; i < n * per_row; i += blockDim.x) {
    const int row = i / per_row, h = i % per_row / chunks, c = i % chunks;
    const int node = P.path.path ? P.path.path[(int64_t)b * P.path.path_stride + row] : row;
    const int page = kv_page(P.c, b, len + row, off);
    if (page < 0 || (unsigned)node >= (unsigned)tok.count) {
      if (P.c.status) P.c.status[b] = UNISON_ERR_RANGE;
      continue;
    }
    const int64_t from = tok.first + node;
    const int4 k = *reinterpret_cast<const int4 *>(static_cast<const T *>(P.s.k_new) + from * P.s.k_token +
                                                   h * P.s.k_head + c * 8);
    const int4 v = *reinterpret_cast<const int4 *>(static_cast<const T *>(P.s.v_new) + from * P.s.v_token +
                                                   h * P.s.v_head + c * 8);
    *reinterpret_cast<int4 *>(static_cast<T *>(P.c.k) + page * P.c.k_page + h * P.c.k_head + off * P.c.k_slot + c * 8) = k;
    *reinterpret_cast<int4 *>(static_cast<T *>(P.c.v) + page * P.c.v_page + h * P.c.v_head + off * P.c.v_slot + c * 8) = v;
    if (c == 0) {
      const int64_t m = page * P.c.m_page + h * P.c.m_head + off * P.c.m_slot;
      if (P.c.mass) P.c.mass[m] = P.s.mass_new ? P.s.mass_new[from * H + h] : 0.f;
      if (P.c.pos) P.c.pos[m] = pos + row;
    }
  }
  if (tid == 0) {
    P.c.length[b] = len + n;
    if (P.c.next_pos) P.c.next_pos[b] = pos + n;
  }
}

// ----------------------------------------------------------------- evict --
struct EvictParams {
  unison_kv_cache c, to;  // to: the cache itself where slots move in place
  const int32_t *keep;
  int32_t sink, recent;
  bool in_place;
  int32_t *from, *into;  // [sessions * heads][slots of a session] moves
  int32_t *count;        // [sessions * heads]
};

constexpr int kSelect = 1024;

// Order of a slot among its session's: protected slots above all, then larger
// mass (the bits of a float, turned so that unsigned order is the numbers'
// order, -0 as 0), NaN and slots without a page below all.
__device__ __forceinline__ uint32_t slot_key(const EvictParams &P, int b, int h, int slot, int next) {
  int off;
  const int page = kv_page(P.c, b, slot, off);
  if (page < 0) return 0;
  const int64_t m = page * P.c.m_page + h * P.c.m_head + off * P.c.m_slot;
  const int pos = P.c.pos ? P.c.pos[m] : slot;
  if (pos < P.sink || (int64_t)pos >= (int64_t)next - P.recent) return ~0u;
  const float x = P.c.mass[m] + 0.f;
  if (isnan(x)) return 0;
  const uint32_t u = __float_as_uint(x);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// How many slots of a session stay.
__device__ __forceinline__ int kept_count(const EvictParams &P, int b, int len) {
  int n = min(len, max(P.keep[b], 0));
  if (!P.in_place) {
    const int room = P.to.max_pages * P.to.page_size;
    if (n > room) {
      n = room;
      if (P.to.status) P.to.status[b] = UNISON_ERR_CAPACITY;
    }
  }
  return n;
}

// One CTA per session and head lists the moves.  The key of the last slot that
// stays is found digit by digit (four counts of 256), then one pass in slot
// order ranks the slots with that very key and pairs sources with targets.
__global__ void __launch_bounds__(kSelect) evict_select_kernel(const EvictParams P) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t prefix, rest;
  __shared__ int64_t part[33];
  const int tid = threadIdx.x;
  const int b = blockIdx.x / P.c.n_heads, h = blockIdx.x % P.c.n_heads;
  const int len = kv_length(P.c, b);
  const int n = kept_count(P, b, len);
  const int next = P.c.pos && P.c.next_pos ? P.c.next_pos[b] : len;
  const int64_t room = (int64_t)P.c.max_pages * P.c.page_size;
  int32_t *from = P.from + blockIdx.x * room, *into = P.into + blockIdx.x * room;
  if (n == 0 || (P.in_place && n == len)) {
    if (tid == 0) P.count[blockIdx.x] = 0;
    return;
  }
  uint32_t last_key = 0;  // of the slots that stay
  int ties = 0;           // slots with that key that stay, the lowest first
  if (n < len) {
    if (tid == 0) prefix = 0, rest = n;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const uint32_t have = prefix;
      for (int s = tid; s < len; s += kSelect) {
        const uint32_t k = slot_key(P, b, h, s, next);
        if (shift == 24 || k >> (shift + 8) == have) atomicAdd(&hist[k >> shift & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        uint32_t left = rest;
        int d = 255;
        while (d > 0 && hist[d] < left) left -= hist[d--];
        rest = left;
        prefix = have << 8 | d;
      }
      __syncthreads();
    }
    last_key = prefix;
    ties = (int)rest;
  }
  int64_t ties_seen = 0, free_seen = 0, moved = 0;
  for (int s0 = 0; s0 < len; s0 += kSelect) {
    const int s = s0 + tid;
    const uint32_t k = s < len ? slot_key(P, b, h, s, next) : 0;
    bool stays = s < len;
    int64_t all;
    if (n < len) {
      const bool tie = s < len && k == last_key;
      const int64_t rank = ties_seen + block_scan(tie, part, all);
      ties_seen += all;
      stays = s < len && (k > last_key || (tie && rank < ties));
    }
    if (P.in_place) {
      const bool target = s < n && !stays, source = s >= n && stays;
      const int64_t r = block_scan((int64_t)target << 32 | source, part, all);
      if (target) into[free_seen + (r >> 32)] = s;
      if (source) from[moved + (r & 0xFFFFFFFF)] = s;
      free_seen += all >> 32;
      moved += all & 0xFFFFFFFF;
    } else {
      const int64_t r = block_scan(stays, part, all);
      if (stays) from[moved + r] = s;
      moved += all;
    }
  }
  if (tid == 0) P.count[blockIdx.x] = (int)(P.in_place ? min(moved, free_seen) : moved);
}

// A warp moves one slot at a time: keys, values, mass and position.
template <typename T>
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictParams P) {
  const int seg = blockIdx.y, lane = threadIdx.x & 31;
  const int b = seg / P.c.n_heads, h = seg % P.c.n_heads;
  const int chunks = P.c.head_dim / 8;
  const int64_t room = (int64_t)P.c.max_pages * P.c.page_size;
  const int32_t *from = P.from + seg * room, *into = P.into + seg * room;
  const int count = P.count[seg];
  const int warps = gridDim.x * (blockDim.x >> 5);
  for (int i = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); i < count; i += warps) {
    int off, to_off;
    const int page = kv_page(P.c, b, from[i], off);
    const int to_page = kv_page(P.to, b, P.in_place ? into[i] : i, to_off);
    if (page < 0 || to_page < 0) continue;
    const T *k = static_cast<const T *>(P.c.k) + page * P.c.k_page + h * P.c.k_head + off * P.c.k_slot;
    const T *v = static_cast<const T *>(P.c.v) + page * P.c.v_page + h * P.c.v_head + off * P.c.v_slot;
    T *tk = static_cast<T *>(P.to.k) + to_page * P.to.k_page + h * P.to.k_head + to_off * P.to.k_slot;
    T *tv = static_cast<T *>(P.to.v) + to_page * P.to.v_page + h * P.to.v_head + to_off * P.to.v_slot;
    for (int c = lane; c < 2 * chunks; c += 32) {
      if (c < chunks)
        reinterpret_cast<int4 *>(tk)[c] = reinterpret_cast<const int4 *>(k)[c];
      else
        reinterpret_cast<int4 *>(tv)[c - chunks] = reinterpret_cast<const int4 *>(v)[c - chunks];
    }
    if (lane == 0) {
      const int64_t m = page * P.c.m_page + h * P.c.m_head + off * P.c.m_slot;
      const int64_t tm = to_page * P.to.m_page + h * P.to.m_head + to_off * P.to.m_slot;
      if (P.to.mass) P.to.mass[tm] = P.c.mass[m];
      if (P.to.pos && P.c.pos) P.to.pos[tm] = P.c.pos[m];
    }
  }
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) {
    P.to.length[b] = kept_count(P, b, kv_length(P.c, b));
    if (!P.in_place && P.to.next_pos && P.c.next_pos) P.to.next_pos[b] = P.c.next_pos[b];
  }
}

uint64_t evict_bytes(const unison_kv_cache *c) {
  const uint64_t segs = (uint64_t)c->n_seqs * c->n_heads;
  return segs * 4 + 2 * segs * c->max_pages * c->page_size * 4;
}

}  // namespace
}  // namespace unison

using namespace unison;

static bool pools_ok(const unison_kv_cache *c) {
  return (c->max_pages == 0 || c->n_pages == 0) || (kv_rows_ok(c->k, c->k_page | c->k_head, c->k_slot) &&
                                                    kv_rows_ok(c->v, c->v_page | c->v_head, c->v_slot));
}

extern "C" int unison_kv_commit(const unison_kv_cache *cache, const unison_kv_tree *tree, const unison_kv_step *step,
                                const unison_kv_path *path, void *cuda_stream) {
  int rc = kv_check_cache(cache);
  if (rc == UNISON_OK) rc = kv_check_tree(tree, cache->n_seqs);
  if (rc != UNISON_OK) return rc;
  if (!step) return UNISON_ERR_ARG;
  if (cache->n_seqs == 0 || tree->n_tokens == 0) return UNISON_OK;
  if (!kv_rows_ok(step->k_new, step->k_token, step->k_head) || !kv_rows_ok(step->v_new, step->v_token, step->v_head) ||
      !pools_ok(cache))
    return UNISON_ERR_ARG;
  if (path && path->path && (!path->n_path || path->path_stride < 0)) return UNISON_ERR_ARG;
  const CommitParams p = {*cache, *tree, *step, path ? *path : unison_kv_path{}};
  // 16-bit types move as they are
  return kv_launch("kv_commit", dim3(cache->n_seqs), dim3(256), 0, cuda_stream, false, commit_kernel<uint16_t>, p);
}

extern "C" uint64_t unison_kv_evict_workspace(const unison_kv_cache *cache) {
  return kv_check_cache(cache) == UNISON_OK ? evict_bytes(cache) : 0;
}

extern "C" int unison_kv_evict(const unison_kv_cache *cache, const unison_kv_cache *into, const int32_t *keep,
                               int32_t sink, int32_t recent, void *workspace, uint64_t workspace_bytes,
                               void *cuda_stream) {
  int rc = kv_check_cache(cache);
  if (rc != UNISON_OK) return rc;
  if (into) {
    rc = kv_check_cache(into);
    if (rc != UNISON_OK) return rc;
    if (into->n_seqs != cache->n_seqs || into->n_heads != cache->n_heads || into->head_dim != cache->head_dim ||
        into->dtype != cache->dtype)
      return UNISON_ERR_ARG;
  }
  if (sink < 0 || recent < 0) return UNISON_ERR_RANGE;
  const uint64_t segs = (uint64_t)cache->n_seqs * cache->n_heads;
  if (segs > 65535) return UNISON_ERR_RANGE;
  if (cache->n_seqs == 0) return UNISON_OK;
  if (!keep || !pools_ok(cache) || (into && !pools_ok(into))) return UNISON_ERR_ARG;
  if (cache->max_pages > 0 && cache->n_pages > 0 && !cache->mass) return UNISON_ERR_ARG;
  if (!workspace || !kv_aligned(workspace, 16) || workspace_bytes < evict_bytes(cache)) return UNISON_ERR_ARG;
  EvictParams p;
  p.c = *cache;
  p.to = into ? *into : *cache;
  p.keep = keep;
  p.sink = sink;
  p.recent = recent;
  p.in_place = into == nullptr;
  p.from = static_cast<int32_t *>(workspace);
  p.into = p.from + segs * cache->max_pages * cache->page_size;
  p.count = p.into + segs * cache->max_pages * cache->page_size;
  rc = kv_launch("kv_evict_select", dim3((unsigned)segs), dim3(kSelect), 0, cuda_stream, false, evict_select_kernel, p);
  if (rc != UNISON_OK) return rc;
  const unsigned per_seg = (unsigned)max((uint64_t)1, ((uint64_t)kv_sm_count() * 8 + segs - 1) / segs);
  return kv_launch("kv_evict_move", dim3(per_seg, (unsigned)segs), dim3(256), 0, cuda_stream, false,
                   evict_move_kernel<uint16_t>, p);
}
