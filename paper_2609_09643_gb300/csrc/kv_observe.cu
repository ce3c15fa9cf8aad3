// Attention weight of accepted tokens on every cached token (unison_kv_observe):
// the variant for head sizes above 128 or more than 512 query rows, which the
// tensor cores' one (kv_observe_tc.cu) has no room for in shared memory.
#include "kv_observe.cuh"

namespace unison {
namespace {

constexpr int kThreads = 128;
constexpr int kTile = 64;   // keys of a tile: 16 of each warp
constexpr int kStages = 3;

template <int DP, int QR>
constexpr int kObserveSmem = kStages *kTile *DP * 2 + QR *DP * 2;

// The keys are the rows of the matrix product and the query rows its columns:
// a thread holds two keys' products with two query rows at a time, and adds up
// their weights without leaving its registers.  Every CTA takes an equal run of
// the call's key tiles.  Query rows beyond QR are loaded again for every tile,
// which bounds it by far then.  16 sessions of 16k keys, 8 KV heads: head size
// 256 with 4 rows 498 us (2.2 TB/s), 32 rows 570, 64 rows 721, 256 rows 9.3 ms;
// 1,024 rows of 64 or 128 elements 17 ms (512 on the tensor cores: 260, 282 us).
template <typename T, int DP, int QR>
__global__ void __launch_bounds__(kThreads) observe_kernel(const ObserveParams P) {
  follow_last_kernel();
  constexpr int kChunks = DP / 8;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ KvRunShared shared_run;
  __shared__ const T *row_k[2][kTile];
  __shared__ int64_t row_m[4][kTile];
  __shared__ float row_lse[QR];
  __shared__ uint64_t row_mask[QR];

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int D = P.c.head_dim, H = P.c.n_heads, G = P.group;
  const uint32_t k_base = smem_u32(smem);
  const uint32_t q_base = k_base + kStages * kTile * DP * 2;

  auto key_tiles_of = [&](int b) -> int { return observe_key_tiles(P, b, kTile); };
  KvRun run;
  if (!kv_find_run(run, shared_run, P.c.n_seqs, gridDim.x, blockIdx.x,
                   [&](int b) { return (int64_t)key_tiles_of(b) * H; }))
    return;
  int b = run.b;
  int64_t at = run.at, seq_begin = run.begin;
  const int64_t end = run.end;
  const float to_log2 = P.s.scale * 1.4426950408889634f;

  while (at < end) {
    int64_t mine = (int64_t)key_tiles_of(b) * H;
    while (at >= seq_begin + mine) {
      seq_begin += mine;
      mine = (int64_t)key_tiles_of(++b) * H;
    }
    const KvRange tok = kv_tokens(P.t, b, nullptr);
    const int len = kv_length(P.c, b);
    const int rows = kv_path_count(P.path, b, tok.count, nullptr) * G;
    const int key_tiles = key_tiles_of(b);
    const int last_tile = key_tiles - 1;
    const int head = (int)((at - seq_begin) / key_tiles);
    const int64_t seg_begin = seq_begin + (int64_t)head * key_tiles;
    const int kt0 = (int)(at - seg_begin);
    const int kt1 = (int)min((int64_t)key_tiles, end - seg_begin);

    auto load_rows = [&](int row0) {  // QR query rows with their statistics
      for (int i = tid; i < QR * kChunks; i += kThreads) {
        const int r = row0 + i / kChunks, c = i % kChunks;
        const int node = r < rows ? observe_node(P, b, tok.count, r / G) : -1;
        const bool ok = node >= 0;
        const T *src = static_cast<const T *>(P.s.q);
        if (ok) src += (tok.first + node) * P.s.q_token + (head * G + r % G) * P.s.q_head;
        cp_async16(swizzled<DP>(q_base, i / kChunks, c), c * 8 < D ? src + c * 8 : src, ok && c * 8 < D);
        if (c == 0) {
          float l = INFINITY;  // no weight from this row
          uint64_t mask = 0;
          if (ok) {
            l = P.s.lse[(int64_t)(tok.first + node) * P.s.n_q_heads + head * G + r % G] * 1.4426950408889634f;
            if (l == -INFINITY) l = INFINITY;
            mask = P.t.mask ? P.t.mask[tok.first + node] : ~0ull >> (63 - node);
          }
          row_lse[i / kChunks] = l;
          row_mask[i / kChunks] = mask;
        }
      }
    };
    auto find_page = [&](int kt, int &off) -> int {
      const int slot = kt * kTile + tid;
      off = 0;
      if (tid >= kTile || kt >= last_tile || slot >= len) return kNoSlot;
      return kv_page_load(P.c, b, slot, off);
    };
    auto put_rows = [&](int kt, int page, int off) {
      if (tid >= kTile) return;
      const T *k = nullptr;
      int64_t m = -1;
      if (kt == last_tile) {
        if (tid < tok.count && P.s.mass_new) {
          k = static_cast<const T *>(P.s.k_new) + (tok.first + tid) * P.s.k_token + head * P.s.k_head;
          m = (int64_t)(tok.first + tid) * H + head;
        }
      } else if ((page = kv_page_ok(P.c, b, page)) >= 0) {
        k = static_cast<const T *>(P.c.k) + page * P.c.k_page + head * P.c.k_head + off * P.c.k_slot;
        m = page * P.c.m_page + head * P.c.m_head + off * P.c.m_slot;
      }
      row_k[kt & 1][tid] = k;
      row_m[kt & 3][tid] = m;
    };
    auto copy_tile = [&](int kt) {
      const uint32_t st = k_base + ((kt - kt0) % kStages) * (kTile * DP * 2);
#pragma unroll
      for (int i = 0; i < kTile * kChunks / kThreads; i++) {
        const int r = (i * kThreads + tid) / kChunks, c = (i * kThreads + tid) % kChunks;
        const T *k = row_k[kt & 1][r];
        const bool ok = k != nullptr && c * 8 < D;
        cp_async16(swizzled<DP>(st, r, c), ok ? k + c * 8 : static_cast<const T *>(P.s.q), ok);
      }
    };

    __syncthreads();
    const bool one_load = rows <= QR;
    load_rows(0);
    cp_commit();
    int page, off;
    for (int s = 0; s < kStages - 1; s++) {
      const int kt = kt0 + s;
      if (kt < kt1) {
        page = find_page(kt, off);
        put_rows(kt, page, off);
      }
      __syncthreads();
      if (kt < kt1) copy_tile(kt);
      cp_commit();
    }
    if (kt0 + kStages - 1 < kt1) {
      page = find_page(kt0 + kStages - 1, off);
      put_rows(kt0 + kStages - 1, page, off);
    }
    page = find_page(kt0 + kStages, off);

    for (int kt = kt0; kt < kt1; kt++) {
      cp_wait<kStages - 2>();
      __syncthreads();
      if (kt + kStages - 1 < kt1) copy_tile(kt + kStages - 1);
      cp_commit();
      const int64_t m0 = row_m[kt & 3][warp * 16 + (lane >> 2)], m1 = row_m[kt & 3][warp * 16 + (lane >> 2) + 8];
      if (kt + kStages < kt1) put_rows(kt + kStages, page, off);
      page = find_page(kt + kStages + 1, off);

      const uint32_t ks = k_base + ((kt - kt0) % kStages) * (kTile * DP * 2);
      uint32_t a[DP / 16][4];
#pragma unroll
      for (int d = 0; d < DP / 16; d++) ldm4(a[d], swizzled<DP>(ks, warp * 16 + (lane & 15), d * 2 + (lane >> 4)));
      float sum0 = 0.f, sum1 = 0.f;
      for (int row0 = 0; row0 < rows; row0 += QR) {
        if (!one_load) {  // more rows than the shared memory holds: round by round
          __syncthreads();
          load_rows(row0);
          cp_commit();
          cp_wait<0>();
          __syncthreads();
        }
        const int n = min(rows - row0, QR);
        for (int r = 0; r < n; r += 16) {
          float c[2][4] = {};
#pragma unroll
          for (int d = 0; d < DP / 16; d++) {
            uint32_t q[4];
            ldm4(q, swizzled<DP>(q_base, r + ((lane >> 4) << 3) + (lane & 7), d * 2 + ((lane >> 3) & 1)));
            mma16816<T>(c[0], a[d], q[0], q[1]);
            mma16816<T>(c[1], a[d], q[2], q[3]);
          }
#pragma unroll
          for (int j = 0; j < 2; j++) {
#pragma unroll
            for (int e = 0; e < 2; e++) {
              const int row = r + j * 8 + (lane & 3) * 2 + e;
              const float l = row_lse[row];
              bool see0 = l != INFINITY, see1 = see0;
              if (kt == last_tile) {
                const uint64_t mask = row_mask[row];
                see0 = see0 && (mask >> (warp * 16 + (lane >> 2)) & 1);
                see1 = see1 && (mask >> (warp * 16 + (lane >> 2) + 8) & 1);
              }
              sum0 += see0 ? exp2_fast(fmaf(c[j][e], to_log2, -l)) : 0.f;
              sum1 += see1 ? exp2_fast(fmaf(c[j][2 + e], to_log2, -l)) : 0.f;
            }
          }
        }
      }
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) {
        sum0 += __shfl_xor_sync(~0u, sum0, d);
        sum1 += __shfl_xor_sync(~0u, sum1, d);
      }
      if ((lane & 3) == 0) {
        if (kt == last_tile) {
          if (m0 >= 0) P.s.mass_new[m0] = sum0;
          if (m1 >= 0) P.s.mass_new[m1] = sum1;
        } else {
          if (m0 >= 0) P.c.mass[m0] += sum0;
          if (m1 >= 0) P.c.mass[m1] += sum1;
        }
      }
    }
    cp_wait<0>();
    at = seg_begin + kt1;
  }
}

template <typename T, int DP, int QR>
int observe_run(const ObserveParams &p, void *stream) {
  static uint64_t done = 0;
  constexpr int smem = kObserveSmem<DP, QR>;
  if (!kv_allow_smem(reinterpret_cast<const void *>(observe_kernel<T, DP, QR>), smem, &done)) return UNISON_ERR_CUDA;
  const int per_sm = max(1, min(4, (220 << 10) / (smem + QR * 12 + 5000)));
  return kv_launch("kv_observe", dim3(kv_sm_count() * per_sm), dim3(kThreads), smem, stream, 1,
                   observe_kernel<T, DP, QR>, p);
}

template <typename T>
int observe_pick(const ObserveParams &p, int max_rows, void *stream) {
  const int d = p.c.head_dim;
  if (d <= 128 && max_rows <= kObserveTcRows)
    return d <= 64 ? observe_tc<T, 64>(p, max_rows, stream) : observe_tc<T, 128>(p, max_rows, stream);
  return d <= 128 ? observe_run<T, 128, 512>(p, stream) : observe_run<T, 256, 192>(p, stream);
}

}  // namespace
}  // namespace unison

using namespace unison;

extern "C" int unison_kv_observe(const unison_kv_cache *cache, const unison_kv_tree *tree, const unison_kv_step *step,
                                 const unison_kv_path *path, void *cuda_stream) {
  int rc = kv_check_cache(cache);
  if (rc == UNISON_OK) rc = kv_check_tree(tree, cache->n_seqs);
  if (rc != UNISON_OK) return rc;
  if (!step) return UNISON_ERR_ARG;
  if (step->n_q_heads < 1 || step->n_q_heads % cache->n_heads || step->n_q_heads / cache->n_heads > 64)
    return UNISON_ERR_RANGE;
  if (cache->n_seqs == 0 || tree->n_tokens == 0) return UNISON_OK;
  if (!kv_rows_ok(step->q, step->q_token, step->q_head) || !step->lse) return UNISON_ERR_ARG;
  if (step->mass_new && !kv_rows_ok(step->k_new, step->k_token, step->k_head)) return UNISON_ERR_ARG;
  if (cache->max_pages > 0 && cache->n_pages > 0 &&
      (!kv_rows_ok(cache->k, cache->k_page | cache->k_head, cache->k_slot) || !cache->mass))
    return UNISON_ERR_ARG;
  if (path && path->path && (!path->n_path || path->path_stride < 0)) return UNISON_ERR_ARG;
  ObserveParams p = {};
  p.c = *cache;
  p.t = *tree;
  p.s = *step;
  p.path = path ? *path : unison_kv_path{};
  p.group = step->n_q_heads / cache->n_heads;
  const int max_rows = tree->max_tokens * p.group;
  return cache->dtype == UNISON_KV_BF16 ? observe_pick<__nv_bfloat16>(p, max_rows, cuda_stream)
                                        : observe_pick<__half>(p, max_rows, cuda_stream);
}
