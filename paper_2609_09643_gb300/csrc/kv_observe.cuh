// What the kernels of unison_kv_observe share.
#pragma once

#include "kv.cuh"

namespace unison {

struct ObserveParams {
  KvCacheArg c;
  unison_kv_tree t;
  unison_kv_step s;
  unison_kv_path path;
  int group;         // query heads of a KV head
  int q_rows, q_buffers, slots;  // tensor cores: query rows that fit, how often, key tiles on their way
};

// Key tiles of a session; the last one holds its new tokens, the only one
// where no token was accepted.
__device__ __forceinline__ int observe_key_tiles(const ObserveParams &P, int b, int tile) {
  const int tokens = kv_tokens(P.t, b, P.c.status).count;
  if (!tokens) return 0;
  return kv_path_count(P.path, b, tokens, P.c.status) ? (kv_length(P.c, b) + tile - 1) / tile + 1 : 1;
}
// Node i of a session's accepted path, or -1, which is reported.
__device__ __forceinline__ int observe_node(const ObserveParams &P, int b, int tokens, int i) {
  const int node = kv_path_node(P.path, b, tokens, i);
  if (node < 0 && P.c.status) P.c.status[b] = UNISON_ERR_RANGE;
  return node;
}

constexpr int kObserveTcRows = 512;  // most query rows per KV head on the tensor cores
template <typename T, int DP>
int observe_tc(ObserveParams p, int max_rows, void *stream);

}  // namespace unison
