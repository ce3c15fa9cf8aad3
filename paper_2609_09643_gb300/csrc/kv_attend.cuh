// What the attention kernels share (kv_attend.cu, kv_attend_tc.cu).
#pragma once

#include "kv.cuh"

namespace unison {

// What a CTA leaves to be joined: the segment (one session, KV head and row
// tile) that begins in its run and goes on in the runs up to `last`.
struct AttendPart {
  int b, head, row_tile, last;  // last < 0: nothing
};

struct AttendParams {
  unison_kv_cache c;
  unison_kv_tree t;
  unison_kv_step s;
  AttendPart *part;  // [grid]
  float *partial;    // [grid][2]: sums [rows][DP], maxima [rows] (log2), sums of weights [rows]
  int group;         // query heads of a KV head
  int rows;          // of a row tile
  int row_groups;    // CTAs of a run, with row tiles of their own
};

// Key tiles of a session; the last one holds its new tokens.
__device__ __forceinline__ int attend_key_tiles(int len, int tokens, int tile) {
  return tokens ? (len + tile - 1) / tile + 1 : 0;
}

constexpr int kTcRows = 256;  // query rows of a CTA on the tensor cores: two tiles of 128
template <typename T, int DP>
int attend_tc(const AttendParams &p, int grid, void *stream);

}  // namespace unison
