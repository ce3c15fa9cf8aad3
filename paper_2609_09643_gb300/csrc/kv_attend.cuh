// What the attention kernels share (kv_attend.cu, kv_attend_tc.cu).
#pragma once

#include "kv.cuh"

namespace unison {

// What a CTA leaves to be joined: the segment (one session, KV head and row
// tile) that begins in its run and goes on in the runs up to `last`.  Whole
// pieces of 16 bytes: the sums follow [grid] of them in the workspace, and are
// read and written 16 bytes at a time.
struct alignas(16) AttendPart {
  int last;                      // < 0: nothing
  int head, first_row, rows;     // of the row tile: its first row, its rows
  int64_t token;                 // the session's first token
};
static_assert(sizeof(AttendPart) % 16 == 0, "an odd number of CTAs leaves the sums aligned");

struct AttendParams {
  KvCacheArg c;
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

// A segment's tiles come in the list of tiles behind kSetup places that stand
// for its beginning (statistics, query rows, an empty pipeline), so that runs
// of many short sessions take as long as runs of few long ones.  (64 sessions of
// 512 to 32k keys: 324 us with 1, 309 with 2, 303 with 3 and with 4; two of
// 128k: 165 to 168 with any.)
constexpr int kSetup = 3;
struct AttendSpan {
  int seg, kt0, kt1;
  int64_t begin;  // of the segment in the list
};
// What a run has of the segment that place `at` lies in; kt0 >= kt1: no tile.
__device__ __forceinline__ AttendSpan attend_span(int64_t at, int64_t end, int64_t seq_begin, int tiles) {
  AttendSpan s;
  s.seg = (int)((at - seq_begin) / (tiles + kSetup));
  s.begin = seq_begin + (int64_t)s.seg * (tiles + kSetup);
  s.kt0 = (int)max(at - s.begin - kSetup, (int64_t)0);
  s.kt1 = (int)max(min(end - s.begin - kSetup, (int64_t)tiles), (int64_t)0);
  return s;
}

constexpr int kTcRows = 256;  // query rows of a CTA on the tensor cores: two tiles of 128
template <typename T, int DP>
int attend_tc(const AttendParams &p, int grid, void *stream);

}  // namespace unison
