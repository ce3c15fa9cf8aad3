// What the attention kernels share (kv_attend.cu, kv_attend_tc.cu, kv_attend_shared.cu).
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

// What the kernels go through:
//   kAlone  the sessions of a call; split segments are joined by attend_join_kernel
//   kList   shared prefixes and then sessions, either of which may be missing.  The
//           query rows of a prefix are those of all its sessions' tokens, and it has no
//           new keys.  Every result stays in 32 bits, unnormalised: a whole segment's
//           in AttendRows, a split one's in the parts.  attend_join_list_kernel joins a
//           row's prefix and its session's own part.
enum AttendUse { kAlone, kList };

struct AttendRows {  // by token and query head
  float *sums;       // [n_tokens][n_q_heads][head_dim], of whole segments
  float2 *stats;     // [n_tokens][n_q_heads]: maximum (log2), sum of weights
  int2 *where;       // [n_tokens][n_q_heads]: first CTA; parts, and the row's place in them (<< 16)
};

struct AttendParams {
  KvCacheArg c;
  unison_kv_tree t;
  unison_kv_step s;
  AttendPart *part;  // [grid]
  float *partial;    // [grid][2]: sums [rows][DP], maxima [rows] (log2), sums of weights [rows]
  int group;         // query heads of a KV head
  int rows;          // of a row tile
  int row_groups;    // CTAs of a run, with row tiles of their own
  // kList
  KvCacheArg prefixes;
  const int32_t *first;        // sessions of a prefix
  int n_prefixes, n_sessions;  // of this launch's list
  AttendRows prefix_rows, own_rows;
};

// A segment's tiles come in the list of tiles behind kSetup places that stand
// for its beginning (statistics, query rows, an empty pipeline), so that runs
// of many short sessions take as long as runs of few long ones.  (64 sessions of
// 512 to 32k keys: 324 us with 1, 309 with 2, 303 with 3 and with 4; two of
// 128k: 165 to 168 with any.)
constexpr int kSetup = 3;
// Key tiles of a session, the last one of which holds its new tokens, or of a prefix.
__device__ __forceinline__ int attend_key_tiles(int len, int tokens, int tile, bool prefix = false) {
  return tokens ? (len + tile - 1) / tile + (prefix ? 0 : 1) : 0;
}
// Tokens of a prefix's sessions.
__device__ __forceinline__ KvRange attend_prefix_tokens(const AttendParams &P, int g, int32_t *status) {
  const int lo = P.first[g], hi = P.first[g + 1];
  const int s0 = min(max(lo, 0), P.t.n_seqs), s1 = min(max(hi, s0), P.t.n_seqs);
  if (status && (lo != s0 || hi != s1)) status[g] = UNISON_ERR_RANGE;
  if (s0 == s1) return {0, 0};
  const int first = min(max(P.t.offsets[s0], 0), P.t.n_tokens);
  return {first, min(max(P.t.offsets[s1], first), P.t.n_tokens) - first};
}
// A prefix's, or a session's, places in the list of tiles.
__device__ __forceinline__ int64_t attend_places(const AttendParams &P, bool prefix, int b, int tile, int rows,
                                                 int groups) {
  const KvCacheArg &c = prefix ? P.prefixes : P.c;
  const int tokens = (prefix ? attend_prefix_tokens(P, b, c.status) : kv_tokens(P.t, b, c.status)).count;
  const int tiles = attend_key_tiles(kv_length(c, b), tokens, tile, prefix);
  if (tiles == 0) return 0;
  const int row_tiles = (tokens * P.group + rows - 1) / rows;
  return (int64_t)(tiles + kSetup) * ((row_tiles + groups - 1) / groups) * c.n_heads;
}

// Runs of a list with prefixes, of `total` places: a run has kLeastPlaces of them
// at least, on average, as what is split has to be joined, row by row.
constexpr int kLeastPlaces = 4;
__device__ __forceinline__ int64_t attend_most_runs(int64_t total) {
  return (total + kLeastPlaces - 1) / kLeastPlaces;
}

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
template <typename T, int DP, int kUse>
int attend_tc(const AttendParams &p, int grid, void *stream);

struct AttendPlan {
  int dp, rows, row_groups, grid;
  bool tc;
  uint64_t bytes;
};
AttendPlan attend_plan(int head_dim, int max_rows);
// Queues the kernel that goes through the call's list.
int attend_list(AttendParams &p, const AttendPlan &plan, void *stream);
int attend_check(const unison_kv_cache *c, const unison_kv_tree *t, int n_q_heads);
bool attend_pools_ok(const unison_kv_cache *c);
bool attend_step_ok(const unison_kv_step *s);

}  // namespace unison
