// Attention of sessions that begin with shared prefixes (unison_kv_attend_shared).
//
// A row's keys are its prefix's and its session's own.  Both go through the
// attention kernels as parts: the rows of all sessions of a prefix meet its
// keys together, so that these are read once, and every part leaves
// its maximum m (in log2 units), its sum l of weights 2^(S - m) and its sums
// o = sum 2^(S - m) v, in 32 bits.  A row is then
//   M = max m,  l = sum l 2^(m - M),  out = sum o 2^(m - M) / l.
//
// Where prefixes and sessions suit the same kernel, both are one list of tiles
// and one launch.  Else (a batch that decodes: hundreds of rows for a prefix, a
// few for a session) the sessions' kernel follows the prefixes'.
//
// 64 sessions of 512 to 8k keys behind 32k shared ones, 8 KV heads of 128 (0.87
// GB, 128 us at the copy rate): 195 us, of which 8 join; all of it on the tensor
// cores as one list: 225.  (Sessions' runs beside the prefixes' on other
// multiprocessors took 174, but such a kernel begins without a wait of its own, and
// what earlier kernels wrote is promised to be seen only behind one.)  Trees of 32
// nodes x 8 heads of 32 sessions behind two prompts of 12k and 24k (0.68 TFLOP): 567
// us, 440 of them the prefixes' products at 1.37 PFLOP/s, 30 the join of 65,536
// rows.  45 sessions of 0 to 2.5k behind six prefixes: 38 us (78 with a kernel and a
// join for each half).
#include "kv_attend.cuh"

namespace unison {
namespace {

// A list of tiles as its kernel has shared it out.
struct AttendList {
  const float *partial;
  int grid, rows, groups;
};
struct AttendJoinParams {
  AttendParams p;
  AttendList prefix, own;
};

// The prefix that a session begins with, or -1: the last one whose range begins
// at the session or before, if it holds it.
__device__ __forceinline__ int attend_prefix_of(const AttendParams &P, int b) {
  int g = 0, end = P.prefixes.n_seqs;
  while (end - g > 1) {
    const int mid = (g + end) / 2;
    if (P.first[mid] <= b)
      g = mid;
    else
      end = mid;
  }
  return end > 0 && P.first[g] <= b && b < P.first[g + 1] ? g : -1;
}

// A row's parts: those of its session, then those of its prefix.
struct RowParts {
  int64_t place;
  int2 own, pre;          // first CTA, parts
  int own_row, pre_row;   // of the row tile
  int count;
  // x, y: what the row's AttendRows::where say (y: of a prefix, if it has one)
  __device__ __forceinline__ RowParts(const AttendJoinParams &J, int64_t at, int2 x, int2 y, bool prefixed)
      : place(at) {
    own = clamped(J.own, x);
    pre = prefixed ? clamped(J.prefix, y) : make_int2(0, 0);
    own_row = min(x.y >> 16 & 0xFF, J.own.rows - 1);
    pre_row = min(y.y >> 16 & 0xFF, J.prefix.rows - 1);
    count = own.y + pre.y;
  }
  // (what a kernel that gave up has not written is not followed out of the scratch)
  static __device__ __forceinline__ int2 clamped(const AttendList &l, int2 at) {
    const int cta = min(max(at.x, 0), l.grid - 1);
    return make_int2(cta, min(at.y & 0xFFFF, (l.grid - 1 - cta) / l.groups + 1));
  }
  // Part i: its maximum and sum of weights, and where its sums lie.
  __device__ __forceinline__ const float *part(const AttendJoinParams &J, int i, int DP, float2 &stat) const {
    const bool is_pre = i >= own.y;
    const AttendList &list = is_pre ? J.prefix : J.own;
    const AttendRows &whole = is_pre ? J.p.prefix_rows : J.p.own_rows;
    const int2 at = is_pre ? pre : own;
    const int row = is_pre ? pre_row : own_row, k = is_pre ? i - own.y : i;
    if (at.y <= 1) {
      stat = whole.stats[place];
      return whole.sums + place * J.p.c.head_dim;
    }
    // (a run's second part is of the segment that begins there)
    const float *s = list.partial + ((int64_t)(at.x + k * list.groups) * 2 + (k ? 0 : 1)) * list.rows * (DP + 2);
    stat = make_float2(s[list.rows * DP + row], s[list.rows * (DP + 1) + row]);
    return s + row * DP;
  }
};

// Joins every row's parts, a warp kRows rows at a time: a lane knows the
// statistics of a part of a row and where its sums lie, and all lanes add those up.
// Four rows at a time where there are many: eight parts of each at most, and
// rows with more go one by one, 32 parts at a time.  Bound by four or five loads
// one after the other: 8 us for 2,048 rows of 20 parts, 30 for 65,536 rows of
// two to four (one row of a warp at a time: 76), with 60 bytes of a thread's 64
// registers' worth in local memory at a head size of 128.
constexpr int kJoin = 256;
template <typename T, int DP, int kRows>
__global__ void __launch_bounds__(kJoin, DP <= 128 ? 4 : 2)
    attend_join_list_kernel(const __grid_constant__ AttendJoinParams J) {
  follow_last_kernel();
  const AttendParams &P = J.p;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.x;
  const int D = P.c.head_dim, Q = P.s.n_q_heads;
  const KvRange tok = kv_tokens(P.t, b, nullptr);
  const int rows = tok.count * Q, row0 = ((int)blockIdx.y * (kJoin / 32) + warp) * kRows;
  if (row0 >= rows) return;
  const int64_t first = (int64_t)tok.first * Q;
  // (asked for before it is known whether there is a prefix)
  constexpr int kEach = 32 / kRows;  // lanes of a row
  const int64_t ahead = first + min(row0 + lane / kEach, rows - 1);
  const int2 own_where = P.own_rows.where[ahead], pre_where = P.prefix_rows.where[ahead];
  const int g = attend_prefix_of(P, b);
  bool prefixed = g >= 0 && kv_length(P.prefixes, max(g, 0)) > 0;
  if (prefixed) {  // (offsets that do not ascend may leave a session outside its prefix's tokens)
    const KvRange all = attend_prefix_tokens(P, g, nullptr);
    prefixed = tok.first >= all.first && tok.first + tok.count <= all.first + all.count;
  }
  constexpr int kPer = DP / 32;               // numbers of a lane
  constexpr int kWide = kPer < 4 ? kPer : 4;  // that lie together
  auto load = [&](const float *from, bool there, float (&y)[kPer]) {
#pragma unroll
    for (int j = 0; j < kPer; j += kWide) {
      const int col = j * 32 + lane * kWide;
      if constexpr (kWide == 4) {
        const float4 v =
            there && col < D ? *reinterpret_cast<const float4 *>(from + col) : make_float4(0.f, 0.f, 0.f, 0.f);
        y[j] = v.x, y[j + 1] = v.y, y[j + 2] = v.z, y[j + 3] = v.w;
      } else {
        const float2 v = there && col < D ? *reinterpret_cast<const float2 *>(from + col) : make_float2(0.f, 0.f);
        y[j] = v.x, y[j + 1] = v.y;
      }
    }
  };
  auto finish = [&](int64_t place, float top, float l, float (&sum)[kPer]) {
    const int64_t token = place / Q;
    const int query = (int)(place - token * Q);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *dst = static_cast<T *>(P.s.out) + token * P.s.out_token + query * P.s.out_head;
#pragma unroll
    for (int j = 0; j < kPer; j += 2) {
      const int col = j / kWide * kWide * 32 + lane * kWide + j % kWide;
      if (col < D) *reinterpret_cast<uint32_t *>(dst + col) = KvType<T>::pack(sum[j] * inv, sum[j + 1] * inv);
    }
    if (lane == 0 && P.s.lse) P.s.lse[place] = (top + log2f(l)) * 0.6931471805599453f;
  };
  auto pointer_of = [](const float *p, int from) {
    return reinterpret_cast<const float *>(__shfl_sync(~0u, reinterpret_cast<unsigned long long>(p), from));
  };

  if constexpr (kRows > 1) {
    const int r = row0 + lane / kEach;
    const RowParts parts(J, ahead, own_where, pre_where, prefixed);
    const int n = r < rows ? parts.count : 0;
    int most_parts = n;
#pragma unroll
    for (int d = 16; d; d >>= 1) most_parts = max(most_parts, __shfl_xor_sync(~0u, most_parts, d));
    if (most_parts <= kEach) {
      float2 stat = make_float2(-INFINITY, 0.f);
      const float *mine = nullptr;
      if (lane % kEach < n) mine = parts.part(J, lane % kEach, DP, stat);
      float top = stat.x;
#pragma unroll
      for (int d = kEach / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
      const float f = exp2_fast(stat.x - (top == -INFINITY ? 0.f : top));
      float l = stat.y * f;
#pragma unroll
      for (int d = kEach / 2; d; d >>= 1) l += __shfl_xor_sync(~0u, l, d);
      float sum[kRows][kPer];
#pragma unroll
      for (int q = 0; q < kRows; q++)
#pragma unroll
        for (int j = 0; j < kPer; j++) sum[q][j] = 0.f;
      for (int i = 0; i < most_parts; i++) {
        float y[kRows][kPer];
#pragma unroll
        for (int q = 0; q < kRows; q++) {
          const float *from = pointer_of(mine, q * kEach + i);
          load(from, from != nullptr, y[q]);
        }
#pragma unroll
        for (int q = 0; q < kRows; q++) {
          const float w = __shfl_sync(~0u, f, q * kEach + i);
#pragma unroll
          for (int j = 0; j < kPer; j++) sum[q][j] += y[q][j] * w;
        }
      }
#pragma unroll
      for (int q = 0; q < kRows; q++) {
        const float top_q = __shfl_sync(~0u, top, q * kEach), l_q = __shfl_sync(~0u, l, q * kEach);
        if (row0 + q < rows) finish(first + row0 + q, top_q, l_q, sum[q]);
      }
      return;
    }
  }

  constexpr int kFlight = 8;
  for (int r = row0; r < min(rows, row0 + kRows); r++) {
    const int from = (r - row0) * kEach;
    const int2 x = make_int2(__shfl_sync(~0u, own_where.x, from), __shfl_sync(~0u, own_where.y, from));
    const int2 y = make_int2(__shfl_sync(~0u, pre_where.x, from), __shfl_sync(~0u, pre_where.y, from));
    const RowParts parts(J, first + r, x, y, prefixed);
    float top = -INFINITY, l = 0.f, sum[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i++) sum[i] = 0.f;
    for (int p0 = 0; p0 < parts.count; p0 += 32) {
      float2 stat = make_float2(-INFINITY, 0.f);
      const float *mine = nullptr;
      if (p0 + lane < parts.count) mine = parts.part(J, p0 + lane, DP, stat);
      float most = fmaxf(top, stat.x);
#pragma unroll
      for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, d));
      const float base = most == -INFINITY ? 0.f : most;
      const float f = exp2_fast(stat.x - base), old = exp2_fast(top - base);  // (more than 32 parts: scaled anew)
      top = most;
      l = l * old + stat.y * f;
#pragma unroll
      for (int i = 0; i < kPer; i++) sum[i] *= old;
      const int n = min(parts.count - p0, 32);
      for (int i0 = 0; i0 < n; i0 += kFlight) {
        float y[kFlight][kPer];
#pragma unroll
        for (int u = 0; u < kFlight; u++) load(pointer_of(mine, (i0 + u) & 31), i0 + u < n, y[u]);
#pragma unroll
        for (int u = 0; u < kFlight; u++) {
          const float w = __shfl_sync(~0u, f, (i0 + u) & 31);
#pragma unroll
          for (int j = 0; j < kPer; j++) sum[j] += i0 + u < n ? y[u][j] * w : 0.f;
        }
      }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(~0u, l, d);
    finish(first + r, top, l, sum);
  }
}

template <typename T, int kRows>
int join_rows(const AttendJoinParams &j, int dp, int max_rows, void *stream) {
  constexpr int kPerCta = kJoin / 32 * kRows;
  const dim3 grid(j.p.t.n_seqs, (max_rows + kPerCta - 1) / kPerCta);
  return kv_launch("kv_attend_join", grid, dim3(kJoin), 0, stream, 1,
                   dp == 64    ? attend_join_list_kernel<T, 64, kRows>
                   : dp == 128 ? attend_join_list_kernel<T, 128, kRows>
                               : attend_join_list_kernel<T, 256, kRows>,
                   j);
}

template <typename T>
int join_list(const AttendJoinParams &j, int dp, int max_rows, void *stream) {
  // one row of a warp where that leaves multiprocessors idle
  const int64_t rows = (int64_t)j.p.t.n_tokens * j.p.s.n_q_heads;
  return rows > (int64_t)kv_sm_count() * 32 ? join_rows<T, 4>(j, dp, max_rows, stream)
                                            : join_rows<T, 1>(j, dp, max_rows, stream);
}

uint64_t parts_bytes(const AttendPlan &p) { return (uint64_t)p.grid * 2 * p.rows * (p.dp + 2) * 4; }

// How a call is done, and its scratch: the parts of one list or two, and the rows
// that prefixes and sessions leave whole.
struct SharedPlan {
  AttendPlan prefix, own;
  bool together;  // one list
  uint64_t own_partial, rows, own_rows, bytes;  // offsets: parts, AttendRows of prefixes and of sessions
};

// Prefixes by the query rows of all of them: a prefix may have nearly all of
// those, and the tensor cores take few rows almost as well as many, while the
// other kernel goes through the keys once for every 32 rows.  As many CTAs share
// keys as a prefix has row tiles on average.
AttendPlan prefix_plan(int head_dim, int64_t rows, int prefixes) {
  const int most = (int)min(rows, (int64_t)4 * kTcRows);
  const int each = (int)min((rows + prefixes - 1) / prefixes, (int64_t)most);
  AttendPlan p = attend_plan(head_dim, most);
  if (p.tc) {
    p.row_groups = min((each + kTcRows - 1) / kTcRows, 4);
    p.grid = kv_sm_count() / p.row_groups * p.row_groups;
  }
  return p;
}

int shared_plan(SharedPlan &s, const unison_kv_cache *c, const unison_kv_prefix *x, const unison_kv_tree *t,
                int n_q_heads) {
  int rc = attend_check(c, t, n_q_heads);
  if (rc != UNISON_OK) return rc;
  if (!x) return UNISON_ERR_ARG;
  rc = kv_check_cache(x->cache);
  if (rc != UNISON_OK) return rc;
  if (x->cache->n_heads != c->n_heads || x->cache->head_dim != c->head_dim || x->cache->dtype != c->dtype)
    return UNISON_ERR_ARG;
  if (x->cache->n_seqs > 0 && !x->first) return UNISON_ERR_ARG;
  if ((int64_t)t->n_tokens * n_q_heads >= 1ll << 31 || (int64_t)t->n_seqs * c->n_heads >= 1ll << 31)
    return UNISON_ERR_RANGE;
  const int group = n_q_heads / c->n_heads;
  s.own = attend_plan(c->head_dim, t->max_tokens * group);
  s.prefix = prefix_plan(c->head_dim, max((int64_t)t->n_tokens, (int64_t)1) * group, max(x->cache->n_seqs, 1));
  const uint64_t alone = s.own.bytes;
  s.together = s.own.tc == s.prefix.tc && s.own.row_groups == 1 && s.prefix.row_groups == 1 &&
               (s.own.rows == s.prefix.rows || s.prefix.rows <= 32);
  if (s.together) {
    if (s.own.rows < s.prefix.rows) s.own = s.prefix;
    s.prefix = s.own;
  }
  const uint64_t rows = (uint64_t)t->n_tokens * n_q_heads;
  auto whole = [](uint64_t n) { return (n + 31) / 32 * 32; };  // stores take 32 bytes
  s.own_partial = s.together ? 0 : whole(parts_bytes(s.prefix));
  s.rows = s.own_partial + whole(parts_bytes(s.own));
  s.own_rows = s.rows + whole(rows * (c->head_dim * 4 + sizeof(float2) + sizeof(int2)));
  s.bytes = max(s.own_rows + (s.own_rows - s.rows) + 16, alone);  // (a workspace may begin 16 bytes off)
  return UNISON_OK;
}

AttendList list_of(const AttendPlan &p, const float *partial) {
  return {partial, p.grid, p.rows, p.row_groups};
}

}  // namespace
}  // namespace unison

using namespace unison;

extern "C" uint64_t unison_kv_attend_shared_workspace(const unison_kv_cache *cache, const unison_kv_prefix *prefix,
                                                      const unison_kv_tree *tree, int n_q_heads) {
  SharedPlan s;
  return shared_plan(s, cache, prefix, tree, n_q_heads) == UNISON_OK ? s.bytes : 0;
}

extern "C" int unison_kv_attend_shared(const unison_kv_cache *cache, const unison_kv_prefix *prefix,
                                       const unison_kv_tree *tree, const unison_kv_step *step, void *workspace,
                                       uint64_t workspace_bytes, void *cuda_stream) {
  if (!step) return UNISON_ERR_ARG;
  SharedPlan s;
  int rc = shared_plan(s, cache, prefix, tree, step->n_q_heads);
  if (rc != UNISON_OK) return rc;
  if (cache->n_seqs == 0 || tree->n_tokens == 0) return UNISON_OK;
  if (prefix->cache->n_seqs == 0)
    return unison_kv_attend(cache, tree, step, workspace, workspace_bytes, cuda_stream);
  if (!attend_step_ok(step) || !attend_pools_ok(cache) || !attend_pools_ok(prefix->cache)) return UNISON_ERR_ARG;
  if (!workspace || !kv_aligned(workspace, 16) || workspace_bytes < s.bytes) return UNISON_ERR_ARG;
  char *base = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(workspace) + 31) & ~(uintptr_t)31);
  AttendJoinParams j = {};
  AttendParams &p = j.p;
  p.c = *cache;
  p.t = *tree;
  p.s = *step;
  p.group = step->n_q_heads / cache->n_heads;
  p.prefixes = *prefix->cache;
  p.first = prefix->first;
  const uint64_t rows = (uint64_t)tree->n_tokens * step->n_q_heads;
  for (AttendRows *r : {&p.prefix_rows, &p.own_rows}) {
    char *at = base + (r == &p.own_rows ? s.own_rows : s.rows);
    r->sums = reinterpret_cast<float *>(at);
    r->stats = reinterpret_cast<float2 *>(at + rows * cache->head_dim * 4);
    r->where = reinterpret_cast<int2 *>(r->stats + rows);
  }
  float *prefix_partial = reinterpret_cast<float *>(base);
  float *own_partial = reinterpret_cast<float *>(base + s.own_partial);
  p.n_prefixes = prefix->cache->n_seqs;
  if (!s.together) {
    p.partial = prefix_partial;
    rc = attend_list(p, s.prefix, cuda_stream);
    if (rc != UNISON_OK) return rc;
    p.n_prefixes = 0;
  }
  p.n_sessions = tree->n_seqs;
  p.partial = own_partial;
  rc = attend_list(p, s.own, cuda_stream);
  if (rc != UNISON_OK) return rc;
  j.prefix = list_of(s.prefix, prefix_partial);
  j.own = list_of(s.own, own_partial);
  const int max_rows = tree->max_tokens * step->n_q_heads;
  return cache->dtype == UNISON_KV_BF16 ? join_list<__nv_bfloat16>(j, s.own.dp, max_rows, cuda_stream)
                                        : join_list<__half>(j, s.own.dp, max_rows, cuda_stream);
}
