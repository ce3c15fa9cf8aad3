// Attention of many query rows per KV head on the tensor cores (the variant of
// unison_kv_attend for trees whose nodes x query heads exceed 32 rows, and head
// sizes up to 128; kv_attend.cu has the formulas).
//
// A CTA takes up to 256 query rows, two tiles of 128, and walks the keys in
// tiles of 128.  Warps have roles:
//   warps 8-11   copy the paged rows of K and V, and the query rows, into
//                shared memory in the swizzled form that the tensor cores read
//   warp 12      issues the products S = Q K^T and O += P V; S, P (over S) and
//                O stay in tensor memory
//   warps 0-3, 4-7  one query tile each: a thread per row turns S into weights
// While one tile's weights are computed, the other tile's products run.  One
// query tile alone takes the keys in two turns instead, each with an O of its
// own, joined at the end (64 rows of 16 sessions of 16k keys, head size 128: 180
// us, in one turn 197).  O is rescaled only when a row's maximum has grown by
// more than 2^8 over the one that their reference was taken from; the sums are 32 bits
// wide, so weights up to 2^8 cost no accuracy.  They are rounded to the cache's
// type for the second product; their sum is of the weights before that.  In fp16
// the reference lies 2^7 below the maximum that it was taken from, as weights may
// be up to 2^15 there: so 2^-32 of the maximum still counts.
//
// Up to 128 rows memory bounds it (5.8 TB/s at 128 rows of that case, 187 us);
// from 256 on the tensor cores and the two warps per scheduler that compute the
// weights: 64 nodes x 8 heads over 32 sessions of 15k to 16k keys, 8 KV heads
// (1.06 PFLOP), take 750 us, 1.41 PFLOP/s, 73% of what a plain matrix product
// reaches here (a long stream of such calls and their joins: 820 to 830 us a
// call, under the power limit).  512 rows' CTAs work in pairs on the same keys,
// which the second finds in the L2 cache.
//
// A wait that runs out ends the CTA (every role sees `dead`) and reports
// UNISON_ERR_TIMEOUT.  Every copying warp waits for every slot, also for those
// that another warp fills: a barrier's parity tells a phase only from the next
// one, and a warp that runs two ahead would take a slot that is being read.
#include "kv_attend.cuh"
#include "kv_copy.cuh"

namespace unison {
namespace {

constexpr int kThreads = 416;
constexpr int kTile = 128;
constexpr int kCopyWarp = 8, kIssueWarp = 12;
constexpr int kSlack = 8;
// Segments whose flags of odd values are kept.  A segment that takes one tile
// passes the second slot's warps by, so nothing else holds the copies back until
// these have read the flags of an earlier one: they wait for that (seg_done).
constexpr int kOddSets = 4;

template <int DP>
constexpr int kSlots = DP == 128 ? 5 : 8;  // tiles of K or V on their way
template <int DP>
constexpr int kTcSmem = 1024 + kTcRows *DP * 2 + kSlots<DP> *kTile *DP * 2;

template <int DP>
struct TcShared {
  KvRunShared run;
  uint64_t kv_full[kSlots<DP>], kv_free[kSlots<DP>], q_full, q_free, s_full[2], p_full[2], pv_done[2], half_full,
      half_free, seg_done[kOddSets], idle;
  alignas(16) uint32_t row_ok[8][4];  // which keys of a tile exist
  bool odd[kOddSets][4];  // whether new values that a copying warp read hold infinities or NaN
  float half[2][128];     // maxima and sums of a single query tile's second half of the keys
  uint32_t tmem;
  volatile int dead;
};

// What every role works out alike for the segment that `at` lies in.
struct Segment {
  bool prefix;
  int b, head, row_tile, rows, tiles, kt0, kt1, len;  // rows <= 0: nothing to do for this CTA
  KvRange tok;
};

// The order in which a run's tiles of keys (0) and values (1) go through the ring,
// n tiles: K0 V0 K1 V1 .. where two query tiles share them, K0 K1 V0 K2 V1 .. where
// one query tile takes the key tiles in two turns.
__device__ __forceinline__ int item_of(int j, int n, bool turns, int &tile) {
  if (!turns || n == 1) {
    tile = j >> 1;
    return j & 1;
  }
  if (j == 0 || j == 2 * n - 1) {
    tile = j ? n - 1 : 0;
    return j ? 1 : 0;
  }
  tile = j & 1 ? (j + 1) >> 1 : (j >> 1) - 1;
  return ~j & 1;
}

struct AttendTcParams : AttendParams {
  KvBoxes k_boxes, v_boxes;                // of the sessions' cache
  KvBoxes k_prefix_boxes, v_prefix_boxes;  // kList
};

template <typename T, int DP, int kUse>
__global__ void __launch_bounds__(kThreads, 1) attend_tc_kernel(const __grid_constant__ AttendTcParams P) {
  follow_last_kernel();
  constexpr uint32_t kTileBytes = kTile * DP * 2, kBlock = kTile * 128;
  constexpr int kLower = KvType<T>::kMostWeight > kSlack ? KvType<T>::kMostWeight - kSlack : 0;
  extern __shared__ unsigned char smem_raw[];
  __shared__ TcShared<DP> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int D = P.c.head_dim, H = P.c.n_heads, G = P.group;
  const uint32_t q_base = (smem_u32(smem_raw) + 1023) & ~1023u, slot_base = q_base + kTcRows * DP * 2;
  const int groups = P.row_groups, rank = blockIdx.x % groups;
  if (kUse == kAlone && tid == 0) P.part[blockIdx.x].last = -1;

  auto seq_tiles = [&](int b) -> int64_t {
    if constexpr (kUse == kList) {
      const bool prefix = b < P.n_prefixes;
      return attend_places(P, prefix, prefix ? b : b - P.n_prefixes, kTile, kTcRows, groups);
    }
    const int tokens = kv_tokens(P.t, b, P.c.status).count;
    const int row_tiles = (tokens * G + kTcRows - 1) / kTcRows;
    return (int64_t)(attend_key_tiles(kv_length(P.c, b), tokens, kTile) + kSetup) *
           ((row_tiles + groups - 1) / groups) * H;
  };
  KvRun run;
  if (!kv_find_run(run, sh.run, kUse == kList ? P.n_prefixes + P.n_sessions : P.c.n_seqs, gridDim.x / groups,
                   blockIdx.x / groups, seq_tiles,
                   [](int64_t total) { return kUse == kList ? attend_most_runs(total) : total; }))
    return;

  if (tid == 0) {
    for (int i = 0; i < kSlots<DP>; i++) {
      bar_init(smem_u32(&sh.kv_full[i]), 4);  // copying warps
      bar_init(smem_u32(&sh.kv_free[i]), 1);
    }
    bar_init(smem_u32(&sh.q_full), 4);
    bar_init(smem_u32(&sh.q_free), 1);
    bar_init(smem_u32(&sh.idle), 1);
    bar_init(smem_u32(&sh.half_full), 4);
    bar_init(smem_u32(&sh.half_free), 4);
    for (int i = 0; i < kOddSets; i++) bar_init(smem_u32(&sh.seg_done[i]), kCopyWarp);  // warps that weigh
    for (int i = 0; i < 2; i++) {
      bar_init(smem_u32(&sh.s_full[i]), 2);
      bar_init(smem_u32(&sh.p_full[i]), 4);  // warps
      bar_init(smem_u32(&sh.pv_done[i]), 2);
    }
    sh.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kIssueWarp) tmem_alloc(smem_u32(&sh.tmem), 512);
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  const uint32_t tmem = sh.tmem;  // S of the two query tiles, then their O

  int b = run.b;
  int64_t at = run.at, seq_begin = run.begin, seg_begin = 0;
  auto next_segment = [&](Segment &g) {
    int64_t mine = seq_tiles(b);
    while (at >= seq_begin + mine) {
      seq_begin += mine;
      mine = seq_tiles(++b);
    }
    g.prefix = kUse == kList && b < P.n_prefixes;
    g.b = kUse == kList && !g.prefix ? b - P.n_prefixes : b;
    g.tok = g.prefix ? attend_prefix_tokens(P, g.b, nullptr) : kv_tokens(P.t, g.b, nullptr);
    g.len = kv_length(g.prefix ? P.prefixes : P.c, g.b);
    g.tiles = attend_key_tiles(g.len, g.tok.count, kTile, g.prefix);
    const int row_tiles = (g.tok.count * G + kTcRows - 1) / kTcRows;
    const int row_groups = (row_tiles + groups - 1) / groups;
    const AttendSpan span = attend_span(at, run.end, seq_begin, g.tiles);
    seg_begin = span.begin;
    g.head = span.seg / row_groups;
    g.row_tile = span.seg % row_groups * groups + rank;
    g.rows = min(g.tok.count * G - g.row_tile * kTcRows, kTcRows);
    g.kt0 = span.kt0;
    g.kt1 = span.kt1;
    if (g.kt0 >= g.kt1) g.rows = 0;
    at = span.begin + kSetup + g.kt1;
  };

  if (warp >= kCopyWarp && warp < kIssueWarp) {
    // ------------------------------------------------------------- copies
    const int w = warp - kCopyWarp;
    KvCopier<T, DP> copier(w, lane, D, P.s.q);
    Ring ring;
    int tile_no = 0, seg_no = 0;
    bool ok = true;
    auto slot_for = [&](uint32_t &bar) -> uint32_t {  // waits until the next slot is free
      ok = copier.wait(smem_u32(&sh.kv_free[ring.at]), ring.turn ^ 1, &sh.dead);
      bar = smem_u32(&sh.kv_full[ring.at]);
      const uint32_t slot = slot_base + ring.at * kTileBytes;
      ring.next(kSlots<DP>);
      return slot;
    };
    while (at < run.end && ok) {
      Segment g;
      next_segment(g);
      if (g.rows <= 0) continue;
      const int last_tile = g.prefix ? g.tiles : g.tiles - 1;  // of new tokens
      const KvCacheArg &cache = g.prefix ? P.prefixes : P.c;
      const KvBoxes &k_boxes = g.prefix ? P.k_prefix_boxes : P.k_boxes;
      const KvBoxes &v_boxes = g.prefix ? P.v_prefix_boxes : P.v_boxes;
      const bool by_boxes = k_boxes.rows && v_boxes.rows;
      BoxSender<DP> sender(w ? v_boxes : k_boxes);
      // the query rows: when the last segment's products have read theirs
      if (seg_no > 0) ok = copier.wait(smem_u32(&sh.q_free), (seg_no - 1) & 1, &sh.dead);
      if (ok && seg_no >= kOddSets)
        ok = copier.wait(smem_u32(&sh.seg_done[seg_no % kOddSets]), (seg_no / kOddSets - 1) & 1, &sh.dead);
      if (!ok) break;
      for (int q = 0; q < (g.rows > 128 ? 2 : 1); q++) {
        const int r = q * 128 + w * 32 + lane, row = g.row_tile * kTcRows + r;
        const T *src = nullptr;
        if (r < g.rows)
          src = static_cast<const T *>(P.s.q) + (g.tok.first + row / G) * P.s.q_token +
                (g.head * G + row % G) * P.s.q_head;
        copier.rows(q_base + q * kTileBytes, src);
      }
      copier.issued(smem_u32(&sh.q_full));
      if (kUse == kList && g.kt0 == 0) {  // (here, because these warps have time to spare)
        const int64_t end = seg_begin + kSetup + g.tiles - 1;
        const int parts = g.kt1 == g.tiles ? 1 : kv_run_of(run, end) - (int)blockIdx.x / groups + 1;
        int2 *where = (g.prefix ? P.prefix_rows : P.own_rows).where;
        for (int r = w * 32 + lane; r < g.rows; r += 128) {
          const int row = g.row_tile * kTcRows + r;
          where[(int64_t)(g.tok.first + row / G) * P.s.n_q_heads + g.head * G + row % G] =
              make_int2(blockIdx.x, parts | r << 16);
        }
      }
      const int n = g.kt1 - g.kt0, j = w * 32 + lane;  // j: this lane's row of a tile
      const int boxed = by_boxes ? g.len / kTile : 0;  // full tiles go by boxes
      sender.reset();
      int page[2], off[2], next_page = kNoSlot, next_off = 0;  // of this lane's row in the last two tiles, the next
      for (int item = 0; item < 2 * n; item++) {
        int tile;
        const int part = item_of(item, n, g.rows <= 128, tile), kt = g.kt0 + tile;
        uint32_t bar;
        if (kt < boxed) {  // the first warp sends the keys, the second one the values
          if (item == 0) copier.landed();
          const bool sends = w == part;
          if (sends) sender.look_up(cache, g.b, kt, g.len);
          const uint32_t dst = slot_for(bar);
          if (!ok) break;
          if (!sends) {
            // (every warp keeps step: a barrier's parity tells only its last phase)
            if (lane == 0) bar_arrive(bar);
          } else {
            if (part == 0) {
              if (!sender.gap) {
                if (lane < 4) sh.row_ok[(tile_no + tile) & 7][lane] = ~0u;
              } else {
                for (int i = 0; i < 4; i++) {
                  const uint32_t word = sender.present(kt, i);
                  if (lane == 0) sh.row_ok[(tile_no + tile) & 7][i] = word;
                }
              }
              __syncwarp();
            }
            sender.send(kt, dst, bar, g.head);
          }
          if (copier.waiting[0] | copier.waiting[1]) copier.issued(0);
          continue;
        }
        // row by row
        const bool last = kt == last_tile, fresh = last && j < g.tok.count;
        auto look_up = [&](int kt, int &o) -> int {
          o = 0;
          return kt < last_tile && kt * kTile + j < g.len ? kv_page_load(cache, g.b, kt * kTile + j, o) : kNoSlot;
        };
        if (part == 0) {
          if (tile == 0 || kt == boxed) next_page = look_up(kt, next_off);
          const int p = kv_page_ok(cache, g.b, next_page);
          if (tile & 1)
            page[1] = p, off[1] = next_off;
          else
            page[0] = p, off[0] = next_off;
          next_page = look_up(kt + 1, next_off);
        }
        const int p = tile & 1 ? page[1] : page[0], o = tile & 1 ? off[1] : off[0];
        const T *src = nullptr;
        if (fresh)
          src = part ? static_cast<const T *>(P.s.v_new) + (g.tok.first + j) * P.s.v_token + g.head * P.s.v_head
                     : static_cast<const T *>(P.s.k_new) + (g.tok.first + j) * P.s.k_token + g.head * P.s.k_head;
        else if (p >= 0)
          src = part ? static_cast<const T *>(cache.v) + p * cache.v_page + g.head * cache.v_head + o * cache.v_slot
                     : static_cast<const T *>(cache.k) + p * cache.k_page + g.head * cache.k_head + o * cache.k_slot;
        const uint32_t there = __ballot_sync(~0u, src != nullptr);
        const uint32_t dst = slot_for(bar);
        if (!ok) break;
        copier.rows(dst, src);
        if (part == 0) {
          if (lane == 0) sh.row_ok[(tile_no + tile) & 7][w] = there;
          copier.issued(bar);
        } else if (!last) {
          copier.issued(bar);
        } else {
          // A new token that a row does not see must not reach it as 0 * inf:
          // such values become 0 here and are put back, row by row, at the end.
          copier.issued(0);
          copier.landed();
          const bool odd = copier.zero_odd_values(dst);
          if (lane == 0) sh.odd[seg_no % kOddSets][w] = odd;
          copier.arrive(bar);
        }
      }
      tile_no += n;
      seg_no++;
    }
    copier.landed();
    if (!ok) copier.give_up();
  } else if (warp >= kIssueWarp) {
    if (warp == kIssueWarp) {
      // --------------------------------------------------------- products
      // (the whole warp goes along, one lane issues)
      const uint32_t shape_s = product_shape(kOperandType<T>, 128, kTile, false, P.s.scale < 0.f);
      const uint32_t shape_o = product_shape(kOperandType<T>, 128, DP, true, false);
      const uint32_t q_rows = smem_operand(q_base, kBlock), slots = smem_operand(slot_base, kBlock);
      const uint32_t tmem = uniform(sh.tmem);
      Ring ring;
      int seg_no = 0, p_no[2] = {0, 0};
      bool ok = true;
      auto take = [&](int &s) -> uint32_t {  // waits for the next slot's tile
        s = ring.at;
        ok = __all_sync(~0u, bar_wait(smem_u32(&sh.kv_full[s]), ring.turn, &sh.dead));
        ring.next(kSlots<DP>);
        return slots + s * (kTileBytes >> 4);
      };
      const bool one = elect_one();
      // Scores of slot `to` from query tile q; weights of slot q with the values.
      auto scores = [&](int to, int q, uint32_t keys) {
        const uint32_t a = q_rows + q * (kTileBytes >> 4);
#pragma unroll
        for (int d = 0; d < DP / 16; d++) {
          const uint32_t at = (d / 4 * kBlock + d % 4 * 32) >> 4;
          product_ss(one, tmem + to * 128, a + at, keys + at, shape_s, d > 0);
        }
        products_done(one, smem_u32(&sh.s_full[to]));
        bar_arrive_by(one, smem_u32(&sh.s_full[to]));  // hands on what the copies of the keys wrote besides (row_ok)
      };
      auto values = [&](int q, uint32_t vals, bool add) {
        ok = __all_sync(~0u, bar_wait(smem_u32(&sh.p_full[q]), p_no[q]++ & 1, &sh.dead));
        if (!ok) return;
        tmem_after_sync();
#pragma unroll
        for (int k = 0; k < kTile / 16; k++)
          product_ts(one, tmem + 256 + q * DP, tmem + q * 128 + k * 8, vals + k * (2048 >> 4), shape_o, add || k > 0);
        products_done(one, smem_u32(&sh.pv_done[q]));
        bar_arrive_by(one, smem_u32(&sh.pv_done[q]));  // and those of the values (odd)
      };
      auto release = [&](uint64_t &bar) { products_done(one, smem_u32(&bar)); };
      while (uniform(at < run.end && ok)) {
        Segment g;
        next_segment(g);
        if (uniform(g.rows) <= 0) continue;
        const int n = uniform(g.kt1 - g.kt0), tiles = uniform(g.rows) > 128 ? 2 : 1;
        int ks, vs;
        uint32_t keys = take(ks);
        if (ok) ok = __all_sync(~0u, bar_wait(smem_u32(&sh.q_full), seg_no & 1, &sh.dead));
        if (!ok) break;
        if (tiles == 2) {  // two query tiles share the keys
          for (int q = 0; q < 2; q++) scores(q, q, keys);
          release(sh.kv_free[ks]);
          if (n == 1) release(sh.q_free);
          for (int i = 0; i < n && ok; i++) {
            const uint32_t vals = take(vs);
            for (int q = 0; q < 2 && ok; q++) {
              values(q, vals, i > 0);
              if (!ok) break;
              if (q == 1) release(sh.kv_free[vs]);
              if (i + 1 < n) {
                if (q == 0) keys = take(ks);
                if (!ok) break;
                scores(q, q, keys);
                if (q == 1) {
                  release(sh.kv_free[ks]);
                  if (i + 2 == n) release(sh.q_free);
                }
              }
            }
          }
        } else {  // one query tile: key tiles in turn to the two slots
          scores(0, 0, keys);
          release(sh.kv_free[ks]);
          if (n > 1) {
            keys = take(ks);
            if (!ok) break;
            scores(1, 0, keys);
            release(sh.kv_free[ks]);
          }
          if (n <= 2) release(sh.q_free);
          for (int i = 0; i < n && ok; i++) {
            const uint32_t vals = take(vs);
            if (ok) values(i & 1, vals, i > 1);
            if (!ok) break;
            release(sh.kv_free[vs]);
            if (i + 2 < n) {
              keys = take(ks);
              if (!ok) break;
              scores(i & 1, 0, keys);
              release(sh.kv_free[ks]);
              if (i + 3 == n) release(sh.q_free);
            }
          }
        }
        seg_no++;
      }
      // nothing may still be at work when tensor memory is freed
      release(sh.idle);
      for (int i = 0; i < 1 << 20 && !__all_sync(~0u, bar_try(smem_u32(&sh.idle), 0)); i++) {
      }
    }
  } else {
    // ------------------------------------------------------------ weights
    const int q = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's quarter of the 128 lanes
    const uint32_t s_addr = tmem + q * 128 + lanes, o_addr = tmem + 256 + q * DP + lanes;
    // (the sign is in the products; not 0, so that -inf stays -inf)
    const float c = fmaxf(fabsf(P.s.scale) * 1.4426950408889634f, 1.2e-38f);
    int s_no = 0, seg_no = 0, tile_no = 0;  // products seen, segments, key tiles of this CTA
    int halves = 0;                          // segments that the slots joined
    bool owed = false;                       // slot 1: its half of the last one may still be read
    bool ok = true;
    auto warp_arrive = [&](uint64_t &bar) {
      __syncwarp();
      if (lane == 0) bar_arrive(smem_u32(&bar));
    };
    while (at < run.end && ok) {
      Segment g;
      next_segment(g);
      if (g.rows <= 0) continue;
      const int mine = seg_no++;
      // Two query tiles: one for each slot.  One: the slots take its key tiles in
      // turn, as two halves that are joined at the end.
      const bool turns = g.rows <= 128;
      const int n = g.kt1 - g.kt0, begin = turns ? g.kt0 + q : g.kt0, step = turns ? 2 : 1;
      const int tiles_before = tile_no;
      tile_no += n;
      if (begin >= g.kt1) {
        warp_arrive(sh.seg_done[mine % kOddSets]);
        continue;
      }
      const int tr = turns ? r : q * 128 + r, row = g.row_tile * kTcRows + tr, node = row / G;
      const bool used = tr < g.rows;
      const uint64_t mask = !used || g.prefix ? 0 : P.t.mask ? P.t.mask[g.tok.first + node] : ~0ull >> (63 - node);
      float m = -INFINITY, l = 0.f;
      for (int kt = begin; kt < g.kt1; kt += step) {
        ok = __all_sync(~0u, bar_wait(smem_u32(&sh.s_full[q]), s_no & 1, &sh.dead));
        if (!ok) break;
        tmem_after_sync();
        uint4 see = *reinterpret_cast<const uint4 *>(sh.row_ok[(tiles_before + kt - g.kt0) & 7]);
        const bool hidden = (see.x & see.y & see.z & see.w) != ~0u;  // the last tile: always (64 tokens at most)
        if (kt == g.tiles - 1 && !g.prefix) {
          see.x &= (uint32_t)mask;
          see.y &= (uint32_t)(mask >> 32);
        }
        const uint64_t cc = pair(c, c);
        uint32_t x[2][32];
        // One pass where the last reference still serves: the weights wait in
        // registers until the tile's maximum is known.  (Two passes cost 700
        // cycles of a tile's 2,400 here.)
        bool done = false;
        if (!hidden && kt > begin) {
          const float base = m == -INFINITY ? 0.f : m;
          const uint64_t bb = pair(-base, -base);
          uint64_t sum[2] = {0, 0};
          float t[2] = {-INFINITY, -INFINITY};
          uint32_t p[64];
          tmem_ld32(x[0], s_addr);
#pragma unroll
          for (int i = 0; i < 4; i++) {
            uint32_t(&v)[32] = x[i & 1];
            tmem_wait_ld(v);
            if (i < 3) tmem_ld32(x[~i & 1], s_addr + i * 32 + 32);
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              float a = __uint_as_float(v[j]), b = __uint_as_float(v[j + 1]);
              t[j >> 1 & 1] = fmaxf(fmaxf(t[j >> 1 & 1], a), b);
              unpair(fma_pair(pair(a, b), cc, bb), a, b);
              a = exp2_fast(a);
              b = exp2_fast(b);
              sum[j >> 1 & 1] = add_pair(sum[j >> 1 & 1], pair(a, b));
              p[i * 16 + j / 2] = KvType<T>::pack(a, b);
            }
          }
          done = !__any_sync(~0u, reference_of<kLower>(fmaxf(t[0], t[1]) * c) > m + kSlack);
          if (done) {
            tmem_st32(s_addr, p);
            tmem_st32(s_addr + 32, p + 32);
            float more, less;
            unpair(add_pair(sum[0], sum[1]), more, less);
            l += more + less;
          }
        }
        if (!done) {
          // Two passes, 32 scores at a time: the maximum, then the weights.
          auto hide = [&](uint32_t(&v)[32], uint32_t word) {
#pragma unroll
            for (int i = 0; i < 32; i++)
              if (!(word >> i & 1)) v[i] = 0xFF800000u;  // -inf
          };
          auto word_of = [&](int i) { return i == 0 ? see.x : i == 1 ? see.y : i == 2 ? see.z : see.w; };
          float t = -INFINITY;
#pragma unroll 1
          for (int i = 0; i < 4; i++) {
            tmem_ld32(x[0], s_addr + i * 32);
            tmem_wait_ld(x[0]);
            if (hidden) hide(x[0], word_of(i));
#pragma unroll
            for (int j = 0; j < 32; j++) t = fmaxf(t, __uint_as_float(x[0][j]));
          }
          const float top = reference_of<kLower>(t * c), to = kt == begin || top > m + kSlack ? top : m;
          if (kt > begin && __any_sync(~0u, to != m)) {
            const float f = m == to ? 1.f : exp2_fast(m - to);
            ok = __all_sync(~0u, bar_wait(smem_u32(&sh.pv_done[q]), (s_no - 1) & 1, &sh.dead));
            if (!ok) break;
            tmem_after_sync();
#pragma unroll 1
            for (int d = 0; d < DP; d += 32) {
              tmem_ld32(x[0], o_addr + d);
              tmem_wait_ld(x[0]);
#pragma unroll
              for (int i = 0; i < 32; i++) x[0][i] = __float_as_uint(__uint_as_float(x[0][i]) * f);
              tmem_st32(o_addr + d, x[0]);
            }
            l *= f;
          }
          m = to;
          const float base = m == -INFINITY ? 0.f : m;
          const uint64_t bb = pair(-base, -base);
          uint64_t sum = 0;
#pragma unroll 1
          for (int i = 0; i < 4; i++) {
            tmem_ld32(x[0], s_addr + i * 32);
            tmem_wait_ld(x[0]);
            if (hidden) hide(x[0], word_of(i));
            uint32_t p[16];
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              float a, b;
              unpair(fma_pair(pair(__uint_as_float(x[0][j]), __uint_as_float(x[0][j + 1])), cc, bb), a, b);
              a = exp2_fast(a);
              b = exp2_fast(b);
              sum = add_pair(sum, pair(a, b));
              p[j / 2] = KvType<T>::pack(a, b);
            }
            tmem_st16(s_addr + i * 16, p);  // over scores that have been read
          }
          float more, less;
          unpair(sum, more, less);
          l += more + less;
        }
        tmem_wait_st();
        tmem_before_sync();
        if (owed) {  // these weights' product overwrites the slot's sums
          ok = __all_sync(~0u, bar_wait(smem_u32(&sh.half_free), (halves - 1) & 1, &sh.dead));
          if (!ok) break;
          owed = false;
        }
        warp_arrive(sh.p_full[q]);
        s_no++;
      }
      if (!ok) break;
      // ---- results: O is complete when the last product with V is
      ok = __all_sync(~0u, bar_wait(smem_u32(&sh.pv_done[q]), (s_no - 1) & 1, &sh.dead));
      if (!ok) break;
      tmem_after_sync();
      const bool join = turns && n > 1;
      float f0 = 1.f, f1 = 0.f;
      if (join) {
        if (q == 1) {
          sh.half[0][r] = m;
          sh.half[1][r] = l;
          tmem_before_sync();
          warp_arrive(sh.half_full);
          warp_arrive(sh.seg_done[mine % kOddSets]);
          halves++;
          owed = true;
          continue;
        }
        ok = __all_sync(~0u, bar_wait(smem_u32(&sh.half_full), halves++ & 1, &sh.dead));
        if (!ok) break;
        tmem_after_sync();
        const float m1 = sh.half[0][r], l1 = sh.half[1][r], top = fmaxf(m, m1), base = top == -INFINITY ? 0.f : top;
        f0 = exp2_fast(m - base);
        f1 = exp2_fast(m1 - base);
        l = l * f0 + l1 * f1;
        m = top;
      }
      const bool whole = g.kt0 == 0 && g.kt1 == g.tiles;
      const bool *flags = sh.odd[mine % kOddSets];
      const bool odd = !g.prefix && g.kt1 == g.tiles && (flags[0] || flags[1] || flags[2] || flags[3]);
      const float inv = l == 0.f ? 0.f : 1.f / l;
      auto place = [&] { return (int64_t)(g.tok.first + node) * P.s.n_q_heads + g.head * G + row % G; };
      auto rows_to = [&]() -> const AttendRows & { return g.prefix ? P.prefix_rows : P.own_rows; };
      float *part = P.partial + ((int64_t)blockIdx.x * 2 + (g.kt0 == 0 ? 1 : 0)) * (kTcRows * (DP + 2));
      T *dst = static_cast<T *>(P.s.out) + (g.tok.first + node) * P.s.out_token + (g.head * G + row % G) * P.s.out_head;
#pragma unroll 1
      for (int d0 = 0; d0 < DP; d0 += 32) {
        uint32_t o[32];
        tmem_ld32(o, o_addr + d0);
        tmem_wait_ld(o);
        if (join) {
          uint32_t o1[32];
          tmem_ld32(o1, o_addr + DP + d0);
          tmem_wait_ld(o1);
#pragma unroll
          for (int i = 0; i < 32; i++)
            o[i] = __float_as_uint(__uint_as_float(o[i]) * f0 + __uint_as_float(o1[i]) * f1);
        }
        if (used && odd) {
          const uint64_t see = mask & (~0ull >> (64 - g.tok.count));
          for (int j = 0; j < g.tok.count; j++) {
            if (!(see >> j & 1)) continue;
            const T *v = static_cast<const T *>(P.s.v_new) + (g.tok.first + j) * P.s.v_token + g.head * P.s.v_head + d0;
#pragma unroll
            for (int i = 0; i < 32; i++) {
              const float y = d0 + i < D ? KvType<T>::to_float(v[i]) : 0.f;
              if (!isfinite(y)) o[i] = __float_as_uint(__uint_as_float(o[i]) + y);
            }
          }
        }
        if (kUse == kList && used) {
          // whole sectors: a thread's row is far from its neighbours'
          float *x = whole ? rows_to().sums + place() * D : part + tr * DP;
#pragma unroll
          for (int i = 0; i < 32; i += 8)
            if (d0 + i < D)
              asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(x + d0 + i), "r"(o[i]),
                           "r"(o[i + 1]), "r"(o[i + 2]), "r"(o[i + 3]), "r"(o[i + 4]), "r"(o[i + 5]), "r"(o[i + 6]),
                           "r"(o[i + 7])
                           : "memory");
        } else if (used && whole) {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (d0 + i < D) {
              uint4 y;
              y.x = KvType<T>::pack(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv);
              y.y = KvType<T>::pack(__uint_as_float(o[i + 2]) * inv, __uint_as_float(o[i + 3]) * inv);
              y.z = KvType<T>::pack(__uint_as_float(o[i + 4]) * inv, __uint_as_float(o[i + 5]) * inv);
              y.w = KvType<T>::pack(__uint_as_float(o[i + 6]) * inv, __uint_as_float(o[i + 7]) * inv);
              *reinterpret_cast<uint4 *>(dst + d0 + i) = y;
            }
          }
        } else if (used) {
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<uint4 *>(part + tr * DP + d0 + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        }
        __syncwarp();  // the next load is one instruction of the whole warp
      }
      if (used) {
        if (!whole) {
          part[kTcRows * DP + tr] = m;
          part[kTcRows * (DP + 1) + tr] = l;
        } else if (kUse == kList) {
          rows_to().stats[place()] = make_float2(m, l);
        } else if (P.s.lse) {
          P.s.lse[place()] = (m + log2f(l)) * 0.6931471805599453f;
        }
      }
      if (kUse == kAlone && !whole && g.kt0 == 0 && r == 0 && q == 0)
        P.part[blockIdx.x] = {kv_run_of(run, seg_begin + kSetup + g.tiles - 1), g.head, g.row_tile * kTcRows, g.rows,
                              g.tok.first};
      __syncwarp();
      tmem_before_sync();  // the next segment's products overwrite O
      if (join && lane == 0) bar_arrive(smem_u32(&sh.half_free));
      if (lane == 0) bar_arrive(smem_u32(&sh.seg_done[mine % kOddSets]));
    }
    if (!ok && r == 0) {
      const bool prefix = kUse == kList && b < P.n_prefixes;
      int32_t *status = prefix ? P.prefixes.status : P.c.status;
      if (status) status[kUse == kList && !prefix ? b - P.n_prefixes : b] = UNISON_ERR_TIMEOUT;
    }
  }
  __syncwarp();
  tmem_before_sync();
  __syncthreads();
  if (warp == kIssueWarp) {
    tmem_after_sync();
    tmem_free(tmem, 512);
  }
}

}  // namespace

template <typename T, int DP, int kUse>
int attend_tc(const AttendParams &p, int grid, void *stream) {
  static uint64_t done = 0;
  const void *kernel = reinterpret_cast<const void *>(attend_tc_kernel<T, DP, kUse>);
  if (!kv_allow_smem(kernel, kTcSmem<DP>, &done)) return UNISON_ERR_CUDA;
  AttendTcParams q;
  static_cast<AttendParams &>(q) = p;
  kv_boxes(q.k_boxes, p.c, p.c.k, p.c.k_page, p.c.k_head, p.c.k_slot, 16);
  kv_boxes(q.v_boxes, p.c, p.c.v, p.c.v_page, p.c.v_head, p.c.v_slot, 16);
  if (kUse == kList && p.n_prefixes) {
    const KvCacheArg &c = p.prefixes;
    kv_boxes(q.k_prefix_boxes, c, c.k, c.k_page, c.k_head, c.k_slot, 16);
    kv_boxes(q.v_prefix_boxes, c, c.v, c.v_page, c.v_head, c.v_slot, 16);
  }
  return kv_launch("kv_attend", dim3(grid), dim3(kThreads), kTcSmem<DP>, stream, 1, attend_tc_kernel<T, DP, kUse>, q);
}

#define UNISON_ATTEND_TC(use)                                                         \
  template int attend_tc<__nv_bfloat16, 64, use>(const AttendParams &, int, void *);  \
  template int attend_tc<__nv_bfloat16, 128, use>(const AttendParams &, int, void *); \
  template int attend_tc<__half, 64, use>(const AttendParams &, int, void *);         \
  template int attend_tc<__half, 128, use>(const AttendParams &, int, void *);
UNISON_ATTEND_TC(kAlone)
UNISON_ATTEND_TC(kList)
#undef UNISON_ATTEND_TC

}  // namespace unison
