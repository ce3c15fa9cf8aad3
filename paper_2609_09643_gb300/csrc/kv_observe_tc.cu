// Attention weight on cached keys by the tensor cores (the variant of
// unison_kv_observe for head sizes up to 128 and up to 512 query rows).
//
// The keys are the rows of the product and the query rows its columns: a
// thread owns a key, reads its scores from tensor memory, and adds their
// weights in its registers, so nothing is exchanged between threads and no
// atomics are needed.  A CTA keeps the query rows of one segment (session and
// KV head) in shared memory and streams tiles of 128 keys past them.  Roles:
//   warps 8-11      find each key's account and, per segment, copy the query
//                   rows; key tiles that are not full, row by row
//   warp 13         full key tiles, by TMA
//   warp 12         issues the products, 128 query rows at a time, into four
//                   buffers of tensor memory
//   warps 0-3, 4-7  turn the scores of a buffer into weights, in turn
//
//   mass[x] += sum over the rows r of exp2(c S[r,x] - log-sum of row r)
//
// with everything in 32 bits: a weight is one fused multiply-add and one exp2.
// Bound by memory up to 128 rows (64 sessions of 512 to 32k keys, 8 KV heads of
// 128, 4 to 16 rows, 1.07 GB: 180 us, 5.9 TB/s), above by the warps that turn
// scores into weights (rows 8 to 512 over 16 sessions of 8k to 32k keys: 209 us).
// They take 1,000 cycles for a chunk of 128 x 128: 622 with nothing but the loads
// and two warps per scheduler (exp2 at 32 a cycle: 512), the rest between chunks
// and tiles (barriers, the sums' exchange).  So what is asked once a segment is
// not asked once a chunk (512 rows took 328 us then).  Not faster: four groups
// of weight warps (249 us where two took 230), scores read as matrix fragments
// so that a log-sum serves four weights, the next scores on their way meanwhile.
#include "kv_copy.cuh"
#include "kv_observe.cuh"

namespace unison {
namespace {

constexpr int kThreads = 448;
constexpr int kTile = 128;
constexpr int kCopyWarp = 8, kIssueWarp = 12, kBoxWarp = 13;
constexpr int kBuffers = 4, kMostSlots = 6;
constexpr int kNodes = UNISON_KV_MAX_TOKENS;
// Tiles whose keys' accounts are kept in shared memory.  The copies for tile t
// wait for the products of tile t - slots, which wait for the scores of tile
// t - slots - kBuffers to be read; accounts are read after that.  So of the last
// two tiles read by then, one of each group where a tile is one chunk, the
// accounts may still be wanted; a group has read those of its tile before.
constexpr int kMoreMarks = kBuffers + 2;
constexpr int kMarkBytes = kTile * 12;

struct ObserveShared {
  KvRunShared run;
  uint64_t k_full[kMostSlots], k_free[kMostSlots], q_full[2], q_free[2], t_full[kBuffers], t_free[kBuffers],
      seg_done[2], part_full[2], part_free[2], idle;
  uint64_t mask[2][kNodes];  // of the accepted nodes
  float part[2][kTile];      // sums of the group that does not write, of two tiles
  bool plain[2][4];          // whether every row that a copying warp read has weight to give
  uint32_t tmem;
  volatile int dead;
};

struct Segment {
  int b, head, rows, tiles, kt0, kt1, len;
  KvRange tok;
};

struct ObserveTcParams : ObserveParams {
  KvBoxes k_boxes;
};

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, 1) observe_tc_kernel(const __grid_constant__ ObserveTcParams P) {
  follow_last_kernel();
  constexpr uint32_t kTileBytes = kTile * DP * 2, kBlock = kTile * 128;
  extern __shared__ unsigned char smem_raw[];
  __shared__ ObserveShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int D = P.c.head_dim, H = P.c.n_heads, G = P.group;
  const uint32_t q_base = (smem_u32(smem_raw) + 1023) & ~1023u, q_bytes = P.q_rows * DP * 2,
                 slot_base = q_base + P.q_buffers * q_bytes;
  // log-sums of the rows, of two segments, in log2 units and negated; -inf: no weight from this row
  float *const lse_base = reinterpret_cast<float *>(smem_raw + (slot_base - smem_u32(smem_raw)) + P.slots * kTileBytes);

  float **const marks_at = reinterpret_cast<float **>(lse_base + 2 * P.q_rows);  // where a key's weight goes
  float *const marks_old = reinterpret_cast<float *>(marks_at + (P.slots + kMoreMarks) * kTile);  // what is there

  // A tile's share of the run, in units of 33 ns: its keys' way here, or the
  // products and weights of its chunks of 128 query rows, where those take
  // longer.  (16 sessions of 16k keys, 8 KV heads, head size 128: 101 us with 8
  // rows, 106 with 128, 154 with 136, 166 with 256, 222 with 384, 282 with 512;
  // head size 64: 81, 88, 146, 161, 212, 259.  Beside sessions of many rows,
  // which leave them the memory, few rows take a fifth less.)
  const int keys_way = DP == 64 ? 20 : P.slots > 2 || P.k_boxes.rows > 8 ? 26 : P.k_boxes.rows ? 40 : 80;
  auto share = [&](int rows) {
    return rows <= 128 ? keys_way + rows / 32 : max(keys_way, 14 + 11 * ((rows + 127) / 128) + rows / 25);
  };
  // A head's beginning (its query rows, an empty pipeline) and the tiles that are
  // not full, in tiles.
  auto setup = [&](int rows) { return max((160 + rows / 4) / share(rows), 1); };
  KvRun run;
  if (!kv_find_run(run, sh.run, P.c.n_seqs, gridDim.x, blockIdx.x, [&](int b) {
        const int tiles = observe_key_tiles(P, b, kTile);
        if (!tiles) return (int64_t)0;
        const int rows = kv_path_count(P.path, b, kv_tokens(P.t, b, nullptr).count, nullptr) * G;
        return (int64_t)(tiles + setup(rows)) * H * share(rows);
      }))
    return;
  if (tid == 0) {
    for (int i = 0; i < kMostSlots; i++) {
      bar_init(smem_u32(&sh.k_full[i]), 5);  // copying warps
      bar_init(smem_u32(&sh.k_free[i]), 1);
    }
    for (int i = 0; i < kBuffers; i++) {
      bar_init(smem_u32(&sh.t_full[i]), 2);
      bar_init(smem_u32(&sh.t_free[i]), 4);  // warps
    }
    for (int i = 0; i < 2; i++) {
      bar_init(smem_u32(&sh.q_full[i]), 4);
      bar_init(smem_u32(&sh.q_free[i]), 1);
      bar_init(smem_u32(&sh.seg_done[i]), kCopyWarp);
      bar_init(smem_u32(&sh.part_full[i]), 4);
      bar_init(smem_u32(&sh.part_free[i]), 4);
    }
    bar_init(smem_u32(&sh.idle), 1);
    sh.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kIssueWarp) tmem_alloc(smem_u32(&sh.tmem), 512);
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  const uint32_t tmem = sh.tmem;

  int b = run.b;
  int64_t at = run.at, seq_begin = run.begin;
  // The next tiles of one head in this run: those whose share begins in it.
  // (A head's tiles come behind the shares that stand for its beginning.)
  auto next_segment = [&](Segment &g) -> bool {
    while (at < run.end) {
      g.tok = kv_tokens(P.t, b, nullptr);
      g.tiles = observe_key_tiles(P, b, kTile);
      g.rows = kv_path_count(P.path, b, g.tok.count, nullptr) * G;
      const int each = share(g.rows), before = setup(g.rows);
      const int64_t per_head = g.tiles ? g.tiles + before : 0;
      const int64_t all = per_head * H;
      const int64_t from = (at - seq_begin + each - 1) / each;
      const int64_t to = min((run.end - seq_begin + each - 1) / each, all);
      if (from >= to) {
        seq_begin += all * each;
        at = max(at, seq_begin);
        b++;
        continue;
      }
      g.head = (int)(from / per_head);
      const int64_t head_begin = g.head * per_head, head_end = min(head_begin + per_head, to);
      at = seq_begin + head_end * each;
      g.kt0 = (int)max(from - head_begin - before, (int64_t)0);
      g.kt1 = (int)max(head_end - head_begin - before, (int64_t)0);
      if (g.kt0 >= g.kt1) continue;
      g.b = b;
      g.len = kv_length(P.c, b);
      return true;
    }
    return false;
  };

  if (warp >= kCopyWarp && warp < kIssueWarp) {
    // ------------------------------------------------------------- copies
    const int w = warp - kCopyWarp;
    KvCopier<T, DP> copier(w, lane, D, P.s.q);
    Ring ring, marks;
    int seg_no = 0;
    bool ok = true;
    Segment g;
    while (ok && next_segment(g)) {
      // The segment's rows: when the products of the last one that was in their
      // place are done, and nobody reads the statistics of the one before last.
      const int buf = seg_no % P.q_buffers, use = seg_no / P.q_buffers;
      if (use > 0) ok = copier.wait(smem_u32(&sh.q_free[buf]), (use - 1) & 1, &sh.dead);
      if (ok && seg_no > 1)
        ok = copier.wait(smem_u32(&sh.seg_done[seg_no & 1]), ((seg_no >> 1) - 1) & 1, &sh.dead);
      if (!ok) break;
      float *lse = lse_base + (seg_no & 1) * P.q_rows;
      const int j = w * 32 + lane;  // this lane's row of a tile
      bool plain = true;
      for (int r0 = 0; r0 < g.rows; r0 += 128) {
        const int r = r0 + j;
        const int node = r < g.rows ? observe_node(P, g.b, g.tok.count, r / G) : -1;
        const T *src = nullptr;
        float l = -INFINITY;
        if (node >= 0) {
          src = static_cast<const T *>(P.s.q) + (g.tok.first + node) * P.s.q_token + (g.head * G + r % G) * P.s.q_head;
          l = P.s.lse[(int64_t)(g.tok.first + node) * P.s.n_q_heads + g.head * G + r % G] * -1.4426950408889634f;
          if (l == INFINITY) l = -INFINITY;
        }
        if (r < g.rows && l == -INFINITY) plain = false;
        lse[r] = l;
        copier.rows(q_base + buf * q_bytes + r0 / 128 * kTileBytes, src);
      }
      if (j < kNodes) {
        const int node = j * G < g.rows ? observe_node(P, g.b, g.tok.count, j) : -1;
        sh.mask[seg_no & 1][j] = node < 0 ? 0 : P.t.mask ? P.t.mask[g.tok.first + node] : ~0ull >> (63 - node);
      }
      plain = __all_sync(~0u, plain);
      if (lane == 0) sh.plain[seg_no & 1][w] = plain;
      copier.issued(smem_u32(&sh.q_full[buf]));

      // a tile's pages are looked up two tiles ahead, the weights there one ahead
      auto find_page = [&](int kt, int &off) -> int {
        off = 0;
        return kt < g.kt1 && kt < g.tiles - 1 && kt * kTile + j < g.len
                   ? kv_page_load(P.c, g.b, kt * kTile + j, off) : kNoSlot;
      };
      auto account = [&](int page, int off) -> float * {
        return page < 0 ? nullptr : P.c.mass + page * P.c.m_page + g.head * P.c.m_head + off * P.c.m_slot;
      };
      int next_off = 0, later_off = 0;
      int next_page = find_page(g.kt0, next_off), later_page = find_page(g.kt0 + 1, later_off);
      next_page = kv_page_ok(P.c, g.b, next_page);
      float *next_m = account(next_page, next_off);
      float next_old = next_m ? *next_m : 0.f;
      const int boxed = P.k_boxes.rows ? g.len / kTile : 0;  // full tiles go by boxes
      for (int kt = g.kt0; kt < g.kt1; kt++) {
        const int page = next_page, off = next_off;
        float *m = next_m;
        const float old = next_old;
        next_page = kv_page_ok(P.c, g.b, later_page), next_off = later_off;
        next_m = account(next_page, next_off);
        next_old = next_m ? *next_m : 0.f;
        later_page = find_page(kt + 2, later_off);
        const int s = ring.at;
        ok = copier.wait(smem_u32(&sh.k_free[s]), ring.turn ^ 1, &sh.dead);
        if (!ok) break;
        ring.next(P.slots);
        const uint32_t bar = smem_u32(&sh.k_full[s]);
        const bool fresh = kt == g.tiles - 1 && j < g.tok.count && P.s.mass_new;
        if (fresh) m = P.s.mass_new + (int64_t)(g.tok.first + j) * H + g.head;
        const int mark = marks.at * kTile + j;
        marks.next(P.slots + kMoreMarks);
        marks_at[mark] = m;
        marks_old[mark] = old;
        __syncwarp();
        if (kt < boxed) {
          if (lane == 0) bar_arrive(bar);
          if (kt == g.kt0) copier.landed();
        } else {
          const T *src = nullptr;
          if (fresh)
            src = static_cast<const T *>(P.s.k_new) + (g.tok.first + j) * P.s.k_token + g.head * P.s.k_head;
          else if (page >= 0)
            src = static_cast<const T *>(P.c.k) + page * P.c.k_page + g.head * P.c.k_head + off * P.c.k_slot;
          copier.rows(slot_base + s * kTileBytes, src);
          copier.issued(bar);
        }
      }
      seg_no++;
    }
    copier.landed();
  } else if (warp == kBoxWarp) {
    // -------------------------------------------------------------- boxes
    Ring ring;
    bool ok = true;
    BoxSender<DP> sender(P.k_boxes);
    Segment g;
    while (ok && next_segment(g)) {
      const int boxed = P.k_boxes.rows ? g.len / kTile : 0;
      sender.reset();
      for (int kt = g.kt0; kt < g.kt1; kt++) {
        const int s = ring.at;
        if (kt < boxed) sender.look_up(P.c, g.b, kt, g.len);
        ok = __all_sync(~0u, bar_wait(smem_u32(&sh.k_free[s]), ring.turn ^ 1, &sh.dead));
        if (!ok) break;
        ring.next(P.slots);
        if (kt < boxed)
          sender.send(kt, slot_base + s * kTileBytes, smem_u32(&sh.k_full[s]), g.head);
        else if (lane == 0)
          bar_arrive(smem_u32(&sh.k_full[s]));
      }
    }
    if (!ok) KvCopier<T, DP>::give_up();
  } else if (warp == kIssueWarp) {
    // ----------------------------------------------------------- products
    // (the whole warp goes along, one lane issues)
    const uint32_t q_rows = smem_operand(q_base, kBlock), slots = smem_operand(slot_base, kBlock);
    Ring ring, buffer;
    int seg_no = 0;
    bool ok = true;
    const bool one = elect_one();
    auto release = [&](uint64_t &bar) { products_done(one, smem_u32(&bar)); };
    const uint32_t tmem = uniform(sh.tmem);
    Segment g;
    while (uniform(ok && next_segment(g))) {
      const int qb = seg_no % P.q_buffers, n_rows = uniform(g.rows), tiles = uniform(g.kt1 - g.kt0);
      for (int kt = 0; kt < tiles && ok; kt++) {
        const int s = ring.at;
        ok = __all_sync(~0u, bar_wait(smem_u32(&sh.k_full[s]), ring.turn, &sh.dead));
        if (ok && kt == 0)
          ok = __all_sync(~0u, bar_wait(smem_u32(&sh.q_full[qb]), (seg_no / P.q_buffers) & 1, &sh.dead));
        ring.next(P.slots);
        const uint32_t keys = slots + s * (kTileBytes >> 4);
        for (int r0 = 0; (r0 == 0 || r0 < n_rows) && ok; r0 += 128) {
          const int buf = buffer.at;
          ok = __all_sync(~0u, bar_wait(smem_u32(&sh.t_free[buf]), buffer.turn ^ 1, &sh.dead));
          if (!ok) break;
          buffer.next(kBuffers);
          tmem_after_sync();
          const int columns = (max(min(n_rows - r0, 128), 1) + 15) & ~15;
          const uint32_t shape = product_shape(kOperandType<T>, kTile, columns, false, false);
          const uint32_t rows = q_rows + ((qb * q_bytes + r0 / 128 * kTileBytes) >> 4);
#pragma unroll
          for (int d = 0; d < DP / 16; d++) {
            const uint32_t o = (d / 4 * kBlock + d % 4 * 32) >> 4;
            product_ss(one, tmem + buf * 128, keys + o, rows + o, shape, d > 0);
          }
          products_done(one, smem_u32(&sh.t_full[buf]));
          bar_arrive_by(one, smem_u32(&sh.t_full[buf]));  // hands on what the copies wrote besides
        }
        release(sh.k_free[s]);
      }
      release(sh.q_free[qb]);
      seg_no++;
    }
    // nothing may still be at work when tensor memory is freed
    release(sh.idle);
    for (int i = 0; i < 1 << 20 && !__all_sync(~0u, bar_try(smem_u32(&sh.idle), 0)); i++) {
    }
  } else if (warp < kCopyWarp) {
    // ------------------------------------------------------------ weights
    const int wg = warp >> 2, key = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's quarter of the 128 lanes
    const float c = P.s.scale * 1.4426950408889634f;
    auto warp_arrive = [&](uint64_t &bar) {
      __syncwarp();
      if (lane == 0) bar_arrive(smem_u32(&bar));
    };
    Ring marks;
    int jobs = 0, seg_no = 0, tile_no = 0, shared_tiles = 0;
    bool ok = true;
    Segment g;
    while (ok && next_segment(g)) {
      const float *lse = lse_base + (seg_no & 1) * P.q_rows;
      const uint64_t *mask = sh.mask[seg_no & 1];
      const int chunks = max((g.rows + 127) / 128, 1);
      int plain = -1;  // whether every row has weight to give, -1: not read yet
      for (int kt = g.kt0; kt < g.kt1; kt++, tile_no++, marks.next(P.slots + kMoreMarks)) {
        const bool last = kt == g.tiles - 1;
        // chunk by chunk in turn, beginning in turn where their number is odd
        const int first = chunks & 1 ? tile_no & 1 : 0;
        const bool writes = wg == first;
        uint64_t sum[2] = {0, 0};
        for (int i = wg ^ first; i < chunks; i += 2) {
          const int job = jobs + i, buf = job % kBuffers;
          ok = __all_sync(~0u, bar_wait(smem_u32(&sh.t_full[buf]), (job / kBuffers) & 1, &sh.dead));
          if (!ok) break;
          tmem_after_sync();
          const int n = min(g.rows - i * 128, 128);
          if (plain < 0) {
            const bool *all = sh.plain[seg_no & 1];
            plain = all[0] && all[1] && all[2] && all[3];
          }
          const bool checked = last || !plain;
          const uint32_t from = tmem + buf * 128 + lanes;
          const float *l = lse + i * 128;
          int r0 = 0;
          if (!checked) {
            const uint64_t cc = pair(c, c);
#pragma unroll 1
            for (; r0 + 32 <= n; r0 += 32) {
              uint32_t v[32];
              tmem_ld32(v, from + r0);
              tmem_wait_ld(v);
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const ulonglong2 y = *reinterpret_cast<const ulonglong2 *>(l + r0 + j);
                float e[4];
                unpair(fma_pair(pair(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), cc, y.x), e[0], e[1]);
                unpair(fma_pair(pair(__uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])), cc, y.y), e[2], e[3]);
                sum[0] = add_pair(sum[0], pair(exp2_fast(e[0]), exp2_fast(e[1])));
                sum[1] = add_pair(sum[1], pair(exp2_fast(e[2]), exp2_fast(e[3])));
              }
            }
          }
          if (r0 < n) {
            // the others 16 at a time, each with the question whether it counts
            const int node = (i * 128 + r0) / G;
            int head = i * 128 + r0 - node * G;
            uint64_t sees = 0;  // the accepted nodes from this one on that see this new token
            if (last && key < 64) {
              for (int j = 0; j < kNodes; j++) sees |= (mask[j] >> key & 1) << j;
              sees >>= min(node, kNodes - 1);
            }
#pragma unroll 1
            for (; r0 < n; r0 += 16) {
              uint32_t v[16], counts = n - r0 < 16 ? (1u << (n - r0)) - 1 : ~0u;
              tmem_ld16(v, from + r0);
              if (last) {
#pragma unroll
                for (int j = 0; j < 16; j++) {
                  if (!(sees & 1)) counts &= ~(1u << j);
                  if (++head == G) head = 0, sees >>= 1;
                }
              }
              __syncwarp();
              tmem_wait_ld(v);
#pragma unroll
              for (int j = 0; j < 16; j += 4) {
                const float4 y = *reinterpret_cast<const float4 *>(l + r0 + j);
                float e[4] = {exp2_fast(fmaf(__uint_as_float(v[j]), c, y.x)),
                              exp2_fast(fmaf(__uint_as_float(v[j + 1]), c, y.y)),
                              exp2_fast(fmaf(__uint_as_float(v[j + 2]), c, y.z)),
                              exp2_fast(fmaf(__uint_as_float(v[j + 3]), c, y.w))};
                e[0] = (counts >> j & 1) && y.x != -INFINITY ? e[0] : 0.f;
                e[1] = (counts >> (j + 1) & 1) && y.y != -INFINITY ? e[1] : 0.f;
                e[2] = (counts >> (j + 2) & 1) && y.z != -INFINITY ? e[2] : 0.f;
                e[3] = (counts >> (j + 3) & 1) && y.w != -INFINITY ? e[3] : 0.f;
                sum[0] = add_pair(sum[0], pair(e[0], e[1]));
                sum[1] = add_pair(sum[1], pair(e[2], e[3]));
              }
            }
          }
          tmem_before_sync();
          warp_arrive(sh.t_free[buf]);
        }
        if (!ok) break;
        jobs += chunks;
        float all, other;
        unpair(add_pair(sum[0], sum[1]), all, other);
        all += other;
        if (chunks > 1) {  // the writer adds the other group's sum
          const int set = shared_tiles & 1, use = shared_tiles >> 1;
          shared_tiles++;
          if (!writes) {
            if (use > 0) ok = __all_sync(~0u, bar_wait(smem_u32(&sh.part_free[set]), (use - 1) & 1, &sh.dead));
            if (!ok) break;
            sh.part[set][key] = all;
            warp_arrive(sh.part_full[set]);
          } else {
            ok = __all_sync(~0u, bar_wait(smem_u32(&sh.part_full[set]), use & 1, &sh.dead));
            if (!ok) break;
            all += sh.part[set][key];
            warp_arrive(sh.part_free[set]);
          }
        }
        if (writes) {
          const int mark = marks.at * kTile + key;
          float *to = marks_at[mark];
          if (to) *to = marks_old[mark] + all;
        }
      }
      if (!ok && key == 0 && P.c.status) P.c.status[g.b] = UNISON_ERR_TIMEOUT;
      warp_arrive(sh.seg_done[seg_no & 1]);
      seg_no++;
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

template <typename T, int DP>
int observe_tc(ObserveParams p, int max_rows, void *stream) {
  constexpr int kTileBytes = kTile * DP * 2;
  static uint64_t done = 0;
  p.q_rows = (max_rows + 127) / 128 * 128;
  p.q_buffers = p.q_rows == 128 ? 2 : 1;  // few rows: the next segment's may come while the last one's are read
  const int fixed = 1024 + p.q_rows * (p.q_buffers * DP * 2 + 8) + kMoreMarks * kMarkBytes;
  const int most = (227 << 10) - (int)sizeof(ObserveShared) - 1024;
  p.slots = min(kMostSlots, (most - fixed) / (kTileBytes + kMarkBytes));
  const int bytes = fixed + p.slots * (kTileBytes + kMarkBytes);
  if (!kv_allow_smem(reinterpret_cast<const void *>(observe_tc_kernel<T, DP>), most, &done))
    return UNISON_ERR_CUDA;
  ObserveTcParams q;
  static_cast<ObserveParams &>(q) = p;
  // Boxes of eight slots where shared memory holds few tiles on their way
  // (kv_copy.cuh has the figures).
  kv_boxes(q.k_boxes, p.c, p.c.k, p.c.k_page, p.c.k_head, p.c.k_slot, p.slots > 2 ? 16 : 8);
  return kv_launch("kv_observe", dim3(kv_sm_count()), dim3(kThreads), max(bytes, 120 << 10), stream, 1,
                   observe_tc_kernel<T, DP>, q);
}

template int observe_tc<__nv_bfloat16, 64>(ObserveParams, int, void *);
template int observe_tc<__nv_bfloat16, 128>(ObserveParams, int, void *);
template int observe_tc<__half, 64>(ObserveParams, int, void *);
template int observe_tc<__half, 128>(ObserveParams, int, void *);

}  // namespace unison
