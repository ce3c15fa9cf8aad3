// Changes of the paged cache: accepted tokens into it (unison_kv_commit), the
// least attended ones out of it (unison_kv_evict).
#include <cooperative_groups.h>

#include "kv.cuh"

namespace unison {
namespace {

// ---------------------------------------------------------------- commit --
struct CommitParams {
  KvCacheArg c;
  unison_kv_tree t;
  unison_kv_step s;
  unison_kv_path path;
};

// One CTA per session; a thread moves 16 bytes at a time.  Bound by latency (two
// dependent look-ups and a copy): 5 us for 64 sessions of up to eight tokens, 8
// KV heads of 128.
template <typename T>
__global__ void __launch_bounds__(256) commit_kernel(const CommitParams P) {
  follow_last_kernel();
  const int b = blockIdx.x, tid = threadIdx.x;
  const int H = P.c.n_heads, chunks = P.c.head_dim / 8;
  const KvRange tok = kv_tokens(P.t, b, P.c.status);
  const int n = kv_path_count(P.path, b, tok.count, P.c.status);
  const int len = kv_length(P.c, b);
  const int pos = P.c.next_pos ? P.c.next_pos[b] : len;
  bool full = len + n > P.c.max_pages * P.c.page_size;
  int off;
  if (!full && tid < n) full = kv_page(P.c, b, len + tid, off) < 0;
  const bool strange = tid < n && kv_path_node(P.path, b, tok.count, tid) < 0;
  // (every thread has also read what the first one will change)
  const bool no_room = __syncthreads_or(full), no_node = __syncthreads_or(strange);
  if (no_room || no_node) {
    if (tid == 0 && P.c.status) P.c.status[b] = no_room ? UNISON_ERR_CAPACITY : UNISON_ERR_RANGE;
    return;
  }
  const int per_row = H * chunks;
  for (int i = tid; i < n * per_row; i += blockDim.x) {
    const int row = i / per_row, h = i % per_row / chunks, c = i % chunks;
    const int node = kv_path_node(P.path, b, tok.count, row);
    const int page = kv_page(P.c, b, len + row, off);
    if (page < 0 || node < 0) continue;  // (asked above)
    const int64_t from = tok.first + node;
    const int4 k = *reinterpret_cast<const int4 *>(static_cast<const T *>(P.s.k_new) + from * P.s.k_token +
                                                   h * P.s.k_head + c * 8);
    const int4 v = *reinterpret_cast<const int4 *>(static_cast<const T *>(P.s.v_new) + from * P.s.v_token +
                                                   h * P.s.v_head + c * 8);
    T *to_k = static_cast<T *>(P.c.k) + page * P.c.k_page + h * P.c.k_head + off * P.c.k_slot;
    T *to_v = static_cast<T *>(P.c.v) + page * P.c.v_page + h * P.c.v_head + off * P.c.v_slot;
    *reinterpret_cast<int4 *>(to_k + c * 8) = k;
    *reinterpret_cast<int4 *>(to_v + c * 8) = v;
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
  KvCacheArg c, to;  // to: the cache itself where slots move in place
  const int32_t *keep;
  int32_t sink, recent;
  bool in_place;
  bool by_pos;     // positions tell what is protected: pos and next_pos are there
  bool by_four;    // mass and pos of four neighbouring slots are 16 aligned bytes
  int hold;        // keys of a thread of the selection in shared memory
  int per_seg;     // CTAs that move one segment's slots
  int32_t *moves;  // [segments][slots of a session]: sources, and from the middle on targets (in place)
  int32_t *count;  // [segments]
};

constexpr int kSelect = 256, kPitch = kSelect + 1;
constexpr int kMaxCluster = 8;
constexpr int kBins = 2048;         // digits of 11, 11 and 10 bits
constexpr int kMostHeld = 192;      // keys of a thread in shared memory

// Order of a slot among its session's: protected slots above all, then larger
// mass (the bits of a float, turned so that unsigned order is the numbers'
// order, -0 as 0), NaN and slots without a page below all.
__device__ __forceinline__ uint32_t order_key(const EvictParams &P, float mass, int pos, int next) {
  const uint32_t u = __float_as_uint(mass + 0.f);
  const uint32_t order = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  if (pos < P.sink || pos >= next) return ~0u;
  return isnan(mass) ? 0 : order;
}
// Keys of kN slots, kStep apart, as far as they are below end: their look-ups
// are on their way together.
template <int kN>
__device__ __forceinline__ void slot_keys(const EvictParams &P, int b, int h, int first, int step, int end, int next,
                                          uint32_t (&key)[kN]) {
  int page[kN], off[kN], pos[kN];
  float mass[kN];
  const int64_t head = h * P.c.m_head;
#pragma unroll
  for (int i = 0; i < kN; i++) {
    page[i] = kNoSlot;
    if (first + i * step < end) page[i] = kv_page_load(P.c, b, first + i * step, off[i]);
  }
#pragma unroll
  for (int i = 0; i < kN; i++) {
    page[i] = kv_page_ok(P.c, b, page[i]);
    const int64_t m = head + page[i] * P.c.m_page + off[i] * P.c.m_slot;
    pos[i] = first + i * step;
    mass[i] = 0.f;
    if (page[i] >= 0) {
      mass[i] = P.c.mass[m];
      if (P.by_pos) pos[i] = P.c.pos[m];
    }
  }
#pragma unroll
  for (int i = 0; i < kN; i++) key[i] = page[i] < 0 ? 0 : order_key(P, mass[i], pos[i], next);
}

// The same of groups of four neighbouring slots (P.by_four): one look-up and two
// loads each.  A group's slots behind `end` lie in the same page.
template <int kN>
__device__ __forceinline__ void slot_keys_by_four(const EvictParams &P, int b, int h, int first, int step, int end,
                                                  int next, uint32_t (&key)[kN][4]) {
  int page[kN], off[kN];
  float4 mass[kN];
  int4 pos[kN];
  const int64_t head = h * P.c.m_head;
#pragma unroll
  for (int i = 0; i < kN; i++) {
    page[i] = kNoSlot;
    if (first + i * step < end) page[i] = kv_page_load(P.c, b, first + i * step, off[i]);
  }
#pragma unroll
  for (int i = 0; i < kN; i++) {
    page[i] = kv_page_ok(P.c, b, page[i]);
    const int64_t m = head + page[i] * P.c.m_page + off[i];
    const int s = first + i * step;
    pos[i] = make_int4(s, s + 1, s + 2, s + 3);
    mass[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (page[i] >= 0) {
      mass[i] = *reinterpret_cast<const float4 *>(P.c.mass + m);
      if (P.by_pos) pos[i] = *reinterpret_cast<const int4 *>(P.c.pos + m);
    }
  }
#pragma unroll
  for (int i = 0; i < kN; i++) {
    const bool no = page[i] < 0;
    key[i][0] = no ? 0 : order_key(P, mass[i].x, pos[i].x, next);
    key[i][1] = no ? 0 : order_key(P, mass[i].y, pos[i].y, next);
    key[i][2] = no ? 0 : order_key(P, mass[i].z, pos[i].z, next);
    key[i][3] = no ? 0 : order_key(P, mass[i].w, pos[i].w, next);
  }
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

// Lists the moves of one segment (session and head); a cluster of CTAs shares
// its slots, in order, and so do a CTA's threads: a thread has a run of them.
// Every key is read once and kept in shared memory, key k of thread t at
// k * kPitch + t (odd: neighbouring slots lie in different banks).  The key of
// the last slot that stays is found digit by digit: each CTA counts its own
// keys, adds up the counts of all (through distributed shared memory) and finds
// the same digit.  Then each thread's slots with that very key are ranked, and
// the moves counted and written.  The counts are whole numbers, so the atomics'
// order changes nothing.  Bound by latency: a chain of dependent steps (table,
// account, three digits with two barriers each, three prefixes), of which only
// the first one reads the 8 bytes of a slot that it has to.  64 sessions x 8
// heads of 4,100 slots: 17 us; 16 x 8 of 8k to 32k: 35 us.
__global__ void __launch_bounds__(kSelect, 4) evict_select_kernel(const EvictParams P) {
  follow_last_kernel();
  namespace cg = cooperative_groups;
  extern __shared__ uint32_t keys[];  // [hold][kPitch]
  __shared__ __align__(16) uint32_t hist[2][kBins];
  __shared__ uint32_t digit, above, inside, part[33];
  __shared__ uint32_t cta_sum[2][kMaxCluster][2];
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank();
  auto sync = [&]() {
    if (ctas > 1)
      cluster.sync();
    else
      __syncthreads();
  };
  const int seg = blockIdx.x / ctas, tid = threadIdx.x;
  const int b = seg / P.c.n_heads, h = seg % P.c.n_heads;
  const int len = kv_length(P.c, b);
  const int n = kept_count(P, b, len);
  // positions from here on are protected
  const int64_t from_pos = (int64_t)(P.by_pos ? P.c.next_pos[b] : len) - P.recent;
  const int next = (int)max(min(from_pos, (int64_t)INT32_MAX), (int64_t)INT32_MIN);
  const int64_t room = (int64_t)P.c.max_pages * P.c.page_size;
  int32_t *from = P.moves + seg * room, *into = from + room / 2;
  if (n == 0 || (P.in_place && n == len)) {  // all CTAs of the cluster
    if (rank == 0 && tid == 0) P.count[seg] = 0;
    return;
  }
  // slots of a thread, of this CTA, of this thread
  const int each = (len + ctas * kSelect - 1) / (ctas * kSelect);
  const int64_t first64 = (int64_t)rank * each * kSelect;
  const int first = (int)min(first64, (int64_t)len), last = (int)min(first64 + each * kSelect, (int64_t)len);
  const int begin = min(first + tid * each, last), mine = min(begin + each, last) - begin;
  const int held = P.hold;  // keys of a thread in shared memory
  // f(k, key) for this thread's slots; the keys come from shared memory four at a time.
  auto each_key = [&](auto f) {
    int k = 0;
    for (; k + 4 <= min(mine, held); k += 4) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; i++) x[i] = keys[(k + i) * kPitch + tid];
#pragma unroll
      for (int i = 0; i < 4; i++) f(k + i, x[i]);
    }
    for (; k < mine; k++) {
      uint32_t x[1] = {0};
      if (k < held)
        x[0] = keys[k * kPitch + tid];
      else if (n < len)
        slot_keys<1>(P, b, h, begin + k, 0, last, next, x);
      f(k, x[0]);
    }
  };

  uint32_t last_key = 0;  // of the slots that stay
  uint32_t ties = 0;      // slots with that key that stay, the lowest first
  if (n < len) {
    // neighbouring threads read neighbouring slots here
    const uint32_t by_each = each == 1 ? 0 : 0xFFFFFFFFu / each + 1;  // (slots of a CTA < 2^16 while they are held)
    auto thread_of = [&](int s) { return each > held ? s / each : each == 1 ? s : (int)__umulhi(s, by_each); };
    if (P.by_four) {
      constexpr int kAtOnce = 4;
      for (int i = tid * 4; i < last - first; i += kSelect * 4 * kAtOnce) {
        uint32_t x[kAtOnce][4];
        slot_keys_by_four<kAtOnce>(P, b, h, first + i, kSelect * 4, last, next, x);
#pragma unroll
        for (int j = 0; j < kAtOnce; j++) {
          int s = i + j * kSelect * 4, t = thread_of(s), k = s - t * each;
#pragma unroll
          for (int e = 0; e < 4; e++, s++) {
            if (first + s < last && k < held) keys[k * kPitch + t] = x[j][e];
            if (++k == each) k = 0, t++;
          }
        }
      }
    } else {
      constexpr int kAtOnce = 8;
      for (int i = tid; i < last - first; i += kSelect * kAtOnce) {
        uint32_t x[kAtOnce];
        slot_keys<kAtOnce>(P, b, h, first + i, kSelect, last, next, x);
#pragma unroll
        for (int j = 0; j < kAtOnce; j++) {
          const int s = i + j * kSelect, t = thread_of(s), k = s - t * each;
          if (first + s < last && k < held) keys[k * kPitch + t] = x[j];
        }
      }
    }
    for (int i = tid; i < kBins; i += kSelect) hist[0][i] = 0;
    __syncthreads();
    uint32_t rest = n;
    int shift = 21, bits = 11;
    for (int pass = 0;; pass++) {
      uint32_t *counts = hist[pass & 1];
      each_key([&](int, uint32_t x) {
        if (pass == 0 || x >> (shift + bits) == last_key) atomicAdd(&counts[x >> shift & ((1u << bits) - 1)], 1u);
      });
      sync();
      // eight bins a thread, from the top: thread 0 has the highest
      const int bin = kBins - 8 - 8 * tid;
      uint32_t of[8] = {0, 0, 0, 0, 0, 0, 0, 0}, sum = 0;
      for (int c0 = 0; c0 < ctas; c0 += 4) {
        uint4 x[4], y[4];
#pragma unroll
        for (int c = 0; c < 4; c++) {
          const uint4 *theirs =
              reinterpret_cast<const uint4 *>(cluster.map_shared_rank(counts, min(c0 + c, ctas - 1)) + bin);
          x[c] = theirs[1], y[c] = theirs[0];
        }
#pragma unroll
        for (int c = 0; c < 4; c++) {
          if (c0 + c >= ctas) break;
          of[0] += x[c].w, of[1] += x[c].z, of[2] += x[c].y, of[3] += x[c].x;
          of[4] += y[c].w, of[5] += y[c].z, of[6] += y[c].y, of[7] += y[c].x;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; i++) sum += of[i];
      for (int i = tid; i < kBins; i += kSelect) hist[~pass & 1][i] = 0;  // of the last pass: read by all
      uint32_t all;
      uint32_t over = block_scan(sum, part, all);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        if (over < rest && rest <= over + of[i]) {
          digit = bin + 7 - i;
          above = over;
          inside = of[i];
        }
        over += of[i];
      }
      __syncthreads();
      last_key = last_key << bits | digit;
      rest -= above;
      if (rest == inside) {  // all with these digits stay
        last_key = (last_key << shift) - 1;
        break;
      }
      if (shift == 0) {
        ties = rest;
        break;
      }
      bits = shift > 10 ? 11 : 10;
      shift -= bits;
      __syncthreads();  // digit, above, inside are read
    }
  }
  if (ctas > 1 && n == len) cluster.sync();  // every CTA has begun: its shared memory may be written to

  // Exclusive prefixes over all CTAs' threads of two counts at once, and their sums.
  int exchanges = 0;
  auto prefix = [&](uint32_t &x, uint32_t &y, uint32_t &all_x, uint32_t &all_y) {
    x = block_scan(x, part, all_x);
    y = block_scan(y, part, all_y);
    if (ctas == 1) return;
    const int slot = exchanges++ & 1;
    if (tid < ctas) {
      uint32_t *theirs = cluster.map_shared_rank(&cta_sum[slot][rank][0], tid);
      theirs[0] = all_x;
      theirs[1] = all_y;
    }
    cluster.sync();
    all_x = all_y = 0;
    for (int c = 0; c < ctas; c++) {
      if (c < rank) x += cta_sum[slot][c][0], y += cta_sum[slot][c][1];
      all_x += cta_sum[slot][c][0];
      all_y += cta_sum[slot][c][1];
    }
  };
  uint32_t tie = 0, none = 0, all, more;
  if (ties) {
    each_key([&](int, uint32_t x) { tie += x == last_key; });
    prefix(tie, none, all, more);
  }
  auto stays = [&](uint32_t x, uint32_t &rank) {
    if (n == len) return true;
    if (ties && x == last_key) return rank++ < ties;
    return x > last_key;
  };
  // (the first 32 slots of a thread are remembered: most sessions have no more)
  uint32_t targets = 0, sources = 0, r = tie, moves = 0;
  each_key([&](int k, uint32_t x) {
    const bool stay = stays(x, r), low = P.in_place && begin + k < n;
    targets += P.in_place && low && !stay;
    sources += stay && !low;
    if (k < 32 && stay != low) moves |= 1u << k;
  });
  prefix(targets, sources, all, more);
  if (rank == 0 && tid == 0) P.count[seg] = (int)(P.in_place ? min(all, more) : more);
  auto write = [&](int k, bool stay) {
    if (stay)
      from[sources++] = begin + k;
    else
      into[targets++] = begin + k;
  };
  for (; moves; moves &= moves - 1) {
    const int k = __ffs(moves) - 1;
    write(k, !(P.in_place && begin + k < n));
  }
  if (mine > 32) {
    r = tie;
    each_key([&](int k, uint32_t x) {
      const bool stay = stays(x, r), low = P.in_place && begin + k < n;
      if (k >= 32 && stay != low) write(k, stay);
    });
  }
}

// Moves the listed slots: keys, values, mass and position.  A warp looks up 32
// moves at once, a lane each, and then copies them row by row, eight loads of 16
// bytes of a lane on their way.  Bound by memory where many slots move (16
// sessions' 8,192 slots into another cache, 8 KV heads of 128: 1.09 GB in 175 us,
// 6.2 TB/s), by latency where few do (6 us).
template <typename T>
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictParams P) {
  follow_last_kernel();
  const int seg = blockIdx.x / P.per_seg, of_seg = blockIdx.x % P.per_seg, lane = threadIdx.x & 31;
  const int b = seg / P.c.n_heads, h = seg % P.c.n_heads;
  const int chunks = P.c.head_dim / 8;
  const int64_t room = (int64_t)P.c.max_pages * P.c.page_size;
  const int32_t *from = P.moves + seg * room, *into = from + room / 2;
  const int count = P.count[seg];
  const int warps = P.per_seg * (blockDim.x >> 5);
  const int width = 2 * chunks;
  const unsigned reciprocal = ((1u << 20) + width - 1) / width;
  const T *k = static_cast<const T *>(P.c.k) + h * P.c.k_head, *v = static_cast<const T *>(P.c.v) + h * P.c.v_head;
  T *to_k = static_cast<T *>(P.to.k) + h * P.to.k_head, *to_v = static_cast<T *>(P.to.v) + h * P.to.v_head;
  for (int i0 = (of_seg * (blockDim.x >> 5) + (threadIdx.x >> 5)) * 32; i0 < count; i0 += warps * 32) {
    int page = -1, to_page = -1, off = 0, to_off = 0;
    if (i0 + lane < count) {
      page = kv_page(P.c, b, from[i0 + lane], off);
      to_page = kv_page(P.to, b, P.in_place ? into[i0 + lane] : i0 + lane, to_off);
    }
    if (page < 0 || to_page < 0) page = to_page = -1;
    if (page >= 0) {
      const int64_t m = page * P.c.m_page + h * P.c.m_head + off * P.c.m_slot;
      const int64_t tm = to_page * P.to.m_page + h * P.to.m_head + to_off * P.to.m_slot;
      if (P.to.mass) P.to.mass[tm] = P.c.mass[m];
      if (P.to.pos && P.c.pos) P.to.pos[tm] = P.c.pos[m];
    }
    // 16 bytes a lane: entry e is chunk e % width of row e / width (the keys'
    // chunks, then the values'); e < 2^11, so the division by multiplication is exact
    constexpr int kFlight = 8;  // loads of a lane on their way at once
    const int entries = min(count - i0, 32) * width;
    for (int e0 = 0; e0 < entries; e0 += 32 * kFlight) {
      int4 x[kFlight];
      T *dst[kFlight];
#pragma unroll
      for (int i = 0; i < kFlight; i++) {
        const int e = e0 + i * 32 + lane;
        const int row = (int)((unsigned)e * reciprocal >> 20) & 31, c = e - row * width;
        const bool key = c < chunks;
        const int64_t p = __shfl_sync(~0u, page, row), o = __shfl_sync(~0u, off, row);
        const int64_t tp = __shfl_sync(~0u, to_page, row), to = __shfl_sync(~0u, to_off, row);
        dst[i] = nullptr;
        if (e < entries && p >= 0) {
          const T *src = key ? k + p * P.c.k_page + o * P.c.k_slot + c * 8
                             : v + p * P.c.v_page + o * P.c.v_slot + (c - chunks) * 8;
          dst[i] = key ? to_k + tp * P.to.k_page + to * P.to.k_slot + c * 8
                       : to_v + tp * P.to.v_page + to * P.to.v_slot + (c - chunks) * 8;
          x[i] = *reinterpret_cast<const int4 *>(src);
        }
      }
#pragma unroll
      for (int i = 0; i < kFlight; i++)
        if (dst[i]) *reinterpret_cast<int4 *>(dst[i]) = x[i];
    }
  }
  if (of_seg == 0 && h == 0 && threadIdx.x == 0) {
    P.to.length[b] = kept_count(P, b, kv_length(P.c, b));
    if (!P.in_place && P.to.next_pos && P.c.next_pos) P.to.next_pos[b] = P.c.next_pos[b];
  }
}

uint64_t evict_bytes(const unison_kv_cache *c) {
  const uint64_t segs = (uint64_t)c->n_seqs * c->n_heads;
  return segs * 4 + segs * c->max_pages * c->page_size * 4;
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
  const CommitParams p = {KvCacheArg(*cache), *tree, *step, path ? *path : unison_kv_path{}};
  // 16-bit types move as they are
  return kv_launch("kv_commit", dim3(cache->n_seqs), dim3(256), 0, cuda_stream, 1, commit_kernel<uint16_t>, p);
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
  if (segs > 1 << 22) return UNISON_ERR_RANGE;
  if (cache->n_seqs == 0) return UNISON_OK;
  if (!keep || !pools_ok(cache) || (into && !pools_ok(into))) return UNISON_ERR_ARG;
  if (cache->max_pages > 0 && cache->n_pages > 0 && !cache->mass) return UNISON_ERR_ARG;
  if (!workspace || !kv_aligned(workspace, 16) || workspace_bytes < evict_bytes(cache)) return UNISON_ERR_ARG;
  const int64_t room = (int64_t)cache->max_pages * cache->page_size;
  EvictParams p;
  p.c = *cache;
  p.to = KvCacheArg(into ? *into : *cache);
  p.keep = keep;
  p.sink = sink;
  p.recent = recent;
  p.in_place = into == nullptr;
  p.by_pos = cache->pos && cache->next_pos;
  p.by_four = cache->m_slot == 1 && cache->page_size % 4 == 0 && (cache->m_page | cache->m_head) % 4 == 0 &&
              kv_aligned(cache->mass, 16) && kv_aligned(cache->pos, 16);
  p.moves = static_cast<int32_t *>(workspace);
  p.count = p.moves + segs * room;
  // CTAs per segment: as many as the segments leave room for (two CTAs on a
  // multiprocessor, though four fit: clusters then wait for places; between events
  // around the launch, which add 4 us, 64 segments of 8k to 32k slots take 32 us
  // against 71, 128 take 39 against 45, and one CTA each 50 and 52), none with less
  // than 2,048 slots.
  const int64_t spare = (int64_t)kv_sm_count() * 2 / (int64_t)segs;
  int ctas = 1;
  while (ctas < kMaxCluster && ctas * 2 <= spare && (int64_t)ctas * 2048 < room) ctas *= 2;
  p.hold = (int)min((room + (int64_t)ctas * kSelect - 1) / ((int64_t)ctas * kSelect), (int64_t)kMostHeld);
  const int bytes = p.hold * kPitch * 4;
  static uint64_t done = 0;
  if (!kv_allow_smem(reinterpret_cast<const void *>(evict_select_kernel), kMostHeld * kPitch * 4, &done))
    return UNISON_ERR_CUDA;
  rc = kv_launch("kv_evict_select", dim3((unsigned)(segs * ctas)), dim3(kSelect), bytes, cuda_stream, ctas,
                 evict_select_kernel, p);
  if (rc != UNISON_OK) return rc;
  // A CTA moves 256 slots at a time.  Enough CTAs for all at once where a cache
  // is copied (16 sessions' 8,192 slots: 179 us between events around the launch,
  // with a fifth of the CTAs 192); few where a session at its budget drops a
  // handful (up to 8 slots of 64 sessions: 10 us, with five times the CTAs 15).
  const int64_t most = into ? min(room, (int64_t)into->max_pages * into->page_size) : room / 2;
  const int64_t fill = ((int64_t)kv_sm_count() * (into ? 32 : 6) + segs - 1) / (int64_t)segs;
  p.per_seg = (int)max((int64_t)1, min((most + 255) / 256, fill));
  return kv_launch("kv_evict_move", dim3((unsigned)(segs * p.per_seg)), dim3(256), 0, cuda_stream, 1,
                   evict_move_kernel<uint16_t>, p);
}
