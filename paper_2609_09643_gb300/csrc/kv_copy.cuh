// Tiles of paged rows on their way into the tensor cores' operands, for the
// four copying warps of a CTA.
//
// Full tiles of caches whose page size is a multiple of 16 go by TMA: one warp
// sends the boxes, and the hardware reports the bytes to the tile's barrier.
// Every other tile (the last one of a session, its new tokens, other page sizes
// or odd strides) and the query rows go by 16-byte copies, which can leave out
// single rows.  128 keys of 128 elements cost the warps about 2,000 cycles by
// copies and next to nothing by TMA; but a box takes the hardware 90 cycles,
// however small.  16 sessions of 16k keys, 8 KV heads, in pages of 8 / 16 / 64
// slots: attention of 64 rows 259 / 203 / 183 us by boxes, 198 by copies (head
// size 128), 178 / 143 / 124 and 159 (64); observation of 8 to 64 rows 169 /
// 112 / 101 by boxes and 120 / 113 / 108 by copies.  So boxes have 16 slots or
// more, except where query rows leave place for two tiles only: 512 rows'
// observation, few of them accepted, takes 168 by boxes of 8 and 343 by copies,
// which are not early enough.
#pragma once

#include <cuda.h>

#include "kv_tc.cuh"

namespace unison {

constexpr int kTileRows = 128;

// The pool of keys or values for TMA: [page][two of slot, head][element].
struct KvBoxes {
  CUtensorMap map;
  int rows;         // of a box, 0: not by TMA
  bool head_first;  // heads lie closer together than slots
};
// On the host; rows = 0 where the pool does not allow boxes of `least` slots
// (8, or a multiple of it).
void kv_boxes(KvBoxes &x, const unison_kv_cache &c, const void *pool, int64_t page, int64_t head, int64_t slot,
              int least);

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {  // an arrival that announces bytes
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void box_copy(uint32_t dst, const KvBoxes &x, uint32_t bar, int col, int slot, int head,
                                         int page) {
  const int c1 = x.head_first ? head : slot, c2 = x.head_first ? slot : head;
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
      "[%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(&x.map)), "r"(col), "r"(c1), "r"(c2), "r"(page), "r"(bar)
      : "memory");
}

// All boxes of full tiles, by one warp: lane i has column block i % (DP / 64) of
// box i / (DP / 64) of the tile.  The pages of the next boxes are looked up 32
// at a time, a lane each, so that most tiles wait for no look-up.  (A warp of
// its own takes five to eight cycles an instruction, and a tile's bytes arrive
// in 1,400: what is the same for every tile is worked out once.)
template <int DP>
struct BoxSender {
  static constexpr int kHalves = DP / 64;
  const KvBoxes &x;
  int rows, per_tile;     // of a box; boxes of a tile
  int box, col, to;       // of this lane: the latter in the tile
  bool sends;
  int page, off, first;   // of box first + lane of the session
  bool gap;               // whether one of those has no page

  __device__ __forceinline__ BoxSender(const KvBoxes &boxes) : x(boxes) {
    const int lane = threadIdx.x & 31;
    rows = x.rows;
    per_tile = rows ? kTileRows / rows : 0;
    box = lane / kHalves;
    col = lane % kHalves * 64;
    sends = box < per_tile;
    to = col * (kTileRows * 2) + box * rows * 128;
  }
  __device__ __forceinline__ void reset() { first = INT32_MIN / 2; }
  // Look-ups for a tile of the session; `end`: its slots.
  __device__ __forceinline__ void look_up(const KvCacheArg &c, int b, int tile, int end) {
    const int wanted = tile * per_tile;
    if (wanted < first || wanted + per_tile > first + 32) {
      first = wanted;
      const int slot = (wanted + (int)(threadIdx.x & 31)) * rows;
      page = kNoSlot;
      off = 0;
      if (slot < end) page = kv_page_ok(c, b, kv_page_load(c, b, slot, off));
      gap = __any_sync(~0u, page < 0 && slot < end);
    }
  }
  // Which of the tile's rows 32 i .. 32 i + 31 have a page.
  __device__ __forceinline__ uint32_t present(int tile, int i) const {
    if (!gap) return ~0u;
    const int of = tile * per_tile - first + (i * 32 + (int)(threadIdx.x & 31)) / rows;
    return __ballot_sync(~0u, __shfl_sync(~0u, page, of) >= 0);
  }
  // Sends the tile.  The warp's arrival at its barrier announces the bytes.
  __device__ __forceinline__ void send(int tile, uint32_t dst, uint32_t bar, int head) const {
    const int of = tile * per_tile - first + box;
    const int p = __shfl_sync(~0u, page, of & 31), o = __shfl_sync(~0u, off, of & 31);
    if ((threadIdx.x & 31) == 0) bar_expect(bar, kTileRows * DP * 2);
    __syncwarp();
    if (sends) box_copy(dst + to, x, bar, col, o, head, p);
    __syncwarp();
  }
};

// A copying warp.  Each item (a tile, or the query rows) ends with one arrival
// of the warp at the item's barrier: two items later, when the copies have
// landed and are fenced.
template <typename T, int DP>
struct KvCopier {
  static constexpr int kChunks = DP / 8, kAtOnce = 32 / kChunks;
  int w, lane, head_dim;
  unsigned long long nowhere;    // an address that may be read: copies of nothing want one all the same
  uint32_t waiting[2] = {0, 0};  // barriers of the copies that are still on their way

  __device__ __forceinline__ KvCopier(int warp, int ln, int dim, const void *any)
      : w(warp), lane(ln), head_dim(dim), nowhere(reinterpret_cast<unsigned long long>(any)) {}

  // This warp's 32 rows of 128; lane i knows row i's address, null: zeros.
  __device__ __forceinline__ void rows(uint32_t dst, const T *mine) {
    const int chunk = lane % kChunks, sub = lane / kChunks;
    const bool inside = chunk * 8 < head_dim;
    constexpr int kBatch = 8;
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += kBatch * kAtOnce) {
      unsigned long long src[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; i++)
        src[i] = __shfl_sync(~0u, reinterpret_cast<unsigned long long>(mine), r0 + i * kAtOnce + sub);
#pragma unroll
      for (int i = 0; i < kBatch; i++) {
        const bool there = src[i] != 0 && inside;
        const T *p = reinterpret_cast<const T *>(there ? src[i] + chunk * 16 : nowhere);
        cp_async16(operand_chunk(dst, kTileRows, w * 32 + r0 + i * kAtOnce + sub, chunk), p, there);
      }
    }
  }

  // The item's copies have all been issued; 0: it needs no arrival of them.
  __device__ __forceinline__ void issued(uint32_t bar) {
    cp_commit();
    if (waiting[0]) {
      cp_wait<2>();
      arrive(waiting[0]);
    }
    waiting[0] = waiting[1];
    waiting[1] = bar;
  }
  __device__ __forceinline__ void landed() {  // all of them
    cp_wait<0>();
    for (int i = 0; i < 2; i++)
      if (waiting[i]) arrive(waiting[i]);
    waiting[0] = waiting[1] = 0;
  }
  // Waits for what others do with earlier items: none of those may be held back.
  __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int *dead) {
    if (__all_sync(~0u, bar_try(bar, parity))) return true;
    landed();
    return __all_sync(~0u, bar_wait(bar, parity, dead));
  }
  // Infinities and NaN in this warp's rows of a tile become 0; whether there were any.
  __device__ __forceinline__ bool zero_odd_values(uint32_t tile) {
    bool odd = false;
    __syncwarp();
    for (int i = lane; i < 32 * kChunks; i += 32) {
      const uint32_t a = operand_chunk(tile, kTileRows, w * 32 + i / kChunks, i % kChunks);
      uint32_t x[4];
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                   : "r"(a)
                   : "memory");
      bool bad = false;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        constexpr uint32_t e = KvType<T>::kExponent;
        if ((x[j] & e) == e) x[j] &= 0xFFFF0000u, bad = true;
        if ((x[j] >> 16 & e) == e) x[j] &= 0xFFFFu, bad = true;
      }
      if (bad) {
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3])
                     : "memory");
        odd = true;
      }
    }
    return __any_sync(~0u, odd);
  }
  // After a wait that ran out: boxes on their way may still arrive for a while.
  static __device__ __forceinline__ void give_up() {
    for (int i = 0; i < 1000; i++) __nanosleep(1000);
  }
  __device__ __forceinline__ void arrive(uint32_t bar) {
    fence_to_tensor();
    __syncwarp();
    if (lane == 0) bar_arrive(bar);
  }
};

}  // namespace unison
