// Attention of drafted tokens over the paged cache (unison_kv_attend): the
// variant for few query rows, and the join of what both variants split.
//
//   S = scale q . k,  m = max S,  l = sum exp(S - m),  out = sum exp(S - m) v / l
//
// in one pass over the keys: when a tile raises the maximum, l and the sums so
// far are scaled by exp(old m - new m).  Two halves of the keys are joined in
// the same way, so the keys may be shared out at will: the call's key tiles are
// one list, every CTA takes an equal run of it, whatever the sessions' lengths
// are, and a second kernel joins what lies in several runs.
#include "kv_attend.cuh"

namespace unison {
namespace {

constexpr int kThreads = 128;
constexpr int kTile = 64;  // keys of a tile

template <int DP>
constexpr int kAttendStages = DP <= 128 ? 3 : 2;
template <int DP, int MT>
constexpr int kAttendSmem = kAttendStages<DP> *kTile *DP * 4 + MT * 16 * DP * 2;

// Up to 32 query rows per KV head (64 with head sizes above 128, row tile by row
// tile): every key meets too few rows for the products to matter, so memory
// bounds it, and the keys go through shared memory by 16-byte copies, which take
// any page size and stride alike.  The query heads of a KV head share its keys;
// the four warps split the rows (MT) and then a tile's keys.  Reads of one
// tile's rows are planned two tiles ahead of their use: first the page ids (into
// a register), then the rows' addresses (shared memory), then the copies.
// Weights are rounded to the cache's type, as the products' operands have to be;
// their sum l is of the weights before that.  In fp16 they are relative to a
// reference 2^15 below the row's maximum, so that 2^-40 of it still counts.
// One token x 4 heads over 64 sessions of 512 to 32k keys (8 KV heads of 128,
// 2.07 GB): 303 us, 6.8 TB/s; 8 tokens over two sessions of 128k keys (1.07 GB):
// 165 us, 6.5 TB/s; one token of one session of 2,100 keys: 8 us.  Heads of 256
// (16 sessions of 16k keys, 8 KV heads, 2.15 GB): 382 us with 4 or 16 rows, 5.6
// TB/s, 515 with 32, 720 with 64, and 720 more for every 64 rows.
template <typename T, int DP, int MT>
__global__ void __launch_bounds__(kThreads, DP <= 128 ? 2 : 1) attend_kernel(const AttendParams P) {
  follow_last_kernel();
  constexpr int kStages = kAttendStages<DP>;
  constexpr int kRows = MT * 16;
  constexpr int kGroups = 4 / MT;      // groups of warps with keys of their own
  constexpr int kWarpKeys = kTile / kGroups;
  constexpr int kLower = KvType<T>::kMostWeight;
  constexpr int kChunks = DP / 8;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ KvRunShared shared_run;
  __shared__ const T *row_k[2][kTile], *row_v[2][kTile];
  __shared__ uint32_t row_ok[8][2];
  __shared__ float merge_m[4][16], merge_l[4][16];
  __shared__ int odd_values;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int D = P.c.head_dim, H = P.c.n_heads, G = P.group;
  const uint32_t kv_base = smem_u32(smem);
  const uint32_t q_base = kv_base + kStages * kTile * DP * 4;
  if (tid == 0) P.part[blockIdx.x].last = -1;

  auto seq_tiles = [&](int b) -> int64_t {
    const int tokens = kv_tokens(P.t, b, P.c.status).count;
    const int row_tiles = (tokens * G + kRows - 1) / kRows;
    return (int64_t)(attend_key_tiles(kv_length(P.c, b), tokens, kTile) + kSetup) * row_tiles * H;
  };
  KvRun run;
  if (!kv_find_run(run, shared_run, P.c.n_seqs, gridDim.x, blockIdx.x, seq_tiles)) return;
  int b = run.b;
  int64_t at = run.at, seq_begin = run.begin;
  const int64_t end = run.end;

  while (at < end) {
    // ---- the segment that `at` lies in
    int64_t mine = seq_tiles(b);
    while (at >= seq_begin + mine) {
      seq_begin += mine;
      mine = seq_tiles(++b);
    }
    const KvRange tok = kv_tokens(P.t, b, nullptr);
    const int len = kv_length(P.c, b);
    const int key_tiles = attend_key_tiles(len, tok.count, kTile);
    const int row_tiles = (tok.count * G + kRows - 1) / kRows;
    const AttendSpan span = attend_span(at, end, seq_begin, key_tiles);
    const int head = span.seg / row_tiles, row_tile = span.seg % row_tiles;
    const int kt0 = span.kt0, kt1 = span.kt1;
    at = span.begin + kSetup + kt1;
    if (kt0 >= kt1) continue;
    const int rows = min(tok.count * G - row_tile * kRows, kRows);
    const int last_tile = key_tiles - 1;

    __syncthreads();  // the last segment's shared memory is free
    if (tid == 0) odd_values = 0;

    // ---- query rows, zeros behind the last and behind head_dim
    for (int i = tid; i < kRows * kChunks; i += kThreads) {
      const int r = i / kChunks, c = i % kChunks;
      const bool ok = r < rows && c * 8 < D;
      const int row = row_tile * kRows + (ok ? r : 0);
      const T *src = static_cast<const T *>(P.s.q) + (tok.first + row / G) * P.s.q_token +
                     (head * G + row % G) * P.s.q_head + (ok ? c * 8 : 0);
      cp_async16(swizzled<DP>(q_base, r, c), src, ok);
    }
    cp_commit();

    auto find_page = [&](int kt, int &off) -> int {  // threads 0 .. kTile-1
      const int slot = kt * kTile + tid;
      off = 0;
      if (tid >= kTile || kt >= last_tile || slot >= len) return kNoSlot;
      return kv_page_load(P.c, b, slot, off);
    };
    auto put_rows = [&](int kt, int page, int off) {
      if (tid >= kTile) return;
      const T *k = nullptr, *v = nullptr;
      if (kt == last_tile) {
        if (tid < tok.count) {
          k = static_cast<const T *>(P.s.k_new) + (tok.first + tid) * P.s.k_token + head * P.s.k_head;
          v = static_cast<const T *>(P.s.v_new) + (tok.first + tid) * P.s.v_token + head * P.s.v_head;
        }
      } else if ((page = kv_page_ok(P.c, b, page)) >= 0) {
        k = static_cast<const T *>(P.c.k) + page * P.c.k_page + head * P.c.k_head + off * P.c.k_slot;
        v = static_cast<const T *>(P.c.v) + page * P.c.v_page + head * P.c.v_head + off * P.c.v_slot;
      }
      row_k[kt & 1][tid] = k;
      row_v[kt & 1][tid] = v;
      const uint32_t bits = __ballot_sync(~0u, k != nullptr);
      if (lane == 0) row_ok[kt & 7][warp] = bits;
    };
    auto copy_tile = [&](int kt) {
      const uint32_t st = kv_base + ((kt - kt0) % kStages) * (kTile * DP * 4);
#pragma unroll
      for (int i = 0; i < kTile * kChunks / kThreads; i++) {
        const int r = (i * kThreads + tid) / kChunks, c = (i * kThreads + tid) % kChunks;
        const T *k = row_k[kt & 1][r], *v = row_v[kt & 1][r];
        const bool ok = k != nullptr && c * 8 < D;
        cp_async16(swizzled<DP>(st, r, c), ok ? k + c * 8 : static_cast<const T *>(P.s.q), ok);
        cp_async16(swizzled<DP>(st + kTile * DP * 2, r, c), ok ? v + c * 8 : static_cast<const T *>(P.s.q), ok);
      }
    };

    // ---- fill the pipeline
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

    const int rt = warp % MT, kg = warp / MT;
    const int r0 = rt * 16 + (lane >> 2), r1 = r0 + 8;
    auto mask_of = [&](int r) -> uint64_t {
      if (r >= rows) return 0;
      const int node = (row_tile * kRows + r) / G;
      return P.t.mask ? P.t.mask[tok.first + node] : ~0ull >> (63 - node);
    };
    const uint64_t mask0 = mask_of(r0), mask1 = mask_of(r1);

    float o[DP / 8][4];
#pragma unroll
    for (int i = 0; i < DP / 8; i++) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;  // reference (log2 units) and sum
    const float to_log2 = P.s.scale * 1.4426950408889634f;

    for (int kt = kt0; kt < kt1; kt++) {
      cp_wait<kStages - 2>();
      __syncthreads();
      if (kt + kStages - 1 < kt1) copy_tile(kt + kStages - 1);
      cp_commit();
      if (kt + kStages < kt1) put_rows(kt + kStages, page, off);
      page = find_page(kt + kStages + 1, off);

      const uint32_t ks = kv_base + ((kt - kt0) % kStages) * (kTile * DP * 4), vs = ks + kTile * DP * 2;
      if (kt == last_tile) {
        // A new token that a row does not see must not reach it as 0 * inf:
        // such values become 0 here and are put back, row by row, at the end.
        const int first = (kt - kt0) % kStages * (kTile * DP * 2) + kTile * DP;
        uint16_t *v = reinterpret_cast<uint16_t *>(smem) + first;
        bool odd = false;
        for (int i = tid; i < kTile * DP; i += kThreads)
          if ((v[i] & KvType<T>::kExponent) == KvType<T>::kExponent) {
            v[i] = 0;
            odd = true;
          }
        if (odd) odd_values = 1;
        __syncthreads();
      }

      // ---- scores of 16 rows and kWarpKeys keys
      float s[kWarpKeys / 8][4];
#pragma unroll
      for (int i = 0; i < kWarpKeys / 8; i++) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
      for (int d = 0; d < DP / 16; d++) {
        uint32_t a[4];
        ldm4(a, swizzled<DP>(q_base, rt * 16 + (lane & 15), d * 2 + (lane >> 4)));
#pragma unroll
        for (int j = 0; j < kWarpKeys / 16; j++) {
          uint32_t kf[4];
          const int key = kg * kWarpKeys + j * 16 + ((lane >> 4) << 3) + (lane & 7);
          ldm4(kf, swizzled<DP>(ks, key, d * 2 + ((lane >> 3) & 1)));
          mma16816<T>(s[2 * j], a, kf[0], kf[1]);
          mma16816<T>(s[2 * j + 1], a, kf[2], kf[3]);
        }
      }
      const uint64_t there = (uint64_t)row_ok[kt & 7][1] << 32 | row_ok[kt & 7][0];
      const uint64_t see0 = kt == last_tile ? there & mask0 : there, see1 = kt == last_tile ? there & mask1 : there;
      float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
      for (int i = 0; i < kWarpKeys / 8; i++) {
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const int key = kg * kWarpKeys + i * 8 + (lane & 3) * 2 + e;
          s[i][e] = see0 >> key & 1 ? s[i][e] * to_log2 : -INFINITY;
          s[i][2 + e] = see1 >> key & 1 ? s[i][2 + e] * to_log2 : -INFINITY;
          t0 = fmaxf(t0, s[i][e]);
          t1 = fmaxf(t1, s[i][2 + e]);
        }
      }
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) {
        t0 = fmaxf(t0, __shfl_xor_sync(~0u, t0, d));
        t1 = fmaxf(t1, __shfl_xor_sync(~0u, t1, d));
      }
      const float n0 = fmaxf(m0, reference_of<kLower>(t0)), n1 = fmaxf(m1, reference_of<kLower>(t1));
      const float u0 = n0 == -INFINITY ? 0.f : n0, u1 = n1 == -INFINITY ? 0.f : n1;
      const float f0 = exp2_fast(m0 - u0), f1 = exp2_fast(m1 - u1);
      m0 = n0;
      m1 = n1;
      l0 *= f0;
      l1 *= f1;
#pragma unroll
      for (int i = 0; i < DP / 8; i++) {
        o[i][0] *= f0;
        o[i][1] *= f0;
        o[i][2] *= f1;
        o[i][3] *= f1;
      }
      // ---- weights, and their products with the values
#pragma unroll
      for (int j = 0; j < kWarpKeys / 16; j++) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          w[e] = exp2_fast(s[2 * j][e] - (e < 2 ? u0 : u1));
          w[4 + e] = exp2_fast(s[2 * j + 1][e] - (e < 2 ? u0 : u1));
        }
        l0 += (w[0] + w[1]) + (w[4] + w[5]);
        l1 += (w[2] + w[3]) + (w[6] + w[7]);
        const uint32_t a[4] = {KvType<T>::pack(w[0], w[1]), KvType<T>::pack(w[2], w[3]),
                               KvType<T>::pack(w[4], w[5]), KvType<T>::pack(w[6], w[7])};
#pragma unroll
        for (int d = 0; d < DP / 16; d++) {
          uint32_t vf[4];
          const int key = kg * kWarpKeys + j * 16 + (lane & 15);
          ldm4t(vf, swizzled<DP>(vs, key, d * 2 + (lane >> 4)));
          mma16816<T>(o[2 * d], a, vf[0], vf[1]);
          mma16816<T>(o[2 * d + 1], a, vf[2], vf[3]);
        }
      }
    }
    cp_wait<0>();

    // ---- join the warps that had keys of their own
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
      l0 += __shfl_xor_sync(~0u, l0, d);
      l1 += __shfl_xor_sync(~0u, l1, d);
    }
    if ((lane & 3) == 0) {
      merge_m[warp][lane >> 2] = m0;
      merge_m[warp][(lane >> 2) + 8] = m1;
      merge_l[warp][lane >> 2] = l0;
      merge_l[warp][(lane >> 2) + 8] = l1;
    }
    __syncthreads();
    float top0 = m0, top1 = m1;
#pragma unroll
    for (int g = 0; g < kGroups; g++) {
      top0 = fmaxf(top0, merge_m[g * MT + rt][lane >> 2]);
      top1 = fmaxf(top1, merge_m[g * MT + rt][(lane >> 2) + 8]);
    }
    const float f0 = exp2_fast(m0 - (top0 == -INFINITY ? 0.f : top0));
    const float f1 = exp2_fast(m1 - (top1 == -INFINITY ? 0.f : top1));
    float *acc = reinterpret_cast<float *>(smem);  // [kGroups][kRows][DP]: the stages are drained
#pragma unroll
    for (int i = 0; i < DP / 8; i++) {
      float *p0 = acc + ((kg * kRows + r0) * DP + i * 8 + (lane & 3) * 2);
      float *p1 = p0 + 8 * DP;
      p0[0] = o[i][0] * f0;
      p0[1] = o[i][1] * f0;
      p1[0] = o[i][2] * f1;
      p1[1] = o[i][3] * f1;
    }
    __syncthreads();
    const bool whole = kt0 == 0 && kt1 == key_tiles;
    const bool starts = kt0 == 0;
    float *part = P.partial + ((int64_t)blockIdx.x * 2 + (starts ? 1 : 0)) * (kRows * (DP + 2));
    float *part_m = part + kRows * DP, *part_l = part_m + kRows;
    for (int i = tid; i < kRows * (DP / 2); i += kThreads) {
      const int r = i / (DP / 2), d = i % (DP / 2) * 2;
      if (r >= rows || d >= D) continue;
      const int rr = r & 15, ww = r >> 4;
      float top = -INFINITY, l = 0.f, x = 0.f, y = 0.f;
#pragma unroll
      for (int g = 0; g < kGroups; g++) top = fmaxf(top, merge_m[g * MT + ww][rr]);
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int g = 0; g < kGroups; g++) {
        l += merge_l[g * MT + ww][rr] * exp2_fast(merge_m[g * MT + ww][rr] - base);
        x += acc[(g * kRows + r) * DP + d];
        y += acc[(g * kRows + r) * DP + d + 1];
      }
      const int row = row_tile * kRows + r, node = row / G;
      if (kt1 == key_tiles && odd_values) {
        const uint64_t mask =
            (P.t.mask ? P.t.mask[tok.first + node] : ~0ull >> (63 - node)) & (~0ull >> (64 - tok.count));
        for (int j = 0; j < tok.count; j++) {
          if (!(mask >> j & 1)) continue;
          const T *v = static_cast<const T *>(P.s.v_new) + (tok.first + j) * P.s.v_token + head * P.s.v_head + d;
          const float vx = KvType<T>::to_float(v[0]), vy = KvType<T>::to_float(v[1]);
          if (!isfinite(vx)) x += vx;
          if (!isfinite(vy)) y += vy;
        }
      }
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T *dst = static_cast<T *>(P.s.out) + (tok.first + node) * P.s.out_token +
                 (head * G + row % G) * P.s.out_head + d;
        *reinterpret_cast<uint32_t *>(dst) = KvType<T>::pack(x * inv, y * inv);
        if (d == 0 && P.s.lse)
          P.s.lse[(int64_t)(tok.first + node) * P.s.n_q_heads + head * G + row % G] =
              (top + log2f(l)) * 0.6931471805599453f;
      } else {
        *reinterpret_cast<float2 *>(part + r * DP + d) = make_float2(x, y);
        if (d == 0) {
          part_m[r] = top;
          part_l[r] = l;
        }
      }
    }
    if (starts && !whole && tid == 0)
      P.part[blockIdx.x] = {kv_run_of(run, span.begin + kSetup + key_tiles - 1), head, row_tile * kRows, rows,
                            tok.first};
  }
}

// Joins the parts of the segments that lie in several runs, each by the CTAs of
// the run that it begins in.
//   up to kFewParts  a warp for each row: it asks for the parts' statistics and
//                    for the row in all of them at once
//   more             four rows at a time: the parts' statistics become weights in
//                    shared memory, in rounds of kParts; the threads of a row
//                    then add up 16 bytes of it each, from parts of their own
//                    where there are threads to spare
// Bound by its loads' latency: 15 us for 304 parts of 256 rows (40 MB; 27 four
// rows at a time), 6 us after two sessions of 128k keys (19 parts a segment).
constexpr int kJoin = 256;
constexpr int kJoinRows = 4;
constexpr int kParts = 256;
constexpr int kFewParts = 4;


template <typename T, int DP>
__global__ void __launch_bounds__(kJoin) attend_join_kernel(const AttendParams P) {
  follow_last_kernel();
  constexpr int kVec = DP / 4;                            // threads of a row
  constexpr int kShares = kJoin / (kJoinRows * kVec);     // that add up different parts
  __shared__ float weight[kJoinRows][kParts];
  __shared__ float4 sums[kShares][kJoinRows][kVec];
  __shared__ float row_l[kJoinRows], row_top[kJoinRows];
  const AttendPart seg = P.part[blockIdx.x];
  if (seg.last < 0) return;
  const int D = P.c.head_dim, G = P.group, R = P.rows, rows = seg.rows;
  const int step = P.row_groups;  // CTAs from one run to the next
  const int parts = seg.last - (int)blockIdx.x / step + 1;
  const int64_t stride = (int64_t)2 * R * (DP + 2) * step;
  // the first run's part is its second one, the others' is their first
  const float *rest = P.partial + (int64_t)blockIdx.x * 2 * R * (DP + 2);
  const float *first = rest + R * (DP + 2);
  auto part = [&](int p) { return p ? rest + p * stride : first; };

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (parts <= kFewParts) {
    constexpr int kPer = DP / 32;  // elements of a lane
    const int col = lane * kPer;
    for (int row = blockIdx.y * (kJoin / 32) + warp; row < rows; row += gridDim.y * (kJoin / 32)) {
      float m = -INFINITY, l = 0.f, x[kFewParts][kPer], sum[kPer];
      if (lane < parts) {
        const float *q = part(lane) + R * DP + row;
        m = q[0], l = q[R];
      }
#pragma unroll
      for (int p = 0; p < kFewParts; p++) {
        const float2 *q = reinterpret_cast<const float2 *>(part(min(p, parts - 1)) + row * DP + col);
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
          const float2 y = p < parts && col < D ? q[i / 2] : make_float2(0.f, 0.f);
          x[p][i] = y.x, x[p][i + 1] = y.y;
        }
      }
      float top = m;
#pragma unroll
      for (int d = kFewParts / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
      top = __shfl_sync(~0u, top, 0);
      const float f = exp2_fast(m - (top == -INFINITY ? 0.f : top));
      l *= f;
#pragma unroll
      for (int d = kFewParts / 2; d; d >>= 1) l += __shfl_xor_sync(~0u, l, d);
      l = __shfl_sync(~0u, l, 0);
#pragma unroll
      for (int i = 0; i < kPer; i++) sum[i] = 0.f;
#pragma unroll
      for (int p = 0; p < kFewParts; p++) {
        const float w = __shfl_sync(~0u, f, p);
#pragma unroll
        for (int i = 0; i < kPer; i++) sum[i] += x[p][i] * w;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int at = seg.first_row + row, head = seg.head * G + at % G;
      const int64_t token = seg.token + at / G;
      T *dst = static_cast<T *>(P.s.out) + token * P.s.out_token + head * P.s.out_head + col;
#pragma unroll
      for (int i = 0; i < kPer; i += 2)
        if (col < D) reinterpret_cast<uint32_t *>(dst)[i / 2] = KvType<T>::pack(sum[i] * inv, sum[i + 1] * inv);
      if (lane == 0 && P.s.lse)
        P.s.lse[token * P.s.n_q_heads + head] = (top + log2f(l)) * 0.6931471805599453f;
    }
    return;
  }
  const int row = threadIdx.x / kVec % kJoinRows, share = threadIdx.x / (kVec * kJoinRows),
            col = threadIdx.x % kVec * 4;
  for (int row0 = blockIdx.y * kJoinRows; row0 < rows; row0 += gridDim.y * kJoinRows) {
    float top = -INFINITY, l = 0.f, one_m = -INFINITY, one_l = 0.f;
    const bool weighs = warp < kJoinRows && row0 + warp < rows;
    if (weighs) {
      const float *q = part(lane) + R * DP + row0 + warp;
      if (lane < parts) one_m = q[0], one_l = q[R];  // (all there is, mostly)
      top = one_m;
      for (int p = lane + 32; p < parts; p += 32) top = fmaxf(top, part(p)[R * DP + row0 + warp]);
#pragma unroll
      for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    }
    const float base = top == -INFINITY ? 0.f : top;
    float4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < parts; p0 += kParts) {
      const int n = min(parts - p0, kParts);
      __syncthreads();
      if (weighs)
        for (int p = lane; p < n; p += 32) {
          const float *q = part(p0 + p) + R * DP + row0 + warp;
          const bool first = p0 + p < 32;
          const float f = exp2_fast((first ? one_m : q[0]) - base);
          weight[warp][p] = f;
          l += (first ? one_l : q[R]) * f;
        }
      __syncthreads();
      if (row0 + row < rows && col < D)
#pragma unroll 8
        for (int p = share; p < n; p += kShares) {
          const float4 x = *reinterpret_cast<const float4 *>(part(p0 + p) + (row0 + row) * DP + col);
          const float f = weight[row][p];
          sum.x += x.x * f, sum.y += x.y * f, sum.z += x.z * f, sum.w += x.w * f;
        }
    }
    if (warp < kJoinRows) {
#pragma unroll
      for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(~0u, l, d);
      if (lane == 0) row_l[warp] = l, row_top[warp] = top;
    }
    sums[share][row][col / 4] = sum;
    __syncthreads();
    if (share == 0 && row0 + row < rows && col < D) {
#pragma unroll
      for (int s = 1; s < kShares; s++) {
        const float4 x = sums[s][row][col / 4];
        sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
      }
      l = row_l[row];
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int at = seg.first_row + row0 + row, head = seg.head * G + at % G;
      const int64_t token = seg.token + at / G;
      T *dst = static_cast<T *>(P.s.out) + token * P.s.out_token + head * P.s.out_head + col;
      *reinterpret_cast<uint2 *>(dst) =
          make_uint2(KvType<T>::pack(sum.x * inv, sum.y * inv), KvType<T>::pack(sum.z * inv, sum.w * inv));
      if (col == 0 && P.s.lse)
        P.s.lse[token * P.s.n_q_heads + head] = (row_top[row] + log2f(l)) * 0.6931471805599453f;
    }
  }
}

struct AttendPlan {
  int dp, rows, row_groups, grid;
  bool tc;
  uint64_t bytes;
};

// Variants, by the query rows per KV head (16 sessions of 16k keys, 8 KV heads):
//   up to 32 the one above: 175 us for 32 rows of 128 elements (the other one:
//            186), 113 of 64 (148)
//   more     tensor cores with sums in tensor memory: 182 us for 48 rows of 128
//            (342 here, row tile by row tile), 124 of 64 (158); 187 and 126 for 128
// Head sizes above 128 do not fit the latter's tensor memory.
AttendPlan attend_plan(int head_dim, int max_rows) {
  AttendPlan p;
  p.dp = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256;
  p.tc = max_rows > 32 && p.dp <= 128;
  p.rows = p.tc ? kTcRows : max_rows <= 16 ? 16 : max_rows <= 32 ? 32 : 64;
  // CTAs that go through the same keys with row tiles of their own
  p.row_groups = p.tc ? min((max_rows + kTcRows - 1) / kTcRows, 4) : 1;
  p.grid = p.tc ? kv_sm_count() / p.row_groups * p.row_groups : kv_sm_count() * (p.dp <= 128 ? 2 : 1);
  p.bytes = (uint64_t)p.grid * (2 * p.rows * (p.dp + 2) * 4 + sizeof(AttendPart));
  return p;
}

template <typename T, int DP>
int attend_join(const AttendParams &p, const AttendPlan &plan, int max_rows, void *stream) {
  const int rounds = (min(max_rows, plan.rows) + kJoinRows - 1) / kJoinRows;
  return kv_launch("kv_attend_join", dim3(plan.grid, min(rounds, plan.tc ? 16 : 8)), dim3(kJoin), 0, stream, 1,
                   attend_join_kernel<T, DP>, p);
}

template <typename T, int DP, int MT>
int attend_run(const AttendParams &p, const AttendPlan &plan, void *stream) {
  static uint64_t done = 0;
  constexpr int smem = kAttendSmem<DP, MT>;
  if (!kv_allow_smem(reinterpret_cast<const void *>(attend_kernel<T, DP, MT>), smem, &done)) return UNISON_ERR_CUDA;
  return kv_launch("kv_attend", dim3(plan.grid), dim3(kThreads), smem, stream, 1, attend_kernel<T, DP, MT>, p);
}

template <typename T, int DP>
int attend_rows(const AttendParams &p, const AttendPlan &plan, int max_rows, void *stream) {
  int rc;
  if constexpr (DP <= 128) {
    if (plan.tc) {
      rc = attend_tc<T, DP>(p, plan.grid, stream);
      return rc == UNISON_OK ? attend_join<T, DP>(p, plan, max_rows, stream) : rc;
    }
  }
  constexpr int kMostTiles = DP <= 128 ? 2 : 4;  // of 16 rows
  rc = plan.rows == 16   ? attend_run<T, DP, 1>(p, plan, stream)
       : plan.rows == 32 ? attend_run<T, DP, 2>(p, plan, stream)
                         : attend_run<T, DP, kMostTiles>(p, plan, stream);
  return rc == UNISON_OK ? attend_join<T, DP>(p, plan, max_rows, stream) : rc;
}

template <typename T>
int attend_pick(const AttendParams &p, const AttendPlan &plan, int max_rows, void *stream) {
  return plan.dp == 64    ? attend_rows<T, 64>(p, plan, max_rows, stream)
         : plan.dp == 128 ? attend_rows<T, 128>(p, plan, max_rows, stream)
                          : attend_rows<T, 256>(p, plan, max_rows, stream);
}

}  // namespace

int kv_sm_count() {
  static int count[64];  // 0: not asked yet; every thread would store the same
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return 1;
  }
  int n = __atomic_load_n(&count[dev], __ATOMIC_RELAXED);
  if (n) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return 1;
  }
  __atomic_store_n(&count[dev], n, __ATOMIC_RELAXED);
  return n;
}

bool kv_allow_smem(const void *kernel, int bytes, uint64_t *done) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return false;
  }
  if (__atomic_load_n(done, __ATOMIC_RELAXED) >> dev & 1) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  __atomic_fetch_or(done, 1ull << dev, __ATOMIC_RELAXED);
  return true;
}

}  // namespace unison

using namespace unison;

static int attend_check(const unison_kv_cache *c, const unison_kv_tree *t, int n_q_heads) {
  int rc = kv_check_cache(c);
  if (rc == UNISON_OK) rc = kv_check_tree(t, c->n_seqs);
  if (rc != UNISON_OK) return rc;
  if (n_q_heads < 1 || n_q_heads % c->n_heads || n_q_heads / c->n_heads > 64) return UNISON_ERR_RANGE;
  return UNISON_OK;
}

extern "C" uint64_t unison_kv_attend_workspace(const unison_kv_cache *cache, const unison_kv_tree *tree,
                                               int n_q_heads) {
  if (attend_check(cache, tree, n_q_heads) != UNISON_OK) return 0;
  return attend_plan(cache->head_dim, tree->max_tokens * (n_q_heads / cache->n_heads)).bytes;
}

extern "C" int unison_kv_attend(const unison_kv_cache *cache, const unison_kv_tree *tree, const unison_kv_step *step,
                                void *workspace, uint64_t workspace_bytes, void *cuda_stream) {
  if (!step) return UNISON_ERR_ARG;
  const int rc = attend_check(cache, tree, step->n_q_heads);
  if (rc != UNISON_OK) return rc;
  if (cache->n_seqs == 0 || tree->n_tokens == 0) return UNISON_OK;
  if (!kv_rows_ok(step->q, step->q_token, step->q_head) || !kv_rows_ok(step->k_new, step->k_token, step->k_head) ||
      !kv_rows_ok(step->v_new, step->v_token, step->v_head) || !kv_rows_ok(step->out, step->out_token, step->out_head))
    return UNISON_ERR_ARG;
  if (cache->max_pages > 0 && cache->n_pages > 0 &&
      (!kv_rows_ok(cache->k, cache->k_page | cache->k_head, cache->k_slot) ||
       !kv_rows_ok(cache->v, cache->v_page | cache->v_head, cache->v_slot)))
    return UNISON_ERR_ARG;
  AttendParams p;
  p.c = *cache;
  p.t = *tree;
  p.s = *step;
  p.group = step->n_q_heads / cache->n_heads;
  const AttendPlan plan = attend_plan(cache->head_dim, tree->max_tokens * p.group);
  if (!workspace || !kv_aligned(workspace, 16) || workspace_bytes < plan.bytes) return UNISON_ERR_ARG;
  p.rows = plan.rows;
  p.row_groups = plan.row_groups;
  p.part = static_cast<AttendPart *>(workspace);
  p.partial = reinterpret_cast<float *>(p.part + plan.grid);
  return cache->dtype == UNISON_KV_BF16 ? attend_pick<__nv_bfloat16>(p, plan, tree->max_tokens * p.group, cuda_stream)
                                        : attend_pick<__half>(p, plan, tree->max_tokens * p.group, cuda_stream);
}
