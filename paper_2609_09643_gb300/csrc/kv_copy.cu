// Tensor maps of the paged pools.
#include "kv_copy.cuh"

namespace unison {

namespace {
using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                            const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                            CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
  static const Encode f = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<Encode>(p);
  }();
  return f;
}
}  // namespace

void kv_boxes(KvBoxes &x, const unison_kv_cache &c, const void *pool, int64_t page, int64_t head, int64_t slot,
              int least) {
  x.rows = 0;
  // A box is the largest power of two of slots that divides a page, up to 128: no
  // box lies in two pages, and its rows are whole repeats of the swizzle.
  const int ps = c.page_size, two = ps & -ps;
  const int rows = two >= least ? (two < kTileRows ? two : kTileRows) : 0;
  if (c.n_heads == 1) head = slot * ps;  // an axis of one: its stride means nothing
  x.head_first = head < slot;
  if (c.n_pages == 1) page = x.head_first ? slot * ps : head * c.n_heads;
  if (!rows || c.n_pages < 1 || !encoder()) return;
  const int64_t s1 = x.head_first ? head : slot, s2 = x.head_first ? slot : head;
  const int64_t n1 = x.head_first ? c.n_heads : ps, n2 = x.head_first ? ps : c.n_heads;
  // axes from the inside out, none overlapping the next
  if (s1 < c.head_dim || s2 < s1 * n1 || page < s2 * n2 || page >= (1ll << 38)) return;
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)n1, (cuuint64_t)n2, (cuuint64_t)c.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)s1 * 2, (cuuint64_t)s2 * 2, (cuuint64_t)page * 2};
  const cuuint32_t box[4] = {64, x.head_first ? 1u : (cuuint32_t)rows, x.head_first ? (cuuint32_t)rows : 1u, 1};
  const cuuint32_t each[4] = {1, 1, 1, 1};
  if (encoder()(&x.map, c.dtype == UNISON_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                4, const_cast<void *>(pool), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS)
    x.rows = rows;
}

}  // namespace unison
