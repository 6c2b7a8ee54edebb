// A paged cache as the kernels that write, read and shorten it see it: addresses of rows, and the checks of what only the
// device knows (lengths, block tables).
#pragma once
#include <stdint.h>

#include "host_common.h"
#include "sm100.cuh"

namespace msd {

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31 by a multiplication (T. Granlund, P. L. Montgomery, Division by invariant integers using multiplication,
// PLDI 1994): with s = ceil(log2 d) and m' = 2^32 + m = floor(2^(32 + s) / d) + 1, m' d lies between 2^(32 + s) + 1 and 2^(32 + s) + 2^s, which is near enough for
// n / d = floor(m' n / 2^(32 + s)) = (mulhi(n, m) + n) >> s (the sum stays below 2^32).
struct FastDiv {
  uint32_t d, mul, shift;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while ((uint64_t{1} << s) < d) ++s;
  return {d, static_cast<uint32_t>(((uint64_t{1} << 32) * ((uint64_t{1} << s) - d)) / d + 1), s};
}
__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) { return (__umulhi(n, f.mul) + n) >> f.shift; }

// Rows of one tensor of the cache (keys, values or their scales): byte strides of blocks, tokens of a block, and heads.
struct PagedRows {
  uint8_t* base;
  int64_t block, token, head;
};
struct PagedCache {
  PagedRows k, v, ks, vs;
  FastDiv page;
  int64_t num_blocks;
  int Hkv, D, Dv;
};

// Whether the rows of a head start less than `most` bytes from one another.
inline bool rows_within(const PagedRows& r, int64_t blocks, int64_t page, int64_t most) {
  return static_cast<__int128>(blocks - 1) * r.block + static_cast<__int128>(page - 1) * r.token < most;
}

__device__ __forceinline__ int64_t row_offset(const PagedRows& r, int32_t blk, uint32_t slot) { return blk * r.block + slot * r.token; }

// Fills in the device's view; MSD_OK or why the cache is refused.
inline msd_status_t paged_cache_view(const msd_paged_cache_t* c, PagedCache* out) {
  if (!c) return MSD_ERR_NULL_POINTER;
  if (c->type != MSD_CACHE_BF16 && c->type != MSD_CACHE_INT8) return MSD_ERR_UNSUPPORTED;
  const bool int8 = c->type == MSD_CACHE_INT8;
  const int es = int8 ? 1 : 2, vec = 16 / es;
  if (c->num_blocks < 1 || c->num_blocks > 0x7FFFFFFF || c->page_size < 1 || c->page_size > 65536 || c->Hkv < 1 || c->Hkv > 65536 || c->D < 1 ||
      c->Dv < 1 || c->D % vec != 0 || c->Dv % vec != 0)
    return MSD_ERR_BAD_SHAPE;
  if (c->D > 256 || c->Dv > 256) return MSD_ERR_UNSUPPORTED;
  if (!c->k || !c->v || (int8 && (!c->k_scale || !c->v_scale))) return MSD_ERR_NULL_POINTER;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return MSD_ERR_BAD_ALIGNMENT;
  if (int8 && (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))) return MSD_ERR_BAD_ALIGNMENT;
  for (int i = 0; i < 3; ++i) {
    if (c->k_stride[i] < 0 || c->v_stride[i] < 0) return MSD_ERR_BAD_SHAPE;
    if (c->k_stride[i] % vec != 0 || c->v_stride[i] % vec != 0) return MSD_ERR_BAD_ALIGNMENT;
    if (int8 && (c->k_scale_stride[i] < 0 || c->v_scale_stride[i] < 0)) return MSD_ERR_BAD_SHAPE;
  }
  out->k = {static_cast<uint8_t*>(c->k), c->k_stride[0] * es, c->k_stride[1] * es, c->k_stride[2] * es};
  out->v = {static_cast<uint8_t*>(c->v), c->v_stride[0] * es, c->v_stride[1] * es, c->v_stride[2] * es};
  out->ks = out->vs = {nullptr, 0, 0, 0};
  if (int8) {
    out->ks = {reinterpret_cast<uint8_t*>(c->k_scale), c->k_scale_stride[0] * 4, c->k_scale_stride[1] * 4, c->k_scale_stride[2] * 4};
    out->vs = {reinterpret_cast<uint8_t*>(c->v_scale), c->v_scale_stride[0] * 4, c->v_scale_stride[1] * 4, c->v_scale_stride[2] * 4};
  }
  out->page = fast_div(static_cast<uint32_t>(c->page_size));
  out->num_blocks = c->num_blocks;
  out->Hkv = c->Hkv;
  out->D = c->D;
  out->Dv = c->Dv;
  return MSD_OK;
}

}  // namespace msd
