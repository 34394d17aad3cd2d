// What the operators over paged caches share: checks of the descriptor, where a block of a page lies.
#pragma once
#include "bass_common.h"

namespace bass {

constexpr int kMaxPagedBatch = 4096;  // sequences, and prefixes, of a plan (its kernel keeps them in LDS)

inline int check_paged(const bass_paged_desc* d) {
  if (!d) return BASS_ERR_INVALID_ARG;
  if (d->B <= 0 || d->kmax <= 0 || d->Hq <= 0 || d->Hkv <= 0 || d->D <= 0 || d->page_tokens <= 0 || d->n_pages <= 0 || d->max_pages <= 0)
    return BASS_ERR_INVALID_ARG;
  if (d->Hq % d->Hkv != 0) return BASS_ERR_INVALID_ARG;
  if (d->dtype != BASS_DTYPE_BF16 && d->dtype != BASS_DTYPE_INT8KV) return BASS_ERR_UNSUPPORTED;
  if ((d->D != 64 && d->D != 128) || d->page_tokens % kBlockTokens != 0) return BASS_ERR_UNSUPPORTED;
  // slots, tokens of a table and blocks of a pool are 32-bit numbers
  if ((int64_t)d->n_pages * d->page_tokens >= (1ll << 31) || (int64_t)d->max_pages * d->page_tokens >= (1ll << 31)) return BASS_ERR_UNSUPPORTED;
  if ((int64_t)d->n_pages * (d->page_tokens / kBlockTokens) * d->Hkv >= (1ll << 31)) return BASS_ERR_UNSUPPORTED;
  return BASS_OK;
}

// Bytes of a block of a pool.
inline size_t page_block_bytes(const bass_paged_desc* d) {
  return d->dtype == BASS_DTYPE_INT8KV ? i8_block_bytes(d->D) : (size_t)kBlockTokens * d->D * 2;
}

// A launch counts its threads in 32 bits; larger ones are refused before anything is enqueued.
inline bool grid_fits(int64_t groups, int threads = 256) { return groups <= ((1ll << 32) - 1) / threads; }

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

#ifdef __HIPCC__
// Block `blk` of kv head `kvh`, counted over the pool's pages (page * blocks per page + block of the page), as the pool has them.
__device__ inline size_t pool_block(int blk, int blocks_per_page, int Hkv, int kvh) {
  const int page = blk / blocks_per_page;
  return ((size_t)page * Hkv + kvh) * blocks_per_page + (blk - page * blocks_per_page);
}
#endif

}  // namespace bass
