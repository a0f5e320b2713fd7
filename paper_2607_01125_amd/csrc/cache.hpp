// What the kernels of the paged 8-bit key/value cache share (zoact_cache.h).
#pragma once
#include "common.hpp"
#include "zoact_cache.h"

namespace zoact {

constexpr int kPage = ZOACT_CACHE_PAGE, kBlock = ZOACT_CACHE_BLOCK, kPageBlocks = kPage / kBlock;

// One entry of a batch as a workgroup sees it.  rows_ok: its rows lie in the buffers; ok: its
// places lie in the cache too.
struct CacheEntry {
  int row0, count, slot, pos;
  bool rows_ok, ok;
};

__device__ __forceinline__ void raise_status(uint32_t* status, uint32_t bit) {
  if (status) atomicOr(status, bit);
}

// (Loads do not wait for one another: where there is no list, a word of pos is read and dropped.)
__device__ __forceinline__ void entry_rows(const zoact_cache_batch& b, int i, CacheEntry& e) {
  const int32_t* const rows = (b.row_begin ? b.row_begin : b.pos) + i;
  const int32_t* const slot = (b.slots ? b.slots : b.pos) + i;
  const int32_t v0 = rows[0], v1 = rows[b.row_begin ? 1 : 0], s = *slot, p = b.pos[i];
  const int64_t r0 = b.row_begin ? v0 : (int64_t)i * b.max_new;
  const int64_t r1 = b.row_begin ? v1 : r0 + b.max_new;
  e.pos = p;
  e.row0 = (int)r0;
  e.count = (int)(r1 - r0);
  e.rows_ok = r0 >= 0 && r1 >= r0 && r1 <= b.rows && r1 - r0 <= b.max_new;
  if (!e.rows_ok) e.count = 0;
  e.slot = b.slots ? s : i;
}

// Entry i with the place extend gave it.  A bad one raises the status bit once (by `report`).
__device__ __forceinline__ CacheEntry read_entry(const zoact_cache& c, const zoact_cache_batch& b, int i, bool report) {
  CacheEntry e;
  entry_rows(b, i, e);
  const bool fits = e.rows_ok && e.slot >= 0 && e.slot < c.n_slots &&
                    (int64_t)e.pos + e.count <= (int64_t)c.max_pages * kPage;
  e.ok = fits && e.pos >= 0;
  if (report && e.pos >= 0 && !fits) raise_status(b.status, ZOACT_STATUS_BAD_ENTRY);
  return e;
}

// Host checks shared by the entry points.
zoact_status check_cache(const zoact_cache* c);
zoact_status check_batch(const zoact_cache_batch* b, const zoact_cache* c);

}  // namespace zoact
