// Index rules of the growing paged cache: which rows and cache slots a call touches, for
// any contents of the device arrays.  Plain functions of integers, so that the host can
// check them (tests/cache_index.cpp).
#pragma once

#include <cstdint>

#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#define C2KV_INDEX_FN __host__ __device__ inline
#else
#define C2KV_INDEX_FN inline
#endif

namespace c2kv {

constexpr int kSlotTile = 64;   // cache slots of one tile; a page holds whole tiles

C2KV_INDEX_FN int imin_(int a, int b) { return a < b ? a : b; }
C2KV_INDEX_FN int imax_(int a, int b) { return a > b ? a : b; }

// One request's chunk: rows [first, first + n) of the chunk tensors; its row t is cache
// index base + t (negative where the chunk is longer than the cache's stated length).
struct Req {
  int first, n, base;
};

// From two neighbouring offsets and a length, whatever they hold: the rows lie in
// [0, n_tokens), base + n is the length (at least 0).
C2KV_INDEX_FN Req clamp_req(int o0, int o1, int len, int n_tokens) {
  Req r;
  r.first = imin_(imax_(o0, 0), n_tokens);
  r.n = imin_(imax_(o1, r.first), n_tokens) - r.first;
  r.base = imax_(len, 0) - r.n;
  return r;
}

// Cache tiles that a chunk's tokens fall in, [t0, t0 + n) of its request, within the
// `limit` tokens that a block-table row names (a multiple of kSlotTile).
struct Tiles {
  int t0, n;
};
C2KV_INDEX_FN Tiles chunk_tiles(const Req& r, int limit) {
  const int lo = imax_(r.base, 0);
  const int hi = imin_(r.base + r.n, limit);
  if (hi <= lo) return {0, 0};
  return {lo / kSlotTile, (hi - 1) / kSlotTile - lo / kSlotTile + 1};
}

// Slots [lo, hi) of a tile of chunk_tiles belong to the chunk; slot s is row row0 + s.
struct TileSlots {
  int lo, hi, row0;
};
C2KV_INDEX_FN TileSlots tile_slots(const Req& r, int tile) {
  const int s0 = tile * kSlotTile;
  return {imax_(r.base - s0, 0), imin_(r.base + r.n - s0, kSlotTile), r.first + s0 - r.base};
}

// A block-table entry, or -1 where it names no page.
C2KV_INDEX_FN int valid_page(int id, int n_pages) {
  return unsigned(id) < unsigned(n_pages) ? id : -1;
}

}  // namespace c2kv
