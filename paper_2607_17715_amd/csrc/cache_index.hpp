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

// ---- launches -----------------------------------------------------------------------

// Workgroups of 256 threads that a launch can have: it counts its threads in 32 bits.
constexpr int64_t kMostGroups = (1ll << 24) - 1;

// The longest chunk of a batch as far as the host knows: its bound, and where none is given all
// tokens, or one where there are no more of them than requests (a step, most likely).
C2KV_INDEX_FN int longest_chunk(int max_chunk, int n_tokens, int batch) {
  if (max_chunk == 0 && n_tokens <= batch) return 1;
  return max_chunk > 0 && max_chunk < n_tokens ? max_chunk : imax_(n_tokens, 1);
}

// A bound on a batch's chunk_tiles, which is the grid of the tile kernels: a chunk of n tokens
// falls in n / kSlotTile + 2 tiles at most.
C2KV_INDEX_FN int64_t most_chunk_tiles(int64_t n_tokens, int64_t batch) {
  return n_tokens / kSlotTile + 2 * batch;
}
// Workgroups of the row kernel: four (token, kv-head) units each.
C2KV_INDEX_FN int64_t row_groups(int64_t n_tokens, int64_t heads) {
  return (n_tokens * heads + 3) / 4;
}
// Whether a write goes by rows.  A wavefront a (token, kv-head) ends soonest where all of them
// run at once, or where a tile would hold few tokens; else tiles, which write whole lines
// (bf16, 8 heads of 128, rows against tiles: 256 tokens 5.4 | 6.1 us, 512 6.8 | 6.3; 128
// requests of 1 token 5.6 | 11.4, of 8 12.1 | 12.2, of 32 26.9 | 18.2).
C2KV_INDEX_FN bool write_by_rows(int64_t n_tokens, int64_t heads, int max_chunk) {
  return n_tokens * heads <= 2048 ||
         (max_chunk <= 8 && row_groups(n_tokens, heads) <= kMostGroups);
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

// ---- attention work ----------------------------------------------------------------
//
// A unit is a block of `rb` query rows of one (request, kv-head); row r of a request's
// chunk is query head r % G of the kv-head's group at token r / G.  Units are ordered by
// request, kv-head, row block; a unit's work is its key tiles, and the tiles of all units
// in that order are one line that the workgroups of a launch share evenly, each a
// contiguous stretch: whatever the lengths, all finish together.  A unit cut by a border
// is joined afterwards.  Rows (n G) and the line's tiles are below 2^31 (the host refuses
// what could have more), so all of this is 32-bit arithmetic: a 64-bit division takes a
// GPU about half a microsecond.

C2KV_INDEX_FN int row_blocks(const Req& r, unsigned G, unsigned rb) {
  return int((unsigned(r.n) * G + rb - 1) / rb);
}
// The row blocks of a chunk in turn; divides once, not per block.
struct UnitWalk {
  unsigned G, step, step_rest;       // tokens from one block's last row to the next's
  unsigned token, rest;              // of the block's last row, as if all blocks were full
  int base, last, limit;

  C2KV_INDEX_FN UnitWalk(const Req& r, unsigned G_, unsigned rb, int limit_, unsigned i = 0)
      : G(G_), step(rb / G_), step_rest(rb % G_), base(r.base), last(r.n - 1), limit(limit_) {
    const unsigned row = (i + 1) * rb - 1;
    token = row / G;
    rest = row % G;
  }
  C2KV_INDEX_FN void next() {
    token += step;
    rest += step_rest;
    if (rest >= G) {
      rest -= G;
      ++token;
    }
  }
  // keys that exist for the block: what its last token sees
  C2KV_INDEX_FN int keys() const {
    const int t = token < unsigned(last) ? int(token) : last;
    return imin_(imax_(0, base + t + 1), limit);
  }
  // its tiles: at least one, so that rows that see no key are answered as well
  C2KV_INDEX_FN int tiles() const { return imax_(1, (keys() + kSlotTile - 1) / kSlotTile); }
};
C2KV_INDEX_FN int unit_keys(const Req& r, unsigned G, unsigned rb, unsigned i, int limit) {
  return UnitWalk(r, G, rb, limit, i).keys();
}
C2KV_INDEX_FN int unit_tiles(const Req& r, unsigned G, unsigned rb, unsigned i, int limit) {
  return UnitWalk(r, G, rb, limit, i).tiles();
}
// Tiles of all row blocks of one kv-head.
C2KV_INDEX_FN unsigned head_tiles(const Req& r, unsigned G, unsigned rb, int limit) {
  unsigned t = 0;
  UnitWalk u(r, G, rb, limit);
  for (int i = row_blocks(r, G, rb); i > 0; --i, u.next()) t += unsigned(u.tiles());
  return t;
}
// A bound on the line's tiles that the host can form: no block has more than the limit's.
C2KV_INDEX_FN int64_t most_tiles(int64_t n_tokens, int64_t batch, int64_t G, int64_t heads,
                                 int64_t rb, int64_t limit) {
  return heads * (n_tokens * G / rb + batch) * imax_(1, int(limit / kSlotTile));
}

// Shares of `groups` workgroups: the first `more` have one tile more than the others.
struct Shares {
  unsigned total, size, more;
  C2KV_INDEX_FN unsigned begin(unsigned w) const { return size * w + (w < more ? w : more); }
  // workgroup whose share holds tile x
  C2KV_INDEX_FN unsigned of(unsigned x) const {
    const unsigned big = more * (size + 1);
    return x < big ? x / (size + 1) : more + (x - big) / size;
  }
};
C2KV_INDEX_FN Shares make_shares(unsigned total, unsigned groups) {
  return {total, total / groups, total % groups};
}

}  // namespace c2kv
