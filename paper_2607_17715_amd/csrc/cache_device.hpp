// Device helpers that the growing cache's kernels share: requests of a batch, pages, turns.
#pragma once

#include <type_traits>

#include "cache.hpp"
#include "device.hpp"

namespace c2kv {

constexpr int ST = kSlotTile;

// ----------------------------------------------------------------------------
// requests and their chunks (the index rules are in cache_index.hpp)
// ----------------------------------------------------------------------------

__device__ inline Req request(const ChunkView& c, int b) {
  return clamp_req(c.tok_off[b], c.tok_off[b + 1], c.kv_len[b], c.n_tokens);
}

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ inline Req lane_req(const Req& r, int src) {
  return {uniform(__shfl(r.first, src)), uniform(__shfl(r.n, src)), uniform(__shfl(r.base, src))};
}

// The request whose chunk holds row `token`, searched by a whole wavefront, 64 requests
// a step; -1 if none does.
__device__ inline int find_row(const ChunkView& c, int token, Req& r) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < c.batch; b0 += 64) {
    const int b = b0 + lane;
    const Req mine = request(c, min(b, c.batch - 1));
    const uint64_t hit =
        __ballot(b < c.batch && token >= mine.first && token < mine.first + mine.n);
    if (hit) {
      const int src = __builtin_ctzll(hit);
      r = lane_req(mine, src);
      return b0 + src;
    }
  }
  return -1;
}

// Page of cache index j >= 0 of request b, or -1 where the block table names none.
__device__ inline int page_of(const ChunkView& c, const PageView& p, int b, int j) {
  const int col = j / p.PS;
  if (col >= c.max_pages) return -1;
  return valid_page(c.table[size_t(b) * c.max_pages + col], p.n_pages);
}

// cos and sin of pos positions' turn of a pair: the angle in whole turns is formed and
// reduced in 64 bits (a far position times a frequency loses its fraction in 32), and the
// instructions take it in turns (within 2^-22.9 over [-1/2, 1/2], measured at 2^20 angles, and
// within 2^-22 with the rounding of the reduced angle; a plan's tables are within 2^-25, but that
// takes polynomials in 64 bits, about 25 operations an angle, which have not been tried here).
__device__ inline void turn_cs(int pos, double turns, float& c, float& s) {
  double x = pos * turns;
  x -= __builtin_rint(x);
  const float f = float(x);
  s = __builtin_amdgcn_sinf(f);
  c = __builtin_amdgcn_cosf(f);
}

// Calls f(T, S, D) as tagged types for a cache or pool of type `store`.
template <typename F>
inline hipError_t with_types(int store, int D, F&& f) {
  auto dim = [&](auto t, auto s) {
    return D == 64 ? f(t, s, std::integral_constant<int, 64>{})
                   : f(t, s, std::integral_constant<int, 128>{});
  };
  if (store == C2KV_F32) return dim(float{}, float{});
  if (store == C2KV_BF16) return dim(__bf16{}, __bf16{});
  return dim(__bf16{}, int8_t{});
}

}  // namespace c2kv
