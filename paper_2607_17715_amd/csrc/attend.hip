// Attention of chunks of new tokens over a growing paged cache, for gfx950 (CDNA4).
//
//   attend_narrow_kernel   one token a unit: every wavefront reads its own keys straight
//                          into MFMA operands
//   attend_wide_kernel     blocks of 128 or 256 query rows: tiles in LDS, shared by the
//                          wavefronts
//   join_kernel            log-sum-exp combine of units that lie in several workgroups
//
// The work of a launch is one line of key tiles (cache_index.hpp), shared evenly by its
// workgroups on the device, where the lengths are.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <utility>

#include "cache.hpp"
#include "cache_device.hpp"

namespace c2kv {

namespace {

typedef float f32x4 __attribute__((__vector_size__(4 * sizeof(float))));
typedef uint32_t u32x4 __attribute__((__vector_size__(4 * sizeof(uint32_t))));

// ----------------------------------------------------------------------------
// a workgroup's share of the line of tiles
// ----------------------------------------------------------------------------

// Inclusive sums over the lanes of a wavefront, by lane moves inside the VALU.  Sums that
// pass 2^32 stay at its end: lengths and offsets may be anything.
__device__ inline unsigned add_sat(unsigned x, unsigned y) {
  return __builtin_elementwise_add_sat(x, y);
}
template <int CTRL, int ROWS>
__device__ inline unsigned add_from(unsigned x) {
  return add_sat(x, unsigned(__builtin_amdgcn_update_dpp(0, int(x), CTRL, ROWS, 0xf, false)));
}
__device__ inline unsigned wave_scan(unsigned x) {
  x = add_from<0x111, 0xf>(x);               // from the lane 1, 2, 4, 8 before, in rows of 16
  x = add_from<0x112, 0xf>(x);
  x = add_from<0x114, 0xf>(x);
  x = add_from<0x118, 0xf>(x);
  x = add_from<0x142, 0xa>(x);               // a row's last lane to the row after it,
  return add_from<0x143, 0xc>(x);            // and lane 31's to the upper half
}

// Where a workgroup is on the line: row block i of (request b, kv-head g), the unit's
// tiles, and the tile at which the workgroup enters it.
struct Place {
  Req r;
  int b, g, i, tiles, tile;
};

// This workgroup's share [p0, p1) of the line and the place of its first tile, the same in
// every wavefront.  A short line goes to as many workgroups as it has tiles, the others get
// an empty share: a block's tiles one after another take longer than their join (128 tokens
// over 100, 32 heads, blocks of 256 rows: 23.4 us in shares of at least two tiles, 15.3 in
// shares of one, the join 7.1 either way; single tokens of three requests, int8, 14.4 us in
// shares of at least four, 10.3; 17 fp32 tokens over two caches 17.6 and 13.2).
struct Share {
  Shares all;
  unsigned p0, p1;
};

// head_tiles of a request that all lanes name, its row blocks dealt to the lanes.
__device__ inline unsigned head_tiles_wave(const Req& r, unsigned G, int rb, int limit) {
  const int lane = threadIdx.x & 63, n = row_blocks(r, G, rb);
  unsigned t = 0;
  for (int i = lane; i < n; i += 64) t += unsigned(unit_tiles(r, G, rb, i, limit));
  return unsigned(__builtin_amdgcn_readlane(int(wave_scan(t)), 63));
}
// The row block of r in which tile `rest` of a kv-head lies; rest becomes the tile in it.
__device__ inline int find_block(const Req& r, unsigned G, int rb, int limit, unsigned& rest,
                                 int& tiles) {
  const int lane = threadIdx.x & 63, n = row_blocks(r, G, rb);
  for (int i0 = 0; i0 < n; i0 += 64) {
    const unsigned t = i0 + lane < n ? unsigned(unit_tiles(r, G, rb, i0 + lane, limit)) : 0;
    const unsigned incl = wave_scan(t);
    const unsigned here = unsigned(__builtin_amdgcn_readlane(int(incl), 63));
    if (rest < here) {
      const int src = __builtin_ctzll(__ballot(incl > rest));
      tiles = __builtin_amdgcn_readlane(int(t), src);
      rest -= unsigned(__builtin_amdgcn_readlane(int(incl - t), src));
      return i0 + src;
    }
    rest -= here;
  }
  tiles = 1;                                 // (not reached: rest is below head_tiles)
  return max(n - 1, 0);
}

__device__ inline Share find_share(const AttendParams& a, int w, int rb, int limit, Place& at) {
  const int lane = threadIdx.x & 63;
  Share s{};
  Req mine{};
  unsigned head = 0, cost = 0, incl = 0;
  auto step = [&](int b0) {
    const int b = b0 + lane;
    mine = request(a.ch, min(b, a.ch.batch - 1));
    // row blocks lane by lane, a request each; few requests of many blocks one by one, their
    // blocks dealt to the lanes (one of 64: 6000 cycles against 400)
    const int blocks = b < a.ch.batch ? row_blocks(mine, a.G, rb) : 0;
    uint64_t some = __ballot(blocks > 0);
    if (__any(blocks > 4 * __builtin_popcountll(some))) {
      head = 0;
      for (; some; some &= some - 1) {
        const int src = __builtin_ctzll(some);
        const Req r = {__builtin_amdgcn_readlane(mine.first, src),
                       __builtin_amdgcn_readlane(mine.n, src),
                       __builtin_amdgcn_readlane(mine.base, src)};
        const unsigned t = head_tiles_wave(r, a.G, rb, limit);
        if (lane == src) head = t;
      }
    } else {
      head = blocks > 0 ? head_tiles(mine, a.G, rb, limit) : 0;
    }
    cost = head * a.pg.Hkv;
    incl = wave_scan(cost);
    return unsigned(__builtin_amdgcn_readlane(int(incl), 63));
  };
  unsigned total = 0;
  for (int b0 = 0; b0 < a.ch.batch; b0 += 64) total = add_sat(total, step(b0));
  // (2^31 tiles cannot be where no two requests share a row)
  if (total == 0 || total >= 1u << 31) return s;
  s.all = make_shares(total, min(total, gridDim.x));
  if (unsigned(w) >= total) return s;
  s.p0 = s.all.begin(w);
  s.p1 = s.all.begin(w + 1);
  unsigned seen = 0;
  for (int b0 = 0; b0 < a.ch.batch; b0 += 64) {
    const unsigned here = a.ch.batch > 64 ? step(b0) : total;
    if (s.p0 - seen < here) {
      const int src = __builtin_ctzll(__ballot(incl > s.p0 - seen));
      auto of = [&](unsigned x) { return unsigned(__builtin_amdgcn_readlane(int(x), src)); };
      at.r = {int(of(mine.first)), int(of(mine.n)), int(of(mine.base))};
      at.b = b0 + src;
      unsigned rest = s.p0 - seen - (of(incl) - of(cost));
      at.g = int(rest / of(head));
      rest -= at.g * of(head);
      at.i = find_block(at.r, a.G, rb, limit, rest, at.tiles);
      at.tile = int(rest);
      return s;
    }
    seen += here;
  }
  return s;
}

// The unit after `at`, entered at its first tile.
__device__ inline void next_unit(const AttendParams& a, int rb, int limit, Place& at) {
  if (++at.i >= row_blocks(at.r, a.G, rb)) {
    at.i = 0;
    if (++at.g >= a.pg.Hkv) {
      at.g = 0;
      do {
        ++at.b;
        const Req r = request(a.ch, at.b);
        at.r = {uniform(r.first), uniform(r.n), uniform(r.base)};
      } while (at.r.n == 0);
    }
  }
  at.tiles = unit_tiles(at.r, a.G, rb, at.i, limit);
  at.tile = 0;
}

// The tiles [t0, t1) of a unit that a workgroup works on.
struct Piece {
  Req r;
  int b, g, t0, t1, tiles, keys, row0, nrows;
  __device__ Piece(const AttendParams& a, int rb, int limit, const Place& at, unsigned left)
      : r(at.r), b(at.b), g(at.g), t0(at.tile),
        t1(int(min(unsigned(at.tiles), at.tile + left))), tiles(at.tiles),
        keys(unit_keys(at.r, a.G, rb, at.i, limit)), row0(at.i * rb),
        nrows(min(rb, at.r.n * a.G - at.i * rb)) {}
  __device__ bool begins() const { return t0 == 0; }
  __device__ bool ends() const { return t1 == tiles; }
  // the join of a unit that begins in this workgroup, whose share ends (at p1) inside it
  __device__ Join cut(const Share& s) const {
    Join j{};
    j.first = r.first;
    j.row0 = row0;
    j.nrows = nrows;
    j.g = g;
    j.last = int(s.all.of(s.p1 + unsigned(tiles - t1) - 1));
    return j;
  }
};

// ----------------------------------------------------------------------------
// rows
// ----------------------------------------------------------------------------

// Turns per position of the pairs, from the kernel's arguments into LDS.
template <int D>
__device__ inline void stage_turns(const AttendParams& a, double* turns) {
  if (threadIdx.x < D / 2) turns[threadIdx.x] = a.rope.turns[threadIdx.x];
}

// Two chunks of N elements of a query row that RoPE pairs, D / 2 apart, turned to pos and
// scaled in fp32.
template <int N>
__device__ inline void turn_chunks(const double* turns, bool on, int pos, float scale,
                                   float (&x)[N], float (&y)[N]) {
  if (on) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float c, s;
      turn_cs(pos, turns[e], c, s);
      rotate_pair(x[e], y[e], c, s);
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    x[e] *= scale;
    y[e] *= scale;
  }
}

__device__ inline bf16x8 bf16_of(const float (&x)[8]) {
  const uint4 u = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                             pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  return __builtin_bit_cast(bf16x8, u);
}
// x as two bf16 numbers, within 2^-16 of itself.  The first is cut short and the second is what
// that leaves and 2^-24 of the first, so that it has the first's sign and is never zero beside it
// (of 2^-100 and more): an infinite key element then gives the one infinity that a single number
// gives, not the NaN of infinity times zero or of two infinities of opposite sign.  An infinity
// stands in both.
__device__ inline void split_bf16(const float (&x)[8], bf16x8& hi, bf16x8& rest) {
  constexpr float most = 0x1.fffffep127f;
  uint32_t w[4];
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float h = __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
    r[e] = __builtin_fmaf(-__builtin_amdgcn_fmed3f(h, -most, most), 1.f - 0x1p-24f, x[e]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]),
                                 0x07060302u);
  hi = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
  rest = bf16_of(r);
}
__device__ inline bf16x8 bf16_of_i8(uint32_t w0, uint32_t w1) {
  const uint32_t w[2] = {w0, w1};
  float x[8];
  raw_to_f8<int8_t>(w, x);
  return bf16_of(x);                       // exact: codes have seven bits
}

// every wavefront, with its LDS accesses done but its loads still in flight
__device__ inline void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// values of the 16 lanes of this lane's group (DPP operands of what uses them)
template <int... K>
__device__ inline void lanes16(float x, float (&v)[16], std::integer_sequence<int, K...>) {
  ((v[K] = __uint_as_float(__builtin_amdgcn_update_dpp(0, int(__float_as_uint(x)), 0x150 + K,
                                                       0xf, 0xf, true))), ...);
}

// Values that are not finite, in tiles where some rows see a key and others do not: a
// probability of zero times an infinity would put a NaN into rows that must not know of it.
// Such elements are taken out of the product, and what they add to the rows that do see them
// comes from products of the same probabilities with where they are: an infinity, or, where
// both signs meet (a NaN counts as both), a NaN.
//
// Class of element i of 16 bytes: bit 2 i: +inf or NaN, bit 2 i + 1: -inf or NaN.  (Whole
// numbers throughout: conditions would be lane masks, which the kernels' loops have no
// scalar registers for.)
template <typename T>
__device__ inline uint32_t not_finite(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t cls = 0;
#pragma unroll
  for (int i = 0; i < 16 / int(sizeof(T)); ++i) {
    const uint32_t u = sizeof(T) == 4 ? w[i] : (i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    const uint32_t m = u & 0x7fffffffu, nan = (m + 0x007fffffu) >> 31, minus = u >> 31;
    const uint32_t odd = (m + 0x00800000u) >> 31;
    cls |= (odd & (nan | (minus ^ 1u))) << (2 * i) | (odd & (nan | minus)) << (2 * i + 1);
  }
  return cls;
}
// Nonzero if 16 bytes hold any: an exponent of all ones carries into the sign's place.
template <typename T>
__device__ inline uint32_t any_not_finite(const uint4& x) {
  constexpr uint32_t exps = sizeof(T) == 4 ? 0x7f800000u : 0x7f807f80u;
  constexpr uint32_t one = sizeof(T) == 4 ? 0x00800000u : 0x00800080u;
  return (((x.x & exps) + one) | ((x.y & exps) + one) | ((x.z & exps) + one) |
          ((x.w & exps) + one)) & ~exps;
}
// the 16 bytes without the elements of `cls`
template <typename T>
__device__ inline uint4 finite_part(const uint4& x, uint32_t cls) {
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 16 / int(sizeof(T)); ++i) {
    const uint32_t keep = (((cls >> (2 * i) & 3u) + 3u) >> 2) - 1u;      // all ones, or zero
    if constexpr (sizeof(T) == 4) w[i] &= keep;
    else w[i / 2] &= i & 1 ? keep | 0x0000ffffu : keep | 0xffff0000u;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// ones where `cls` has bit `sign` of an element
template <typename T>
__device__ inline uint4 ones_at(uint32_t cls, int sign) {
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16 / int(sizeof(T)); ++i) {
    const uint32_t on = cls >> (2 * i + sign) & 1u;
    if constexpr (sizeof(T) == 4) w[i] = on * 0x3f800000u;
    else w[i / 2] |= on * (i & 1 ? 0x3f800000u : 0x3f80u);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// what a row's share of such elements adds
__device__ inline float infinity_of(float share, int sign) {
  return share > 0.f ? (sign ? -__builtin_huge_valf() : __builtin_huge_valf()) : 0.f;
}

// ----------------------------------------------------------------------------
// single tokens
// ----------------------------------------------------------------------------

// A unit is up to 16 NB query rows of ONE token, so that all of them see the same keys and
// nothing but the cache's end is masked; a workgroup's four wavefronts take contiguous
// quarters of its tiles and meet only at a unit's end.  Scores are computed transposed, keys x rows,
// in 16x16x32 MFMAs: lane l has column (query row) l % 16 and, of the 8 U keys that its
// group j = l / 16 holds, all of a step's scores.  Keys are dealt to MFMA rows so that
// these are 8 U consecutive keys, which is what the lane feeds to the P*V product, against
// 16 bytes of a transposed value row: operands go from memory to the MFMA without LDS and
// without a lane exchange.  A step is 8 KB of keys and 8 KB of values (D = 128); two are
// in flight (one where 32 rows leave no registers for the second).
//
// int8 codes become bf16 exactly; key scales multiply the scores, value scales the
// probabilities, in fp32.  Turned queries and probabilities are held as two bf16 numbers each, the
// second what the first leaves: the output is then off by its own rounding (2-norm of a batch's
// error 0.0017 of the output's; with queries rounded to one 0.0041, with probabilities 0.0023, in
// int8 0.0025).  Queries come from LDS every step, and the MFMAs that the second numbers add are
// idle time here (24 requests of 1200 to 6200 tokens: 79.1 us with probabilities in one, 79.4 in
// two; 512 of 200 to 900 in int8 181 and 184).  Sums and outputs stay in fp32.
//
// Bound by memory: with up to 16 rows 256 KB are in flight a CU (D = 128), and the rest hides under
// them.  24 requests of 1200 to 6200 tokens (bf16, 373 MB) in pages of 128: 71 to 77 us, 5.2 to
// 4.8 TB/s of the 6.0 that a read of contiguous memory reaches (pages of 64: 70); one of 128k in
// int8 (277 MB): 57, 4.9; eight of those 376 us, 5.9.  With up to 32 rows one workgroup a CU has
// 64 KB in flight: the first of these with 32 heads a kv-head 85 us and 24 of joining.
template <typename S, int D, int NB>
__global__ __launch_bounds__(256, 2) void attend_narrow_kernel(AttendParams a) {
  using T = __bf16;
  constexpr bool I8 = sizeof(S) == 1;
  constexpr int SZ = sizeof(S);
  constexpr int U = I8 ? 2 : 1;              // 32-key groups of a step
  constexpr int KS = 32 * U, SPT = ST / KS;  // keys of a step, steps of a tile
  constexpr int RB = 16 * NB, NW = 4;
  constexpr int NKC = D / (I8 ? 64 : 32);    // 16-byte pieces of a key a lane holds
  constexpr int NKF = 2 * U * NKC, NVF = D / 16, NQC = D / 32;
  constexpr int SETS = NB == 1 ? 2 : 1;
  constexpr int LDO = D + 4;

  __shared__ __attribute__((aligned(16))) float s_o[NW * RB * LDO];
  __shared__ float s_m[NW * RB], s_l[NW * RB];
  __shared__ double s_turns[D / 2];
  __shared__ bf16x8 s_q[NB * NQC * 64], s_rest[NB * NQC * 64];   // (every wavefront's the same)

  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const int col = lane & 15, j = lane >> 4;
  const int PS = a.pg.PS, limit = a.ch.max_pages * PS, rb = a.rb;
  stage_turns<D>(a, s_turns);
  Place at;
  const Share share = find_share(a, blockIdx.x, rb, limit, at);
  Join join{};
  if (share.p0 == share.p1) {
    if (tid == 0) a.joins[blockIdx.x] = join;
    return;
  }
  unsigned p = share.p0;
  Piece cur(a, rb, limit, at, share.p1 - p);

  // ---- loads of this wavefront's steps [s0, s1) of the current piece
  struct Set {
    u32x4 k[NKF], v[NVF];
    float ks, vs;
    int page;
  } set[SETS];
  int s0 = 0, s1 = 0;
  int ids = -1, ids_from = 0;                // pages of tiles ids_from + lane
  const int kofs = (8 * U * (col >> 2) + (col & 3)) * D * SZ + 16 * j;
  const int vofs = col * PS * SZ + 16 * j;
  auto fetch_ids = [&](int tile) __attribute__((always_inline)) {
    ids_from = tile;
    ids = valid_page(a.ch.table[size_t(cur.b) * a.ch.max_pages +
                                min(int(unsigned((tile + lane) * ST) / unsigned(PS)),
                                    a.ch.max_pages - 1)],
                     a.pg.n_pages);
  };
  // past the last step, and where there is no page: descriptors without extent, whose loads
  // give zeros and touch no memory
  auto rsrc = [&](const void* p, bool real, int bytes) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, real ? bytes : 0,
                                             kBufferFlags);
  };
  auto fetch_k = [&](int step, Set& x) __attribute__((always_inline)) {
    const int tile = step / SPT;
    if (tile - ids_from >= 64) fetch_ids(tile);
    x.page = __builtin_amdgcn_readlane(ids, tile - ids_from);
    const bool real = step >= s0 && step < s1 && x.page >= 0;
    const size_t ph = size_t(real ? x.page : 0) * a.pg.Hkv + cur.g;
    const int off = unsigned(step * KS) % unsigned(PS);
    const __amdgpu_buffer_rsrc_t kr =
        rsrc(static_cast<S*>(a.pg.k) + (ph * PS + off) * D, real, KS * D * SZ);
#pragma unroll
    for (int m = 0; m < 2 * U; ++m)
#pragma unroll
      for (int c = 0; c < NKC; ++c)
        x.k[m * NKC + c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
            kr, kofs + 4 * m * D * SZ + 64 * c, 0, 0));
    if constexpr (I8) {
      const __amdgpu_buffer_rsrc_t ksr = rsrc(a.pg.k_scale + ph * PS + off, real, KS * 4);
      const __amdgpu_buffer_rsrc_t vsr = rsrc(a.pg.v_scale + ph * PS + off, real, KS * 4);
      x.ks = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(ksr, 4 * lane, 0, 0));
      x.vs = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(vsr, 4 * lane, 0, 0));
    }
  };
  // The values of both sets, whose keys are being fetched.  A step has half a line of each
  // value row; asked for a step apart, by the time of the second half the L2 had often let
  // the line go (24 requests of 1200 to 6200 tokens: 3.41 million lines read, 2.96 in pairs,
  // 2.91 their number; 80.8 -> 77.3 us, and 73.6 -> 70.0 in pages of 64).
  auto fetch_v = [&](int step) __attribute__((always_inline)) {
    __amdgpu_buffer_rsrc_t vr[SETS];
#pragma unroll
    for (int k = 0; k < SETS; ++k) {
      const bool real = step + k >= s0 && step + k < s1 && set[k].page >= 0;
      const size_t ph = size_t(real ? set[k].page : 0) * a.pg.Hkv + cur.g;
      vr[k] = rsrc(static_cast<S*>(a.pg.v) + ph * D * PS + unsigned((step + k) * KS) % unsigned(PS),
                   real, ((D - 1) * PS + KS) * SZ);
    }
#pragma unroll
    for (int db = 0; db < NVF; ++db)
#pragma unroll
      for (int k = 0; k < SETS; ++k)
        set[k].v[db] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
            vr[k], vofs + 16 * db * PS * SZ, 0, 0));
  };
  // query chunk c of a lane: elements qd(c) .. + 7, following the keys' 16-byte pieces; its
  // partner is chunk c + NQP of the lane, or, where two lanes hold the pair, only loaded
  constexpr int NQP = I8 && D == 64 ? NQC : NQC / 2;
  auto qd = [&](int c) __attribute__((always_inline)) {
    return I8 ? 64 * (c / 2) + 16 * j + 8 * (c % 2) : 32 * c + 8 * j;
  };
  uint32_t qx[NB][NQP][4], qy[NB][NQP][4];
  int qpos[NB];
  // a piece's queries and first steps
  auto enter = [&]() __attribute__((always_inline)) {
    // quarters of the piece's steps, in pairs where every wavefront gets one
    const int a0 = cur.t0 * SPT, a1 = cur.t1 * SPT, sh = a1 - a0 <= NW ? 0 : SETS - 1;
    const int from = a0 >> sh << sh, n = (a1 - from + sh) >> sh;
    s0 = max(a0, from + (n * wave / NW << sh));
    s1 = min(a1, from + (n * (wave + 1) / NW << sh));
    fetch_ids(s0 / SETS * SETS / SPT);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const unsigned row = cur.row0 + min(16 * nb + col, cur.nrows - 1);
      const int t = row / unsigned(a.G);
      const T* qrow = static_cast<const T*>(a.q) + (cur.r.first + t) * a.q_stride +
                      size_t(cur.g * a.G + row - t * a.G) * D;
      qpos[nb] = a.rope.pos ? a.rope.pos[cur.r.first + t] : 0;
#pragma unroll
      for (int c = 0; c < NQP; ++c) {
        raw_load8<T>(qx[nb][c], qrow + qd(c) % (D / 2));
        raw_load8<T>(qy[nb][c], qrow + qd(c) % (D / 2) + D / 2);
      }
    }
#pragma unroll
    for (int k = 0; k < SETS; ++k) fetch_k(s0 / SETS * SETS + k, set[k]);
    fetch_v(s0 / SETS * SETS);
  };
  enter();
  lds_barrier();                             // the turns are there

  while (true) {
    // ---- queries: turned by their tokens' positions, the softmax scale folded in
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int c = 0; c < NQP; ++c) {
        float x[8], y[8];
        raw_to_f8<T>(qx[nb][c], x);
        raw_to_f8<T>(qy[nb][c], y);
        turn_chunks<8>(s_turns + qd(c) % (D / 2), a.rope.pos, qpos[nb], a.qscale, x, y);
        auto put = [&](int i, const float (&v)[8]) __attribute__((always_inline)) {
          split_bf16(v, s_q[(nb * NQC + i) * 64 + lane], s_rest[(nb * NQC + i) * 64 + lane]);
        };
        if constexpr (NQP < NQC) {
          put(c, x);
          put(c + NQP, y);
        } else {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = qd(c) < D / 2 ? x[e] : y[e];
          put(c, v);
        }
      }
    }
    const int keys = cur.keys;

    float m_run[NB], m_ref[NB], l_run[NB];
    f32x4 o[NB][NVF];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m_run[nb] = kNegInf;
      m_ref[nb] = l_run[nb] = 0.f;
#pragma unroll
      for (int db = 0; db < NVF; ++db) o[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    auto compute = [&](int step, Set& x) __attribute__((always_inline)) {
      const int key0 = step * KS;
      const bool partial = key0 + KS > keys || x.page < 0;
      bf16x8 pb[NB][U], pr_rest[NB][U];
      f32x4 s[NB][2 * U];
#pragma unroll
      for (int m = 0; m < 2 * U; ++m)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          // bf16: scores leave the product relative to the reference
          const float z = I8 ? 0.f : -m_ref[nb];
          s[nb][m] = f32x4{z, z, z, z};
        }
#pragma unroll
      for (int c = 0; c < NQC; ++c) {
        bf16x8 q[NB], rest[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          q[nb] = s_q[(nb * NQC + c) * 64 + lane];
          rest[nb] = s_rest[(nb * NQC + c) * 64 + lane];
        }
#pragma unroll
        for (int m = 0; m < 2 * U; ++m) {
          bf16x8 kf;
          if constexpr (I8) {
            const u32x4 w = x.k[m * NKC + c / 2];
            kf = bf16_of_i8(w[2 * (c % 2)], w[2 * (c % 2) + 1]);
          } else {
            kf = __builtin_bit_cast(bf16x8, x.k[m * NKC + c]);
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            s[nb][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[nb], s[nb][m], 0, 0, 0);
            s[nb][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, rest[nb], s[nb][m], 0, 0, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);     // (one chunk's queries at a time)
      }
      if constexpr (I8) {
        // lane l has the scale of key key0 + l, and scores of its group's 16 keys
        float ks[16];
        lanes16(x.ks, ks, std::make_integer_sequence<int, 16>{});
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int k = 0; k < 16; ++k)
            s[nb][k / 4][k % 4] = __builtin_fmaf(s[nb][k / 4][k % 4], ks[k], -m_ref[nb]);
      }
      if (partial) {
        const int n = x.page < 0 ? 0 : keys - key0 - 8 * U * j;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int k = 0; k < 8 * U; ++k)
            if (k >= n) s[nb][k / 4][k % 4] = kNegInf;
        // what lies behind the last key may be anything
        if constexpr (I8) {
          if (key0 + lane >= keys) x.vs = 0.f;
        } else if (key0 + KS > keys) {
#pragma unroll
          for (int db = 0; db < NVF; ++db) {
            const uint4 v = keep_first<T>(__builtin_bit_cast(uint4, x.v[db]),
                                          max(keys - key0 - 8 * j, 0));
            x.v[db] = __builtin_bit_cast(u32x4, v);
          }
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float mx = s[nb][0][0];
#pragma unroll
        for (int k = 1; k < 8 * U; ++k) mx = fmaxf(mx, s[nb][k / 4][k % 4]);
        // the reference moves where a score outgrows it by more than kLazyLog2
        if (__any(mx + m_ref[nb] > m_run[nb] + kLazyLog2)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          const float m_new = fmaxf(m_run[nb], mx + m_ref[nb]);
          const float ref = m_new == kNegInf ? 0.f : m_new;
          const float keep = __builtin_amdgcn_exp2f(m_run[nb] - ref);
          const float d = ref - m_ref[nb];
          l_run[nb] *= keep;
#pragma unroll
          for (int db = 0; db < NVF; ++db) o[nb][db] *= keep;
#pragma unroll
          for (int k = 0; k < 8 * U; ++k) s[nb][k / 4][k % 4] -= d;
          m_run[nb] = m_new;
          m_ref[nb] = ref;
        }
        float pr[8 * U], sum = 0.f;
#pragma unroll
        for (int k = 0; k < 8 * U; ++k) {
          pr[k] = __builtin_amdgcn_exp2f(s[nb][k / 4][k % 4]);
          sum += pr[k];
        }
        l_run[nb] += sum;
        if constexpr (I8) {
          float vs[16];
          lanes16(x.vs, vs, std::make_integer_sequence<int, 16>{});
#pragma unroll
          for (int k = 0; k < 16; ++k) pr[k] *= vs[k];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float (&x8)[8] = reinterpret_cast<const float (&)[8]>(pr[8 * u]);
          split_bf16(x8, pb[nb][u], pr_rest[nb][u]);
        }
      }
#pragma unroll
      for (int db = 0; db < NVF; ++db)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          bf16x8 vf;
          if constexpr (I8) vf = bf16_of_i8(x.v[db][2 * u], x.v[db][2 * u + 1]);
          else vf = __builtin_bit_cast(bf16x8, x.v[db]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[nb][u], o[nb][db], 0, 0, 0);
            o[nb][db] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pr_rest[nb][u], o[nb][db], 0, 0, 0);
          }
        }
    };
    for (int step = s0 / SETS * SETS; step < s1; step += SETS) {
#pragma unroll
      for (int k = 0; k < SETS; ++k) {
        if (step + k >= s0 && step + k < s1) compute(step + k, set[k]);
        fetch_k(step + k + SETS, set[k]);
      }
      fetch_v(step + SETS);
    }

    // ---- the next piece's first loads, under the end of this one
    const Piece old = cur;
    p += old.t1 - old.t0;
    const bool more = p < share.p1;
    if (more) {
      next_unit(a, rb, limit, at);
      cur = Piece(a, rb, limit, at, share.p1 - p);
      enter();
    }

    // ---- the wavefronts' parts meet
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float l = l_run[nb];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      const int r = wave * RB + 16 * nb + col;
      if (j == 0) {
        s_m[r] = m_run[nb];
        s_l[r] = l;
      }
#pragma unroll
      for (int db = 0; db < NVF; ++db)
        *reinterpret_cast<f32x4*>(s_o + r * LDO + 16 * db + 4 * j) = o[nb][db];
    }
    lds_barrier();
    if (old.begins() && !old.ends()) join = old.cut(share);
    constexpr int TPR = 256 / RB, EPT = D / TPR;    // threads a row, elements a thread
    const int row = tid / TPR, d0 = tid % TPR * EPT;
    if (row < old.nrows) {
      float m = kNegInf, l = 0.f, x[EPT] = {};
#pragma unroll
      for (int w = 0; w < NW; ++w) m = fmaxf(m, s_m[w * RB + row]);
      const float ref = m == kNegInf ? 0.f : m;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_m[w * RB + row] - ref);
        l += f * s_l[w * RB + row];
#pragma unroll
        for (int e = 0; e < EPT; ++e) x[e] += f * s_o[(w * RB + row) * LDO + d0 + e];
      }
      if (old.begins() && old.ends()) {
        const unsigned r = old.row0 + row, t = r / unsigned(a.G);
        const size_t oh = size_t(old.r.first + t) * a.Hq + old.g * a.G + (r - t * a.G);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* out = static_cast<T*>(a.out) + oh * D + d0;
#pragma unroll
        for (int e = 0; e < EPT; e += 4)
          *reinterpret_cast<uint2*>(out + e) =
              make_uint2(pack_bf16(x[e] * inv, x[e + 1] * inv),
                         pack_bf16(x[e + 2] * inv, x[e + 3] * inv));
        if (a.lse && d0 == 0)
          a.lse[oh] = l == 0.f ? kNegInf : (ref + __builtin_amdgcn_logf(l)) * kLn2;
      } else {
        const size_t part = (size_t(2) * blockIdx.x + (old.begins() ? 1 : 0)) * RB + row;
#pragma unroll
        for (int e = 0; e < EPT; e += 4)
          *reinterpret_cast<float4*>(a.part_o + part * D + d0 + e) =
              make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        if (d0 == 0) a.part_ml[part] = make_float2(m, l);
      }
    }
    if (!more) break;
    lds_barrier();                           // LDS of this piece is read
  }
  if (tid == 0) a.joins[blockIdx.x] = join;
}

// ----------------------------------------------------------------------------
// blocks of rows
// ----------------------------------------------------------------------------

// Tiles of keys and transposed values in LDS, as 16-byte chunks of rows of D (keys) or 64
// (values) elements; a row's chunks are permuted by its index, so that the operand reads
// of 32 rows at one column fall on distinct banks without padding.
template <typename T, int D>
struct WideTile {
  static constexpr int EPC = 16 / int(sizeof(T));
  static constexpr int CK = D / EPC, CV = ST / EPC;        // chunks of a row
  static constexpr int MK = (CK < 16 ? CK : 16) - 1, MV = (CV < 16 ? CV : 16) - 1;
  static constexpr int KBYTES = ST * D * int(sizeof(T)), BYTES = 2 * KBYTES;
  __device__ static int k_at(int key, int ch) { return (key * CK + (ch ^ (key & MK))) * 16; }
  __device__ static int v_at(int d, int ch) { return KBYTES + (d * CV + (ch ^ (d & MV))) * 16; }
};

// 64 lanes' 16 bytes each from base + off (per lane) to LDS at `lds` + 16 * lane, in flight
// until the wavefront's vector-memory count says otherwise (wait_loads).  Written out
// because the compiler would wait for every such load before any LDS read.
__device__ inline void load_to_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(off), "s"(base) : "m0", "memory");
}
// until at most N of this wavefront's loads are in flight, then every wavefront's
template <int N>
__device__ inline void wait_loads_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// 512 threads: RG groups of 32 query rows, and 8 / RG parts of a tile's keys for each.
// Scores transposed (keys x rows) in 32x32 MFMAs: a lane has one row's scores, for bf16 of
// 8 consecutive keys at a time (keys are dealt to the MFMA's rows with bits 2 and 3 of
// their index exchanged), the operand of the P*V product.
//
// int8 codes go through registers.  Keys become bf16 exactly and their scales multiply the
// scores in fp32; values are decoded there (code * scale in fp32) and rounded once, as
// c2kv_compose rounds them.  (2048 tokens over 32k, 32 query heads: 1.20 to 1.30 ms, 0.95 to 0.87
// PFLOP/s, and 26 us of joining: after a tile's barrier all wavefronts decode the next one while the
// MFMAs, busy 41 % of the time, wait.  Keys decoded and rounded too: 12 % faster, but the 2-norm of
// the error is then 0.0052 of the output's, not 0.0045; value scales applied to the probabilities
// instead: 4 % slower, and 0.0042.)
//
// Bound by the MFMAs' share of a wavefront pair's time: 2048 tokens over 32k (64 query heads,
// 2.27 TFLOP) in 1.97 to 2.03 ms, 1.15 to 1.12 PFLOP/s, where a library product of 8192 cubed
// reaches 1.21; the MFMAs are busy 57 % of the time, the softmax and the operands' LDS reads the
// rest.  A wavefront that runs the scores of one tile beside the softmax of the tile before spills;
// values' rows exchanged so that no LDS read meets a conflict (a third do) change nothing.
// fp32: 1024 tokens over 1024, 32 heads, 239 to 268 us, 108 to 96 TFLOP/s of the 147 that a library
// product of 4096 cubed reaches, the MFMAs busy 76 % of the time.
//
// Few rows over a long cache leave most wavefronts and the MFMAs idle (busy 16 %), and one workgroup
// a CU nothing to hide a tile's chain under, about 2 us of barrier, LDS reads, products and softmax:
// 81 drafts of 16 requests over 329 MB of bf16 take 87 us, over 171 MB of int8 95 to 100, single
// fp32 tokens of 16 requests over 593 MB 317.
template <typename T, typename S, int D, int RG>
__global__ __launch_bounds__(512, 2) void attend_wide_kernel(AttendParams a) {
  using M = Mma<T>;
  using W = WideTile<T, D>;
  constexpr bool F32 = sizeof(T) == 4, I8 = sizeof(S) == 1;
  constexpr int SZ = sizeof(T), NTH = 512;
  constexpr int KG = 8 / RG, NKB = 2 / KG;       // key parts, 32-key blocks of a wavefront
  static_assert(KG <= 2, "a wavefront has a 32-key block at least");
  constexpr int RB = 32 * RG;
  // Queries held as two bf16 numbers, as for single tokens, where 128 rows a workgroup leave
  // the MFMAs idle (16 requests of 3 to 7 drafts: 81 -> 84 us).  256 rows would pay half as
  // many products again for the scores (2048 tokens over 32k: 1.06 -> 1.43 ms): there a turned
  // and scaled query is rounded once, as c2kv_attend's are.  Probabilities are rounded once in
  // both (two numbers in 128 rows: drafts' error 0.0022 -> 0.0017 of the output's 2-norm, 88 -> 91
  // us with 32 query heads and 87 -> 95 with 64; int8 0.0027 -> 0.0023, 90 -> 102).
  constexpr bool TWO = !F32 && RG == 4;
  constexpr int NST = F32 || I8 ? 2 : TWO ? 3 : 4;   // tiles in LDS
  constexpr int LK = ST * W::CK / NTH, LV = D * W::CV / NTH, LPT = LK + LV;
  constexpr int NQC = W::CK / 2;                 // query chunks of a lane (its half's)
  constexpr int NPC = 16 * NKB / W::EPC;         // probability chunks of a lane
  constexpr int NDB = D / 32;
  static_assert(LK >= 1 && LV >= 1 && (NTH / W::CK) % (W::MK + 1) == 0 &&
                    (NTH / W::CV) % (W::MV + 1) == 0,
                "a thread's chunks of one tile lie in rows of one permutation");

  // After the tiles the stages serve the key parts' exchange (XW floats a lane) and the way
  // of the rows out (OUT bytes a wavefront).
  constexpr int XW = 4 + 16 * NDB, OUT = 32 * 64 * 4;
  constexpr int XBYTES = KG == 2 ? RG * 64 * XW * 4 : 8 * OUT;
  static_assert(KG == 1 || 64 * XW * 4 >= OUT, "a row group's exchange holds its rows' way out");
  __shared__ __attribute__((aligned(1024)))
  uint8_t lds[NST * W::BYTES > XBYTES ? NST * W::BYTES : XBYTES];
  __shared__ double s_turns[D / 2];
  __shared__ int s_odd[8];                       // a wavefront's values that are not finite
  __shared__ bf16x8 s_rest[TWO ? RG * NQC * 64 : 1];
  __shared__ float s_scale[I8 ? NST * ST : 1];   // int8: of a tile's keys
  const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) uint8_t*)lds));

  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const int col = lane & 31, half = lane >> 5;
  const int rg = wave % RG, kg = wave / RG;
  const int PS = a.pg.PS, limit = a.ch.max_pages * PS;
  // workgroups of one XCD (every eighth) take neighbouring shares, which read the same keys
  const int nx = gridDim.x / 8;
  const int w = gridDim.x % 8 == 0 ? int(blockIdx.x % 8) * nx + int(blockIdx.x / 8)
                                   : int(blockIdx.x);
  stage_turns<D>(a, s_turns);
  Place at;
  const Share share = find_share(a, w, RB, limit, at);
  Join join{};
  unsigned p = share.p0;
  lds_barrier();                                 // the turns are there

  // this thread's chunks of a tile: chunk tid + i * 512 of the keys, and of the values
  const int kkey = tid / W::CK, kch = (tid % W::CK) ^ (kkey & W::MK);
  const int vrow = tid / W::CV, vch = (tid % W::CV) ^ (vrow & W::MV);
  const uint32_t kofs = uint32_t(kkey * D * SZ + kch * 16);
  const uint32_t vofs = uint32_t(vrow * PS * SZ + vch * 16);

  while (p < share.p1) {
    const Piece cur(a, RB, limit, at, share.p1 - p);
    const int t0 = cur.t0, t1 = cur.t1, row0 = cur.row0, nrows = cur.nrows, keys = cur.keys;
    const int32_t* table = a.ch.table + size_t(at.b) * a.ch.max_pages;
    int ids = -1, ids_from = -(1 << 30);         // pages of tiles ids_from + lane

    auto page_id = [&](int tile) __attribute__((always_inline)) {
      if (unsigned(tile - ids_from) >= 64u) {
        ids_from = tile;
        ids = valid_page(table[min((tile + lane) * ST / PS, a.ch.max_pages - 1)], a.pg.n_pages);
      }
      return __builtin_amdgcn_readlane(ids, tile - ids_from);
    };
    // a tile without a page is loaded from page 0: its scores are masked, its values zeroed
    auto load = [&](int tile) __attribute__((always_inline)) {
      const int page = max(page_id(tile), 0), off = tile * ST % PS;
      const size_t ph = size_t(page) * a.pg.Hkv + at.g;
      const T* kp = static_cast<const T*>(a.pg.k) + (ph * PS + off) * D;
      const T* vp = static_cast<const T*>(a.pg.v) + ph * D * PS + off;
      const uint32_t to = lds0 + (tile - t0) % NST * W::BYTES + wave * 1024;
#pragma unroll
      for (int i = 0; i < LK; ++i)
        load_to_lds(kp + size_t(i) * (NTH / W::CK) * D, kofs, to + i * NTH * 16);
#pragma unroll
      for (int i = 0; i < LV; ++i)
        load_to_lds(vp + size_t(i) * (NTH / W::CV) * PS, vofs, to + W::KBYTES + i * NTH * 16);
    };

    auto stage = [&](int tile) { return lds + (tile - t0) % NST * W::BYTES; };
    // keys of a tile that exist
    auto there = [&](int tile, int page) { return page < 0 ? 0 : min(max(keys - tile * ST, 0), ST); };

    // int8: BPT codes of a key (elements ikd ..) and of a value row (keys ivk ..) a thread;
    // lane l has the scales of key l
    constexpr int BPT = ST * D / NTH;
    const int ikey = tid / (D / BPT), ikd = tid % (D / BPT) * BPT;
    const int ivd = wave * BPT + lane % BPT, ivk = lane / BPT * BPT;
    uint32_t kraw[BPT / 4], vraw[BPT / 4];
    float kscale = 0.f, vscale = 0.f;
    auto load_i8 = [&](int tile) __attribute__((always_inline)) {
      const int page = max(page_id(tile), 0), off = tile * ST % PS;
      const size_t ph = size_t(page) * a.pg.Hkv + at.g;
      const int8_t* kp = static_cast<const int8_t*>(a.pg.k) + (ph * PS + off + ikey) * D + ikd;
      const int8_t* vp = static_cast<const int8_t*>(a.pg.v) + (ph * D + ivd) * PS + off + ivk;
#pragma unroll
      for (int i = 0; i < BPT / 8; ++i) {
        raw_load8<int8_t>(kraw + 2 * i, kp + 8 * i);
        raw_load8<int8_t>(vraw + 2 * i, vp + 8 * i);
      }
      vscale = a.pg.v_scale[ph * PS + off + lane];
      kscale = a.pg.k_scale[ph * PS + off + lane];
    };
    auto commit_i8 = [&](int tile) __attribute__((always_inline)) {
      const int n = there(tile, page_id(tile));
      // (a scale behind the last key may be anything)
      float vs[16];
      lanes16(lane < n ? vscale : 0.f, vs, std::make_integer_sequence<int, 16>{});
      if (wave == 0) s_scale[unsigned(tile - t0) % NST * ST + lane] = kscale;
      uint8_t* st = stage(tile);
#pragma unroll
      for (int i = 0; i < BPT / 8; ++i) {
        *reinterpret_cast<bf16x8*>(st + W::k_at(ikey, ikd / 8 + i)) =
            bf16_of_i8(kraw[2 * i], kraw[2 * i + 1]);
        float y[8];
        raw_to_f8<int8_t>(vraw + 2 * i, y);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          y[e] *= BPT == 16 ? vs[8 * i + e] : lane & 8 ? vs[8 + e] : vs[e];
        *reinterpret_cast<bf16x8*>(st + W::v_at(ivd, ivk / 8 + i)) = bf16_of(y);
      }
    };

    // ---- the first tiles
    if constexpr (I8) {
      load_i8(t0);
    } else {
#pragma unroll
      for (int k = 0; k < NST - 1; ++k)
        if (t0 + k < t1) load(t0 + k);
    }

    // ---- this wavefront's rows
    const bool rows_here = 32 * rg < nrows;
    const unsigned row = row0 + min(32 * rg + col, nrows - 1), t = row / unsigned(a.G);
    const int sees = min(max(at.r.base + int(t) + 1, 0), limit);
    // every row's keys, and any row's
    auto token_of = [&](int r) { return int(unsigned(row0 + min(r, nrows - 1)) / unsigned(a.G)); };
    const int sees_all = min(max(at.r.base + token_of(32 * rg) + 1, 0), limit);
    const int sees_any = min(max(at.r.base + token_of(32 * rg + 31) + 1, 0), limit);
    const int sees_first = min(max(at.r.base + token_of(0) + 1, 0), limit);   // all rows' keys
    // tiles [t0, end) have keys that rows of this wavefront see
    const int end = rows_here ? (sees_any + ST - 1) / ST : t0;
    typename M::Op q[NQC * (F32 ? 4 : 1)];
    {
      const T* qrow = static_cast<const T*>(a.q) + (at.r.first + t) * a.q_stride +
                      size_t(at.g * a.G + row % a.G) * D;
      const int pos = a.rope.pos ? a.rope.pos[at.r.first + t] : 0;
      // chunk 2 c + half of the row; its partner D / 2 away is chunk c + NQC / 2's
      uint4 qx[NQC / 2], qy[NQC / 2];
#pragma unroll
      for (int c = 0; c < NQC / 2; ++c) {
        const T* from = qrow + (2 * c + half) * W::EPC;
        qx[c] = *reinterpret_cast<const uint4*>(from);
        qy[c] = *reinterpret_cast<const uint4*>(from + D / 2);
      }
#pragma unroll
      for (int c = 0; c < NQC / 2; ++c) {
        float x[W::EPC], y[W::EPC];
        if constexpr (F32) {
          const float xs[4] = {__uint_as_float(qx[c].x), __uint_as_float(qx[c].y),
                               __uint_as_float(qx[c].z), __uint_as_float(qx[c].w)};
          const float ys[4] = {__uint_as_float(qy[c].x), __uint_as_float(qy[c].y),
                               __uint_as_float(qy[c].z), __uint_as_float(qy[c].w)};
#pragma unroll
          for (int e = 0; e < 4; ++e) { x[e] = xs[e]; y[e] = ys[e]; }
        } else {
          const uint32_t xs[4] = {qx[c].x, qx[c].y, qx[c].z, qx[c].w};
          const uint32_t ys[4] = {qy[c].x, qy[c].y, qy[c].z, qy[c].w};
          raw_to_f8<T>(xs, x);
          raw_to_f8<T>(ys, y);
        }
        turn_chunks<W::EPC>(s_turns + (2 * c + half) * W::EPC, a.rope.pos, pos, a.qscale, x, y);
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            q[4 * c + e] = x[e];
            q[4 * (c + NQC / 2) + e] = y[e];
          }
        } else {
          if constexpr (TWO) {                   // (the same from both key parts)
            split_bf16(x, q[c], s_rest[(rg * NQC + c) * 64 + lane]);
            split_bf16(y, q[c + NQC / 2], s_rest[(rg * NQC + c + NQC / 2) * 64 + lane]);
          } else {
            q[c] = bf16_of(x);
            q[c + NQC / 2] = bf16_of(y);
          }
        }
      }
    }

    float m_run = kNegInf, m_ref = 0.f, l_run = 0.f;
    f32x16 o[NDB], bias;
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[v] = 0.f;
#pragma unroll
    for (int db = 0; db < NDB; ++db) o[db] = bias;

    // value v of a 32-key block is its key 16 (v / 8) + 8 half + v % 8 (fp32: 8 (v / 4) +
    // 4 half + v % 4); block b of this wavefront's part of the tile
    auto mask = [&](int tile, int b, int page, f32x16& s) __attribute__((always_inline)) {
      const int k0 = tile * ST + 32 * (kg * NKB + b);
      if (k0 + 32 <= sees_all && page >= 0) return;
      const int lim = page < 0 ? -64 : sees - k0 - (F32 ? 4 : 8) * half - 1;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = F32 ? 8 * (v >> 2) + (v & 3) : 16 * (v >> 3) + (v & 7);
        const uint32_t hide = uint32_t((lim - key) >> 31);
        const uint32_t x = __float_as_uint(s[v]);
        s[v] = __uint_as_float((x & ~hide) | (0xff800000u & hide));
      }
    };
    // the reference moves where a score outgrows it (by mx) by over kLazyLog2; scores are
    // relative to it: the MFMA chains begin with `bias`, minus it
    auto rebase = [&](float mx, f32x16 (&s)[NKB]) __attribute__((always_inline)) {
      if (__any(mx + m_ref > m_run + kLazyLog2)) {
        const float m_new = fmaxf(m_run, half_pair_max(mx) + m_ref);
        const float ref = m_new == kNegInf ? 0.f : m_new;
        const float keep = __builtin_amdgcn_exp2f(m_run - ref), d = ref - m_ref;
        l_run *= keep;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][v] *= keep;
#pragma unroll
        for (int b = 0; b < NKB; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) s[b][v] -= d;
        if constexpr (!I8) {
#pragma unroll
          for (int v = 0; v < 16; ++v) bias[v] = -ref;
        }
        m_run = m_new;
        m_ref = ref;
      }
    };
    // what lies behind the last key may be anything: zero values there
    auto clean = [&](int tile, int page) __attribute__((always_inline)) {
      const int n = there(tile, page);
      if (n == ST) return;
#pragma unroll
      for (int i = 0; i < LV; ++i) {
        uint4* v = reinterpret_cast<uint4*>(stage(tile) + W::KBYTES + (tid + i * NTH) * 16);
        if (vch * W::EPC + W::EPC > n) *v = keep_first<T>(*v, max(n - vch * W::EPC, 0));
      }
      lds_barrier();
    };
    // Takes values that are not finite out of a tile that some rows see and others do not;
    // this thread's are `odd`, two bits an element.  True (for all wavefronts) if there are any.
    uint32_t odd = 0;
    static_assert(LV * W::EPC <= 16, "two bits for every element of a thread's chunks");
    auto own_chunk = [&](int tile, int i) {
      return reinterpret_cast<uint4*>(stage(tile) + W::KBYTES + (tid + i * NTH) * 16);
    };
    auto take_odd = [&](int tile) __attribute__((always_inline)) {
      if ((tile + 1) * ST <= sees_first || sees_first >= keys) return false;
      uint32_t quick = 0;
#pragma unroll
      for (int i = 0; i < LV; ++i) quick |= any_not_finite<T>(*own_chunk(tile, i));
      const bool here = __any(quick);
      if (lane == 0) s_odd[wave] = here;
      lds_barrier();
      int any = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) any |= s_odd[i];
      if (!uniform(any)) return false;
      odd = 0;
#pragma unroll
      for (int i = 0; i < LV; ++i) {
        const uint32_t cls = not_finite<T>(*own_chunk(tile, i));
        *own_chunk(tile, i) = finite_part<T>(*own_chunk(tile, i), cls);
        odd |= cls << (2 * W::EPC * i);
      }
      lds_barrier();
      return true;
    };
    // puts ones where they were
    auto put_ones = [&](int tile, int sign) __attribute__((always_inline)) {
      lds_barrier();
#pragma unroll
      for (int i = 0; i < LV; ++i)
        *own_chunk(tile, i) = ones_at<T>(odd >> (2 * W::EPC * i), sign);
      lds_barrier();
    };

    // ---- one tile: scores, probabilities, P*V
    auto compute = [&](int tile, int page, const uint8_t* st, bool strange)
        __attribute__((always_inline)) {
      f32x16 s[NKB];
      if constexpr (F32) {
        static_assert(!F32 || NKB == 1, "an fp32 wavefront has one block of a tile");
        s[0] = bias;
#pragma unroll
        for (int c = 0; c < NQC; ++c) {
          const float4 f =
              *reinterpret_cast<const float4*>(st + W::k_at(32 * kg + col, 2 * c + half));
          s[0] = M::run(f.x, q[4 * c], s[0]);
          s[0] = M::run(f.y, q[4 * c + 1], s[0]);
          s[0] = M::run(f.z, q[4 * c + 2], s[0]);
          s[0] = M::run(f.w, q[4 * c + 3], s[0]);
        }
      } else {
        // operands in a ring AH ahead of their MFMAs; the scheduling fences hold the order
        constexpr int NF = NKB * NQC, AH = 4;
        const int kr = 32 * kg * NKB + ((col & ~12) | (col & 4) << 1 | (col & 8) >> 1);
        auto frag = [&](int f) __attribute__((always_inline)) {
          return *reinterpret_cast<const bf16x8*>(
              st + W::k_at(kr + 32 * (f / NQC), 2 * (f % NQC) + half));
        };
        bf16x8 kf[AH], rf[AH];
#pragma unroll
        for (int f = 0; f < AH; ++f) {
          kf[f] = frag(f);
          if constexpr (TWO) rf[f] = s_rest[(rg * NQC + f % NQC) * 64 + lane];
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);           // matrix work before the other's softmax
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const int b = f / NQC, c = f % NQC;
          s[b] = M::run(kf[f % AH], q[c], c == 0 ? bias : s[b]);
          if constexpr (TWO) {
            s[b] = M::run(kf[f % AH], rf[f % AH], s[b]);
            if (f + AH < NF) rf[f % AH] = s_rest[(rg * NQC + (f + AH) % NQC) * 64 + lane];
          }
          if (f + AH < NF) kf[f % AH] = frag(f + AH);
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
      }
      if constexpr (I8) {
#pragma unroll
        for (int b = 0; b < NKB; ++b) {
          // of this lane's 16 scores, from its group of 16 lanes
          float ks[16];
          lanes16(s_scale[unsigned(tile - t0) % NST * ST + 32 * (kg * NKB + b) +
                          16 * (lane >> 3 & 1) + 8 * half + (lane & 7)],
                  ks, std::make_integer_sequence<int, 16>{});
#pragma unroll
          for (int v = 0; v < 16; ++v) s[b][v] = __builtin_fmaf(s[b][v], ks[v], -m_ref);
        }
      }
#pragma unroll
      for (int b = 0; b < NKB; ++b) mask(tile, b, page, s[b]);
      float mx = s[0][0];
#pragma unroll
      for (int i = 1; i < 16 * NKB; ++i) mx = fmaxf(mx, s[i / 16][i % 16]);
      rebase(mx, s);
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[0][i] = __builtin_amdgcn_exp2f(s[0][i]);
          sum[i % 4] += s[0][i];
        }
        // a tile's sum apart, then added: the rounding of a long sum grows with the tiles
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          f32x16 part;
#pragma unroll
          for (int v = 0; v < 16; ++v) part[v] = 0.f;
#pragma unroll
          for (int c = 0; c < NPC; ++c) {
            const float4 f = *reinterpret_cast<const float4*>(
                st + W::v_at(32 * db + col, 2 * (kg * NPC + c) + half));
            part = M::run(f.x, s[0][4 * c], part);
            part = M::run(f.y, s[0][4 * c + 1], part);
            part = M::run(f.z, s[0][4 * c + 2], part);
            part = M::run(f.w, s[0][4 * c + 3], part);
          }
          o[db] += part;
        }
        if (strange) {
          for (int sign = 0; sign < 2; ++sign) {
            put_ones(tile, sign);
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
              f32x16 part;
#pragma unroll
              for (int v = 0; v < 16; ++v) part[v] = 0.f;
#pragma unroll
              for (int c = 0; c < NPC; ++c) {
                const float4 f = *reinterpret_cast<const float4*>(
                    st + W::v_at(32 * db + col, 2 * (kg * NPC + c) + half));
                const float fs[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) part = M::run(fs[e], s[0][4 * c + e], part);
              }
#pragma unroll
              for (int v = 0; v < 16; ++v) o[db][v] += infinity_of(part[v], sign);
            }
          }
        }
      } else {
        bf16x8 pb[NPC];
        const bf16x2 ones = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
#pragma unroll
        for (int b = 0; b < NKB; ++b) {
#pragma unroll
          for (int v = 0; v < 16; v += 2) {
            const f32x2 x = {__builtin_amdgcn_exp2f(s[b][v]), __builtin_amdgcn_exp2f(s[b][v + 1])};
            const bf16x2 w = __builtin_convertvector(x, bf16x2);
            pb[2 * b + v / 8][v % 8] = w[0];
            pb[2 * b + v / 8][v % 8 + 1] = w[1];
            // the sum of the rounded values that the product uses
            sum[v / 2 % 4] = __builtin_amdgcn_fdot2_f32_bf16(w, ones, sum[v / 2 % 4], false);
          }
        }
        constexpr int NF = NPC * NDB, AH = 4;
        auto frag = [&](int f) __attribute__((always_inline)) {
          return *reinterpret_cast<const bf16x8*>(
              st + W::v_at(32 * (f % NDB) + col, 2 * (kg * NPC + f / NDB) + half));
        };
        bf16x8 vf[AH];
#pragma unroll
        for (int f = 0; f < AH; ++f) vf[f] = frag(f);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          o[f % NDB] = M::run(vf[f % AH], pb[f / NDB], o[f % NDB]);
          if (f + AH < NF) vf[f % AH] = frag(f + AH);
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (strange) {
          for (int sign = 0; sign < 2; ++sign) {
            put_ones(tile, sign);
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
              f32x16 part;
#pragma unroll
              for (int v = 0; v < 16; ++v) part[v] = 0.f;
#pragma unroll
              for (int c = 0; c < NPC; ++c)
                part = M::run(*reinterpret_cast<const bf16x8*>(
                                  st + W::v_at(32 * db + col, 2 * (kg * NPC + c) + half)),
                              pb[c], part);
#pragma unroll
              for (int v = 0; v < 16; ++v) o[db][v] += infinity_of(part[v], sign);
            }
          }
        }
      }
      l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    // a tile that has arrived, by all wavefronts
    auto work = [&](int tile, int page) __attribute__((always_inline)) {
      const bool strange = take_odd(tile);
      if (tile < end) {
        compute(tile, page, stage(tile), strange);
      } else if (strange) {
        put_ones(tile, 0);
        put_ones(tile, 1);
      }
    };

    if constexpr (I8) {
      commit_i8(t0);
      if (t0 + 1 < t1) load_i8(t0 + 1);
      for (int tile = t0; tile < t1; ++tile) {
        lds_barrier();                           // this tile is there, the one before is read
        if (tile + 1 < t1) commit_i8(tile + 1);
        if (tile + 2 < t1) load_i8(tile + 2);
        work(tile, page_id(tile));
      }
    } else for (int tile = t0; tile < t1; ++tile) {
      // this tile's loads are done where only those of the tiles after it are in flight
      const int after = min(t1 - 1 - tile, NST - 2);
      if (after >= 2) wait_loads_barrier<2 * LPT>();
      else if (after == 1) wait_loads_barrier<LPT>();
      else wait_loads_barrier<0>();
      // (every wavefront is past the tile before, whose place the next load takes)
      if (tile + NST - 1 < t1) load(tile + NST - 1);
      const int page = page_id(tile);
      clean(tile, page);
      work(tile, page);
    }

    // ---- the key parts of a row group meet
    lds_barrier();                               // the tiles are read
    float l_tot = half_pair_sum(l_run);
    if constexpr (KG == 2) {
      float* mine = reinterpret_cast<float*>(lds) + (rg * 64 + lane) * XW;
      if (kg == 1) {
        *reinterpret_cast<float2*>(mine) = make_float2(m_run, l_tot);
#pragma unroll
        for (int i = 0; i < 4 * NDB; ++i) {
          const int v = 4 * (i % 4);
          const f32x16& b = o[i / 4];
          *reinterpret_cast<float4*>(mine + 4 + 4 * i) =
              make_float4(b[v], b[v + 1], b[v + 2], b[v + 3]);
        }
      }
      lds_barrier();
      if (kg == 0) {
        const float2 ml = *reinterpret_cast<const float2*>(mine);
        const float m = fmaxf(m_run, ml.x), ref = m == kNegInf ? 0.f : m;
        const float f0 = __builtin_amdgcn_exp2f(m_run - ref);
        const float f1 = __builtin_amdgcn_exp2f(ml.x - ref);
        l_tot = l_tot * f0 + ml.y * f1;
        m_run = m;
#pragma unroll
        for (int i = 0; i < 4 * NDB; ++i) {
          const float4 x = *reinterpret_cast<const float4*>(mine + 4 + 4 * i);
          const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[i / 4][4 * (i % 4) + e] = o[i / 4][4 * (i % 4) + e] * f0 + xs[e] * f1;
        }
      }
    }

    // ---- the rows leave, 64 columns at a time, through LDS of the wavefront's own, so that a
    // store writes whole lines (a lane's own values are 16 bytes of each of 32 rows: 8000
    // cycles a unit of 256 rows).  Values 4 i .. 4 i + 3 of block db are elements 32 db + 8 i +
    // 4 half + 0 .. 3; a row's 16-byte chunks are permuted by its index.
    const bool begins = cur.begins(), ends = cur.ends(), whole = begins && ends;
    if (begins && !ends) join = cur.cut(share);
    if (kg == 0 && rows_here) {
      const float ref = m_run == kNegInf ? 0.f : m_run;
      const float inv = !whole ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
      uint8_t* way = lds + (KG == 2 ? rg * 64 * XW * 4 : wave * OUT);
      const int rows = min(32, nrows - 32 * rg);
      if (half == 0 && col < rows) {
        if (!whole)
          a.part_ml[(size_t(2) * w + (begins ? 1 : 0)) * RB + 32 * rg + col] =
              make_float2(m_run, l_tot);
        else if (a.lse)
          a.lse[size_t(at.r.first + int(t)) * a.Hq + at.g * a.G + row % a.G] =
              l_tot == 0.f ? kNegInf : (ref + __builtin_amdgcn_logf(l_tot)) * kLn2;
      }
#pragma unroll
      for (int d0 = 0; d0 < D; d0 += 64) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const f32x16& b = o[d0 / 32 + i / 4];
          const int v = 4 * (i % 4);
          *reinterpret_cast<float4*>(way + col * 256 + ((2 * i + half) ^ (col & 15)) * 16) =
              make_float4(b[v] * inv, b[v + 1] * inv, b[v + 2] * inv, b[v + 3] * inv);
        }
        // (the wavefront's LDS accesses are in order)
        __builtin_amdgcn_wave_barrier();
        constexpr int CPR = 16;                  // chunks of four elements
        if (F32 || !whole) {
#pragma unroll
          for (int i = 0; i < 32 * CPR / 64; ++i) {
            const int r = (i * 64 + lane) / CPR, c = lane % CPR;
            const float4 x =
                *reinterpret_cast<const float4*>(way + r * 256 + (c ^ (r & 15)) * 16);
            if (r >= rows) continue;
            const int rr = row0 + 32 * rg + r;
            float* to;
            if (!whole) {
              to = a.part_o + ((size_t(2) * w + (begins ? 1 : 0)) * RB + 32 * rg + r) * D;
            } else {
              const unsigned tk = unsigned(rr) / unsigned(a.G);
              to = static_cast<float*>(a.out) +
                   (size_t(at.r.first + int(tk)) * a.Hq + at.g * a.G + (rr - tk * a.G)) * D;
            }
            *reinterpret_cast<float4*>(to + d0 + 4 * c) = x;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32 * CPR / 2 / 64; ++i) {
            const int r = (i * 64 + lane) / (CPR / 2), c = 2 * (lane % (CPR / 2));
            const uint8_t* from = way + r * 256;
            const float4 x = *reinterpret_cast<const float4*>(from + (c ^ (r & 15)) * 16);
            const float4 y = *reinterpret_cast<const float4*>(from + ((c + 1) ^ (r & 15)) * 16);
            if (r >= rows) continue;
            const unsigned rr = row0 + 32 * rg + r, tk = rr / unsigned(a.G);
            T* to = static_cast<T*>(a.out) +
                    (size_t(at.r.first + int(tk)) * a.Hq + at.g * a.G + (rr - tk * a.G)) * D;
            *reinterpret_cast<uint4*>(to + d0 + 4 * c) =
                make_uint4(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w), pack_bf16(y.x, y.y),
                           pack_bf16(y.z, y.w));
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
    p += t1 - t0;
    if (p < share.p1) next_unit(a, RB, limit, at);
    lds_barrier();                               // LDS of this unit is read
  }
  if (tid == 0) a.joins[w] = join;
}

// ----------------------------------------------------------------------------
// join
// ----------------------------------------------------------------------------

// Units that lie in several workgroups.  A set of PW wavefronts takes a row, its wavefronts
// every PW-th piece, a lane D / 64 columns.  Bound by dependent loads (the join, the pieces)
// and the partials' bytes.  Units of few rows have many pieces: PW = 4, and workgroup
// (w, y) takes rows y, y + gridDim.y, .. of the unit that workgroup w began (24 single
// tokens: 5.5 us; an empty launch takes 4).  Blocks have many rows, and how many of them are
// cut depends on the lengths: PW = 1, and all their rows, in one line, are shared evenly (512
// rows of a kv-head over 4128 tokens, 16 pieces each: 30.0 us with workgroups for every share's
// unit, cut or not, 10.1 so; 128 tokens over 100: 7.8 and 4.4; drafts with 32 query heads 4.7 and
// 4.6.  Where most shares are cut, finding the rows costs: drafts with 64 heads 6.4 and 6.0, 2048
// tokens of 64 heads 20.6 and 25.4 of 150 us before them, over 32k 26.5 and 30.6 of 2.0 ms.  1024
// workgroups; 512: 36.5, 2048: the same, but drafts 6.3; 8192: 32.3).
template <typename T, int D, int RB, int PW>
__global__ __launch_bounds__(256) void join_kernel(AttendParams a) {
  constexpr int CPL = D / 64, NW = 4, N = PW > 1 ? 16 : 8;   // columns of a lane; pieces in flight
  constexpr int JPL = 4;                       // joins of a lane, PW = 1
  __shared__ float s_x[NW][D];
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int mine = wave % PW;
  unsigned nrows[JPL] = {}, incl = 0, rows;
  if constexpr (PW > 1) {
    rows = unsigned(a.joins[blockIdx.x].nrows);
  } else {
#pragma unroll
    for (int i = 0; i < JPL; ++i)
      if (JPL * lane + i < a.groups) nrows[i] = unsigned(a.joins[JPL * lane + i].nrows);
    incl = wave_scan((nrows[0] + nrows[1]) + (nrows[2] + nrows[3]));
    rows = unsigned(__builtin_amdgcn_readlane(int(incl), 63));
  }
  // PW = 1: neighbouring rows to a set, so that the join is mostly the one before
  const unsigned set = blockIdx.x * NW + wave, sets = gridDim.x * NW;
  const unsigned each = (rows + sets - 1) / sets;
  const unsigned first = PW > 1 ? blockIdx.y : set * each;
  const unsigned last = PW > 1 ? rows : min(rows, first + each);
  int w0 = blockIdx.x, row = int(first);
  Join jn{};
  if constexpr (PW > 1) jn = a.joins[w0];
  for (unsigned at_row = first; at_row < last; at_row += PW > 1 ? gridDim.y : 1) {
    if constexpr (PW > 1) {
      row = int(at_row);
    } else if (++row >= jn.nrows) {
      const int src = __builtin_ctzll(__ballot(incl > at_row));
      unsigned n[JPL], before = unsigned(__builtin_amdgcn_readlane(int(incl), src));
#pragma unroll
      for (int i = 0; i < JPL; ++i) {
        n[i] = unsigned(__builtin_amdgcn_readlane(int(nrows[i]), src));
        before -= n[i];
      }
      w0 = JPL * src;
      unsigned rest = at_row - before;
#pragma unroll
      for (int i = 0; i < JPL - 1; ++i)
        if (w0 == JPL * src + i && rest >= n[i]) {
          rest -= n[i];
          ++w0;
        }
      row = int(rest);
      jn = a.joins[w0];
    }
    const int pieces = jn.last - w0 + 1;
    // piece k: the second partial of w0, then the first ones of those after it
    auto at = [&](int k, int r) {
      return (size_t(2) * (w0 + k) + (k == 0 ? 1 : 0)) * RB + r;
    };
    float x[CPL] = {}, m = kNegInf, l = 0.f;
    for (int k0 = 0; k0 < pieces; k0 += PW * N) {
      float v[N][CPL];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float* o = a.part_o + at(min(k0 + PW * i + mine, pieces - 1), row) * D + lane * CPL;
#pragma unroll
        for (int e = 0; e < CPL; ++e) v[i][e] = o[e];
      }
      // lane k has the maximum and the sum of piece k0 + k
      float2 ml = make_float2(kNegInf, 0.f);
      if (lane < PW * N && k0 + lane < pieces) ml = a.part_ml[at(k0 + lane, row)];
      float m_new = ml.x;
#pragma unroll
      for (int d = 1; d < PW * N; d *= 2) m_new = fmaxf(m_new, __shfl_xor(m_new, d));
      m_new = fmaxf(m, __shfl(m_new, 0));
      const float ref = m_new == kNegInf ? 0.f : m_new;
      const float keep = __builtin_amdgcn_exp2f(m - ref);
      const float f = __builtin_amdgcn_exp2f(ml.x - ref);
      float sum = f * ml.y;
#pragma unroll
      for (int d = 1; d < PW * N; d *= 2) sum += __shfl_xor(sum, d);
      l = l * keep + __shfl(sum, 0);
      m = m_new;
#pragma unroll
      for (int e = 0; e < CPL; ++e) x[e] *= keep;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (k0 + PW * i + mine >= pieces) continue;
        const float g = __shfl(f, PW * i + mine);
#pragma unroll
        for (int e = 0; e < CPL; ++e) x[e] = __builtin_fmaf(g, v[i][e], x[e]);
      }
    }
    if constexpr (PW > 1) {
      static_assert(PW == NW, "one row a workgroup and turn");
#pragma unroll
      for (int e = 0; e < CPL; ++e) s_x[wave][lane * CPL + e] = x[e];
      __syncthreads();
#pragma unroll
      for (int e = 0; e < CPL; ++e) {
        const int d = lane * CPL + e;
        x[e] = (s_x[0][d] + s_x[1][d]) + (s_x[2][d] + s_x[3][d]);
      }
      __syncthreads();
    }
    if (mine == 0) {
      const unsigned r = jn.row0 + row, t = r / unsigned(a.G);
      const size_t oh = size_t(jn.first + t) * a.Hq + jn.g * a.G + (r - t * a.G);
      const float inv = l == 0.f ? 0.f : 1.f / l;
      T* out = static_cast<T*>(a.out) + oh * D + lane * CPL;
#pragma unroll
      for (int e = 0; e < CPL; ++e) out[e] = from_f<T>(x[e] * inv);
      if (a.lse && lane == 0)
        a.lse[oh] = l == 0.f ? kNegInf
                             : ((m == kNegInf ? 0.f : m) + __builtin_amdgcn_logf(l)) * kLn2;
    }
  }
}

template <typename K>
const void* fn(K* k) { return reinterpret_cast<const void*>(k); }

template <typename T, typename S, int D>
const void* attend_fn(int rows) {
  if constexpr (sizeof(S) == 4) {
    return fn(&attend_wide_kernel<T, S, D, 4>);
  } else {
    if (rows == 16) return fn(&attend_narrow_kernel<S, D, 1>);
    if (rows == 32) return fn(&attend_narrow_kernel<S, D, 2>);
    return rows == 128 ? fn(&attend_wide_kernel<T, S, D, 4>) : fn(&attend_wide_kernel<T, S, D, 8>);
  }
}

template <typename T, int D>
const void* join_fn(int rows) {
  if constexpr (sizeof(T) == 4) {
    return fn(&join_kernel<T, D, 128, 1>);
  } else {
    return rows == 16    ? fn(&join_kernel<T, D, 16, 4>)
           : rows == 32  ? fn(&join_kernel<T, D, 32, 4>)
           : rows == 128 ? fn(&join_kernel<T, D, 128, 1>)
                         : fn(&join_kernel<T, D, 256, 1>);
  }
}

}  // namespace

AttendShape attend_shape(int store, int D, int64_t rows_max, int64_t max_chunk, int64_t batch,
                         int64_t heads, int64_t kv_max) {
  AttendShape s{};
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  const int64_t G = rows_max / max_chunk;
  // Single tokens of up to 32 heads a kv-head: a unit is the token's rows.  Of more heads it would
  // be a part of them, and each part reads the cache again: that pays for int8 alone, whose blocks
  // are slow, and for two parts (24 requests of 1200 to 6200 tokens, with the join, parts | blocks,
  // D = 128: bf16 272 heads over 8 152 | 104 us, 512 over 8 162 | 106, 296 over 8, which 37 parts
  // would divide, 1926 | 104; int8 116 | 109, 128 | 114, 1105 | 111; D = 64: bf16 79 | 68, 92 | 71,
  // 1019 | 69; int8 64 | 135, 77 | 138, 590 | 136).  Chunks of a few tokens run faster in blocks as
  // well, which read the keys once for all of them: 16 requests of 3 to 7 drafts, 4 query heads a
  // kv-head, 95 us in units of 32 mixed rows and their join, 88 in blocks of 128.  fp32 has the
  // 128-row kernel only.
  const int64_t parts = G <= 32 ? 1 : 2;
  if (store != C2KV_F32 && max_chunk == 1 && G <= 32 * parts && G % parts == 0 &&
      (parts == 1 || store == C2KV_I8)) {
    s.unit_rows = int(G / parts);
    s.rows = s.unit_rows <= 16 ? 16 : 32;
  } else {
    s.rows = s.unit_rows = store == C2KV_F32 || rows_max <= 128 ? 128 : 256;
  }
  const double tiles = double(batch) * double(heads) *
                       double((rows_max + s.unit_rows - 1) / s.unit_rows) *
                       double((kv_max + ST - 1) / ST);   // (may pass 64 bits)
  // Two workgroups a CU, or one (4 a lane: joins): of the 32-row kernel two fit at D = 64 only (85
  // KB of LDS at 128; 24 requests of 1200 to 6200 tokens, 256 heads over 8, 512 | 256 workgroups,
  // with the join: D = 128 bf16 118 | 109 us, int8 96 | 83; D = 64 bf16 59 | 62, int8 49 | 53).
  const int64_t most = s.rows == 16 || (s.rows == 32 && D == 64) ? 512 : 256;
  s.groups = int(tiles < most ? tiles : most);
  size_t at = 0;
  s.part_o = at;
  at = up(at + size_t(2) * s.groups * s.rows * D * sizeof(float));
  s.part_ml = at;
  at = up(at + size_t(2) * s.groups * s.rows * sizeof(float2));
  s.joins = at;
  s.total = up(at + size_t(s.groups) * sizeof(Join));
  return s;
}

hipError_t launch_cache_attend(const AttendParams& p, const AttendShape& sh, int store, int D,
                               hipStream_t st, hipEvent_t e0, hipEvent_t e1) {
  return with_types(store, D, [&](auto t, auto s, auto d) {
    return launch(attend_fn<decltype(t), decltype(s), decltype(d)::value>(sh.rows),
                  dim3(unsigned(sh.groups)), dim3(sh.rows <= 32 ? 256 : 512), st, p, e0, e1);
  });
}

hipError_t launch_cache_merge(const AttendParams& p, const AttendShape& sh, int store, int D,
                              hipStream_t st, hipEvent_t e0, hipEvent_t e1) {
  return with_types(store, D, [&](auto t, auto, auto d) {
    return launch(join_fn<decltype(t), decltype(d)::value>(sh.rows),
                  sh.rows <= 32 ? dim3(unsigned(sh.groups), 4)
                                : dim3(unsigned(min(1024, sh.groups * (sh.rows / 4)))),
                  dim3(256), st, p, e0, e1);
  });
}

}  // namespace c2kv
