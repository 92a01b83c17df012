// HIP kernels of the growing paged cache for gfx950 (CDNA4).
//
//   write_rows_kernel   new tokens into pages, a wavefront per (token, kv-head)
//   write_tile_kernel   the same for chunks, a workgroup per 64 cache slots
//   read_tile_kernel    cached tokens back to rows
//   pool_write_kernel   rows into the chunk pool
//
// Lengths, offsets and page numbers are read on the device, so that a captured step
// can be replayed as they grow.  They are clamped to the buffers that the host named:
// whatever they hold, nothing outside those is touched.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "cache.hpp"
#include "cache_device.hpp"

namespace c2kv {

namespace {

// Unit u of the batch, where each request has as many units as its chunk has tiles.
// Searched by a whole wavefront; -1 past the last.
__device__ inline int find_tile(const ChunkView& c, int limit, int u, Req& r, int& tile) {
  const int lane = threadIdx.x & 63;
  int seen = 0;
  for (int b0 = 0; b0 < c.batch; b0 += 64) {
    const int b = b0 + lane;
    const Req mine = request(c, min(b, c.batch - 1));
    const Tiles t = b < c.batch ? chunk_tiles(mine, limit) : Tiles{0, 0};
    int incl = t.n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int x = __shfl_up(incl, d);
      if (lane >= d) incl += x;
    }
    const uint64_t past = __ballot(seen + incl > u);
    if (past) {
      const int src = __builtin_ctzll(past);
      r = lane_req(mine, src);
      tile = uniform(__shfl(t.t0 + u - (seen + incl - t.n), src));
      return b0 + src;
    }
    seen += uniform(__shfl(incl, 63));
  }
  return -1;
}

// ----------------------------------------------------------------------------
// stores
// ----------------------------------------------------------------------------

// Stores of whole 128-byte lines (16 bytes a lane of rows of bf16, and of value pages) are
// marked as not read again soon: the lines stream out instead of waiting in the L2s beside
// what is still read.  16384 tokens, bf16: written in 34 -> 24.4 us (5.5 TB/s), read back in
// 32.8 -> 23.6, stored in a pool in 30 -> 22.4; int8 tokens written in 32 -> 23 and, not
// found in the L2s, read back in 21 instead of 19.  Not for fp32, whose lanes write half a
// line at a time (61 -> 73 us), nor the 8-byte rows of int8 codes (65536 into a pool 107 ->
// 115).
__device__ inline void stream16(void* p, uint4 v) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 x = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(x, static_cast<u32x4*>(p));
}
__device__ inline void stream8(float* p, const float (&x)[8]) { store8(p, x); }
__device__ inline void stream8(__bf16* p, const float (&x)[8]) {
  stream16(p, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                         pack_bf16(x[6], x[7])));
}

// ----------------------------------------------------------------------------
// RoPE and int8
// ----------------------------------------------------------------------------

// Largest magnitude of what has been seen; a NaN stays.
__device__ inline float max_mag(float m, float x, float y) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, __builtin_fabsf(x)),
                                       __builtin_fabsf(y));
}
// its maximum over groups of LANES neighbouring lanes, by lane moves inside the VALU up to 16
template <int CTRL>
__device__ inline float max_with(float m) {
  return __builtin_elementwise_maximum(
      m, __uint_as_float(__builtin_amdgcn_update_dpp(0, int(__float_as_uint(m)), CTRL, 0xf, 0xf,
                                                     true)));
}
template <int LANES>
__device__ inline float lanes_max(float m) {
  m = max_with<0xb1>(m);                      // lane ^ 1
  m = max_with<0x4e>(m);                      // lane ^ 2
  if constexpr (LANES >= 8) m = max_with<0x141>(m);    // the other four of eight (mirrored)
  if constexpr (LANES >= 16) m = max_with<0x140>(m);   // the other eight of sixteen
#pragma unroll
  for (int d = 16; d < LANES; d *= 2) m = __builtin_elementwise_maximum(m, __shfl_xor(m, d));
  return m;
}

// Symmetric int8 of a row whose largest magnitude is m: scale = m / 127, code = x / scale, the
// quotient rounded to fp32 and then to the nearest whole number (halves to the even one).  The
// quotient is a product with the scale's reciprocal and one correction by what that leaves of x,
// which is the division's own result: both remainders are exact in a fused multiply-add (tried
// over all pairs of bf16 numbers and 6e8 fp32 ones next to halves, the reciprocal off by one unit
// either way).  Adding 1.5 * 2^23 rounds it to a whole number, in the low bits of the sum in two's
// complement.  No |quotient| passes 127.5, so nothing is clamped.  (16384 tokens written in 21.1
// us, in 20.7 without the correction, which rounds 53 of those 155712 bf16 pairs otherwise; the
// compiler's division an element bounded these kernels, 41 us against 32 before their stores
// streamed.)  A row below 2^-100, whose
// reciprocal would leave the range, is stored as zeros; one with an infinity or a NaN gets a NaN
// scale, whatever its codes.
struct I8Row {
  float scale, inv;
  __device__ explicit I8Row(float m) {
    const float c = 1.f / 127.f;
    float s = m * c;
    s = __builtin_fmaf(__builtin_fmaf(-s, 127.f, m), c, s);      // correctly rounded
    float r = __builtin_amdgcn_rcpf(s);
    r = __builtin_fmaf(__builtin_fmaf(-s, r, 1.f), r, r);
    const bool tiny = m < 0x1p-100f;
    scale = m < __builtin_huge_valf() ? (tiny ? 1.f : s) : __builtin_nanf("");
    inv = tiny ? 0.f : r;
  }
  // the code as the low byte of a word
  __device__ uint32_t code(float x) const {
    const float q = x * inv;
    return __float_as_uint(__builtin_fmaf(__builtin_fmaf(-q, scale, x), inv, q) + 12582912.f);
  }
  __device__ uint32_t pack4(const float* x) const {
    const uint32_t lo = __builtin_amdgcn_perm(code(x[1]), code(x[0]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(code(x[3]), code(x[2]), 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
  }
};

// 8 floats -> 8 consecutive stored elements
template <typename S>
__device__ inline void put8(S* p, const float (&x)[8], const I8Row& row) {
  if constexpr (sizeof(S) == 1)
    *reinterpret_cast<uint2*>(p) = make_uint2(row.pack4(x), row.pack4(x + 4));
  else
    stream8(p, x);
}

// the word of one element of two neighbouring tokens
template <typename S> struct PairOf { using type = uint32_t; };
template <> struct PairOf<float> { using type = float2; };
template <> struct PairOf<int8_t> { using type = uint16_t; };
template <typename S>
__device__ inline typename PairOf<S>::type pair_of(float a, float b, const I8Row& ra,
                                                   const I8Row& rb) {
  if constexpr (sizeof(S) == 4) return make_float2(a, b);
  else if constexpr (sizeof(S) == 2) return pack_bf16(a, b);
  else return uint16_t(__builtin_amdgcn_perm(rb.code(b), ra.code(a), 0x0c0c0400u));
}

// LDS tile of transposed values: D rows of ST tokens, each row's 16-byte blocks permuted
// by the row / 16, which spreads the columns that a wavefront's rows write over the banks.
template <typename S, int D>
struct ValueTile {
  static constexpr int EPV = 16 / int(sizeof(S));    // tokens per block
  static constexpr int BLOCKS = ST / EPV;
  static constexpr int LD = ST + EPV;
  __device__ static int col(int d, int token) {
    return token ^ (EPV * ((d >> 4) & (BLOCKS - 1)));
  }
};

// ----------------------------------------------------------------------------
// write
// ----------------------------------------------------------------------------

// A wavefront per (token, kv-head): lane i holds the key pair (i, i + D/2).  For few tokens,
// or few of each request: bound by latency (two dependent loads: the requests, the page; 24
// requests' tokens, 8 heads of 128 in bf16: 4.0 us, an empty launch's time).
template <typename T, typename S, int D>
__global__ __launch_bounds__(256) void write_rows_kernel(WriteParams a) {
  constexpr int VPL = D / 64;                // values per lane
  const int lane = threadIdx.x & 63;
  const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int token = unit / a.pg.Hkv, g = unit % a.pg.Hkv;
  if (token >= a.ch.n_tokens) return;
  const T* krow = static_cast<const T*>(a.k) + token * a.k_stride + g * D;
  const T* vrow = static_cast<const T*>(a.v) + token * a.v_stride + g * D;
  const int i = lane & (D / 2 - 1);
  float x = to_f(krow[i]), y = to_f(krow[i + D / 2]);
  float v[VPL];
#pragma unroll
  for (int e = 0; e < VPL; ++e) v[e] = to_f(vrow[lane * VPL + e]);
  const int pos = a.rope.pos ? a.rope.pos[token] : 0;

  Req r;
  const int b = find_row(a.ch, token, r);
  if (b < 0) return;
  const int j = r.base + token - r.first;
  if (j < 0) return;
  const int page = page_of(a.ch, a.pg, b, j);
  if (page < 0) return;
  const size_t ph = size_t(page) * a.pg.Hkv + g;
  const int off = j % a.pg.PS;

  if (a.rope.pos) {
    float c, s;
    turn_cs(pos, a.rope.turns[i], c, s);
    rotate_pair(x, y, c, s);
  }
  S* kp = static_cast<S*>(a.pg.k) + (ph * a.pg.PS + off) * D;
  S* vp = static_cast<S*>(a.pg.v) + ph * D * a.pg.PS + off;
  if constexpr (sizeof(S) == 1) {
    const I8Row ks(lanes_max<64>(max_mag(0.f, x, y)));
    const I8Row vs(lanes_max<64>(max_mag(0.f, v[0], v[VPL - 1])));
    if (lane == 0) {
      a.pg.k_scale[ph * a.pg.PS + off] = ks.scale;
      a.pg.v_scale[ph * a.pg.PS + off] = vs.scale;
    }
    if (lane < D / 2) {
      kp[i] = int8_t(ks.code(x));
      kp[i + D / 2] = int8_t(ks.code(y));
    }
#pragma unroll
    for (int e = 0; e < VPL; ++e) vp[size_t(lane * VPL + e) * a.pg.PS] = int8_t(vs.code(v[e]));
  } else {
    if (lane < D / 2) {
      kp[i] = from_f<S>(x);
      kp[i + D / 2] = from_f<S>(y);
    }
#pragma unroll
    for (int e = 0; e < VPL; ++e) vp[size_t(lane * VPL + e) * a.pg.PS] = from_f<S>(v[e]);
  }
}

// A workgroup per 64-slot tile of a request that its chunk touches, for the kv-heads
// blockIdx.y, blockIdx.y + gridDim.y, ...: keys by rows, values transposed through LDS.
// The turn of a (token, 8 pairs) unit is formed once for all of a workgroup's heads.  Bound by
// HBM: 16384 tokens of 8 heads of 128 in bf16 (134 MB), 24.5 us = 5.5 TB/s, a 1 GiB copy 5.2;
// int8, 9400 tokens of ragged prompts (58 MB): 16 us, 3.6 TB/s, 4 us of it the launch.
template <typename T, typename S, int D>
__global__ __launch_bounds__(256) void write_tile_kernel(WriteParams a) {
  constexpr int NTH = 256;
  constexpr int KU = D / 16, NKU = ST * KU / NTH;
  constexpr int VU = D / 8, NVU = ST / 2 * VU / NTH;
  using VT = ValueTile<S, D>;
  __shared__ __attribute__((aligned(16))) S sV[D * VT::LD];
  const int tid = threadIdx.x, PS = a.pg.PS;
  Req r;
  int tile;
  const int b = find_tile(a.ch, a.ch.max_pages * PS, blockIdx.x, r, tile);
  if (b < 0) return;
  const int page = page_of(a.ch, a.pg, b, tile * ST);
  if (page < 0) return;
  const int off = tile * ST % PS;
  const auto [lo, hi, row0] = tile_slots(r, tile);

  float kc[NKU][8], kn[NKU][8];
  if (a.rope.pos) {
#pragma unroll
    for (int i = 0; i < NKU; ++i) {
      const int u = tid + i * NTH;
      const int pos = a.rope.pos[row0 + min(max(u / KU, lo), hi - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        turn_cs(pos, a.rope.turns[8 * (u % KU) + e], kc[i][e], kn[i][e]);
    }
  }

  for (int g = blockIdx.y; g < a.pg.Hkv; g += gridDim.y) {
    const size_t ph = size_t(page) * a.pg.Hkv + g;
    S* kp = static_cast<S*>(a.pg.k) + (ph * PS + off) * D;
    S* vp = static_cast<S*>(a.pg.v) + ph * D * PS + off;
    float x[NKU][8], y[NKU][8], v[NVU][2][8];
#pragma unroll
    for (int i = 0; i < NKU; ++i) {
      const int u = tid + i * NTH;
      const T* src = static_cast<const T*>(a.k) + g * D + 8 * (u % KU) +
                     (row0 + min(max(u / KU, lo), hi - 1)) * a.k_stride;
      load8(src, x[i]);
      load8(src + D / 2, y[i]);
    }
#pragma unroll
    for (int i = 0; i < NVU; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int u = tid + i * NTH;
        load8(static_cast<const T*>(a.v) + g * D + 8 * (u % VU) +
                  (row0 + min(max(2 * (u / VU) + j, lo), hi - 1)) * a.v_stride,
              v[i][j]);
      }
    // ---- keys
#pragma unroll
    for (int i = 0; i < NKU; ++i) {
      const int u = tid + i * NTH;
      const int slot = u / KU, c = u % KU;
      if (a.rope.pos) rotate8(x[i], y[i], kc[i], kn[i]);
      float m = 0.f;
      if constexpr (sizeof(S) == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max_mag(m, x[i][e], y[i][e]);
        m = lanes_max<KU>(m);
      }
      const I8Row q(m);
      if (slot >= lo && slot < hi) {
        if (sizeof(S) == 1 && c == 0) a.pg.k_scale[ph * PS + off + slot] = q.scale;
        put8(kp + slot * D + 8 * c, x[i], q);
        put8(kp + slot * D + 8 * c + D / 2, y[i], q);
      }
    }
    // ---- values: words of two tokens into LDS rows, then rows of 16-byte blocks out
#pragma unroll
    for (int i = 0; i < NVU; ++i) {
      const int u = tid + i * NTH;
      const int slot = 2 * (u / VU), c = u % VU;
      float m[2] = {0.f, 0.f};
      if constexpr (sizeof(S) == 1) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) m[j] = max_mag(m[j], v[i][j][e], v[i][j][e + 1]);
          m[j] = lanes_max<VU>(m[j]);
        }
      }
      const I8Row q0(m[0]), q1(m[1]);
      if (sizeof(S) == 1 && c == 0) {
        if (slot >= lo && slot < hi) a.pg.v_scale[ph * PS + off + slot] = q0.scale;
        if (slot + 1 >= lo && slot + 1 < hi) a.pg.v_scale[ph * PS + off + slot + 1] = q1.scale;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = 8 * c + e;
        *reinterpret_cast<typename PairOf<S>::type*>(sV + d * VT::LD + VT::col(d, slot)) =
            pair_of<S>(v[i][0][e], v[i][1][e], q0, q1);
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < D * VT::BLOCKS / NTH; ++i) {
      const int u = tid + i * NTH;
      const int d = u / VT::BLOCKS, s0 = u % VT::BLOCKS * VT::EPV;
      const S* from = sV + d * VT::LD + VT::col(d, s0);
      S* to = vp + size_t(d) * PS + s0;
      if (s0 >= lo && s0 + VT::EPV <= hi) {
        const uint4 v16 = *reinterpret_cast<const uint4*>(from);
        if constexpr (sizeof(S) == 4) *reinterpret_cast<uint4*>(to) = v16;
        else stream16(to, v16);
      } else {
#pragma unroll
        for (int e = 0; e < VT::EPV; ++e)
          if (s0 + e >= lo && s0 + e < hi) to[e] = from[e];
      }
    }
    __syncthreads();
  }
}

// ----------------------------------------------------------------------------
// read
// ----------------------------------------------------------------------------

// The tiles of write_tile_kernel the other way: rows in the activation type, int8 decoded
// and keys turned in fp32, rounded once.  Bound by HBM: 32768 int8 tokens (204 MB) in 33 us =
// 6.1 TB/s.
template <typename T, typename S, int D>
__global__ __launch_bounds__(256) void read_tile_kernel(ReadParams a) {
  constexpr int NTH = 256;
  constexpr int KU = D / 16, NKU = ST * KU / NTH;
  constexpr int VU = D / 8, NVU = ST / 2 * VU / NTH;
  using VT = ValueTile<S, D>;
  constexpr int NB = D * VT::BLOCKS / NTH;
  __shared__ __attribute__((aligned(16))) S sV[D * VT::LD];
  const int tid = threadIdx.x, PS = a.pg.PS;
  Req r;
  int tile;
  const int b = find_tile(a.ch, a.ch.max_pages * PS, blockIdx.x, r, tile);
  if (b < 0) return;
  const int page = page_of(a.ch, a.pg, b, tile * ST);
  if (page < 0) return;
  const int off = tile * ST % PS;
  const auto [lo, hi, row0] = tile_slots(r, tile);

  float kc[NKU][8], kn[NKU][8];
  if (a.rope.pos) {
#pragma unroll
    for (int i = 0; i < NKU; ++i) {
      const int u = tid + i * NTH;
      const int pos = a.rope.pos[row0 + min(max(u / KU, lo), hi - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        turn_cs(pos, a.rope.turns[8 * (u % KU) + e], kc[i][e], kn[i][e]);
    }
  }

  for (int g = blockIdx.y; g < a.pg.Hkv; g += gridDim.y) {
    const size_t ph = size_t(page) * a.pg.Hkv + g;
    const S* kp = static_cast<const S*>(a.pg.k) + (ph * PS + off) * D;
    const S* vp = static_cast<const S*>(a.pg.v) + ph * D * PS + off;
    uint4 blocks[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int u = tid + i * NTH;
      blocks[i] = *reinterpret_cast<const uint4*>(vp + size_t(u / VT::BLOCKS) * PS +
                                                  u % VT::BLOCKS * VT::EPV);
    }
    float x[NKU][8], y[NKU][8];
#pragma unroll
    for (int i = 0; i < NKU; ++i) {
      const int u = tid + i * NTH;
      const S* src = kp + (u / KU) * D + 8 * (u % KU);
      load8(src, x[i]);
      load8(src + D / 2, y[i]);
      if constexpr (sizeof(S) == 1) {
        const float scale = a.pg.k_scale[ph * PS + off + u / KU];
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[i][e] *= scale; y[i][e] *= scale; }
      }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int u = tid + i * NTH;
      const int d = u / VT::BLOCKS;
      *reinterpret_cast<uint4*>(sV + d * VT::LD + VT::col(d, u % VT::BLOCKS * VT::EPV)) =
          blocks[i];
    }
#pragma unroll
    for (int i = 0; i < NKU; ++i) {
      const int u = tid + i * NTH;
      const int slot = u / KU;
      if (a.rope.pos) rotate8(x[i], y[i], kc[i], kn[i]);
      if (slot >= lo && slot < hi) {
        T* to = static_cast<T*>(a.k) + (size_t(row0 + slot) * a.pg.Hkv + g) * D + 8 * (u % KU);
        stream8(to, x[i]);
        stream8(to + D / 2, y[i]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NVU; ++i) {
      const int u = tid + i * NTH;
      const int slot = 2 * (u / VU), c = u % VU;
      float v[2][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = 8 * c + e;
        const S* from = sV + d * VT::LD + VT::col(d, slot);
        if constexpr (sizeof(S) == 1) {
          v[0][e] = float(from[0]);
          v[1][e] = float(from[1]);
        } else {
          v[0][e] = to_f(from[0]);
          v[1][e] = to_f(from[1]);
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (slot + j < lo || slot + j >= hi) continue;
        if constexpr (sizeof(S) == 1) {
          const float scale = a.pg.v_scale[ph * PS + off + slot + j];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[j][e] *= scale;
        }
        stream8(static_cast<T*>(a.v) + (size_t(row0 + slot + j) * a.pg.Hkv + g) * D + 8 * c, v[j]);
      }
    }
    __syncthreads();
  }
}

// ----------------------------------------------------------------------------
// pool write
// ----------------------------------------------------------------------------

// A thread per (token, 8 pairs): the unit's keys (and the values of the same columns) for
// the kv-heads blockIdx.y, blockIdx.y + gridDim.y, ..., its turn formed once for all.  Bound by
// HBM: 65536 tokens into int8 (407 MB) in 106 us = 3.9 TB/s; their codes leave as 8 bytes a
// thread (exchanged into 16 first: no faster), a 4-byte scale a row beside them.
template <typename T, typename S, int D>
__global__ __launch_bounds__(256) void pool_write_kernel(PoolWriteParams a) {
  constexpr int KU = D / 16, TOKENS = 256 / KU;
  const int c = threadIdx.x % KU;
  const int64_t token = int64_t(blockIdx.x) * TOKENS + threadIdx.x / KU;
  const bool in = token < a.n;
  const int64_t t = in ? token : a.n - 1;
  const int64_t row = a.row[t];
  const bool ok = in && row >= 0 && row < a.n_rows;
  float kc[8], kn[8];
  if (a.rope.pos) {
    const int pos = a.rope.pos[t];
#pragma unroll
    for (int e = 0; e < 8; ++e) turn_cs(pos, a.rope.turns[8 * c + e], kc[e], kn[e]);
  }
  for (int g = blockIdx.y; g < a.Hkv; g += gridDim.y) {
    float x[2][8], y[2][8];                    // keys, values
    const T* k = static_cast<const T*>(a.k) + t * a.k_stride + g * D + 8 * c;
    const T* v = static_cast<const T*>(a.v) + t * a.v_stride + g * D + 8 * c;
    load8(k, x[0]);
    load8(k + D / 2, y[0]);
    load8(v, x[1]);
    load8(v + D / 2, y[1]);
    if (a.rope.pos) rotate8(x[0], y[0], kc, kn);
    float m[2] = {0.f, 0.f};
    if constexpr (sizeof(S) == 1) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m[j] = max_mag(m[j], x[j][e], y[j][e]);
        m[j] = lanes_max<KU>(m[j]);
      }
    }
    const I8Row qk(m[0]), qv(m[1]);
    if (!ok) continue;
    const size_t rh = size_t(row) * a.Hkv + g;
    S* pk = static_cast<S*>(a.pool_k) + rh * D + 8 * c;
    S* pv = static_cast<S*>(a.pool_v) + rh * D + 8 * c;
    put8(pk, x[0], qk);
    put8(pk + D / 2, y[0], qk);
    put8(pv, x[1], qv);
    put8(pv + D / 2, y[1], qv);
    if constexpr (sizeof(S) == 1) {
      if (c == 0) {
        a.k_scale[rh] = qk.scale;
        a.v_scale[rh] = qv.scale;
      }
    }
  }
}

}  // namespace

// ----------------------------------------------------------------------------
// launchers
// ----------------------------------------------------------------------------

namespace {

// Heads one workgroup runs through: all of them where the tiles alone fill the GPU four
// times over, fewer where they do not (the turns are then formed again per workgroup).
int head_groups(int64_t tiles, int heads) {
  const int64_t want = (4 * 256 + tiles - 1) / (tiles > 0 ? tiles : 1);
  return int(want < 1 ? 1 : want > heads ? heads : want);
}

}  // namespace

hipError_t launch_cache_write(const WriteParams& p, int store, int D, int max_chunk,
                              hipStream_t st, hipEvent_t e0, hipEvent_t e1) {
  return with_types(store, D, [&](auto t, auto s, auto d) {
    using T = decltype(t);
    using S = decltype(s);
    constexpr int kD = decltype(d)::value;
    if (write_by_rows(p.ch.n_tokens, p.pg.Hkv, max_chunk)) {
      return launch(reinterpret_cast<const void*>(&write_rows_kernel<T, S, kD>),
                    dim3(unsigned(row_groups(p.ch.n_tokens, p.pg.Hkv))), dim3(256), st, p, e0, e1);
    }
    const int64_t tiles = most_chunk_tiles(p.ch.n_tokens, p.ch.batch);
    return launch(reinterpret_cast<const void*>(&write_tile_kernel<T, S, kD>),
                  dim3(unsigned(tiles), head_groups(tiles, p.pg.Hkv)), dim3(256), st, p, e0, e1);
  });
}

hipError_t launch_cache_read(const ReadParams& p, int store, int D, hipStream_t st,
                             hipEvent_t e0, hipEvent_t e1) {
  return with_types(store, D, [&](auto t, auto s, auto d) {
    using T = decltype(t);
    using S = decltype(s);
    const int64_t tiles = most_chunk_tiles(p.ch.n_tokens, p.ch.batch);
    return launch(reinterpret_cast<const void*>(&read_tile_kernel<T, S, decltype(d)::value>),
                  dim3(unsigned(tiles), head_groups(tiles, p.pg.Hkv)), dim3(256), st, p, e0, e1);
  });
}

hipError_t launch_pool_write(const PoolWriteParams& p, int store, int D, hipStream_t st,
                             hipEvent_t e0, hipEvent_t e1) {
  return with_types(store, D, [&](auto t, auto s, auto d) {
    using T = decltype(t);
    using S = decltype(s);
    constexpr int kD = decltype(d)::value, kTokens = 256 / (kD / 16);
    const int64_t blocks = (int64_t(p.n) + kTokens - 1) / kTokens;
    return launch(reinterpret_cast<const void*>(&pool_write_kernel<T, S, kD>),
                  dim3(unsigned(blocks), head_groups(blocks, p.Hkv)), dim3(256), st, p, e0, e1);
  });
}

}  // namespace c2kv
