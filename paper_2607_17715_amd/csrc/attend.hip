// Attention of chunks of new tokens over a growing paged cache, for gfx950 (CDNA4).
//
//   attend_narrow_kernel   few query rows a unit (single tokens, drafts): every wavefront
//                          reads its own keys straight into MFMA operands
//   join_kernel            log-sum-exp combine of units that lie in several workgroups
//
// The work of a launch is one line of key tiles (cache_index.hpp), shared evenly by its
// workgroups on the device, where the lengths are.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache.hpp"
#include "cache_device.hpp"

namespace c2kv {

namespace {

typedef float f32x4 __attribute__((__vector_size__(4 * sizeof(float))));
typedef uint32_t u32x4 __attribute__((__vector_size__(4 * sizeof(uint32_t))));

// ----------------------------------------------------------------------------
// a workgroup's share of the line of tiles
// ----------------------------------------------------------------------------

template <typename N>
__device__ inline N wave_scan(N x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const N y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}
__device__ inline int64_t uniform64(int64_t x) {
  return int64_t(uint64_t(uint32_t(uniform(int(x >> 32)))) << 32 | uint32_t(uniform(int(x))));
}

// Where a workgroup is on the line: unit (b, g, i) with row block i, the unit's tiles, and
// the tile at which the workgroup enters it.
struct Place {
  Req r;
  int b, g, i, tiles, tile;
};

// The launch's tiles in all, and the place of the first tile of this workgroup's share
// [p0, p1); the same in every wavefront.  A share is at least `least` tiles where the line
// is that long; workgroups past the last share get an empty one.
struct Share {
  int64_t total, p0, p1;
  int groups;
};

template <int RB>
__device__ inline Share find_share(const AttendParams& a, int limit, int least, Place& at) {
  const int lane = threadIdx.x & 63;
  Share s{};
  Req mine{};
  int64_t cost = 0, incl = 0;
  auto step = [&](int b0) {
    const int b = b0 + lane;
    mine = request(a.ch, min(b, a.ch.batch - 1));
    cost = b < a.ch.batch ? head_tiles(mine, a.G, RB, limit) * a.pg.Hkv : 0;
    incl = wave_scan(cost);
    return uniform64(__shfl(incl, 63));
  };
  for (int b0 = 0; b0 < a.ch.batch; b0 += 64) s.total += step(b0);
  if (s.total == 0) return s;
  const int64_t most = (s.total + least - 1) / least;
  s.groups = int(most < gridDim.x ? most : int64_t(gridDim.x));
  const int w = blockIdx.x;
  if (w >= s.groups) return s;
  s.p0 = share_begin(s.total, s.groups, w);
  s.p1 = share_begin(s.total, s.groups, w + 1);
  int64_t seen = 0;
  for (int b0 = 0; b0 < a.ch.batch; b0 += 64) {
    const int64_t here = a.ch.batch > 64 ? step(b0) : s.total;
    if (s.p0 < seen + here) {
      const int src = __builtin_ctzll(__ballot(seen + incl > s.p0));
      at.r = lane_req(mine, src);
      at.b = b0 + src;
      int64_t rest = s.p0 - uniform64(__shfl(seen + incl - cost, src));
      const int64_t per_head = uniform64(__shfl(cost, src)) / a.pg.Hkv;
      at.g = int(rest / per_head);
      rest -= at.g * per_head;
      at.i = 0;
      while (rest >= (at.tiles = unit_tiles(at.r, a.G, RB, at.i, limit))) {
        rest -= at.tiles;
        ++at.i;
      }
      at.tile = int(rest);
      return s;
    }
    seen += here;
  }
  return s;
}

// The unit after `at`, entered at its first tile.
template <int RB>
__device__ inline void next_unit(const AttendParams& a, int limit, Place& at) {
  if (++at.i >= row_blocks(at.r, a.G, RB)) {
    at.i = 0;
    if (++at.g >= a.pg.Hkv) {
      at.g = 0;
      do {
        ++at.b;
        at.r = request(a.ch, at.b);
      } while (at.r.n == 0);
    }
  }
  at.tiles = unit_tiles(at.r, a.G, RB, at.i, limit);
  at.tile = 0;
}

// The join of the unit that this workgroup's share begins, and ends inside before tile t1.
template <int RB>
__device__ inline Join cut_unit(const AttendParams& a, const Share& s, const Place& at, int t1) {
  Join j{};
  j.first = at.r.first;
  j.row0 = at.i * RB;
  j.nrows = int(min(int64_t(RB), int64_t(at.r.n) * a.G - j.row0));
  j.g = at.g;
  j.last = share_of(s.total, s.groups, s.p1 + (at.tiles - t1) - 1);
  return j;
}

// ----------------------------------------------------------------------------
// rows
// ----------------------------------------------------------------------------

// cos and sin of the turns of a unit's tokens, [token - first token][pair]
template <int RB, int D>
__device__ inline void unit_turns(const AttendParams& a, const Place& at, int row0, int nrows,
                                  float2* cs) {
  const int t0 = row0 / a.G, nt = (row0 + nrows - 1) / a.G - t0 + 1;
  for (int i = threadIdx.x; i < nt * (D / 2); i += blockDim.x) {
    float c, s;
    turn_cs(a.rope.pos[at.r.first + t0 + i / (D / 2)], a.rope.turns[i % (D / 2)], c, s);
    cs[i] = make_float2(c, s);
  }
}

// 8 consecutive elements d0 .. d0 + 7 of a query row, turned and scaled
template <typename T, int D>
__device__ inline void query8(const T* row, int d0, const float2* cs, float scale,
                              float (&out)[8]) {
  const int lo = d0 % (D / 2);
  if (!cs) {
    load8(row + d0, out);
  } else {
    float x[8], y[8];
    load8(row + lo, x);
    load8(row + lo + D / 2, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 w = cs[lo + e];
      rotate_pair(x[e], y[e], w.x, w.y);
      out[e] = d0 < D / 2 ? x[e] : y[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] *= scale;
}

__device__ inline bf16x8 bf16_of(const float (&x)[8]) {
  const uint4 u = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                             pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  return __builtin_bit_cast(bf16x8, u);
}
__device__ inline bf16x8 bf16_of_i8(uint32_t w0, uint32_t w1) {
  const uint32_t w[2] = {w0, w1};
  float x[8];
  raw_to_f8<int8_t>(w, x);
  return bf16_of(x);                       // exact: codes have seven bits
}

// value of lane k of this lane's group of 16 (a DPP operand of what uses it)
template <int K>
__device__ inline float lane16(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, int(__float_as_uint(x)), 0x150 + K, 0xf,
                                                     0xf, true));
}

// ----------------------------------------------------------------------------
// few rows
// ----------------------------------------------------------------------------

// A unit is 16 NB query rows; a workgroup's four wavefronts take contiguous quarters of
// its tiles and meet only at a unit's end.  Scores are computed transposed, keys x rows,
// in 16x16x32 MFMAs: lane l has column (query row) l % 16 and, of the 8 U keys that its
// group j = l / 16 holds, all of a step's scores.  Keys are dealt to MFMA rows so that
// these are 8 U consecutive keys, which is what the lane feeds to the P*V product, against
// 16 bytes of a transposed value row: operands go from memory to the MFMA without LDS and
// without a lane exchange.  A step is 8 KB of keys and 8 KB of values (D = 128); two are
// in flight (one where 32 rows leave no registers for the second).
//
// int8 codes become bf16 exactly; key scales multiply the scores, value scales the
// probabilities, in fp32.
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
  __shared__ float2 s_cs[RB * (D / 2)];

  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const int col = lane & 15, j = lane >> 4;
  const int PS = a.pg.PS, limit = a.ch.max_pages * PS;
  // two tiles a workgroup at least: fewer leave wavefronts without a step
  Place at;
  const Share share = find_share<RB>(a, limit, I8 ? 4 : 2, at);
  Join join{};
  int64_t p = share.p0;

  while (p < share.p1) {
    const int row0 = at.i * RB;
    const int nrows = int(min(int64_t(RB), int64_t(at.r.n) * a.G - row0));
    const int t0 = at.tile;
    const int t1 = int(min(int64_t(at.tiles), t0 + (share.p1 - p)));
    const int keys = unit_keys(at.r, a.G, RB, at.i, limit);

    // ---- this wavefront's steps and their loads
    const int n_steps = (t1 - t0) * SPT;
    const int s0 = t0 * SPT + n_steps * wave / NW, s1 = t0 * SPT + n_steps * (wave + 1) / NW;
    const int32_t* table = a.ch.table + size_t(at.b) * a.ch.max_pages;
    int ids = -1, ids_from = -(1 << 30);     // pages of tiles ids_from + lane
    struct Set {
      u32x4 k[NKF], v[NVF];
      float ks, vs;
      int page;
    } set[SETS];
    auto fetch = [&](int step, Set& x) __attribute__((always_inline)) {
      const int tile = step / SPT;
      if (unsigned(tile - ids_from) >= 64u) {
        ids_from = tile;
        const int c = (tile + lane) * ST / PS;
        ids = valid_page(table[min(c, a.ch.max_pages - 1)], a.pg.n_pages);
      }
      x.page = __builtin_amdgcn_readlane(ids, tile - ids_from);
      // past the last step, and where there is no page: descriptors without extent, whose
      // loads give zeros and touch no memory
      const bool real = step < s1 && x.page >= 0;
      const size_t ph = size_t(real ? x.page : 0) * a.pg.Hkv + at.g;
      const int off = (step * KS) % PS;
      const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(
          static_cast<S*>(a.pg.k) + (ph * PS + off) * D, 0, real ? KS * D * SZ : 0, kBufferFlags);
      const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(
          static_cast<S*>(a.pg.v) + ph * D * PS + off, 0,
          real ? ((D - 1) * PS + KS) * SZ : 0, kBufferFlags);
      const int kofs = (8 * U * (col >> 2) + (col & 3)) * D * SZ + 16 * j;
#pragma unroll
      for (int m = 0; m < 2 * U; ++m)
#pragma unroll
        for (int c = 0; c < NKC; ++c)
          x.k[m * NKC + c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
              kr, kofs + 4 * m * D * SZ + 64 * c, 0, 0));
#pragma unroll
      for (int db = 0; db < NVF; ++db)
        x.v[db] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
            vr, (16 * db + col) * PS * SZ + 16 * j, 0, 0));
      if constexpr (I8) {
        const __amdgpu_buffer_rsrc_t ksr = __builtin_amdgcn_make_buffer_rsrc(
            a.pg.k_scale + ph * PS + off, 0, real ? KS * 4 : 0, kBufferFlags);
        const __amdgpu_buffer_rsrc_t vsr = __builtin_amdgcn_make_buffer_rsrc(
            a.pg.v_scale + ph * PS + off, 0, real ? KS * 4 : 0, kBufferFlags);
        x.ks = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(ksr, 4 * lane, 0, 0));
        x.vs = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(vsr, 4 * lane, 0, 0));
      }
    };
#pragma unroll
    for (int k = 0; k < SETS; ++k) fetch(min(s0 + k, max(s1 - 1, s0)), set[k]);

    // ---- queries: turned by their tokens' positions, the softmax scale folded in
    if (a.rope.pos) {
      unit_turns<RB, D>(a, at, row0, nrows, s_cs);
      __syncthreads();
    }
    bf16x8 q[NB][NQC];
    int sees[NB];                            // keys that this lane's rows see
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int row = row0 + min(16 * nb + col, nrows - 1);
      const int t = row / a.G;
      sees[nb] = min(max(at.r.base + t + 1, 0), limit);
      const T* qrow = static_cast<const T*>(a.q) + (at.r.first + t) * a.q_stride +
                      size_t(at.g * a.G + row % a.G) * D;
      const float2* cs = a.rope.pos ? s_cs + (t - row0 / a.G) * (D / 2) : nullptr;
#pragma unroll
      for (int c = 0; c < NQC; ++c) {
        float x[8];
        // the contraction index follows the keys' 16-byte pieces
        query8<T, D>(qrow, I8 ? 64 * (c / 2) + 16 * j + 8 * (c % 2) : 32 * c + 8 * j, cs,
                     a.qscale, x);
        q[nb][c] = bf16_of(x);
      }
    }
    const int sees_all = min(max(at.r.base + row0 / a.G + 1, 0), limit);   // every row's keys

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
      const bool partial = key0 + KS > sees_all || x.page < 0;
      bf16x8 pb[NB][U];
      f32x4 s[NB][2 * U];
#pragma unroll
      for (int m = 0; m < 2 * U; ++m) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          // bf16: scores leave the product relative to the reference
          const float z = I8 ? 0.f : -m_ref[nb];
          s[nb][m] = f32x4{z, z, z, z};
        }
#pragma unroll
        for (int c = 0; c < NKC; ++c) {
          const u32x4 w = x.k[m * NKC + c];
          if constexpr (I8) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const bf16x8 kf = bf16_of_i8(w[2 * h], w[2 * h + 1]);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb)
                s[nb][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[nb][2 * c + h], s[nb][m],
                                                                   0, 0, 0);
            }
          } else {
            const bf16x8 kf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              s[nb][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[nb][c], s[nb][m], 0, 0, 0);
          }
        }
      }
      if constexpr (I8) {
        // lane l has the scale of key key0 + l, and scores of its group's 16 keys
        auto scaled = [&](auto k_c) __attribute__((always_inline)) {
          constexpr int k = decltype(k_c)::value;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            s[nb][k / 4][k % 4] =
                __builtin_fmaf(s[nb][k / 4][k % 4], lane16<k>(x.ks), -m_ref[nb]);
        };
        [&]<int... k>(std::integer_sequence<int, k...>) __attribute__((always_inline)) {
          (scaled(std::integral_constant<int, k>{}), ...);
        }(std::make_integer_sequence<int, 16>{});
      }
      if (partial) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int n = x.page < 0 ? 0 : sees[nb] - key0 - 8 * U * j;
#pragma unroll
          for (int k = 0; k < 8 * U; ++k)
            if (k >= n) s[nb][k / 4][k % 4] = kNegInf;
        }
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
          [&]<int... k>(std::integer_sequence<int, k...>) __attribute__((always_inline)) {
            ((pr[k] *= lane16<k>(x.vs)), ...);
          }(std::make_integer_sequence<int, 16>{});
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float (&x8)[8] = reinterpret_cast<const float (&)[8]>(pr[8 * u]);
          pb[nb][u] = bf16_of(x8);
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
          for (int nb = 0; nb < NB; ++nb)
            o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[nb][u], o[nb][db], 0, 0, 0);
        }
    };
    for (int step = s0; step < s1; step += SETS) {
#pragma unroll
      for (int k = 0; k < SETS; ++k) {
        if (step + k < s1) compute(step + k, set[k]);
        fetch(step + k + SETS, set[k]);
      }
    }

    // ---- the wavefronts' pieces meet
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
    __syncthreads();
    const bool begins = t0 == 0, ends = t1 == at.tiles;
    if (begins && !ends) join = cut_unit<RB>(a, share, at, t1);
    constexpr int TPR = 256 / RB, EPT = D / TPR;    // threads a row, elements a thread
    const int row = tid / TPR, d0 = tid % TPR * EPT;
    if (row < nrows) {
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
      if (begins && ends) {
        const int r = row0 + row, token = at.r.first + r / a.G, h = at.g * a.G + r % a.G;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* out = static_cast<T*>(a.out) + (size_t(token) * a.Hq + h) * D + d0;
#pragma unroll
        for (int e = 0; e < EPT; e += 4)
          *reinterpret_cast<uint2*>(out + e) =
              make_uint2(pack_bf16(x[e] * inv, x[e + 1] * inv),
                         pack_bf16(x[e + 2] * inv, x[e + 3] * inv));
        if (a.lse && d0 == 0)
          a.lse[size_t(token) * a.Hq + h] =
              l == 0.f ? kNegInf : (ref + __builtin_amdgcn_logf(l)) * kLn2;
      } else {
        const size_t part = (size_t(2) * blockIdx.x + (begins ? 1 : 0)) * RB + row;
#pragma unroll
        for (int e = 0; e < EPT; e += 4)
          *reinterpret_cast<float4*>(a.part_o + part * D + d0 + e) =
              make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        if (d0 == 0) a.part_ml[part] = make_float2(m, l);
      }
    }
    p += t1 - t0;
    if (p < share.p1) {
      next_unit<RB>(a, limit, at);
      __syncthreads();                       // LDS of this unit is read
    }
  }
  if (tid == 0) a.joins[blockIdx.x] = join;
}

// ----------------------------------------------------------------------------
// join
// ----------------------------------------------------------------------------

// Rows blockIdx.y, blockIdx.y + gridDim.y, ... of the unit that workgroup blockIdx.x began
// and others finished: the four wavefronts take every fourth piece, a lane two columns.
template <typename T, int D, int RB>
__global__ __launch_bounds__(256) void join_kernel(AttendParams a) {
  constexpr int CPL = D / 64;                // columns of a lane
  __shared__ float s_x[4][D];
  const int w0 = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const Join jn = a.joins[w0];
  const int pieces = jn.last - w0 + 1;
  // piece k: the second partial of w0, then the first ones of those after it
  auto slot = [&](int k) { return size_t(2) * (w0 + k) + (k == 0 ? 1 : 0); };
  for (int row = blockIdx.y; row < jn.nrows; row += gridDim.y) {
    float m = kNegInf;
    for (int k = lane; k < pieces; k += 64) m = fmaxf(m, a.part_ml[slot(k) * RB + row].x);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    const float ref = m == kNegInf ? 0.f : m;
    float l = 0.f;
    for (int k = lane; k < pieces; k += 64) {
      const float2 ml = a.part_ml[slot(k) * RB + row];
      l += ml.y * __builtin_amdgcn_exp2f(ml.x - ref);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
    float x[CPL] = {};
    constexpr int N = 8;
    for (int k0 = wave; k0 < pieces; k0 += 4 * N) {
      float v[N][CPL], f[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int k = min(k0 + 4 * i, pieces - 1);
        const float* o = a.part_o + (slot(k) * RB + row) * D + lane * CPL;
#pragma unroll
        for (int e = 0; e < CPL; ++e) v[i][e] = o[e];
        f[i] = a.part_ml[slot(k) * RB + row].x;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (k0 + 4 * i >= pieces) continue;
        const float g = __builtin_amdgcn_exp2f(f[i] - ref);
#pragma unroll
        for (int e = 0; e < CPL; ++e) x[e] = __builtin_fmaf(g, v[i][e], x[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < CPL; ++e) s_x[wave][lane * CPL + e] = x[e];
    __syncthreads();
    if (tid < D) {
      const int r = jn.row0 + row, token = jn.first + r / a.G, h = jn.g * a.G + r % a.G;
      const float sum = (s_x[0][tid] + s_x[1][tid]) + (s_x[2][tid] + s_x[3][tid]);
      static_cast<T*>(a.out)[(size_t(token) * a.Hq + h) * D + tid] =
          from_f<T>(l == 0.f ? 0.f : sum / l);
      if (a.lse && tid == 0)
        a.lse[size_t(token) * a.Hq + h] =
            l == 0.f ? kNegInf : (ref + __builtin_amdgcn_logf(l)) * kLn2;
    }
    __syncthreads();
  }
}

// A wavefront per (token, query head): 64 keys a step, a lane a key for the scores and a
// column (or two) of the values for the sum.
template <typename T, typename S, int D>
__global__ __launch_bounds__(64) void attend_token_kernel(AttendParams a) {
  constexpr int VPL = D / 64;
  __shared__ float sQ[D], sP[ST];
  const int lane = threadIdx.x, token = blockIdx.x, h = blockIdx.y, g = h / a.G;
  const int PS = a.pg.PS;
  Req r;
  const int b = find_row(a.ch, token, r);
  if (b < 0) return;
  if (lane < D / 2) {
    const T* q = static_cast<const T*>(a.q) + token * a.q_stride + h * D;
    float x = to_f(q[lane]), y = to_f(q[lane + D / 2]);
    if (a.rope.pos) {
      float c, s;
      turn_cs(a.rope.pos[token], a.rope.turns[lane], c, s);
      rotate_pair(x, y, c, s);
    }
    sQ[lane] = x * a.qscale;
    sQ[lane + D / 2] = y * a.qscale;
  }
  __syncthreads();
  const int sees = min(r.base + (token - r.first) + 1, a.ch.max_pages * PS);
  float m = kNegInf, l = 0.f, acc[VPL] = {};
  for (int k0 = 0; k0 < sees; k0 += ST) {
    const int page = page_of(a.ch, a.pg, b, k0);
    if (page < 0) continue;
    const size_t ph = size_t(page) * a.pg.Hkv + g;
    const int off = k0 % PS, n = min(ST, sees - k0);
    const S* kp = static_cast<const S*>(a.pg.k) + (ph * PS + off + min(lane, n - 1)) * D;
    float s = 0.f;
    for (int d = 0; d < D; d += 8) {
      float x[8];
      load8(kp + d, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = __builtin_fmaf(x[e], sQ[d + e], s);
    }
    const size_t at = ph * PS + off + min(lane, n - 1);
    if constexpr (sizeof(S) == 1) s *= a.pg.k_scale[at];
    if (lane >= n) s = kNegInf;
    float mt = s;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) mt = fmaxf(mt, __shfl_xor(mt, d));
    const float m_new = fmaxf(m, mt), ref = m_new == kNegInf ? 0.f : m_new;
    const float keep = exp2f(m - ref);
    float p = exp2f(s - ref);
    l = l * keep + p;
    m = m_new;
    if constexpr (sizeof(S) == 1) p *= lane < n ? a.pg.v_scale[at] : 0.f;
    sP[lane] = p;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VPL; ++e) {
      const S* vp = static_cast<const S*>(a.pg.v) + (ph * D + lane + 64 * e) * PS + off;
      acc[e] *= keep;
      for (int j = 0; j < n; ++j) acc[e] = __builtin_fmaf(sP[j], float(vp[j]), acc[e]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* out = static_cast<T*>(a.out) + (size_t(token) * a.Hq + h) * D;
#pragma unroll
  for (int e = 0; e < VPL; ++e) out[lane + 64 * e] = from_f<T>(acc[e] * inv);
  if (a.lse && lane == 0)
    a.lse[size_t(token) * a.Hq + h] = l == 0.f ? kNegInf : (m + log2f(l)) * kLn2;
}

// the kernel of a shape: narrow by rows, else token by token
template <typename S, int D>
const void* narrow_kernel(int rows) {
  return rows == 16 ? reinterpret_cast<const void*>(&attend_narrow_kernel<S, D, 1>)
                    : reinterpret_cast<const void*>(&attend_narrow_kernel<S, D, 2>);
}

}  // namespace

AttendShape attend_shape(int store, int D, int64_t rows_max, int64_t batch, int64_t heads,
                         int64_t kv_max) {
  AttendShape s{};
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  if (store == C2KV_F32 || rows_max > 32) return s;
  s.rows = rows_max <= 16 ? 16 : 32;
  const int64_t tiles = batch * heads * ((kv_max + ST - 1) / ST);
  s.groups = int(tiles < 512 ? tiles : 512);
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
  if (sh.groups > 0) {
    const void* k = store == C2KV_I8 ? (D == 64 ? narrow_kernel<int8_t, 64>(sh.rows)
                                                : narrow_kernel<int8_t, 128>(sh.rows))
                                     : (D == 64 ? narrow_kernel<__bf16, 64>(sh.rows)
                                                : narrow_kernel<__bf16, 128>(sh.rows));
    return launch(k, dim3(unsigned(sh.groups)), dim3(256), st, p, e0, e1);
  }
  return with_types(store, D, [&](auto t, auto s, auto d) {
    using T = decltype(t);
    using S = decltype(s);
    return launch(reinterpret_cast<const void*>(&attend_token_kernel<T, S, decltype(d)::value>),
                  dim3(unsigned(p.ch.n_tokens), unsigned(p.Hq)), dim3(64), st, p, e0, e1);
  });
}

hipError_t launch_cache_merge(const AttendParams& p, const AttendShape& sh, int store, int D,
                              hipStream_t st, hipEvent_t e0, hipEvent_t e1) {
  (void)store;
  const void* k =
      D == 64 ? (sh.rows == 16 ? reinterpret_cast<const void*>(&join_kernel<__bf16, 64, 16>)
                               : reinterpret_cast<const void*>(&join_kernel<__bf16, 64, 32>))
              : (sh.rows == 16 ? reinterpret_cast<const void*>(&join_kernel<__bf16, 128, 16>)
                               : reinterpret_cast<const void*>(&join_kernel<__bf16, 128, 32>));
  return launch(k, dim3(unsigned(sh.groups), 4), dim3(256), st, p, e0, e1);
}

}  // namespace c2kv
