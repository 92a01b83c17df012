// The growing paged cache: parameters of its kernels and their launchers (defined in
// cache.hip, those of attention in attend.hip), called by the C ABI in api.cpp.  Non-null events are stamped at the
// kernel's start and end.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "c2kv.h"
#include "cache_index.hpp"

namespace c2kv {

// Chunks of new tokens (c2kv_chunks): device arrays.
struct ChunkView {
  const int32_t* tok_off;
  const int32_t* kv_len;
  const int32_t* table;
  int32_t batch, n_tokens, max_pages;
};

// The cache's pages (c2kv_cache) of one layer.
struct PageView {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int32_t n_pages, PS, Hkv;
};

// RoPE: turns[i] full turns of pair (i, i + D/2) per position, in 64 bits; pos == NULL: no turn.
struct RopeView {
  const int32_t* pos;
  double turns[64];
};

struct WriteParams {
  ChunkView ch;
  PageView pg;
  RopeView rope;
  const void* k;
  const void* v;
  int64_t k_stride, v_stride;   // elements between tokens
};

struct ReadParams {
  ChunkView ch;
  PageView pg;
  RopeView rope;
  void* k;
  void* v;
};

struct PoolWriteParams {
  RopeView rope;
  const int64_t* row;
  int32_t n, Hkv;
  int64_t n_rows;
  const void* k;
  const void* v;
  int64_t k_stride, v_stride;
  void* pool_k;
  void* pool_v;
  float* k_scale;
  float* v_scale;
};

struct AttendParams {
  ChunkView ch;
  PageView pg;
  RopeView rope;
  int32_t Hq, G;
  int32_t rb;                   // query rows of a unit
  float qscale;                 // softmax scale * log2(e)
  const void* q;
  int64_t q_stride;
  void* out;
  float* lse;                   // [n_tokens][Hq] or NULL
  // workspace: what the workgroups of one launch leave for the joining one
  float* part_o;                // [2 * groups][RB][D]
  float2* part_ml;              // [2 * groups][RB] reference maximum (base 2), sum
  struct Join* joins;           // [groups]
  int32_t groups;
};

// A unit cut by a border between workgroups (joins[w]: the one that begins in workgroup
// w), nrows 0 where there is none: its pieces are the second partial of workgroup w and
// the first ones of w + 1 .. last.
struct Join {
  int32_t first, row0, nrows, g, last, pad[3];
};

// How an attention call is launched, and what its workspace holds.
struct AttendShape {
  int32_t rows;                 // RB: query rows that a kernel's unit has room for
  int32_t unit_rows;            // rows of a unit here, at most RB
  int32_t groups;               // workgroups
  size_t part_o, part_ml, joins, total;   // byte offsets
};
// rows_max: bound on the (token, query head) rows of one (request, kv-head), those of
// max_chunk tokens; kv_max: bound on a request's cached tokens
AttendShape attend_shape(int store, int D, int64_t rows_max, int64_t max_chunk, int64_t batch,
                         int64_t heads, int64_t kv_max);

// `store`: type of the cache or pool; its activations are F32 for F32, else BF16.
hipError_t launch_cache_write(const WriteParams& p, int store, int D, int max_chunk,
                              hipStream_t st, hipEvent_t e0, hipEvent_t e1);
hipError_t launch_cache_read(const ReadParams& p, int store, int D, hipStream_t st,
                             hipEvent_t e0, hipEvent_t e1);
hipError_t launch_pool_write(const PoolWriteParams& p, int store, int D, hipStream_t st,
                             hipEvent_t e0, hipEvent_t e1);
hipError_t launch_cache_attend(const AttendParams& p, const AttendShape& sh, int store, int D,
                               hipStream_t st, hipEvent_t e0, hipEvent_t e1);
hipError_t launch_cache_merge(const AttendParams& p, const AttendShape& sh, int store, int D,
                              hipStream_t st, hipEvent_t e0, hipEvent_t e1);

}  // namespace c2kv
