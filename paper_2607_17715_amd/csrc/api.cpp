// C ABI of the compose-and-attend path (declared in include/c2kv.h): argument
// checks, workspace binding, kernel launches on the caller's stream, optional
// per-kernel event timing, and the thread-local error text.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <map>
#include <mutex>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "c2kv.h"
#include "cache.hpp"
#include "launch.hpp"
#include "plan.hpp"

namespace {

thread_local std::string g_last_error;

c2kv_status fail(c2kv_status st, std::string msg) {
  g_last_error = std::move(msg);
  return st;
}

c2kv_status hip_fail(hipError_t e, const char* what) {
  return fail(C2KV_E_HIP, std::string(what) + ": " + hipGetErrorName(e) + " (" +
                              hipGetErrorString(e) + ")");
}

// ---- optional per-kernel timing --------------------------------------------
struct Timing {
  std::mutex mu;
  bool on = false;
  struct Rec { hipEvent_t a, b; };
  std::map<std::string, std::vector<Rec>> recs;
  std::vector<hipEvent_t> spare;
};
Timing g_timing;

hipEvent_t take_event() {
  if (!g_timing.spare.empty()) {
    hipEvent_t e = g_timing.spare.back();
    g_timing.spare.pop_back();
    return e;
  }
  hipEvent_t e = nullptr;
  if (hipEventCreate(&e) != hipSuccess) return nullptr;
  return e;
}

// Runs `launch(ev0, ev1)`; when timing is on, the events (stamped by the
// kernel's own dispatch at its start and end) are filed under `name`.
template <typename F>
hipError_t timed(const char* name, F&& launch) {
  bool on;
  {
    std::lock_guard<std::mutex> lk(g_timing.mu);
    on = g_timing.on;
  }
  if (!on) return launch(nullptr, nullptr);
  hipEvent_t a, b;
  {
    std::lock_guard<std::mutex> lk(g_timing.mu);
    a = take_event();
    b = take_event();
  }
  hipError_t e = a && b ? launch(a, b) : hipErrorOutOfMemory;
  std::lock_guard<std::mutex> lk(g_timing.mu);
  if (e != hipSuccess) {
    // events of a launch that did not happen go back to the spare list
    if (a) g_timing.spare.push_back(a);
    if (b) g_timing.spare.push_back(b);
    return e;
  }
  g_timing.recs[name].push_back({a, b});
  return hipSuccess;
}

bool check_plan(const c2kv_plan* plan, c2kv_status* st) {
  if (!plan) { *st = fail(C2KV_E_INVAL, "plan is NULL"); return false; }
  if (!plan->p.d_workspace) {
    *st = fail(C2KV_E_STATE, "plan is not uploaded (call c2kv_plan_upload first)");
    return false;
  }
  return true;
}

bool check_pool(const c2kv::Plan& p, const c2kv_pool* pool, c2kv_status* st) {
  if (!pool || !pool->k || !pool->v) {
    *st = fail(C2KV_E_INVAL, "pool or its K/V pointer is NULL");
    return false;
  }
  if (pool->dtype != C2KV_F32 && pool->dtype != C2KV_BF16 && pool->dtype != C2KV_I8) {
    *st = fail(C2KV_E_INVAL, "pool dtype must be F32, BF16 or I8");
    return false;
  }
  const bool ok_combo = (pool->dtype == C2KV_F32 && p.cfg.act_dtype == C2KV_F32) ||
                        (pool->dtype == C2KV_BF16 && p.cfg.act_dtype == C2KV_BF16) ||
                        (pool->dtype == C2KV_I8 && p.cfg.act_dtype == C2KV_BF16);
  if (!ok_combo) {
    *st = fail(C2KV_E_UNSUPPORTED,
               "pool/act dtype combination not built (F32/F32, BF16/BF16, I8/BF16)");
    return false;
  }
  if (pool->dtype == C2KV_I8 && (!pool->k_scale || !pool->v_scale)) {
    *st = fail(C2KV_E_INVAL, "I8 pool needs k_scale and v_scale");
    return false;
  }
  if (p.max_src_row >= pool->n_rows) {
    *st = fail(C2KV_E_INVAL, "a kept token reads pool row " + std::to_string(p.max_src_row) +
                                 " but the pool has " + std::to_string(pool->n_rows) + " rows");
    return false;
  }
  return true;
}

bool check_io(const void* q, const void* ks, const void* vs, const void* out,
              c2kv_status* st) {
  if (!q || !ks || !vs || !out) {
    *st = fail(C2KV_E_INVAL, "q, k_suf, v_suf and out must not be NULL");
    return false;
  }
  return true;
}

// ---- the growing cache ------------------------------------------------------

// Runs a call's body; nothing thrown in it (a failed host allocation) leaves the C entry.
template <typename F>
c2kv_status guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    g_last_error.clear();
    return C2KV_E_NOMEM;
  }
}

bool on16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

c2kv_status check_shape(const c2kv_attn_cfg* cfg) {
  if (!cfg) return fail(C2KV_E_INVAL, "cfg is NULL");
  std::string err;
  const c2kv_status st = c2kv::check_cfg(*cfg, err);
  if (st != C2KV_OK) return fail(st, err);
  if (cfg->n_q_heads > 65535)
    return fail(C2KV_E_UNSUPPORTED, "more than 65535 query heads are not built");
  return C2KV_OK;
}

c2kv_status check_store(const char* what, c2kv_dtype store, const c2kv_attn_cfg& cfg,
                        const void* k, const void* v, const void* ks, const void* vs) {
  if (!k || !v) return fail(C2KV_E_INVAL, std::string(what) + "'s K/V pointer is NULL");
  if (store != C2KV_F32 && store != C2KV_BF16 && store != C2KV_I8)
    return fail(C2KV_E_INVAL, std::string(what) + " dtype must be F32, BF16 or I8");
  if ((store == C2KV_F32) != (cfg.act_dtype == C2KV_F32))
    return fail(C2KV_E_UNSUPPORTED, std::string(what) + "/act dtype combination not built "
                                                        "(F32/F32, BF16/BF16, I8/BF16)");
  if (store == C2KV_I8 && (!ks || !vs))
    return fail(C2KV_E_INVAL, "I8 " + std::string(what) + " needs k_scale and v_scale");
  if (!on16(k) || !on16(v) || (store == C2KV_I8 && (!on16(ks) || !on16(vs))))
    return fail(C2KV_E_INVAL, std::string(what) + " memory must lie on 16 bytes");
  return C2KV_OK;
}

c2kv_status check_cache(const c2kv_attn_cfg* cfg, const c2kv_cache* cache,
                        const c2kv_chunks* ch) {
  c2kv_status st = check_shape(cfg);
  if (st != C2KV_OK) return st;
  if (!cache || !ch) return fail(C2KV_E_INVAL, "cache and chunks must not be NULL");
  st = check_store("cache", cache->dtype, *cfg, cache->k, cache->v, cache->k_scale,
                   cache->v_scale);
  if (st != C2KV_OK) return st;
  if (cache->n_pages < 1) return fail(C2KV_E_INVAL, "n_pages must be >= 1");
  if (cache->page_size < 1 || cache->page_size % c2kv::kSlotTile != 0)
    return fail(C2KV_E_INVAL, "page_size must be a positive multiple of " +
                                  std::to_string(c2kv::kSlotTile) + ", got " +
                                  std::to_string(cache->page_size));
  if (cache->page_size > 65536)
    return fail(C2KV_E_UNSUPPORTED, "pages of more than 65536 tokens are not built");
  if (ch->batch < 1) return fail(C2KV_E_INVAL, "batch must be >= 1");
  if (ch->n_tokens < 0 || ch->max_chunk < 0 || ch->max_kv < 0)
    return fail(C2KV_E_INVAL, "n_tokens, max_chunk and max_kv must be >= 0");
  if (ch->max_pages < 1) return fail(C2KV_E_INVAL, "max_pages must be >= 1");
  if (!ch->tok_off || !ch->kv_len || !ch->block_table)
    return fail(C2KV_E_INVAL, "tok_off, kv_len and block_table must not be NULL");
  if (int64_t(ch->max_pages) * cache->page_size > (1ll << 30))
    return fail(C2KV_E_UNSUPPORTED, "block tables of more than 2^30 tokens are not built");
  if (int64_t(ch->n_tokens) * cfg->n_q_heads > (1ll << 31) - 1)
    return fail(C2KV_E_UNSUPPORTED, "chunks of 2^31 (token, head) rows or more are not built");
  if (ch->n_tokens > 1 << 29)
    return fail(C2KV_E_UNSUPPORTED, "chunks of more than 2^29 tokens are not built");
  if (ch->batch > 1 << 22)
    return fail(C2KV_E_UNSUPPORTED, "batches of more than 2^22 requests are not built");
  return C2KV_OK;
}

// Refuses batches whose tiles of tokens a launch cannot count.
c2kv_status check_tiles(const c2kv_chunks& ch) {
  if (c2kv::most_chunk_tiles(ch.n_tokens, ch.batch) > c2kv::kMostGroups)
    return fail(C2KV_E_UNSUPPORTED, "batches that may fill 2^24 tiles of tokens are not built");
  return C2KV_OK;
}

// rows of `heads` heads, `stride` elements between tokens (0: dense)
c2kv_status check_rows(const char* what, const c2kv_attn_cfg& cfg, const void* p, int heads,
                       int64_t& stride) {
  if (!p) return fail(C2KV_E_INVAL, std::string(what) + " must not be NULL");
  const int64_t dense = int64_t(heads) * cfg.head_dim;
  if (stride == 0) stride = dense;
  if (stride < dense)
    return fail(C2KV_E_INVAL, std::string(what) + "'s stride is smaller than a token");
  if (!on16(p) || stride * (cfg.act_dtype == C2KV_F32 ? 4 : 2) % 16 != 0)
    return fail(C2KV_E_INVAL, std::string(what) + "'s tokens must lie on 16 bytes");
  return C2KV_OK;
}

c2kv::ChunkView view(const c2kv_chunks& c) {
  return {c.tok_off, c.kv_len, c.block_table, c.batch, c.n_tokens, c.max_pages};
}
c2kv::PageView view(const c2kv_cache& c, const c2kv_attn_cfg& cfg) {
  return {c.k, c.v, c.k_scale, c.v_scale, c.n_pages, c.page_size, cfg.n_kv_heads};
}
// theta_i = base^(-2i/D) as turns per position, by powers of the first ratio: 63 products
// of 64-bit numbers, exact to 1e-14
c2kv::RopeView rope(const c2kv_attn_cfg& cfg, const int32_t* pos) {
  c2kv::RopeView r{};
  r.pos = pos;
  if (!pos) return r;
  const double ratio = std::pow(cfg.rope_base, -2.0 / cfg.head_dim);
  double t = 0.15915494309189533577;          // 1 / (2 pi)
  for (int i = 0; i < cfg.head_dim / 2; ++i, t *= ratio) r.turns[i] = t;
  return r;
}
int longest_chunk(const c2kv_chunks& c) {
  return c2kv::longest_chunk(c.max_chunk, c.n_tokens, c.batch);
}
// Launch shape of an attention call, from the bounds that the host knows.
c2kv::AttendShape attend_shape(const c2kv_attn_cfg& cfg, const c2kv_cache& cache,
                               const c2kv_chunks& ch) {
  const int64_t G = cfg.n_q_heads / cfg.n_kv_heads;
  const int64_t longest = longest_chunk(ch);
  const int64_t room = int64_t(ch.max_pages) * cache.page_size;
  const int64_t kv = ch.max_kv > 0 && ch.max_kv < room ? ch.max_kv : room;
  return c2kv::attend_shape(cache.dtype, cfg.head_dim, longest * G, longest, ch.batch,
                            cfg.n_kv_heads, kv);
}

// Whether the line of key tiles that the device may find passes 32 bits.
bool too_long(const c2kv::AttendShape& sh, const c2kv_attn_cfg& cfg, const c2kv_cache& cache,
              const c2kv_chunks& ch) {
  return c2kv::most_tiles(ch.n_tokens, ch.batch, cfg.n_q_heads / cfg.n_kv_heads, cfg.n_kv_heads,
                          sh.unit_rows, int64_t(ch.max_pages) * cache.page_size) >= 1ll << 31;
}
const char kTooLong[] = "batches that may hold 2^31 key tiles are not built";

}  // namespace

extern "C" {

const char* c2kv_last_error(void) { return g_last_error.c_str(); }

const char* c2kv_version(void) { return "c2kv 0.1.0 gfx950"; }

c2kv_status c2kv_plan_create(const c2kv_attn_cfg* cfg, const c2kv_compose_desc* desc,
                             int32_t suffix_len, const c2kv_plan_opts* opts,
                             c2kv_plan** out) {
  if (!cfg || !desc || !out) return fail(C2KV_E_INVAL, "cfg, desc and out must not be NULL");
  c2kv_plan* plan = new (std::nothrow) c2kv_plan;
  if (!plan) return fail(C2KV_E_NOMEM, "cannot allocate plan");
  std::string err;
  c2kv_status st;
  try {
    st = c2kv::build_plan(*cfg, *desc, suffix_len, opts, plan->p, err);
  } catch (const std::bad_alloc&) {
    st = C2KV_E_NOMEM;
    err = "host allocation failed while building the plan";
  }
  if (st != C2KV_OK) {
    delete plan;
    return fail(st, err);
  }
  *out = plan;
  return C2KV_OK;
}

c2kv_status c2kv_sif_plan_create(const c2kv_attn_cfg* cfg, int32_t batch, int32_t n_tokens,
                                 int32_t block, int32_t sink, const c2kv_plan_opts* opts,
                                 c2kv_plan** out) {
  if (!cfg || !out) return fail(C2KV_E_INVAL, "cfg and out must not be NULL");
  c2kv_plan* plan = new (std::nothrow) c2kv_plan;
  if (!plan) return fail(C2KV_E_NOMEM, "cannot allocate plan");
  std::string err;
  c2kv_status st;
  try {
    st = c2kv::build_sif_plan(*cfg, batch, n_tokens, block, sink, opts, plan->p, err);
  } catch (const std::bad_alloc&) {
    st = C2KV_E_NOMEM;
    err = "host allocation failed while building the plan";
  }
  if (st != C2KV_OK) {
    delete plan;
    return fail(st, err);
  }
  *out = plan;
  return C2KV_OK;
}

void c2kv_plan_destroy(c2kv_plan* plan) { delete plan; }

c2kv_status c2kv_plan_get_info(const c2kv_plan* plan, c2kv_plan_info* info) {
  if (!plan || !info) return fail(C2KV_E_INVAL, "plan and info must not be NULL");
  const c2kv::Plan& p = plan->p;
  info->batch = p.batch;
  info->suffix_len = p.suffix_len;
  info->page_size = p.page_size;
  info->n_pages = p.n_pages;
  info->max_pages = p.max_pages;
  info->n_segments = p.n_segments;
  info->total_slots = static_cast<int64_t>(p.slot_src.size());
  info->max_src_row = p.max_src_row;
  info->workspace_bytes = p.ws.total;
  info->rows_per_block = p.rows_per_block;
  info->n_work_items = static_cast<int32_t>(p.items.size());
  info->n_merge_groups = static_cast<int32_t>(p.merges.size());
  info->max_splits = p.max_splits;
  return C2KV_OK;
}

c2kv_status c2kv_plan_get_requests(const c2kv_plan* plan, int32_t* composed_len,
                                   int32_t* span_end) {
  if (!plan) return fail(C2KV_E_INVAL, "plan is NULL");
  const c2kv::Plan& p = plan->p;
  for (int b = 0; b < p.batch; ++b) {
    if (composed_len) composed_len[b] = p.req_slot0[b + 1] - p.req_slot0[b];
    if (span_end) span_end[b] = p.span_end[b];
  }
  return C2KV_OK;
}

c2kv_status c2kv_plan_get_slots(const c2kv_plan* plan, int64_t* src_row, int32_t* p_new,
                                int32_t* delta) {
  if (!plan) return fail(C2KV_E_INVAL, "plan is NULL");
  const c2kv::Plan& p = plan->p;
  const size_t n = p.slot_src.size();
  for (size_t i = 0; i < n; ++i) {
    if (src_row) src_row[i] = p.slot_src[i];
    if (p_new) p_new[i] = p.slot_pos[i];
    if (delta) delta[i] = p.slot_delta[i];
  }
  return C2KV_OK;
}

c2kv_status c2kv_plan_get_block_table(const c2kv_plan* plan, int32_t* block_table) {
  if (!plan || !block_table) return fail(C2KV_E_INVAL, "plan and block_table must not be NULL");
  std::memcpy(block_table, plan->p.block_table.data(),
              plan->p.block_table.size() * sizeof(int32_t));
  return C2KV_OK;
}

c2kv_status c2kv_plan_upload(c2kv_plan* plan, void* workspace, size_t workspace_bytes,
                             void* stream) {
  if (!plan) return fail(C2KV_E_INVAL, "plan is NULL");
  c2kv::Plan& p = plan->p;
  if (!workspace) return fail(C2KV_E_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return fail(C2KV_E_WORKSPACE, "workspace must be 256-byte aligned");
  if (workspace_bytes < p.ws.total)
    return fail(C2KV_E_WORKSPACE, "workspace has " + std::to_string(workspace_bytes) +
                                      " bytes, plan needs " + std::to_string(p.ws.total));
  hipError_t e = hipMemcpyAsync(workspace, p.image.data(), p.image.size(),
                                hipMemcpyHostToDevice, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "hipMemcpyAsync (plan upload)");
  p.d_workspace = workspace;
  p.d_workspace_bytes = workspace_bytes;
  return C2KV_OK;
}

c2kv_status c2kv_compose(const c2kv_plan* plan, const c2kv_pool* pool, void* k_pages,
                         void* v_pages, int64_t* slot_src_row, int32_t* slot_pos,
                         int32_t* block_table, void* stream) {
  c2kv_status st;
  if (!check_plan(plan, &st)) return st;
  const c2kv::Plan& p = plan->p;
  if (!check_pool(p, pool, &st)) return st;
  if ((!k_pages || !v_pages) && p.n_pages > 0)
    return fail(C2KV_E_INVAL, "k_pages and v_pages must not be NULL");
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = timed("compose", [&](hipEvent_t e0, hipEvent_t e1) {
    return c2kv::launch_compose(p, p.d_workspace, pool->dtype, pool->k, pool->v, pool->k_scale,
                                pool->v_scale, k_pages, v_pages, slot_src_row, slot_pos, s, e0, e1);
  });
  if (e != hipSuccess) return hip_fail(e, "compose launch");
  if (block_table) {
    e = hipMemcpyAsync(block_table,
                       static_cast<const uint8_t*>(p.d_workspace) + p.ws.block_table,
                       p.block_table.size() * sizeof(int32_t), hipMemcpyDeviceToDevice, s);
    if (e != hipSuccess) return hip_fail(e, "hipMemcpyAsync (block table)");
  }
  return C2KV_OK;
}

static c2kv_status run_attention(const c2kv::Plan& p, void* ws, int src_kind, const char* name,
                                 const void* k, const void* v, const float* ks,
                                 const float* vs, const void* q, const void* k_suf,
                                 const void* v_suf, void* out, float* lse, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = timed(name, [&](hipEvent_t e0, hipEvent_t e1) {
    return c2kv::launch_attention(p, ws, src_kind, k, v, ks, vs, q, k_suf, v_suf, out, lse, s, e0,
                                  e1);
  });
  if (e != hipSuccess) return hip_fail(e, "attention launch");
  if (!p.merges.empty() && !p.merge_in_kernel) {
    e = timed("merge", [&](hipEvent_t e0, hipEvent_t e1) {
      return c2kv::launch_merge(p, ws, out, lse, s, e0, e1);
    });
    if (e != hipSuccess) return hip_fail(e, "merge launch");
  }
  return C2KV_OK;
}

c2kv_status c2kv_attend(const c2kv_plan* plan, const void* k_pages, const void* v_pages,
                        const void* q, const void* k_suf, const void* v_suf, void* out,
                        float* lse, void* stream) {
  c2kv_status st;
  if (!check_plan(plan, &st)) return st;
  if (!check_io(q, k_suf, v_suf, out, &st)) return st;
  const c2kv::Plan& p = plan->p;
  if ((!k_pages || !v_pages) && p.n_pages > 0)
    return fail(C2KV_E_INVAL, "k_pages and v_pages must not be NULL");
  return run_attention(p, p.d_workspace, c2kv::kSrcPaged, "attn_paged", k_pages, v_pages,
                       nullptr, nullptr, q, k_suf, v_suf, out, lse, stream);
}

c2kv_status c2kv_compose_attend(const c2kv_plan* plan, const c2kv_pool* pool, const void* q,
                                const void* k_suf, const void* v_suf, void* out, float* lse,
                                void* stream) {
  c2kv_status st;
  if (!check_plan(plan, &st)) return st;
  const c2kv::Plan& p = plan->p;
  if (!check_pool(p, pool, &st)) return st;
  if (!check_io(q, k_suf, v_suf, out, &st)) return st;
  const int kind = pool->dtype == C2KV_I8 ? c2kv::kSrcPoolI8 : c2kv::kSrcPool;
  return run_attention(p, p.d_workspace, kind, "attn_pool", pool->k, pool->v, pool->k_scale,
                       pool->v_scale, q, k_suf, v_suf, out, lse, stream);
}

c2kv_status c2kv_compose_attend_static(const c2kv_plan* plan, const c2kv_pool* pool,
                                       const void* q, const void* k_suf, const void* v_suf,
                                       void* out, float* lse, void* stream) {
  if (!plan) return fail(C2KV_E_INVAL, "plan is NULL");
  const c2kv::Plan& p = plan->p;
  // checked before any HIP call: the tables and partials must fit the array
  if (p.ws.total > C2KV_STATIC_SCRATCH_BYTES)
    return fail(C2KV_E_WORKSPACE,
                "plan needs " + std::to_string(p.ws.total) + " bytes of scratch; the static "
                "array holds " + std::to_string(size_t(C2KV_STATIC_SCRATCH_BYTES)) +
                " (use c2kv_compose_attend with a workspace)");
  c2kv_status st;
  if (!check_pool(p, pool, &st)) return st;
  if (!check_io(q, k_suf, v_suf, out, &st)) return st;
  void* ws = nullptr;
  hipError_t e = c2kv::static_scratch(&ws);
  if (e != hipSuccess) return hip_fail(e, "hipGetSymbolAddress (static scratch)");
  // this call's tables, over whatever the last call on this GPU left; the image
  // carries the zeroed merge counters as well
  e = hipMemcpyAsync(ws, p.image.data(), p.image.size(), hipMemcpyHostToDevice,
                     static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "hipMemcpyAsync (tables into static scratch)");
  const int kind = pool->dtype == C2KV_I8 ? c2kv::kSrcPoolI8 : c2kv::kSrcPool;
  return run_attention(p, ws, kind, "attn_pool", pool->k, pool->v, pool->k_scale,
                       pool->v_scale, q, k_suf, v_suf, out, lse, stream);
}

c2kv_status c2kv_host_alloc(size_t bytes, void** host, void** device) {
  if (!host || !device || bytes == 0) return fail(C2KV_E_INVAL, "host_alloc: bad arguments");
  *host = nullptr;
  *device = nullptr;
  void* h = nullptr;
  hipError_t e = hipHostMalloc(&h, bytes, hipHostMallocMapped);
  if (e != hipSuccess) return hip_fail(e, "hipHostMalloc");
  void* d = nullptr;
  e = hipHostGetDevicePointer(&d, h, 0);
  if (e != hipSuccess) {
    (void)hipHostFree(h);
    return hip_fail(e, "hipHostGetDevicePointer");
  }
  *host = h;
  *device = d;
  return C2KV_OK;
}

c2kv_status c2kv_host_free(void* host) {
  if (!host) return C2KV_OK;
  const hipError_t e = hipHostFree(host);
  return e == hipSuccess ? C2KV_OK : hip_fail(e, "hipHostFree");
}

c2kv_status c2kv_load(const c2kv_plan* plan, const c2kv_pool* src, const c2kv_pool* dst,
                      void* stream) {
  c2kv_status st;
  if (!check_plan(plan, &st)) return st;
  const c2kv::Plan& p = plan->p;
  if (!check_pool(p, src, &st) || !check_pool(p, dst, &st)) return st;
  if (src->dtype != dst->dtype) return fail(C2KV_E_INVAL, "load: pools of different dtypes");
  const size_t esz = src->dtype == C2KV_F32 ? 4 : src->dtype == C2KV_BF16 ? 2 : 1;
  const size_t row_bytes = esz * size_t(p.cfg.n_kv_heads) * size_t(p.cfg.head_dim);
  const size_t scale_bytes = sizeof(float) * size_t(p.cfg.n_kv_heads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto copy = [&](const void* from, void* to, size_t per_row, int64_t r0, int64_t r1) {
    return hipMemcpyAsync(static_cast<uint8_t*>(to) + size_t(r0) * per_row,
                          static_cast<const uint8_t*>(from) + size_t(r0) * per_row,
                          size_t(r1 - r0) * per_row, hipMemcpyDefault, s);
  };
  for (const auto& r : p.load_rows) {
    hipError_t e = copy(src->k, const_cast<void*>(dst->k), row_bytes, r.first, r.second);
    if (e == hipSuccess) e = copy(src->v, const_cast<void*>(dst->v), row_bytes, r.first, r.second);
    if (e == hipSuccess && src->dtype == C2KV_I8) {
      e = copy(src->k_scale, const_cast<float*>(dst->k_scale), scale_bytes, r.first, r.second);
      if (e == hipSuccess)
        e = copy(src->v_scale, const_cast<float*>(dst->v_scale), scale_bytes, r.first, r.second);
    }
    if (e != hipSuccess) return hip_fail(e, "hipMemcpyAsync (load)");
  }
  return C2KV_OK;
}

c2kv_status c2kv_cache_write(const c2kv_attn_cfg* cfg, const c2kv_cache* cache,
                             const c2kv_chunks* chunks, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, const int32_t* pos,
                             void* stream) {
  return guarded([&] {
    c2kv_status st = check_cache(cfg, cache, chunks);
    if (st == C2KV_OK && chunks->n_tokens == 0) return C2KV_OK;
    if (st == C2KV_OK) st = check_tiles(*chunks);
    if (st == C2KV_OK) st = check_rows("k", *cfg, k, cfg->n_kv_heads, k_stride);
    if (st == C2KV_OK) st = check_rows("v", *cfg, v, cfg->n_kv_heads, v_stride);
    if (st != C2KV_OK) return st;
    const c2kv::WriteParams p{view(*chunks), view(*cache, *cfg), rope(*cfg, pos), k, v,
                              k_stride, v_stride};
    hipError_t e = timed("cache_write", [&](hipEvent_t e0, hipEvent_t e1) {
      return c2kv::launch_cache_write(p, cache->dtype, cfg->head_dim, longest_chunk(*chunks),
                                      static_cast<hipStream_t>(stream), e0, e1);
    });
    return e == hipSuccess ? C2KV_OK : hip_fail(e, "cache write launch");
  });
}

c2kv_status c2kv_cache_read(const c2kv_attn_cfg* cfg, const c2kv_cache* cache,
                            const c2kv_chunks* chunks, const int32_t* turn, void* k, void* v,
                            void* stream) {
  return guarded([&] {
    c2kv_status st = check_cache(cfg, cache, chunks);
    if (st == C2KV_OK && chunks->n_tokens == 0) return C2KV_OK;
    if (st == C2KV_OK) st = check_tiles(*chunks);
    int64_t dense = 0;
    if (st == C2KV_OK) st = check_rows("k", *cfg, k, cfg->n_kv_heads, dense);
    if (st == C2KV_OK) st = check_rows("v", *cfg, v, cfg->n_kv_heads, dense);
    if (st != C2KV_OK) return st;
    const c2kv::ReadParams p{view(*chunks), view(*cache, *cfg), rope(*cfg, turn), k, v};
    hipError_t e = timed("cache_read", [&](hipEvent_t e0, hipEvent_t e1) {
      return c2kv::launch_cache_read(p, cache->dtype, cfg->head_dim,
                                     static_cast<hipStream_t>(stream), e0, e1);
    });
    return e == hipSuccess ? C2KV_OK : hip_fail(e, "cache read launch");
  });
}

c2kv_status c2kv_cache_attend_workspace(const c2kv_attn_cfg* cfg, const c2kv_cache* cache,
                                        const c2kv_chunks* chunks, size_t* bytes) {
  return guarded([&] {
    const c2kv_status st = check_cache(cfg, cache, chunks);
    if (st != C2KV_OK) return st;
    if (!bytes) return fail(C2KV_E_INVAL, "bytes must not be NULL");
    const c2kv::AttendShape sh = attend_shape(*cfg, *cache, *chunks);
    if (too_long(sh, *cfg, *cache, *chunks)) return fail(C2KV_E_UNSUPPORTED, kTooLong);
    *bytes = sh.total;
    return C2KV_OK;
  });
}

c2kv_status c2kv_cache_attend(const c2kv_attn_cfg* cfg, const c2kv_cache* cache,
                              const c2kv_chunks* chunks, const void* q, int64_t q_stride,
                              const int32_t* pos, void* out, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream) {
  return guarded([&] {
    c2kv_status st = check_cache(cfg, cache, chunks);
    if (st == C2KV_OK && chunks->n_tokens == 0) return C2KV_OK;
    int64_t dense = 0;
    if (st == C2KV_OK) st = check_rows("q", *cfg, q, cfg->n_q_heads, q_stride);
    if (st == C2KV_OK) st = check_rows("out", *cfg, out, cfg->n_q_heads, dense);
    if (st != C2KV_OK) return st;
    const c2kv::AttendShape sh = attend_shape(*cfg, *cache, *chunks);
    if (too_long(sh, *cfg, *cache, *chunks)) return fail(C2KV_E_UNSUPPORTED, kTooLong);
    if (!workspace) return fail(C2KV_E_WORKSPACE, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
      return fail(C2KV_E_WORKSPACE, "workspace must be 256-byte aligned");
    if (workspace_bytes < sh.total)
      return fail(C2KV_E_WORKSPACE, "workspace has " + std::to_string(workspace_bytes) +
                                        " bytes, the call needs " + std::to_string(sh.total));
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const float scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale
                                                 : float(1.0 / std::sqrt(double(cfg->head_dim)));
    c2kv::AttendParams p{};
    p.ch = view(*chunks);
    p.pg = view(*cache, *cfg);
    p.rope = rope(*cfg, pos);
    p.Hq = cfg->n_q_heads;
    p.G = cfg->n_q_heads / cfg->n_kv_heads;
    p.rb = sh.unit_rows;
    p.qscale = float(double(scale) * 1.4426950408889634074);
    p.q = q;
    p.q_stride = q_stride;
    p.out = out;
    p.lse = lse;
    p.part_o = reinterpret_cast<float*>(ws + sh.part_o);
    p.part_ml = reinterpret_cast<float2*>(ws + sh.part_ml);
    p.joins = reinterpret_cast<c2kv::Join*>(ws + sh.joins);
    p.groups = sh.groups;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = timed("cache_attend", [&](hipEvent_t e0, hipEvent_t e1) {
      return c2kv::launch_cache_attend(p, sh, cache->dtype, cfg->head_dim, s, e0, e1);
    });
    if (e != hipSuccess) return hip_fail(e, "cache attention launch");
    if (sh.groups > 1) {
      e = timed("cache_merge", [&](hipEvent_t e0, hipEvent_t e1) {
        return c2kv::launch_cache_merge(p, sh, cache->dtype, cfg->head_dim, s, e0, e1);
      });
      if (e != hipSuccess) return hip_fail(e, "cache merge launch");
    }
    return C2KV_OK;
  });
}

c2kv_status c2kv_pool_write(const c2kv_attn_cfg* cfg, const c2kv_pool* pool, int32_t n,
                            const int64_t* row, const void* k, int64_t k_stride,
                            const void* v, int64_t v_stride, const int32_t* pos,
                            void* stream) {
  return guarded([&] {
    c2kv_status st = check_shape(cfg);
    if (st != C2KV_OK) return st;
    if (!pool) return fail(C2KV_E_INVAL, "pool is NULL");
    st = check_store("pool", pool->dtype, *cfg, pool->k, pool->v, pool->k_scale, pool->v_scale);
    if (st != C2KV_OK) return st;
    if (n < 0 || pool->n_rows < 0) return fail(C2KV_E_INVAL, "n and n_rows must be >= 0");
    if (n == 0) return C2KV_OK;
    if (n > 1 << 28) return fail(C2KV_E_UNSUPPORTED, "more than 2^28 rows a call are not built");
    if (!row) return fail(C2KV_E_INVAL, "row must not be NULL");
    st = check_rows("k", *cfg, k, cfg->n_kv_heads, k_stride);
    if (st == C2KV_OK) st = check_rows("v", *cfg, v, cfg->n_kv_heads, v_stride);
    if (st != C2KV_OK) return st;
    const c2kv::PoolWriteParams p{rope(*cfg, pos), row, n, cfg->n_kv_heads, pool->n_rows, k, v,
                                  k_stride, v_stride, const_cast<void*>(pool->k),
                                  const_cast<void*>(pool->v), const_cast<float*>(pool->k_scale),
                                  const_cast<float*>(pool->v_scale)};
    hipError_t e = timed("pool_write", [&](hipEvent_t e0, hipEvent_t e1) {
      return c2kv::launch_pool_write(p, pool->dtype, cfg->head_dim,
                                     static_cast<hipStream_t>(stream), e0, e1);
    });
    return e == hipSuccess ? C2KV_OK : hip_fail(e, "pool write launch");
  });
}

c2kv_status c2kv_timing_enable(int32_t on) {
  std::lock_guard<std::mutex> lk(g_timing.mu);
  g_timing.on = on != 0;
  return C2KV_OK;
}

c2kv_status c2kv_timing_reset(void) {
  std::lock_guard<std::mutex> lk(g_timing.mu);
  for (auto& kv : g_timing.recs)
    for (auto& r : kv.second) {
      g_timing.spare.push_back(r.a);
      g_timing.spare.push_back(r.b);
    }
  g_timing.recs.clear();
  return C2KV_OK;
}

c2kv_status c2kv_timing_read(const char* name, double* total_ms, int64_t* launches) {
  if (!name || !total_ms || !launches) return fail(C2KV_E_INVAL, "NULL argument");
  std::lock_guard<std::mutex> lk(g_timing.mu);
  *total_ms = 0.0;
  *launches = 0;
  auto it = g_timing.recs.find(name);
  if (it == g_timing.recs.end()) return C2KV_OK;
  for (auto& r : it->second) {
    hipError_t e = hipEventSynchronize(r.b);
    if (e != hipSuccess) return hip_fail(e, "hipEventSynchronize");
    float ms = 0.f;
    e = hipEventElapsedTime(&ms, r.a, r.b);
    if (e != hipSuccess) return hip_fail(e, "hipEventElapsedTime");
    *total_ms += ms;
    ++*launches;
  }
  return C2KV_OK;
}

}  // extern "C"
