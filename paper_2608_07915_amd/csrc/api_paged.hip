// C entry points of the paged cache: argument checks and launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "api_common.hpp"
#include "paged.hpp"
#include "splits.hpp"

using namespace spectra;
using spectra_dev::PagedAttnArgs;
using spectra_dev::PagedCache;
using spectra_dev::PagedEncodeArgs;
using spectra_dev::PageMap;
using spectra_dev::PageMoves;
using spectra_dev::PoolList;

namespace {

constexpr int64_t kMaxBatch = 16384;
constexpr int64_t kMost = (int64_t)1 << 30;       // slots of a row, query rows of a call: counted in 32 bits
constexpr int32_t kMostPage = 1 << 20;            // slots of a page: a record's place in it too
constexpr int64_t kMostGroups = (int64_t)1 << 18;  // sequences times KV heads: 16 workgroups each at most

spectra_status check_map(const spectra_pages* m, const char* name, bool with_refs) {
  if (!m) return fail(SPECTRA_EINVAL, "%s: null page map", name);
  if (m->n_pages <= 0 || m->n_pages >= ((int64_t)1 << 31) - 1)
    return fail(SPECTRA_EINVAL, "%s: n_pages=%lld out of range", name, (long long)m->n_pages);
  if (m->page_tokens <= 0 || m->page_tokens % 64 != 0 || m->page_tokens > kMostPage)
    return fail(SPECTRA_EINVAL, "%s: page_tokens=%d must be a positive multiple of 64 up to 2^20", name, m->page_tokens);
  if (m->rows <= 0 || m->rows > 65535) return fail(SPECTRA_EINVAL, "%s: rows=%d out of range [1, 65535]", name, m->rows);
  if (m->row_pages <= 0 || (int64_t)m->row_pages * m->page_tokens > kMost)
    return fail(SPECTRA_EINVAL, "%s: row_pages=%d must be positive and a row's slots at most 2^30", name, m->row_pages);
  if (!m->table || !m->lens || !aligned(m->table, 4) || !aligned(m->lens, 4))
    return fail(SPECTRA_EINVAL, "%s: table and lens must be non-null and 4-byte aligned", name);
  if (with_refs && (!m->refs || !aligned(m->refs, 4)))
    return fail(SPECTRA_EINVAL, "%s: refs must be non-null and 4-byte aligned", name);
  return SPECTRA_OK;
}

PageMap map_of(const spectra_pages* m) {
  return PageMap{m->table, m->lens, m->refs, (int32_t)m->n_pages, m->page_tokens, m->rows, m->row_pages};
}

spectra_status check_list(const char* name, int32_t n, const void* a, const void* b) {
  if (n < 0 || n > spectra_dev::PAGES_LIST)
    return fail(SPECTRA_EINVAL, "%s: n=%d out of range [0, %d]", name, n, spectra_dev::PAGES_LIST);
  if (n > 0 && (!a || !b || !aligned(a, 4) || !aligned(b, 4)))
    return fail(SPECTRA_EINVAL, "%s: lists must be non-null and 4-byte aligned", name);
  return SPECTRA_OK;
}

spectra_status check_pools(const char* name, const spectra_pool* pools, int32_t n_pools) {
  if (n_pools < 0 || (n_pools > 0 && !pools)) return fail(SPECTRA_EINVAL, "%s: n_pools=%d, or null pools", name, n_pools);
  for (int i = 0; i < n_pools; ++i) {
    if (pools[i].page_words < 0 || pools[i].page_words % 64 != 0 || pools[i].page_words >= ((int64_t)1 << 40))
      return fail(SPECTRA_EINVAL, "%s: pool %d: page_words=%lld must be a multiple of 64", name, i, (long long)pools[i].page_words);
    if (pools[i].page_words > 0 && (!pools[i].base || !aligned(pools[i].base, 16)))
      return fail(SPECTRA_EINVAL, "%s: pool %d must be non-null and 16-byte aligned", name, i);
  }
  return SPECTRA_OK;
}

spectra_status check_moves(const char* name, const spectra_pages* m, void* workspace, size_t ws_bytes, PageMoves* mv) {
  if (!workspace || !aligned(workspace, 256)) return fail(SPECTRA_EINVAL, "%s: workspace must be 256-byte aligned", name);
  const size_t need = spectra_pages_workspace_bytes(m);
  if (ws_bytes < need) return fail(SPECTRA_EWORKSPACE, "%s: workspace %zu < %zu bytes", name, ws_bytes, need);
  mv->count = static_cast<int32_t*>(workspace);
  mv->src = mv->count + 64;
  mv->dst = mv->src + m->n_pages;
  return SPECTRA_OK;
}

hipError_t copy_pages(const spectra_pool* pools, int32_t n_pools, const PageMoves& mv, int64_t most, hipStream_t st) {
  for (int i = 0; i < n_pools; i += spectra_dev::PAGES_POOLS) {
    PoolList l{};
    for (l.n = 0; l.n < spectra_dev::PAGES_POOLS && i + l.n < n_pools; ++l.n) {
      l.base[l.n] = pools[i + l.n].base;
      l.words[l.n] = pools[i + l.n].page_words;
    }
    const hipError_t e = launch_page_copies(l, mv, most, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Checks shared by append and attention; fills the cache part.
spectra_status check_cache(const char* name, const spectra_pages* m, const spectra_codec* ck, const spectra_codec* cv,
                           const void* pool_k, const void* pool_v, const int32_t* rows, const int32_t* ends,
                           const int32_t* cu_new, int32_t batch, int64_t n_new, PagedCache* c) {
  spectra_status st = check_map(m, name, false);
  if (st != SPECTRA_OK) return st;
  if ((st = check_codec(ck, name)) != SPECTRA_OK) return st;
  if ((st = check_codec(cv, name)) != SPECTRA_OK) return st;
  if (ck->n_streams != cv->n_streams)
    return fail(SPECTRA_EINVAL, "%s: the codecs hold %lld and %lld KV heads", name, (long long)ck->n_streams, (long long)cv->n_streams);
  if (batch < 0 || batch > kMaxBatch) return fail(SPECTRA_EINVAL, "%s: batch=%d out of range [0, %lld]", name, batch, (long long)kMaxBatch);
  if (!rows && batch > m->rows) return fail(SPECTRA_EINVAL, "%s: batch=%d exceeds the map's %d rows", name, batch, m->rows);
  if (n_new < 0 || n_new >= ((int64_t)1 << 31)) return fail(SPECTRA_EINVAL, "%s: n_new=%lld out of range", name, (long long)n_new);
  if (batch > 0 && (!cu_new || !aligned(cu_new, 4))) return fail(SPECTRA_EINVAL, "%s: cu_new must be non-null and 4-byte aligned", name);
  if ((rows && !aligned(rows, 4)) || (ends && !aligned(ends, 4)))
    return fail(SPECTRA_EINVAL, "%s: rows and ends must be 4-byte aligned", name);
  if ((ck->record_words > 0 && (!pool_k || !aligned(pool_k, 16))) || (cv->record_words > 0 && (!pool_v || !aligned(pool_v, 16))))
    return fail(SPECTRA_EINVAL, "%s: pool_k / pool_v must be non-null and 16-byte aligned", name);
  *c = PagedCache{m->table, m->lens, ends, rows, cu_new, n_new, (int32_t)m->n_pages, m->page_tokens, m->rows, m->row_pages, batch,
                  (int32_t)ck->n_streams};
  return SPECTRA_OK;
}

// Token rows x[t * token_stride + head * head_stride + c].
spectra_status check_rows(const char* name, const char* what, const void* x, spectra_dtype dt, int64_t token_stride,
                          int64_t head_stride) {
  if (dt != SPECTRA_F32 && dt != SPECTRA_BF16) return fail(SPECTRA_EINVAL, "%s: dtype %d not supported", name, (int)dt);
  const int64_t vec = dt == SPECTRA_F32 ? 4 : 8;  // elements per 16 bytes
  if (!x || !aligned(x, 16)) return fail(SPECTRA_EINVAL, "%s: %s must be non-null and 16-byte aligned", name, what);
  if (token_stride < 0 || head_stride < 0 || token_stride % vec || head_stride % vec)
    return fail(SPECTRA_EINVAL, "%s: %s: strides must be non-negative multiples of %lld elements", name, what, (long long)vec);
  return SPECTRA_OK;
}

}  // namespace

extern "C" {

int64_t spectra_paged_pool_words(const spectra_pages* m, const spectra_codec* c) {
  if (!m || !c || m->n_pages <= 0 || m->page_tokens <= 0 || c->n_streams <= 0) return 0;
  return m->n_pages * m->page_tokens * c->n_streams * c->record_words;
}

size_t spectra_pages_workspace_bytes(const spectra_pages* m) {
  if (!m || m->n_pages <= 0) return 0;
  return 256 + round256((size_t)m->n_pages * 2 * sizeof(int32_t));
}

spectra_status spectra_pages_extend(const spectra_pages* m, const int32_t* rows, const int32_t* counts, int32_t n,
                                    const spectra_pool* pools, int32_t n_pools, int32_t* ends, void* workspace,
                                    size_t ws_bytes, void* stream) {
  const char* name = "pages_extend";
  spectra_status st = check_map(m, name, true);
  if (st != SPECTRA_OK) return st;
  if ((st = check_list(name, n, rows, counts)) != SPECTRA_OK) return st;
  if ((st = check_list(name, n, ends, ends)) != SPECTRA_OK) return st;
  if ((st = check_pools(name, pools, n_pools)) != SPECTRA_OK) return st;
  PageMoves mv{};
  if ((st = check_moves(name, m, workspace, ws_bytes, &mv)) != SPECTRA_OK) return st;
  if (n == 0) return SPECTRA_OK;
  hipError_t e = launch_pages_extend(map_of(m), rows, counts, n, ends, mv, (hipStream_t)stream);
  if (e == hipSuccess) e = copy_pages(pools, n_pools, mv, n < m->n_pages ? n : m->n_pages, (hipStream_t)stream);
  return e == hipSuccess ? SPECTRA_OK : hip_fail(e, "pages_extend launch");
}

spectra_status spectra_pages_fork(const spectra_pages* m, const int32_t* parents, const int32_t* children, int32_t n,
                                  int32_t* ends, void* stream) {
  const char* name = "pages_fork";
  spectra_status st = check_map(m, name, true);
  if (st != SPECTRA_OK) return st;
  if ((st = check_list(name, n, parents, children)) != SPECTRA_OK) return st;
  if ((st = check_list(name, n, ends, ends)) != SPECTRA_OK) return st;
  if (n == 0) return SPECTRA_OK;
  const hipError_t e = launch_pages_fork(map_of(m), parents, children, n, ends, (hipStream_t)stream);
  return e == hipSuccess ? SPECTRA_OK : hip_fail(e, "pages_fork launch");
}

spectra_status spectra_pages_truncate(const spectra_pages* m, const int32_t* rows, const int32_t* keep, int32_t n, void* stream) {
  const char* name = "pages_truncate";
  spectra_status st = check_map(m, name, true);
  if (st != SPECTRA_OK) return st;
  if ((st = check_list(name, n, rows, keep ? keep : rows)) != SPECTRA_OK) return st;
  if (n == 0) return SPECTRA_OK;
  const hipError_t e = launch_pages_truncate(map_of(m), rows, keep, n, (hipStream_t)stream);
  return e == hipSuccess ? SPECTRA_OK : hip_fail(e, "pages_truncate launch");
}

spectra_status spectra_pages_compact(const spectra_pages* m, const spectra_pool* pools, int32_t n_pools, int32_t* moved,
                                     void* workspace, size_t ws_bytes, void* stream) {
  const char* name = "pages_compact";
  spectra_status st = check_map(m, name, true);
  if (st != SPECTRA_OK) return st;
  if ((st = check_pools(name, pools, n_pools)) != SPECTRA_OK) return st;
  if (!moved || !aligned(moved, 4)) return fail(SPECTRA_EINVAL, "%s: moved must be non-null and 4-byte aligned", name);
  PageMoves mv{};
  if ((st = check_moves(name, m, workspace, ws_bytes, &mv)) != SPECTRA_OK) return st;
  hipError_t e = launch_pages_compact(map_of(m), moved, mv, (hipStream_t)stream);
  if (e == hipSuccess) e = copy_pages(pools, n_pools, mv, m->n_pages / 2, (hipStream_t)stream);
  return e == hipSuccess ? SPECTRA_OK : hip_fail(e, "pages_compact launch");
}

spectra_status spectra_paged_encode(const spectra_pages* m, const spectra_codec* ck, const spectra_codec* cv, uint32_t* pool_k,
                                    uint32_t* pool_v, const int32_t* rows, const int32_t* ends, const int32_t* cu_new,
                                    int32_t batch, int64_t n_new, const void* k, int64_t k_token_stride, int64_t k_head_stride,
                                    const void* v, int64_t v_token_stride, int64_t v_head_stride, spectra_dtype dt, void* stream) {
  const char* name = "paged_encode";
  PagedEncodeArgs a{};
  spectra_status st = check_cache(name, m, ck, cv, pool_k, pool_v, rows, ends, cu_new, batch, n_new, &a.c);
  if (st != SPECTRA_OK) return st;
  if (batch == 0 || n_new == 0) return SPECTRA_OK;
  if ((st = check_rows(name, "k", k, dt, k_token_stride, k_head_stride)) != SPECTRA_OK) return st;
  if ((st = check_rows(name, "v", v, dt, v_token_stride, v_head_stride)) != SPECTRA_OK) return st;
  if (a.c.n_kv > 32767) return fail(SPECTRA_EUNSUPPORTED, "%s: more than 32767 KV heads", name);
  const spectra_codec* c[2] = {ck, cv};
  uint32_t* pool[2] = {pool_k, pool_v};
  for (int i = 0; i < 2; ++i) {
    a.x[i] = i ? v : k;
    a.token_stride[i] = i ? v_token_stride : k_token_stride;
    a.head_stride[i] = i ? v_head_stride : k_head_stride;
    a.basis[i] = c[i]->basis;
    a.mean[i] = c[i]->mean;
    a.bits[i] = c[i]->bits;
    a.pool[i] = pool[i];
    a.W[i] = c[i]->record_words;
  }
  const hipError_t e = launch_paged_encode(a, dt == SPECTRA_F32, (hipStream_t)stream);
  return e == hipSuccess ? SPECTRA_OK : hip_fail(e, "paged_encode launch");
}

size_t spectra_paged_attention_workspace_bytes(int32_t batch, int64_t n_new, int32_t n_q_heads, int32_t n_kv_heads,
                                               int32_t max_new, int64_t max_tokens) {
  if (batch <= 0 || batch > kMaxBatch || n_new <= 0 || n_new > kMost || max_new <= 0 || max_tokens <= 0 || max_tokens > kMost) return 0;
  if (n_kv_heads <= 0 || n_kv_heads > 65535 || n_q_heads <= 0 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 16) return 0;
  return paged_workspace_bytes(batch, n_new, n_q_heads, n_kv_heads, max_new, max_tokens);
}

spectra_status spectra_paged_attention(const spectra_pages* m, const spectra_codec* ck, const spectra_codec* cv,
                                       const uint32_t* pool_k, const uint32_t* pool_v, const int32_t* rows, const int32_t* ends,
                                       const int32_t* cu_new, int32_t batch, int64_t n_new, int32_t max_new, int64_t max_tokens,
                                       const void* q, spectra_dtype q_dt, int64_t q_token_stride, int64_t q_head_stride,
                                       int32_t n_q_heads, float softmax_scale, void* out, spectra_dtype out_dt, float* lse,
                                       void* workspace, size_t ws_bytes, void* stream) {
  const char* name = "paged_attention";
  PagedAttnArgs a{};
  spectra_status st = check_cache(name, m, ck, cv, pool_k, pool_v, rows, ends, cu_new, batch, n_new, &a.c);
  if (st != SPECTRA_OK) return st;
  if (n_q_heads <= 0 || n_q_heads % a.c.n_kv != 0)
    return fail(SPECTRA_EINVAL, "%s: n_q_heads=%d must be a positive multiple of the codecs' %d KV heads", name, n_q_heads, a.c.n_kv);
  if (n_q_heads / a.c.n_kv > 16) return fail(SPECTRA_EUNSUPPORTED, "%s: more than 16 query heads per KV head", name);
  if (max_new < 0 || max_tokens < 0 || max_tokens > kMost || (int64_t)max_new * n_q_heads > kMost)
    return fail(SPECTRA_EINVAL, "%s: max_new=%d or max_tokens=%lld out of range", name, max_new, (long long)max_tokens);
  if (n_new * n_q_heads > kMost || (int64_t)batch * a.c.n_kv >= kMostGroups)
    return fail(SPECTRA_EINVAL, "%s: n_new=%lld times %d query heads passes 2^30, or batch=%d times %d KV heads 2^18", name,
                (long long)n_new, n_q_heads, batch, a.c.n_kv);
  if (!(softmax_scale == softmax_scale) || std::isinf(softmax_scale)) return fail(SPECTRA_EINVAL, "%s: softmax_scale not finite", name);
  if (out_dt != SPECTRA_F32 && out_dt != SPECTRA_BF16) return fail(SPECTRA_EINVAL, "%s: output dtype %d not supported", name, (int)out_dt);
  if (batch == 0 || n_new == 0 || max_new == 0 || max_tokens == 0) return SPECTRA_OK;
  if ((st = check_rows(name, "q", q, q_dt, q_token_stride, q_head_stride)) != SPECTRA_OK) return st;
  if (!out || !aligned(out, 16) || (lse && !aligned(lse, 4)))
    return fail(SPECTRA_EINVAL, "%s: out must be non-null and 16-byte aligned, lse 4-byte aligned", name);
  const size_t need = spectra_paged_attention_workspace_bytes(batch, n_new, n_q_heads, a.c.n_kv, max_new, max_tokens);
  if (!workspace || !aligned(workspace, 256)) return fail(SPECTRA_EINVAL, "%s: workspace must be 256-byte aligned", name);
  if (ws_bytes < need) return fail(SPECTRA_EWORKSPACE, "%s: workspace %zu < %zu bytes", name, ws_bytes, need);
  a.pool_k = pool_k;
  a.pool_v = pool_v;
  a.basis_k = ck->basis;
  a.basis_v = cv->basis;
  a.mean_k = ck->mean;
  a.mean_v = cv->mean;
  a.bits_k = ck->bits;
  a.bits_v = cv->bits;
  a.q = q;
  a.q_token_stride = q_token_stride;
  a.q_head_stride = q_head_stride;
  a.q_f32 = q_dt == SPECTRA_F32;
  a.out_f32 = out_dt == SPECTRA_F32;
  a.n_q_heads = n_q_heads;
  a.n_qh = n_q_heads / a.c.n_kv;
  a.max_new = max_new;
  a.max_tokens = max_tokens;
  a.Wk = ck->record_words;
  a.Wv = cv->record_words;
  a.scale_log2 = (softmax_scale > 0.0f ? softmax_scale : 1.0f / std::sqrt(128.0f)) * 1.4426950408889634f;
  a.out = out;
  a.lse = lse;
  const hipError_t e = launch_paged_attention(a, workspace, (hipStream_t)stream);
  return e == hipSuccess ? SPECTRA_OK : hip_fail(e, "paged_attention launch");
}

}  // extern "C"
