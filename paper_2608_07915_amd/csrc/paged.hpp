// Argument blocks and launchers of the paged cache (host and device visible).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "spectra.h"

namespace spectra_dev {

constexpr int PAGES_LIST = 1024;  // entries of one page-map call
constexpr int PAGES_POOLS = 64;   // pools of one copy launch

// The page map as kernels see it (spectra_pages).
struct PageMap {
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int32_t n_pages, page_tokens, rows, row_pages;
};

struct PoolList {
  uint32_t* base[PAGES_POOLS];
  int64_t words[PAGES_POOLS];  // of a page
  int32_t n;
};

// Workspace of the page-map calls: the number of pages to copy, then their sources and their
// destinations (n_pages of each).
struct PageMoves {
  int32_t* count;
  int32_t* src;
  int32_t* dst;
};

// A cache as the append and the attention see it: pages, and which sequences take part.
struct PagedCache {
  const int32_t* table;
  const int32_t* lens;  // by map row
  const int32_t* ends;  // by sequence of the call, or null: lens of its row
  const int32_t* rows;  // map row of each sequence, or null: sequence b is row b
  const int32_t* cu;    // [batch + 1] first new token of each sequence
  int64_t n_new;        // rows of the token arrays
  int32_t n_pages, page_tokens, n_rows, row_pages;
  int32_t batch, n_kv;
};

struct PagedEncodeArgs {
  PagedCache c;
  const void* x[2];  // keys, values
  int64_t token_stride[2], head_stride[2];
  const float* basis[2];
  const float* mean[2];
  const uint8_t* bits[2];
  uint32_t* pool[2];
  int32_t W[2];
};

struct PagedAttnArgs {
  PagedCache c;
  const uint32_t* pool_k;
  const uint32_t* pool_v;
  const float* basis_k;
  const float* basis_v;
  const float* mean_k;
  const float* mean_v;
  const uint8_t* bits_k;
  const uint8_t* bits_v;
  const void* q;
  int64_t q_token_stride, q_head_stride;
  int32_t q_f32, out_f32;
  int32_t n_q_heads, n_qh;
  int32_t max_new;
  int32_t scan_tokens;  // sequences with at most so many new tokens are the scan kernel's
  int32_t scan_items, scan_least;  // its workgroups per KV head, and the fewest tiles of one
  int32_t* scan_plan;   // workspace: [batch][2], a sequence's first item and how many it has
  int32_t Wk, Wv;
  int64_t max_tokens;
  float scale_log2;  // softmax scale * log2(e)
  void* out;         // [n_new][n_q_heads][128]
  float* lse;        // [n_new][n_q_heads] or null
  float* lse_u;      // workspace: scale V_K m_K of each KV head
  // chunk kernel: the slots of a part, parts, and their results (joined when a unit has several)
  int64_t part_slots;
  int32_t parts;
  float* partial;
};

}  // namespace spectra_dev

namespace spectra {
hipError_t launch_pages_extend(const spectra_dev::PageMap& m, const int32_t* rows, const int32_t* counts, int32_t n,
                               int32_t* ends, const spectra_dev::PageMoves& mv, hipStream_t st);
hipError_t launch_pages_fork(const spectra_dev::PageMap& m, const int32_t* parents, const int32_t* children, int32_t n,
                             int32_t* ends, hipStream_t st);
hipError_t launch_pages_truncate(const spectra_dev::PageMap& m, const int32_t* rows, const int32_t* keep, int32_t n,
                                 hipStream_t st);
hipError_t launch_pages_compact(const spectra_dev::PageMap& m, int32_t* moved, const spectra_dev::PageMoves& mv,
                                hipStream_t st);
// Copies the listed pages in every pool, most_moves of them at most.
hipError_t launch_page_copies(const spectra_dev::PoolList& pools, const spectra_dev::PageMoves& mv, int64_t most_moves,
                              hipStream_t st);
hipError_t launch_paged_encode(const spectra_dev::PagedEncodeArgs& a, bool f32_input, hipStream_t st);
// Sequences of at most a.scan_tokens new tokens (a.scan_tokens * n_qh <= scan_rows): chunks into partial, and their join.
void launch_paged_scan(const spectra_dev::PagedAttnArgs& a, float* partial, hipStream_t st);
hipError_t launch_paged_combine(const spectra_dev::PagedAttnArgs& a, float* partial, hipStream_t st);
hipError_t launch_paged_attention(const spectra_dev::PagedAttnArgs& a, void* workspace, hipStream_t st);
}  // namespace spectra
