// Device helpers of the paged cache: which slots a sequence's new tokens take, and where a
// slot's record lies. What device arrays hold is never trusted: sequences are cut to the token
// arrays, lengths to the row's slots, and pages outside the pool are not touched.
#pragma once
#include "device_common.hpp"
#include "paged.hpp"

namespace spectra_dev {

struct PagedSeq {
  int64_t first;  // its first new token
  int64_t n;      // new tokens
  int64_t len;    // slots, new tokens included; 0 where the sequence takes no part
  int row;        // of the table
};

__device__ __forceinline__ PagedSeq paged_seq(const PagedCache& c, int b) {
  PagedSeq s;
  int64_t lo = c.cu[b], hi = c.cu[b + 1];
  lo = lo < 0 ? 0 : (lo > c.n_new ? c.n_new : lo);
  hi = hi < lo ? lo : (hi > c.n_new ? c.n_new : hi);
  s.first = lo;
  s.n = hi - lo;
  s.row = c.rows ? c.rows[b] : b;
  s.len = 0;
  if (s.row >= 0 && s.row < c.n_rows) {
    const int64_t cap = (int64_t)c.row_pages * c.page_tokens;
    const int64_t len = c.ends ? c.ends[b] : c.lens[s.row];
    s.len = len < 0 ? 0 : (len > cap ? cap : len);
  }
  return s;
}

// Word 0 of token 0 of KV head kv's records of 64-slot tile `tile` (of W words), or null where
// the row has no page of the pool there. tile < row_pages * page_tokens / 64.
template <typename Word>
__device__ __forceinline__ Word* paged_tile(const PagedCache& c, Word* pool, int W, int row, int64_t tile, int kv) {
  const int tpp = c.page_tokens >> 6;
  const int64_t at = tile / tpp;
  const int page = c.table[(int64_t)row * c.row_pages + at];
  if (page < 0 || page >= c.n_pages) return nullptr;
  return pool + (((int64_t)page * c.n_kv + kv) * tpp + (tile - at * tpp)) * (int64_t)(TILE * W);
}

// Sequences past the call's bounds are left out, their rows as they were.
__device__ __forceinline__ bool attended(const PagedAttnArgs& a, const PagedSeq& s) {
  return s.n <= a.max_new && s.len <= a.max_tokens;
}
// Few new tokens: the scan's; the others are the chunk kernel's.
__device__ __forceinline__ bool scanned(const PagedAttnArgs& a, const PagedSeq& s) {
  return s.n > 0 && s.n <= a.scan_tokens && attended(a, s);
}

__device__ __forceinline__ float query_at(const PagedAttnArgs& a, int64_t i) {
  return a.q_f32 ? reinterpret_cast<const float*>(a.q)[i] : bf2f(reinterpret_cast<const uint16_t*>(a.q)[i]);
}

// A metadata word, 0 where its scale or zero point is NaN or infinite.
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t m) {
  return (m & 0x7C00u) == 0x7C00u || (m & 0x7C000000u) == 0x7C000000u ? 0u : m;
}

constexpr float LN2 = 0.69314718055994531f;

}  // namespace spectra_dev
