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

constexpr int DRAFT = 64;  // drafted tokens of a sequence at most
// Of lane i < n: the drafted tokens that token i sees, its ancestors and itself, as bits. By doubled steps:
// after k of them a lane holds its 2^k nearest. A parent that is no earlier token counts as none.
__device__ __forceinline__ uint64_t ancestors(const int32_t* __restrict__ parents, int64_t first, int n, int lane) {
  int up = lane < n ? parents[first + lane] : -1;
  if (up < 0 || up >= lane) up = -1;
  uint64_t seen = (uint64_t)1 << lane;
#pragma unroll
  for (int k = 0; k < 6; ++k) {
    const int src = up < 0 ? lane : up;
    const uint64_t more = __shfl(seen, src);
    const int next = __shfl(up, src);
    if (up >= 0) {
      seen |= more;
      up = next;
    }
  }
  return seen;
}
// Which of the 64 slots from t0 on are seen by a row that sees all slots before `past`, and behind those the
// ones of `own`.
__device__ __forceinline__ uint64_t seen_slots(int64_t t0, int64_t past, uint64_t own) {
  const int64_t rel = t0 - past;
  return rel >= 64 ? 0u : rel >= 0 ? own >> rel : rel > -64 ? (own << -rel) | (((uint64_t)1 << -rel) - 1) : ~(uint64_t)0;
}

// Where the scan's work lies: chunks of tiles_per_chunk tiles, the sequences' one after the
// other (items), about as many as the call has workgroups for (p.scan_items). The length of a
// chunk comes from what the sequences hold, not from the longest that the call allows.
struct ScanPlace {
  int b, chunk;    // of an item; b < 0: none
  int n_chunks;    // of its sequence
  int tiles_per_chunk;
};
struct ScanScratch {
  int64_t part[4];
  int64_t total;
  int32_t b, at, n;
};
// Of an item; the same in every thread of a workgroup of 256.
__device__ __forceinline__ ScanPlace scan_place(const PagedAttnArgs& p, int item, ScanScratch& s) {
  constexpr int NT = 256;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto tiles_of = [&](int b) -> int64_t {
    if (b >= p.c.batch) return 0;
    const PagedSeq q = paged_seq(p.c, b);
    return scanned(p, q) ? (q.len + TILE - 1) / TILE : 0;
  };
  // inclusive sum of v over the workgroup; the total in s.total
  auto sum = [&](int64_t v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t u = __shfl_up(v, o);
      if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 63) s.part[wave] = v;
    __syncthreads();
    int64_t before = 0;
    for (int w = 0; w < wave; ++w) before += s.part[w];
    if (tid == NT - 1) s.total = before + v;
    __syncthreads();
    return before + v;
  };
  const int64_t mine = tiles_of(tid);  // of the first NT sequences
  int64_t total = 0;
  if (p.c.batch == 1) {
    total = tiles_of(0);
  } else {
    int64_t v = mine;
    for (int b = tid + NT; b < p.c.batch; b += NT) v += tiles_of(b);
    sum(v);
    total = s.total;
  }
  ScanPlace r;
  // every sequence ends in half a chunk on average: those count too
  const int64_t whole = p.scan_items - (p.c.batch < p.scan_items ? p.c.batch : p.scan_items) / 2;
  int64_t tpc = (total + whole - 1) / whole;
  tpc = (tpc + 3) & ~(int64_t)3;  // whole steps of four wavefronts
  constexpr int64_t most = (int64_t)1 << 24;  // tiles of the longest row
  r.tiles_per_chunk = (int)(tpc < p.scan_least ? p.scan_least : tpc < most ? tpc : most);
  if (p.c.batch == 1) {
    r.n_chunks = (int)((total + r.tiles_per_chunk - 1) / r.tiles_per_chunk);
    r.chunk = item;
    r.b = item < r.n_chunks ? 0 : -1;
    return r;
  }
  if (tid == 0) s.b = -1;
  int base = 0;
  for (int b0 = 0; b0 < p.c.batch; b0 += NT) {
    const int64_t t = b0 == 0 ? mine : tiles_of(b0 + tid);
    const int n = (int)((t + r.tiles_per_chunk - 1) / r.tiles_per_chunk);
    const int lo = base + (int)sum(n) - n;
    if (item >= lo && item < lo + n) {
      s.b = b0 + tid;
      s.at = lo;
      s.n = n;
    }
    __syncthreads();
    if (s.b >= 0) break;
    base += (int)s.total;
    __syncthreads();
  }
  r.b = __builtin_amdgcn_readfirstlane(s.b);
  r.n_chunks = __builtin_amdgcn_readfirstlane(s.n);
  r.chunk = item - __builtin_amdgcn_readfirstlane(s.at);
  return r;
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
