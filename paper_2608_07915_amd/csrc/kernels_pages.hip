// Page maps of packed caches: making room, branching, dropping and compacting sequences.
// Whole numbers only. Every result is a function of the arguments alone: free pages are taken
// lowest first, list entries served in their order, and the only atomics add to counts.
#include "paged.hpp"

namespace spectra_dev {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int PLAN = 1024;  // threads of a planning workgroup
static_assert(PAGES_LIST == PLAN, "an entry per thread");

__device__ __forceinline__ int64_t ceil_pages(int64_t tokens, int page_tokens) {
  return (tokens + page_tokens - 1) / page_tokens;
}

// A row's length where it is one that the row can hold, otherwise -1.
__device__ __forceinline__ int64_t row_len(const PageMap& m, int row) {
  if (row < 0 || row >= m.rows) return -1;
  const int64_t len = m.lens[row];
  return len >= 0 && len <= (int64_t)m.row_pages * m.page_tokens ? len : -1;
}

// Inclusive sum over the workgroup's threads; part: LDS of one entry per wavefront.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();  // part's last readers are done
  if (lane == 63) part[wave] = v;
  __syncthreads();
  int64_t base = 0;
  for (int w = 0; w < wave; ++w) base += part[w];
  return base + v;
}

// Pages of [lo, hi) that `take` accepts, in ascending order: out[k] is the k-th, k < most; the
// return value, the same in every thread, is how many there are (counted no further than the
// round in which they reach `most`). A thread looks at 16 neighbouring pages a round.
template <typename Take>
__device__ __forceinline__ int64_t list_pages(const int32_t* __restrict__ refs, int64_t lo, int64_t hi, int64_t most,
                                              int32_t* __restrict__ out, int64_t* part, Take&& take) {
  constexpr int EACH = 16;
  __shared__ int64_t total_s;
  int64_t found = 0;
  for (int64_t p0 = lo; p0 < hi && found < most; p0 += PLAN * EACH) {
    const int64_t p = p0 + (int64_t)threadIdx.x * EACH;
    uint32_t mask = 0u;
    if (p + EACH <= hi && (reinterpret_cast<uintptr_t>(refs + p) & 15) == 0) {
      i32x4 r[EACH / 4];
#pragma unroll
      for (int i = 0; i < EACH / 4; ++i) r[i] = reinterpret_cast<const i32x4*>(refs + p)[i];
#pragma unroll
      for (int i = 0; i < EACH; ++i) mask |= take(r[i >> 2][i & 3]) ? 1u << i : 0u;
    } else {
#pragma unroll
      for (int i = 0; i < EACH; ++i) mask |= (p + i < hi && take(refs[p + i])) ? 1u << i : 0u;
    }
    const int mine = __popc(mask);
    const int64_t upto = block_scan(mine, part);
    if (threadIdx.x == PLAN - 1) total_s = upto;
    int64_t k = found + upto - mine;
    while (mask) {
      if (k < most) out[k] = (int32_t)(p + __ffs(mask) - 1);
      mask &= mask - 1;
      ++k;
    }
    __syncthreads();
    found += total_s;
  }
  return found;
}

// ---------------------------------------------------------------------------
// Room for new tokens. One workgroup, a list entry per thread: what every entry needs (new
// pages, and a copy of a partly filled last page that has other owners), their running sum,
// the lowest free pages, and who gets them. 2 n loads and one pass over the counts until
// enough free pages are found: bound by latency (the pool's first 16 k counts are one round).
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(PLAN) void pages_extend_kernel(PageMap m, const int32_t* __restrict__ rows,
                                                            const int32_t* __restrict__ counts, int n,
                                                            int32_t* __restrict__ ends, PageMoves mv) {
  __shared__ int32_t row_s[PLAN], last_s[PLAN];
  __shared__ int64_t upto_s[PLAN], part[PLAN / 64];
  __shared__ int32_t start_s[PLAN], copy_s[PLAN];
  __shared__ int64_t granted_s;
  const int t = threadIdx.x;
  const int row = t < n ? rows[t] : -1;
  const int64_t add = t < n ? counts[t] : -1;
  row_s[t] = row;
  if (t == 0) granted_s = 0;
  const int64_t len = row_len(m, row);
  bool ok = t < n && len >= 0 && add >= 0 && len + add <= (int64_t)m.row_pages * m.page_tokens;
  int last = -1;
  if (ok && add > 0 && len % m.page_tokens != 0) {
    last = m.table[(int64_t)row * m.row_pages + len / m.page_tokens];
    if (last < 0 || last >= m.n_pages) ok = false;
  }
  const int owners = ok && last >= 0 ? m.refs[last] : 0;
  __syncthreads();
  for (int j = 0; j < t && t < n; ++j) ok = ok && row_s[j] != row;  // a row listed again is refused
  last_s[t] = ok ? last : -1;
  __syncthreads();
  // owners ahead in the list have left the page by then, each with a copy of its own
  int ahead = 0;
  if (ok && last >= 0)
    for (int j = 0; j < t; ++j) ahead += last_s[j] == last ? 1 : 0;
  const bool copies = ok && last >= 0 && owners - ahead > 1;
  const int64_t start = ok ? ceil_pages(len, m.page_tokens) - (copies ? 1 : 0) : 0;
  const int64_t want = ok ? ceil_pages(len + add, m.page_tokens) - start : 0;
  const int64_t upto = block_scan(want, part);
  upto_s[t] = upto;
  start_s[t] = (int32_t)start;
  __syncthreads();
  const int64_t wanted = upto_s[PLAN - 1];
  int64_t avail = 0;
  // the free pages go to the move list's second half, which is written from its start below
  if (wanted > 0)
    avail = list_pages(m.refs, 0, m.n_pages, wanted < m.n_pages ? wanted : m.n_pages, mv.dst, part,
                       [](int32_t r) { return r == 0; });
  // served in the order listed; from the first that finds too few, whoever needs a page, or
  // counted on an entry before it to leave one, is refused
  const bool granted = ok && ((want == 0 && ahead == 0) || upto <= avail);
  copy_s[t] = granted && copies ? last : -1;
  if (granted && want > 0) atomicMax(reinterpret_cast<unsigned long long*>(&granted_s), (unsigned long long)upto);
  if (t < n) ends[t] = granted ? (int32_t)(len + add) : -1;
  if (granted) m.lens[row] = (int32_t)(len + add);
  const int64_t n_copies = block_scan(granted && copies ? 1 : 0, part);
  __syncthreads();
  for (int64_t k = t; k < granted_s; k += PLAN) {
    int lo = 0, hi = PLAN - 1;  // the first entry whose sum passes k
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (upto_s[mid] > k) hi = mid; else lo = mid + 1;
    }
    const int64_t before = lo > 0 ? upto_s[lo - 1] : 0;
    const int32_t page = mv.dst[k];
    m.table[(int64_t)row_s[lo] * m.row_pages + start_s[lo] + (k - before)] = page;
    m.refs[page] = 1;
  }
  // the copies: the entry's first page takes its old last page's records
  int32_t to = -1;
  if (granted && copies) {
    to = mv.dst[upto - want];
    atomicSub(&m.refs[last], 1);
  }
  __syncthreads();  // the free list has been read
  if (granted && copies) {
    mv.src[n_copies - 1] = last;
    mv.dst[n_copies - 1] = to;
  }
  if (t == PLAN - 1) *mv.count = (int32_t)n_copies;
}

// ---------------------------------------------------------------------------
// Branching: entry i's child becomes another owner of its parent's pages. A workgroup per
// entry. A child must be empty and listed once, and no parent; so the rows that are read and
// the rows that are written are different ones and the entries need no order.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pages_fork_kernel(PageMap m, const int32_t* __restrict__ parents,
                                                         const int32_t* __restrict__ children, int n,
                                                         int32_t* __restrict__ ends) {
  const int i = blockIdx.x, t = threadIdx.x;
  const int parent = parents[i], child = children[i];
  bool bad = child < 0 || child >= m.rows || parent < 0 || parent >= m.rows;
  for (int j = t; j < n; j += 256) {
    const int c = children[j];
    bad = bad || c == parent || (j < i && c == child);
  }
  bad = __syncthreads_or(bad) != 0;
  // row `child` is written by this workgroup alone, and row `parent` by none
  const int64_t len = bad ? -1 : row_len(m, parent);
  const int64_t old = bad ? -1 : m.lens[child];
  __syncthreads();
  if (len < 0 || old != 0) {
    if (t == 0) ends[i] = -1;
    return;
  }
  const int32_t* src = m.table + (int64_t)parent * m.row_pages;
  int32_t* dst = m.table + (int64_t)child * m.row_pages;
  const int64_t pages = ceil_pages(len, m.page_tokens);
  for (int64_t k = t; k < pages; k += 256) {
    const int32_t p = src[k];
    dst[k] = p;
    if (p >= 0 && p < m.n_pages) atomicAdd(&m.refs[p], 1);
  }
  if (t == 0) {
    m.lens[child] = (int32_t)len;
    ends[i] = (int32_t)len;
  }
}

// ---------------------------------------------------------------------------
// Dropping the slots from keep[i] on (all of them without keep). A workgroup per entry; of a
// row listed more than once the first entry does it, with the smallest length listed.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pages_truncate_kernel(PageMap m, const int32_t* __restrict__ rows,
                                                             const int32_t* __restrict__ keep, int n) {
  __shared__ int32_t least_s;
  const int i = blockIdx.x, t = threadIdx.x, row = rows[i];
  if (t == 0) least_s = 0x7FFFFFFF;
  __syncthreads();
  bool again = false;
  int32_t least = 0x7FFFFFFF;
  for (int j = t; j < n; j += 256)
    if (rows[j] == row) {
      again = again || j < i;
      const int32_t k = keep ? keep[j] : 0;
      least = k < least ? k : least;
    }
  atomicMin(&least_s, least < 0 ? 0 : least);
  if (__syncthreads_or(again)) return;
  const int64_t len = row_len(m, row);
  const int64_t left = least_s;
  __syncthreads();  // every thread has the row's length
  if (len < 0 || left >= len) return;
  int32_t* tab = m.table + (int64_t)row * m.row_pages;
  for (int64_t k = ceil_pages(left, m.page_tokens) + t; k < ceil_pages(len, m.page_tokens); k += 256) {
    const int32_t p = tab[k];
    tab[k] = -1;
    if (p >= 0 && p < m.n_pages) atomicSub(&m.refs[p], 1);
  }
  if (t == 0) m.lens[row] = (int32_t)left;
}

// ---------------------------------------------------------------------------
// Compaction: with U used pages, the k-th used page at or past U moves to the k-th free page
// before U. Sources and destinations are disjoint, so the copies need no order. The plan is
// one workgroup's two passes over the counts (16 k pages a round).
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(PLAN) void pages_compact_kernel(PageMap m, int32_t* __restrict__ moved, PageMoves mv) {
  __shared__ int64_t part[PLAN / 64];
  __shared__ int64_t used_s;
  const int t = threadIdx.x;
  int64_t mine = 0;
  for (int64_t p0 = 0; p0 < m.n_pages; p0 += 8 * PLAN) {
    int32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = p0 + t + PLAN * i < m.n_pages ? m.refs[p0 + t + PLAN * i] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mine += r[i] > 0 ? 1 : 0;
      if (p0 + t + PLAN * i < m.n_pages) moved[p0 + t + PLAN * i] = (int32_t)(p0 + t + PLAN * i);
    }
  }
  const int64_t upto = block_scan(mine, part);
  if (t == PLAN - 1) used_s = upto;
  __syncthreads();
  const int64_t used = used_s;
  const int64_t holes = list_pages(m.refs, 0, used, used, mv.dst, part, [](int32_t r) { return r <= 0; });
  list_pages(m.refs, used, m.n_pages, holes, mv.src, part, [](int32_t r) { return r > 0; });
  __syncthreads();
  for (int64_t k0 = t; k0 < holes; k0 += 8 * PLAN) {
    int32_t s[8], d[8], r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t k = k0 + PLAN * i;
      s[i] = k < holes ? mv.src[k] : -1;
      d[i] = k < holes ? mv.dst[k] : -1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = s[i] >= 0 ? m.refs[s[i]] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (s[i] >= 0) {
        moved[s[i]] = d[i];
        m.refs[d[i]] = r[i];
        m.refs[s[i]] = 0;
      }
  }
  if (t == 0) {
    moved[m.n_pages] = (int32_t)used;
    *mv.count = (int32_t)holes;
  }
}

__global__ __launch_bounds__(256) void pages_retable_kernel(PageMap m, const int32_t* __restrict__ moved) {
  const int row = blockIdx.y;
  const int64_t len = row_len(m, row);
  const int64_t pages = len < 0 ? 0 : ceil_pages(len, m.page_tokens);
  int32_t* tab = m.table + (int64_t)row * m.row_pages;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < pages; k += (int64_t)gridDim.x * 256) {
    const int32_t p = tab[k];
    if (p >= 0 && p < m.n_pages) tab[k] = moved[p];
  }
}

// ---------------------------------------------------------------------------
// Page copies: work item = (move, pool, piece of 8 KB). Bound by HBM, read and write.
// ---------------------------------------------------------------------------
constexpr int PIECE = 2048;  // words
__global__ __launch_bounds__(256) void page_copy_kernel(PoolList pools, PageMoves mv, int32_t pieces) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const int64_t per = (int64_t)pools.n * pieces, items = (int64_t)*mv.count * per;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t k = it / per;
    const int r = (int)(it % per), pool = r / pieces;
    const int64_t words = pools.words[pool], w0 = (int64_t)(r % pieces) * PIECE;
    const u32x4* src = reinterpret_cast<const u32x4*>(pools.base[pool] + mv.src[k] * words + w0);
    u32x4* dst = reinterpret_cast<u32x4*>(pools.base[pool] + mv.dst[k] * words + w0);
    u32x4 v[PIECE / 1024];
#pragma unroll
    for (int i = 0; i < PIECE / 1024; ++i)
      if (w0 + 4 * (threadIdx.x + 256 * i) < words) v[i] = src[threadIdx.x + 256 * i];
#pragma unroll
    for (int i = 0; i < PIECE / 1024; ++i)
      if (w0 + 4 * (threadIdx.x + 256 * i) < words) dst[threadIdx.x + 256 * i] = v[i];
  }
}

}  // namespace spectra_dev

namespace spectra {
using namespace spectra_dev;

hipError_t launch_pages_extend(const PageMap& m, const int32_t* rows, const int32_t* counts, int32_t n, int32_t* ends,
                               const PageMoves& mv, hipStream_t st) {
  hipLaunchKernelGGL(pages_extend_kernel, dim3(1), dim3(PLAN), 0, st, m, rows, counts, n, ends, mv);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PageMap& m, const int32_t* parents, const int32_t* children, int32_t n, int32_t* ends,
                             hipStream_t st) {
  hipLaunchKernelGGL(pages_fork_kernel, dim3(n), dim3(256), 0, st, m, parents, children, n, ends);
  return hipGetLastError();
}

hipError_t launch_pages_truncate(const PageMap& m, const int32_t* rows, const int32_t* keep, int32_t n, hipStream_t st) {
  hipLaunchKernelGGL(pages_truncate_kernel, dim3(n), dim3(256), 0, st, m, rows, keep, n);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PageMap& m, int32_t* moved, const PageMoves& mv, hipStream_t st) {
  hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(PLAN), 0, st, m, moved, mv);
  const int64_t blocks = ((int64_t)m.row_pages + 255) / 256;
  hipLaunchKernelGGL(pages_retable_kernel, dim3(blocks < 64 ? blocks : 64, m.rows), dim3(256), 0, st, m, moved);
  return hipGetLastError();
}

hipError_t launch_page_copies(const PoolList& pools, const PageMoves& mv, int64_t most_moves, hipStream_t st) {
  int64_t most = 0;
  for (int i = 0; i < pools.n; ++i) most = pools.words[i] > most ? pools.words[i] : most;
  const int64_t pieces = (most + PIECE - 1) / PIECE;
  if (pieces == 0 || most_moves <= 0) return hipSuccess;
  const int64_t items = most_moves * pools.n * pieces;
  hipLaunchKernelGGL(page_copy_kernel, dim3(items < 4096 ? items : 4096), dim3(256), 0, st, pools, mv, (int32_t)pieces);
  return hipGetLastError();
}

}  // namespace spectra
