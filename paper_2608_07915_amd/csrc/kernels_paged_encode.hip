// Encode of the new tokens of many sequences into their pages (Sec. 3.2-3.3): the steps of
// encode_dev.hpp with a destination per token.
//
// The codec state is one KV head's whatever the sequence, so a work item is 64 neighbouring
// rows of the token array: a decode step's single tokens of 64 sequences are one item, and a
// ragged batch leaves no partly filled tiles. Every lane finds the sequence of its own token by
// bisection of the sequence starts.
#include "encode_dev.hpp"
#include "paged_dev.hpp"

namespace spectra_dev {

// The next item's rows (into registers) and destinations (the last wavefront) are loaded while
// this one's are projected: 32k prompt tokens of eight heads (152 MB) take 58 us, with the loads in
// front of each item 87. Bound by the wait for a row that only two workgroups per CU hide: the
// basis of a group is 96 registers of each lane, and three per CU spill (79 us).
constexpr int PE_ROWS = 64;
constexpr int PE_STARTS = 1024;  // sequence starts held in LDS

template <bool F32IN>
__global__ __launch_bounds__(256, 2) void paged_encode_kernel(PagedEncodeArgs a) {
  constexpr int ESZ = F32IN ? 4 : 2;
  constexpr int ROWB = D * ESZ + 16;  // padded LDS row (bank spread)
  constexpr int CPR = D * ESZ / 16;   // 16-byte pieces of a row
  constexpr int PRE = PE_ROWS * CPR / 256;
  __shared__ __attribute__((aligned(16))) uint8_t xs[PE_ROWS * ROWB];
  __shared__ uint32_t* rec_s[2][PE_ROWS];
  __shared__ int32_t cu_s[PE_STARTS];
  const int kv = (int)(blockIdx.y % (unsigned)a.c.n_kv), which = (int)(blockIdx.y / (unsigned)a.c.n_kv);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, col = lane & 31;
  const int W = a.W[which];
  const char* x = reinterpret_cast<const char*>(a.x[which]) + kv * a.head_stride[which] * ESZ;
  const int64_t row_bytes = a.token_stride[which] * ESZ;
  const int64_t n_items = (a.c.n_new + PE_ROWS - 1) / PE_ROWS;
  u32x4 pre[PRE];
  auto load_rows = [&](int64_t it) {
#pragma unroll
    for (int i = 0; i < PRE; ++i) {
      const int c = tid + 256 * i, row = c / CPR, part = c % CPR;
      pre[i] = u32x4{0u, 0u, 0u, 0u};
      if (it * PE_ROWS + row < a.c.n_new) pre[i] = *reinterpret_cast<const u32x4*>(x + (it * PE_ROWS + row) * row_bytes + part * 16);
    }
  };
  // where lane's row of the item goes: word 0 of its record, or null
  auto destination = [&](int64_t it) -> uint32_t* {
    const int64_t r = it * PE_ROWS + lane;
    if (r >= a.c.n_new) return nullptr;
    int lo = 0, hi = a.c.batch;  // the last sequence that starts at or before r
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((mid < PE_STARTS ? cu_s[mid] : a.c.cu[mid]) <= r) lo = mid; else hi = mid;
    }
    const PagedSeq s = paged_seq(a.c, lo);
    const int64_t t = s.len - s.n + (r - s.first);
    if (r < s.first || r >= s.first + s.n || t < 0 || s.len <= 0) return nullptr;
    uint32_t* rec = paged_tile(a.c, a.pool[which], W, s.row, t >> 6, kv);
    return rec ? rec + (t & 63) : nullptr;
  };
  int64_t it = blockIdx.x;
  if (it < n_items) load_rows(it);
  const Kept K = read_kept(a.bits[which] + kv * NG);
  if (!K.ok || K.used > W) return;  // width table inconsistent with the record: write nothing
  for (int i = tid; i < PE_STARTS && i < a.c.batch; i += 256) cu_s[i] = a.c.cu[i];
  const int wpg = K.n ? 4 / K.n : 0;
  const bool active = K.n > 0 && wave < K.n * wpg;
  const int slot = active ? wave / wpg : 0, phase = active ? wave % wpg : 0;
  const int grp = pick4(K.grp, slot), gbits = pick4(K.bits, slot), gpay = pick4(K.pay, slot);
  bf16x8 Va[3][8];
  f32x16 nm;
  if (active) load_group_operands(a.basis[which] + (int64_t)kv * D * D, a.mean[which] + kv * D, grp, col, h, Va, nm);
  __syncthreads();  // the starts
  if (wave == 3 && it < n_items) rec_s[0][lane] = destination(it);
  for (int buf = 0; it < n_items; buf ^= 1) {
#pragma unroll
    for (int i = 0; i < PRE; ++i) {
      const int c = tid + 256 * i, row = c / CPR, part = c % CPR;
      *reinterpret_cast<u32x4*>(xs + row * ROWB + part * 16) = pre[i];
    }
    __syncthreads();  // rows and destinations
    const int64_t next = it + gridDim.x;
    if (next < n_items) {
      load_rows(next);
      if (wave == 3) rec_s[buf ^ 1][lane] = destination(next);
    }
    if (active) {
      for (int beta = phase; beta < PE_ROWS / 32; beta += wpg) {
        const f32x16 acc = project_block<F32IN, ROWB>(xs, beta, col, h, nm, [&](int p, int k) { return Va[p][k]; });
        uint32_t* rec = rec_s[buf][32 * beta + col];
        store_block(acc, rec, rec != nullptr, h, slot, gbits, gpay);
      }
    }
    for (int c = tid; c < PE_ROWS * (W - K.used); c += 256) {  // padding words are zero
      uint32_t* rec = rec_s[buf][c % PE_ROWS];
      if (rec) rec[(K.used + c / PE_ROWS) * TILE] = 0u;
    }
    it = next;
    __syncthreads();  // the rows are used
  }
}

}  // namespace spectra_dev

namespace spectra {
using namespace spectra_dev;

hipError_t launch_paged_encode(const PagedEncodeArgs& a, bool f32_input, hipStream_t st) {
  const int64_t items = (a.c.n_new + PE_ROWS - 1) / PE_ROWS, heads = 2 * (int64_t)a.c.n_kv;
  int64_t nx = (512 + heads - 1) / heads;  // two workgroups per CU (three: 79 us for 61)
  if (nx > items) nx = items;
  const dim3 grid((unsigned)nx, (unsigned)heads);
  if (f32_input)
    hipLaunchKernelGGL((paged_encode_kernel<true>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((paged_encode_kernel<false>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace spectra
