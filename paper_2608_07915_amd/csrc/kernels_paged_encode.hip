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

constexpr int PE_ROWS = 64;

template <bool F32IN>
__global__ __launch_bounds__(256, 2) void paged_encode_kernel(PagedEncodeArgs a) {
  constexpr int ESZ = F32IN ? 4 : 2;
  constexpr int ROWB = D * ESZ + 16;  // padded LDS row (bank spread)
  constexpr int CPR = D * ESZ / 16;   // 16-byte pieces of a row
  __shared__ __attribute__((aligned(16))) uint8_t xs[PE_ROWS * ROWB];
  __shared__ uint32_t* rec_s[PE_ROWS];
  const int kv = (int)(blockIdx.y % (unsigned)a.c.n_kv), which = (int)(blockIdx.y / (unsigned)a.c.n_kv);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, col = lane & 31;
  const int W = a.W[which];
  const Kept K = read_kept(a.bits[which] + kv * NG);
  if (!K.ok || K.used > W) return;  // width table inconsistent with the record: write nothing
  const int wpg = K.n ? 4 / K.n : 0;
  const bool active = K.n > 0 && wave < K.n * wpg;
  const int slot = active ? wave / wpg : 0, phase = active ? wave % wpg : 0;
  const int grp = pick4(K.grp, slot), gbits = pick4(K.bits, slot), gpay = pick4(K.pay, slot);
  bf16x8 Va[3][8];
  f32x16 nm;
  if (active) load_group_operands(a.basis[which] + (int64_t)kv * D * D, a.mean[which] + kv * D, grp, col, h, Va, nm);
  const char* x = reinterpret_cast<const char*>(a.x[which]) + kv * a.head_stride[which] * ESZ;
  const int64_t n_items = (a.c.n_new + PE_ROWS - 1) / PE_ROWS;
  for (int64_t it = blockIdx.x; it < n_items; it += gridDim.x) {
    const int64_t r0 = it * PE_ROWS;
    for (int c = tid; c < PE_ROWS * CPR; c += 256) {
      const int row = c / CPR, part = c % CPR;
      u32x4 v = u32x4{0u, 0u, 0u, 0u};
      if (r0 + row < a.c.n_new) v = *reinterpret_cast<const u32x4*>(x + (r0 + row) * a.token_stride[which] * ESZ + part * 16);
      *reinterpret_cast<u32x4*>(xs + row * ROWB + part * 16) = v;
    }
    if (tid < PE_ROWS) {
      const int64_t r = r0 + tid;
      uint32_t* rec = nullptr;
      if (r < a.c.n_new) {
        int lo = 0, hi = a.c.batch;  // the last sequence that starts at or before r
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (a.c.cu[mid] <= r) lo = mid; else hi = mid;
        }
        const PagedSeq s = paged_seq(a.c, lo);
        const int64_t t = s.len - s.n + (r - s.first);
        if (r >= s.first && r < s.first + s.n && t >= 0 && s.len > 0) {
          rec = paged_tile(a.c, a.pool[which], W, s.row, t >> 6, kv);
          if (rec) rec += t & 63;
        }
      }
      rec_s[tid] = rec;
    }
    __syncthreads();
    if (active) {
      for (int beta = phase; beta < PE_ROWS / 32; beta += wpg) {
        const f32x16 acc = project_block<F32IN, ROWB>(xs, beta, col, h, nm, [&](int p, int k) { return Va[p][k]; });
        uint32_t* rec = rec_s[32 * beta + col];
        store_block(acc, rec, rec != nullptr, h, slot, gbits, gpay);
      }
    }
    for (int c = tid; c < PE_ROWS * (W - K.used); c += 256) {  // padding words are zero
      uint32_t* rec = rec_s[c % PE_ROWS];
      if (rec) rec[(K.used + c / PE_ROWS) * TILE] = 0u;
    }
    __syncthreads();
  }
}

}  // namespace spectra_dev

namespace spectra {
using namespace spectra_dev;

hipError_t launch_paged_encode(const PagedEncodeArgs& a, bool f32_input, hipStream_t st) {
  const int64_t items = (a.c.n_new + PE_ROWS - 1) / PE_ROWS, heads = 2 * (int64_t)a.c.n_kv;
  int64_t nx = (512 + heads - 1) / heads;  // two workgroups per CU
  if (nx > items) nx = items;
  const dim3 grid((unsigned)nx, (unsigned)heads);
  if (f32_input)
    hipLaunchKernelGGL((paged_encode_kernel<true>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((paged_encode_kernel<false>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace spectra
