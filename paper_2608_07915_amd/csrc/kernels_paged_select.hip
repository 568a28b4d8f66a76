// Blocks of a paged cache for sparse attention: the boxes of the keys' coefficients, and the best
// blocks of every new token and KV head.
//
// A block is a tile of 64 slots. Its box holds, for every kept coefficient j of the keys, least_j and
// largest_j over its slots. For a query q' = q V_K and any slot of the block
//   q' . c <= B = sum_j max(q'_j least_j, q'_j largest_j) = sum_j min(q'_j, 0) least_j + max(q'_j, 0) largest_j,
// a matrix product of the queries with the boxes.
#include "code_operands.hpp"
#include "encode_dev.hpp"
#include "paged_coef.hpp"
#include "paged_dev.hpp"

namespace spectra_dev {

constexpr int BOX = 2 * G;             // fp16 of a group in a box: the least, then the largest
constexpr int BOX_WORDS = NG * BOX / 2;  // words of a block's box

// The sequence that new token `t` belongs to (the last one that begins at or before it), -1: none.
// cu is searched by halves: log2(batch) dependent loads, a lane's own.
__device__ __forceinline__ int sequence_of(const PagedCache& c, int64_t t) {
  int lo = 0, hi = c.batch;  // first b with cu[b] > t lies in (lo, hi]
  if (c.batch == 0 || c.cu[0] > t) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (c.cu[mid] <= t) lo = mid; else hi = mid;
  }
  return t < c.cu[lo + 1] ? lo : -1;
}

// ---------------------------------------------------------------------------
// Boxes. A wavefront takes `tokens` neighbouring new tokens of one KV head; those that are the
// first of their sequence in a block stand for it, so each block is made once. A lane then
// holds one slot's coefficients, fp16 pairs as the attention kernels make them, and the 64 slots
// are reduced by halving: at each of four exchanges a lane keeps half of its coefficients, the last
// two within quads (per group 34 exchanges instead of 192). Words of HBM once, 128 bytes written
// a group.
// ---------------------------------------------------------------------------
__device__ __forceinline__ f16x2 pk_min(f16x2 a, f16x2 b) { return __builtin_elementwise_min(a, b); }
__device__ __forceinline__ f16x2 pk_max(f16x2 a, f16x2 b) { return __builtin_elementwise_max(a, b); }
template <int CTRL>
__device__ __forceinline__ f16x2 dpp_pair(f16x2 v) {
  return __builtin_bit_cast(f16x2, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}

// r[x], x < 16: codes x and x + 16 of the lane's slot. Returns the pair x = lane / 4 over all lanes.
template <typename Op>
__device__ __forceinline__ f16x2 reduce_slots(const f16x2 (&r)[16], int lane, Op&& op) {
  f16x2 a[8], b[4], c[2];
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // halves of the wavefront: the upper one keeps pairs 8 ..
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, r[i]), __builtin_bit_cast(uint32_t, r[i + 8]), false, false);
    const uint32_t s0 = s[0], s1 = s[1];  // (a bit cast of a vector's element reads its first)
    a[i] = op(__builtin_bit_cast(f16x2, s0), __builtin_bit_cast(f16x2, s1));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // rows of 16 lanes
    const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a[i]), __builtin_bit_cast(uint32_t, a[i + 4]), false, false);
    const uint32_t s0 = s[0], s1 = s[1];
    b[i] = op(__builtin_bit_cast(f16x2, s0), __builtin_bit_cast(f16x2, s1));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {  // lane ^ 8 (row_ror:8)
    const f16x2 keep = lane & 8 ? b[i + 2] : b[i], send = lane & 8 ? b[i] : b[i + 2];
    c[i] = op(keep, dpp_pair<0x128>(send));
  }
  const f16x2 keep = lane & 4 ? c[1] : c[0], send = lane & 4 ? c[0] : c[1];  // lane ^ 7 (row_half_mirror)
  f16x2 d = op(keep, dpp_pair<0x141>(send));
  d = op(d, dpp_pair<0xB1>(d));  // lane ^ 1, lane ^ 2
  return op(d, dpp_pair<0x4E>(d));
}

__global__ __launch_bounds__(256) void paged_bounds_kernel(PagedBoundsArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv = (int)(w % a.c.n_kv);
  const int64_t t = w / a.c.n_kv * a.tokens + lane;
  int row = 0, slot = 0, len = 0;
  bool starts = false;
  if (lane < a.tokens && t < a.c.n_new) {
    const int b = sequence_of(a.c, t);
    if (b >= 0) {
      const PagedSeq s = paged_seq(a.c, b);
      const int64_t at = s.len - s.n + (t - s.first);
      starts = s.len > 0 && at >= 0 && t >= s.first && t < s.first + s.n && (t == s.first || at % TILE == 0);
      row = s.row;
      slot = (int)at;
      len = (int)s.len;
    }
  }
  Kept K = read_kept(a.bits_k + kv * NG);
  if (!K.ok || K.used > a.Wk) return;  // width table inconsistent with the record: write nothing
  const int tpp = a.c.page_tokens >> 6;
  uint32_t magic = 0x64006400u;  // exponent of 1024 in both halves, in a VGPR
  asm volatile("" : "+v"(magic));
  uint64_t todo = __ballot(starts);
  while (todo) {
    const int l = __builtin_ctzll(todo);
    todo &= todo - 1;
    const int tile = __builtin_amdgcn_readlane(slot, l) >> 6, end = __builtin_amdgcn_readlane(len, l);
    const int table_row = __builtin_amdgcn_readlane(row, l), at = tile / tpp;
    const int page = __builtin_amdgcn_readfirstlane(a.c.table[(int64_t)table_row * a.c.row_pages + at]);
    if (page < 0 || page >= a.c.n_pages) continue;
    const int64_t blk = ((int64_t)page * a.c.n_kv + kv) * tpp + (tile - at * tpp);
    const uint32_t* rec = a.pool_k + blk * (TILE * a.Wk) + lane;
    uint16_t* box = reinterpret_cast<uint16_t*>(a.bounds + blk * BOX_WORDS);
    const bool live = tile * TILE + lane < end;
#pragma unroll
    for (int sl = 0; sl < NG; ++sl) {
      if (sl >= K.n) break;
      const int b = K.bits[sl];
      uint32_t words[8];
      const uint32_t meta = finite_meta(rec[sl * TILE], b);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < b) words[i] = rec[(K.pay[sl] + i) * TILE];
      f16x2 least[16], most[16];
      with_bits(b, [&](auto bc) __attribute__((always_inline)) {
        constexpr int B = decltype(bc)::value;
        uint32_t Z[8];
        join_halves<B>(words, Z);
        const _Float16 s = __builtin_bit_cast(_Float16, (uint16_t)meta), z = __builtin_bit_cast(_Float16, (uint16_t)(meta >> 16));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f16x8 c = codes_f16<B, false>(Z, k, magic);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            least[4 * k + i] = __builtin_elementwise_fma(f16x2{s, s}, f16x2{c[2 * i], c[2 * i + 1]}, f16x2{z, z});
        }
      });
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        most[i] = live ? least[i] : __builtin_bit_cast(f16x2, 0xFC00FC00u);
        least[i] = live ? least[i] : __builtin_bit_cast(f16x2, 0x7C007C00u);
      }
      const f16x2 lo = reduce_slots(least, lane, pk_min), hi = reduce_slots(most, lane, pk_max);
      // lanes of a quad hold the same: each writes one of least x, least x + 16, largest x, largest x + 16
      const uint32_t pair = __builtin_bit_cast(uint32_t, lane & 2 ? hi : lo);
      box[BOX * sl + G * ((lane >> 1) & 1) + 16 * (lane & 1) + (lane >> 2)] = (uint16_t)(lane & 1 ? pair >> 16 : pair);
    }
  }
}

// ---------------------------------------------------------------------------
// Scores. A unit is the query rows (token, query head on the KV head) of TG = 16 NB / n_qh
// neighbouring new tokens of one sequence, the columns of 16 x 16 x 32 products whose rows are 16
// blocks: a lane reads 8 fp16 of a block's box, the register operand as it lies in memory. q' is
// scaled by 2^E and cut into two fp16 parts, each split by sign into the part against the least
// values and the one against the largest; the boxes are exact, so a score is off by about 2^-22 of
// sum_j |q'_j box_j| and the sums' roundings.
// Sequence b's units begin at first_b / TG + b: those of two sequences never meet, and a workgroup
// finds its own without a sum over the others.
// ---------------------------------------------------------------------------
struct UnitScratch {
  int32_t b;
};
// The sequence of unit u and the unit's place in it; the same in every thread. b < 0: none.
template <int NT>
__device__ __forceinline__ int find_token_unit(const PagedCache& c, int64_t u, int tg, UnitScratch& s, int64_t& at) {
  if (threadIdx.x == 0) s.b = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < c.batch; b += NT) {
    const PagedSeq q = paged_seq(c, b);
    const int64_t base = q.first / tg + b;
    if (u >= base && u < base + (q.n + tg - 1) / tg) atomicMax(&s.b, b);
  }
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(s.b);
  if (b >= 0) at = u - (paged_seq(c, b).first / tg + b);
  return b;
}

template <int NB>
__global__ __launch_bounds__(256) void paged_block_scores_kernel(PagedSelectArgs a, int tiles_per_chunk) {
  __shared__ UnitScratch unit_s;
  __shared__ float most_s[NG][16 * NB];
  __shared__ __attribute__((aligned(16))) uint8_t q_s[NG][NB][4][64 * 16];  // against least: hi, lo; against largest: hi, lo
  __shared__ float un_s[16 * NB];
  const int tg = 16 * NB / a.n_qh;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int64_t at = 0;
  const int b = find_token_unit<256>(a.c, blockIdx.x / (unsigned)a.c.n_kv, tg, unit_s, at);
  if (b < 0) return;
  const PagedSeq seq = paged_seq(a.c, b);
  if (seq.len > a.max_tokens) return;
  const int64_t tok0 = at * tg;
  const int n_rows = (int)(seq.n - tok0 < tg ? seq.n - tok0 : tg) * a.n_qh;
  // slots that the unit's last token sees: the blocks of the others are among its
  const int64_t past = seq.len - seq.n + tok0 + 1, see = past + n_rows / a.n_qh - 1;
  const int n_blocks = see > 0 ? (int)((see + TILE - 1) / TILE) : 0;
  const int begin = blockIdx.y * tiles_per_chunk;
  int end = (n_blocks + 15) / 16;
  end = end < begin + tiles_per_chunk ? end : begin + tiles_per_chunk;
  if (begin >= end) return;
  Kept K = read_kept(a.bits_k + kv * NG);
  if (!K.ok || K.used > a.Wk) K.n = 0;  // width table inconsistent with the record

  // q' of kept group sl and row block nb: element e of quarter p is coefficient 8 p + e
  constexpr int PAIRS = NB;  // NG NB over four wavefronts
  f32x4 acc[PAIRS][2];
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    const int pair = wave + 4 * i, sl = pair & 3, nb = pair >> 2;
    acc[i][0] = acc[i][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (sl < K.n) {
      const int row = 16 * nb + col < n_rows ? 16 * nb + col : 0, tok = row / a.n_qh, head = row - tok * a.n_qh;
      const int64_t qoff = (seq.first + tok0 + tok) * a.q_token_stride + (kv * a.n_qh + head) * a.q_head_stride + 8 * quarter;
      const float* V = a.basis_k + (int64_t)kv * D * D + (8 * quarter) * D + G * pick4(K.grp, sl) + 8 * (col >> 2) + (col & 3);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float v[2][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[0][e] = V[(32 * k + e) * D];
          v[1][e] = V[(32 * k + e) * D + 4];
        }
        bf16x8 qq[3];
        if (a.q_f32) {
          const f32x4* qp = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.q) + qoff + 32 * k);
          const f32x4 q0 = qp[0], q1 = qp[1];
          const float qv[8] = {q0[0], q0[1], q0[2], q0[3], q1[0], q1[1], q1[2], q1[3]};
          split8<3>(qv, qq);
        } else {
          qq[0] = as_bf16x8(*reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + qoff + 32 * k));
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          bf16x8 vp[3];
          split8<3>(v[x], vp);
#pragma unroll
          for (int p = 0; p < 3; ++p) acc[i][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[p], qq[0], acc[i][x], 0, 0, 0);
          if (a.q_f32) {
            acc[i][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[0], qq[1], acc[i][x], 0, 0, 0);
            acc[i][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[1], qq[1], acc[i][x], 0, 0, 0);
            acc[i][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[0], qq[2], acc[i][x], 0, 0, 0);
          }
        }
      }
    }
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, __builtin_fabsf(acc[i][e >> 2][e & 3]));
    most = __builtin_fmaxf(most, __shfl_xor(most, 16));
    most = __builtin_fmaxf(most, other_half(most));
    if (quarter == 0) most_s[sl][16 * nb + col] = most;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    const int pair = wave + 4 * i, sl = pair & 3, nb = pair >> 2, row = 16 * nb + col;
    const float most = __builtin_fmaxf(__builtin_fmaxf(most_s[0][row], most_s[1][row]), __builtin_fmaxf(most_s[2][row], most_s[3][row]));
    const float up = __builtin_ldexpf(1.0f, 9 - scale_exponent(most));
    if (sl == 0 && quarter == 0) un_s[row] = 1.0f / up;
    u32x4 r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 x = f32x2{acc[i][j >> 1][2 * (j & 1)] * up, acc[i][j >> 1][2 * (j & 1) + 1] * up};
      const f16x2 hi = __builtin_convertvector(x, f16x2);
      const uint32_t h = __builtin_bit_cast(uint32_t, hi);
      const uint32_t l = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{(x[0] - (float)hi[0]) * CA_LO, (x[1] - (float)hi[1]) * CA_LO}, f16x2));
      const uint32_t below = (x[0] < 0.0f ? 0xFFFFu : 0u) | (x[1] < 0.0f ? 0xFFFF0000u : 0u);
      r[0][j] = h & below;
      r[1][j] = l & below;
      r[2][j] = h & ~below;
      r[3][j] = l & ~below;
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) *reinterpret_cast<u32x4*>(q_s[sl][nb][p] + 16 * lane) = r[p];
  }
  __syncthreads();

  const int tpp = a.c.page_tokens >> 6;
  float* out[NB];
  int lim[NB];  // blocks that the lane's row sees
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int row = 16 * nb + col, tok = row / a.n_qh, head = row - tok * a.n_qh;
    out[nb] = row < n_rows ? a.scores + ((seq.first + tok0 + tok) * a.n_q_heads + kv * a.n_qh + head) * a.most_blocks : nullptr;
    const int64_t l = past + tok;
    lim[nb] = l > 0 ? (int)((l + TILE - 1) / TILE) : 0;
  }
  for (int bt = begin + wave; bt < end; bt += 4) {
    const int blk = 16 * bt + col, idx = blk / tpp;
    const int page = blk < n_blocks ? a.c.table[(int64_t)seq.row * a.c.row_pages + idx] : -1;
    const bool ok = page >= 0 && page < a.c.n_pages;
    const uint32_t* box = a.bounds + (((int64_t)(ok ? page : 0) * a.c.n_kv + kv) * tpp + (ok ? blk - idx * tpp : 0)) * BOX_WORDS + 4 * quarter;
    u32x4 x[NG][2];
#pragma unroll
    for (int sl = 0; sl < NG; ++sl)
#pragma unroll
      for (int side = 0; side < 2; ++side)
        x[sl][side] = sl < K.n && ok ? *reinterpret_cast<const u32x4*>(box + (sl * 2 + side) * (G / 2)) : u32x4{0u, 0u, 0u, 0u};
    f32x4 hi[NB], lo[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) hi[nb] = lo[nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int sl = 0; sl < NG; ++sl) {
      if (sl >= K.n) continue;
#pragma unroll
      for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const f16x8 qh = as_f16x8(*reinterpret_cast<const u32x4*>(q_s[sl][nb][2 * side] + 16 * lane));
          const f16x8 ql = as_f16x8(*reinterpret_cast<const u32x4*>(q_s[sl][nb][2 * side + 1] + 16 * lane));
          hi[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(x[sl][side]), qh, hi[nb], 0, 0, 0);
          lo[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(x[sl][side]), ql, lo[nb], 0, 0, 0);
        }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (out[nb] == nullptr) continue;
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = 16 * bt + 4 * quarter + i < lim[nb] ? __builtin_fmaf(lo[nb][i], 1.0f / CA_LO, hi[nb][i]) * un_s[16 * nb + col] : -__builtin_inff();
      *reinterpret_cast<f32x4*>(out[nb] + 16 * bt + 4 * quarter) = v;
    }
  }
}

// ---------------------------------------------------------------------------
// The best blocks of a (token, KV head): a workgroup makes a key of every block, an unsigned number
// that orders as its value does, finds the n-th largest by four rounds of counts of 8 bits, and
// writes those above it and, of those equal to it, the first, in ascending order. Keys lie in LDS, or in the
// place of the first head's scores.
// ---------------------------------------------------------------------------
constexpr int PICK = 256;
constexpr int PICK_LDS = 16384;  // blocks whose keys LDS takes
template <bool IN_LDS>
__global__ __launch_bounds__(PICK) void paged_pick_kernel(PagedSelectArgs a) {
  extern __shared__ uint32_t keys_s[];
  __shared__ int32_t b_s;
  __shared__ float top_s[16][PICK / 64];
  __shared__ int32_t hist_s[256], part_s[PICK / 64], part2_s[PICK / 64], found_s[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int64_t t = blockIdx.x / (unsigned)a.c.n_kv;
  if (tid == 0) b_s = -1;
  __syncthreads();
  for (int b = tid; b < a.c.batch; b += PICK) {
    const PagedSeq q = paged_seq(a.c, b);
    if (t >= q.first && t < q.first + q.n) atomicMax(&b_s, b);
  }
  __syncthreads();
  if (b_s < 0) return;
  const PagedSeq seq = paged_seq(a.c, b_s);
  if (seq.len > a.max_tokens) return;
  const int64_t see = seq.len - seq.n + (t - seq.first) + 1;
  const int have = see > 0 ? (int)((see + TILE - 1) / TILE) : 0, want = a.n_blocks;
  int32_t* out = a.blocks + (t * a.c.n_kv + kv) * want;
  if (have <= want) {
    for (int i = tid; i < want; i += PICK) out[i] = i < have ? i : -1;
    return;
  }
  float* rows = a.scores + (t * a.n_q_heads + kv * a.n_qh) * (int64_t)a.most_blocks;
  uint32_t* keys = IN_LDS ? keys_s : reinterpret_cast<uint32_t*>(rows);
  for (int h = 0; h < a.n_qh; ++h) {
    float top = -__builtin_inff();
    for (int i = tid; i < have; i += PICK) top = __builtin_fmaxf(top, rows[(int64_t)h * a.most_blocks + i]);
    top = wave_max(top);
    if (lane == 0) top_s[h][wave] = top;
  }
  __syncthreads();
  for (int i = tid; i < have; i += PICK) {
    float v = -__builtin_inff();
    for (int h = 0; h < a.n_qh; ++h) {
      const float top = __builtin_fmaxf(__builtin_fmaxf(top_s[h][0], top_s[h][1]), __builtin_fmaxf(top_s[h][2], top_s[h][3]));
      const float d = rows[(int64_t)h * a.most_blocks + i] - top;  // NaN where the head has no number
      v = __builtin_fmaxf(v, d == d ? d : -__builtin_inff());
    }
    const uint32_t u = __float_as_uint(v), key = u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
    keys[i] = i < a.first || i >= have - a.last ? 0xFFFFFFFFu : key;
  }
  uint32_t prefix = 0u, mask = 0u;
  int left = want;
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist_s[tid] = 0;
    __syncthreads();
    for (int i = tid; i < have; i += PICK) {
      const uint32_t k = keys[i];
      if ((k & mask) == prefix) atomicAdd(&hist_s[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    const int mine = hist_s[255 - tid];  // the largest digits first
    int v = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(v, o);
      if (lane >= o) v += u;
    }
    if (lane == 63) part_s[wave] = v;
    __syncthreads();
    for (int w = 0; w < wave; ++w) v += part_s[w];
    if (v >= left && v - mine < left) {
      found_s[0] = 255 - tid;
      found_s[1] = left - (v - mine);
    }
    __syncthreads();
    prefix |= (uint32_t)found_s[0] << shift;
    mask |= 255u << shift;
    left = found_s[1];
    __syncthreads();
  }
  // neighbouring blocks to a thread: how many above and equal, then their places
  const int each = (have + PICK - 1) / PICK, from = tid * each, to = from + each < have ? from + each : have;
  int above = 0, equal = 0;
  for (int i = from; i < to; ++i) {
    const uint32_t k = keys[i];
    above += k > prefix ? 1 : 0;
    equal += k == prefix ? 1 : 0;
  }
  int va = above, ve = equal;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int ua = __shfl_up(va, o), ue = __shfl_up(ve, o);
    if (lane >= o) {
      va += ua;
      ve += ue;
    }
  }
  if (lane == 63) {
    part_s[wave] = va;
    part2_s[wave] = ve;
  }
  __syncthreads();
  for (int w = 0; w < wave; ++w) {
    va += part_s[w];
    ve += part2_s[w];
  }
  int eq = ve - equal, place = va - above + (eq < left ? eq : left);
  for (int i = from; i < to; ++i) {
    const uint32_t k = keys[i];
    bool take = k > prefix;
    if (k == prefix) take = eq++ < left;
    if (take) out[place++] = i;
  }
}

}  // namespace spectra_dev

namespace spectra {
using namespace spectra_dev;

hipError_t launch_paged_bounds(const PagedBoundsArgs& args, hipStream_t st) {
  PagedBoundsArgs a = args;
  // a token a wavefront as long as the card holds them all at once (a decode step), then more
  a.tokens = 1;
  while (a.tokens < 64 && (a.c.n_new + a.tokens - 1) / a.tokens * a.c.n_kv > 16384) a.tokens *= 2;
  const int64_t waves = (a.c.n_new + a.tokens - 1) / a.tokens * a.c.n_kv;
  hipLaunchKernelGGL(paged_bounds_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}

static int64_t score_pitch(int64_t max_tokens) { return (max_tokens + 16 * TILE - 1) / (16 * TILE) * 16; }

size_t paged_select_bytes(int64_t n_new, int32_t n_q_heads, int32_t n_kv, int64_t max_tokens) {
  (void)n_kv;
  return (size_t)(n_new * n_q_heads * score_pitch(max_tokens)) * sizeof(float);
}

hipError_t launch_paged_select(const PagedSelectArgs& args, void* workspace, hipStream_t st) {
  PagedSelectArgs a = args;
  a.scores = static_cast<float*>(workspace);
  a.most_blocks = (int32_t)score_pitch(a.max_tokens);
  const bool many = a.c.n_new * a.n_qh > 64;
  const int nb = many ? 4 : 1, tg = 16 * nb / a.n_qh;
  const int64_t units = a.c.n_new / tg + a.c.batch, tiles = (a.most_blocks + 15) / 16;
  int64_t n = 1024 / (units * a.c.n_kv);
  if (n < 1) n = 1;
  int64_t per = (tiles + n - 1) / n;
  per = (per + 3) / 4 * 4;
  const dim3 grid((unsigned)(units * a.c.n_kv), (unsigned)((tiles + per - 1) / per));
  if (many)
    hipLaunchKernelGGL((paged_block_scores_kernel<4>), grid, dim3(256), 0, st, a, (int)per);
  else
    hipLaunchKernelGGL((paged_block_scores_kernel<1>), grid, dim3(256), 0, st, a, (int)per);
  const dim3 rows((unsigned)(a.c.n_new * a.c.n_kv));
  if (a.most_blocks <= PICK_LDS)
    hipLaunchKernelGGL((paged_pick_kernel<true>), rows, dim3(PICK), a.most_blocks * sizeof(uint32_t), st, a);
  else
    hipLaunchKernelGGL((paged_pick_kernel<false>), rows, dim3(PICK), 0, st, a);
  return hipGetLastError();
}

}  // namespace spectra
