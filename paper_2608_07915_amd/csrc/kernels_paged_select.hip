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
#include "splits.hpp"

namespace spectra_dev {

constexpr int BOX = 2 * G;             // fp16 of a group in a box: the least, then the largest
constexpr int BOX_WORDS = NG * BOX / 2;  // words of a block's box

// The sequence that new token `t` belongs to (the last one that begins at or before it), -1: none; starts(b) is
// cu[b]. Searched by halves, a lane for itself.
template <typename Starts>
__device__ __forceinline__ int sequence_of(int batch, int64_t t, Starts&& starts) {
  int lo = 0, hi = batch;  // first b with cu[b] > t lies in (lo, hi]
  if (batch == 0 || starts(0) > t) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts(mid) <= t) lo = mid; else hi = mid;
  }
  return t < starts(lo + 1) ? lo : -1;
}

// ---------------------------------------------------------------------------
// Boxes. A wavefront takes `tokens` neighbouring new tokens of one KV head; those that are the
// first of their sequence in a block stand for it, so each block is made once. A lane then
// holds one slot's coefficients, fp16 pairs as the attention kernels make them, and the 64 slots
// are reduced by halving: at each of four exchanges a lane keeps half of its coefficients, the last
// two within quads (per group 34 exchanges instead of 192). Words of HBM once, 128 bytes written
// a group. The starts of up to BOX_STARTS sequences are searched in LDS.
// Measured: 131072 prompt slots of 8 KV heads 23 to 25 us (38 MB, 1.5 TB/s), by the vector unit, which making the
// coefficients and the exchanges keep busy 85% of the time that a CU holds work; the newest blocks of 64 sequences 10 us,
// a launch and one chain of loads.
// ---------------------------------------------------------------------------
// (as instructions: the compiler first makes every operand quiet, which doubles them; nothing here is NaN)
__device__ __forceinline__ f16x2 pk_min(f16x2 a, f16x2 b) {
  f16x2 d;
  asm("v_pk_min_f16 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
  return d;
}
__device__ __forceinline__ f16x2 pk_max(f16x2 a, f16x2 b) {
  f16x2 d;
  asm("v_pk_max_f16 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
  return d;
}
constexpr int BOX_STARTS = 512;
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
  // an exchange of rows reads what was written two wait states ago or more; the compiler does not count from op's assembly
  asm volatile("s_nop 1" : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(a[4]), "+v"(a[5]), "+v"(a[6]), "+v"(a[7]));
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
  __shared__ int32_t starts_s[BOX_STARTS];
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv = (int)(w % a.c.n_kv);
  const int64_t t = w / a.c.n_kv * a.tokens + lane;
  const bool in_lds = a.c.batch < BOX_STARTS;
  if (in_lds) {
    for (int i = threadIdx.x; i <= a.c.batch; i += 256) starts_s[i] = a.c.cu[i];
    __syncthreads();
  }
  int row = 0, slot = 0, len = 0;
  bool starts = false;
  if (lane < a.tokens && t < a.c.n_new) {
    const int b = in_lds ? sequence_of(a.c.batch, t, [&](int i) { return starts_s[i]; }) : sequence_of(a.c.batch, t, [&](int i) { return a.c.cu[i]; });
    if (b >= 0) {
      const PagedSeq s = paged_seq(a.c, b);
      const int64_t at = s.len - s.n + (t - s.first);
      starts = s.len > 0 && at >= 0 && t >= s.first && t < s.first + s.n && (t == s.first || at % TILE == 0);
      row = s.row;
      slot = (int)at;
      len = (int)s.len;
    }
  }
  const Kept K = read_kept(a.bits_k + kv * NG);
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
    const bool whole = tile * TILE + TILE <= end, live = tile * TILE + lane < end;
    int pay = K.n;
#pragma unroll 1
    for (int sl = 0; sl < K.n; ++sl) {
      const int b = pick4(K.bits, sl);
      uint32_t words[8];
      const uint32_t word = rec[sl * TILE];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < b) words[i] = rec[(pay + i) * TILE];
      pay += b;
      const uint32_t meta = finite_meta(word, b);
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
      for (int i = 0; i < 16; ++i) most[i] = least[i];
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          most[i] = live ? most[i] : __builtin_bit_cast(f16x2, 0xFC00FC00u);
          least[i] = live ? least[i] : __builtin_bit_cast(f16x2, 0x7C007C00u);
        }
      }
      const f16x2 lo = reduce_slots(least, lane, pk_min), hi = reduce_slots(most, lane, pk_max);
      // lanes of a quad hold the same: each writes one of least x, least x + 16, largest x, largest x + 16
      const uint32_t pair = __builtin_bit_cast(uint32_t, lane & 2 ? hi : lo);
      box[BOX * sl + G * ((lane >> 1) & 1) + 16 * (lane & 1) + (lane >> 2)] = (uint16_t)(lane & 1 ? pair >> 16 : pair);
    }
  }
}

// ---------------------------------------------------------------------------
// Scores. A unit is the query rows of TG neighbouring new tokens of one sequence and KV head, a token's
// heads on 2^p columns (the last ones repeat the first head), TG tokens to 16 NB columns of
// 16 x 16 x 32 products whose rows are 16 blocks: a lane reads 8 fp16 of a block's box, the
// register operand as it lies in memory. q' is scaled by 2^E and cut into two fp16 parts, each split by
// sign into the part against the least values and the one against the largest; the boxes are exact, so a
// score is off by about 2^-22 of sum_j |q'_j box_j| and the sums' roundings.
// Sequence b's units begin at first_b / TG + b: those of two sequences never meet, and a workgroup
// finds its own without a sum over the others. A launch is of the new tokens from .. to, as many as the scores' room holds:
// to it a sequence is its tokens among those, and its end the slot of the last.
//
// Few tokens: HEADS writes every head's scores and the best of its chunk of blocks, the rest is
// paged_pick_kernel's. Many: TOPS finds the heads' best alone, VALUES makes the scores again and writes
// the blocks' values, a KV head's instead of all its heads'; with units enough for the card, BOTH in turn.
//
// Measured, 8 KV heads of four: one token over 1M slots 17 us (34 MB of boxes, 2 TB/s; the prologue's chain and the
// memory's latency, DEEP units under way: wavefronts wait 64% of their time, the vector unit is busy 17%); 512 tokens over
// 100k slots 67 us (27 GFLOP in both sweeps, two parts each, 0.4 PFLOP/s; matrix cores 27% busy, vector unit 35, half of the
// wavefronts' time waiting). The latter waits for operands: without the boxes' loads 23 us less, with one of two parts 25 less; four
// block tiles a step, which halve the reads of q', came to 76 (fewer steps to share, spills), one sum for both
// parts to 67.
// ---------------------------------------------------------------------------
struct UnitScratch {
  int32_t b;
};
// Sequence b as this launch has it; n = 0 where it has none of its tokens, or more slots than the call allows.
__device__ __forceinline__ PagedSeq launched(const PagedSelectArgs& a, int b) {
  PagedSeq s = paged_seq(a.c, b);
  const int64_t end = s.first + s.n, lo = s.first < a.from ? a.from : s.first, hi = end < a.to ? end : a.to;
  s.n = lo < hi && s.len <= a.max_tokens ? hi - lo : 0;
  s.first = lo;
  s.len -= end - hi;  // (below 0: it sees nothing)
  return s;
}
// The sequence of unit u and the unit's place in it; the same in every thread. b < 0: none.
template <int NT>
__device__ __forceinline__ int find_token_unit(const PagedSelectArgs& a, int64_t u, int tg, UnitScratch& s, int64_t& at) {
  if (a.c.batch == 1) {
    const PagedSeq q = launched(a, 0);
    at = u - (q.first - a.from) / tg;
    return at >= 0 && at < (q.n + tg - 1) / tg ? 0 : -1;
  }
  if (threadIdx.x == 0) s.b = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < a.c.batch; b += NT) {
    const PagedSeq q = launched(a, b);
    const int64_t base = (q.first - a.from) / tg + b;
    if (u >= base && u < base + (q.n + tg - 1) / tg) atomicMax(&s.b, b);
  }
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(s.b);
  if (b >= 0) at = u - ((launched(a, b).first - a.from) / tg + b);
  return b;
}

// What a page out of range and places past the last block read as.
__device__ const u32x4 empty_box[BOX_WORDS / 4] = {};

enum SelectMode { HEADS, TOPS, VALUES, BOTH };
constexpr int PAIR = 2;  // block tiles of a wavefront's step: an operand of q' is read once for both
static_assert(16 * PAIR == spectra::SELECT_STEP, "whole steps in a row of scores");

template <int NB, int NW, SelectMode MODE>
__global__ __launch_bounds__(64 * NW, 2) void paged_block_scores_kernel(PagedSelectArgs a, int steps) {
  constexpr int COLS = 16 * NB, NT = 64 * NW, SHARE = NW / 4, HALF = NB / SHARE;  // of a group's row blocks a wavefront makes HALF
  constexpr int DEEP = NB == 1 ? 4 : 3;
  __shared__ UnitScratch unit_s;
  __shared__ float most_s[NG][COLS];
  __shared__ __attribute__((aligned(16))) uint8_t q_s[NG][NB][4][64 * 16];  // against least: hi, lo; against largest: hi, lo
  __shared__ float un_s[COLS], top_s[MODE == VALUES ? 1 : NW][COLS];
  const int tg = COLS >> a.pitch_log2;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int64_t at = 0;
  const int b = find_token_unit<NT>(a, blockIdx.x / (unsigned)a.c.n_kv, tg, unit_s, at);
  if (b < 0) return;
  const PagedSeq seq = launched(a, b);
  const int64_t tok0 = at * tg;
  const int n_tok = (int)(seq.n - tok0 < tg ? seq.n - tok0 : tg);
  // slots that the unit's last token sees: the blocks of the others are among its
  const int64_t past = seq.len - seq.n + tok0 + 1, see = past + n_tok - 1;
  const int n_blocks = see > 0 ? (int)((see + TILE - 1) / TILE) : 0;
  const int begin = blockIdx.y * steps;
  int end = (n_blocks + 16 * PAIR - 1) / (16 * PAIR);
  end = end < begin + steps ? end : begin + steps;
  // what a lane's column stands for
  auto column = [&](int nb, int& tok, int& head) __attribute__((always_inline)) {
    const int c = 16 * nb + col;
    tok = c >> a.pitch_log2;
    head = c & ((1 << a.pitch_log2) - 1);
    const bool live = tok < n_tok && head < a.n_qh;
    tok = tok < n_tok ? tok : 0;
    head = head < a.n_qh ? head : 0;
    return live;
  };
  const int64_t row0 = seq.first - a.from + tok0;  // of the unit's first token among the launch's
  auto row_of = [&](int tok, int head) { return (row0 + tok) * a.n_q_heads + kv * a.n_qh + head; };
  if (begin >= end) {
    if constexpr (MODE == HEADS || MODE == TOPS) {  // nothing here: no best
      for (int c = tid; c < COLS; c += NT) {
        const int tok = c >> a.pitch_log2, head = c & ((1 << a.pitch_log2) - 1);
        if (tok < n_tok && head < a.n_qh) a.tops[row_of(tok, head) * a.n_chunks + blockIdx.y] = -__builtin_inff();
      }
    }
    return;
  }
  Kept K = read_kept(a.bits_k + kv * NG);
  if (!K.ok || K.used > a.Wk) K.n = 0;  // width table inconsistent with the record
  const int tpp = a.c.page_tokens >> 6;
  // the walk over pages: of the lane's block in each tile of the step to load next, whose page is looked up
  // a step ahead
  int idx[PAIR], in_page[PAIR], page[PAIR], at_blk;
  const int walk = 16 * PAIR * NW, walk_pages = walk / tpp, walk_rest = walk - walk_pages * tpp;
  auto look_up = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < PAIR; ++t)
      page[t] = at_blk + 16 * t < n_blocks ? a.c.table[(int64_t)seq.row * a.c.row_pages + idx[t]] : -1;
  };
  auto start = [&]() __attribute__((always_inline)) {
    at_blk = 16 * PAIR * (begin + wave) + col;
#pragma unroll
    for (int t = 0; t < PAIR; ++t) {
      idx[t] = (at_blk + 16 * t) / tpp;
      in_page[t] = at_blk + 16 * t - idx[t] * tpp;
    }
    look_up();
  };
  // A unit is a kept group of a step's tiles; DEEP units' boxes are under way.
  const int n_sl = K.n > 0 ? K.n : 1, n_steps = end - begin > wave ? (end - begin - wave + NW - 1) / NW : 0, n_units = n_steps * n_sl;
  const u32x4* box[PAIR];
  int load_sl = n_sl;
  u32x4 x[DEEP][PAIR][2];
  auto load = [&](u32x4 (&y)[PAIR][2]) __attribute__((always_inline)) {
    if (load_sl == n_sl) {  // the next step
#pragma unroll
      for (int t = 0; t < PAIR; ++t) {
        const bool ok = page[t] >= 0 && page[t] < a.c.n_pages && K.n > 0;
        const int64_t at = (((int64_t)page[t] * a.c.n_kv + kv) * tpp + in_page[t]) * (BOX_WORDS / 4);
        box[t] = (ok ? reinterpret_cast<const u32x4*>(a.bounds) + at : empty_box) + quarter;
        in_page[t] += walk_rest;
        const bool next = in_page[t] >= tpp;
        in_page[t] -= next ? tpp : 0;
        idx[t] += walk_pages + (next ? 1 : 0);
      }
      at_blk += walk;
      look_up();
      load_sl = 0;
    }
#pragma unroll
    for (int t = 0; t < PAIR; ++t)
#pragma unroll
      for (int side = 0; side < 2; ++side) y[t][side] = box[t][(load_sl * 2 + side) * (G / 8)];
    ++load_sl;
  };
  start();
#pragma unroll
  for (int d = 0; d < DEEP; ++d) load(x[d]);  // under way while q' is made

  // q' of kept group `slot` and row blocks nb0 ..: element e of quarter p is coefficient 8 p + e. The
  // group's basis is cut into parts once for them.
  const int slot = wave & 3, nb0 = (wave >> 2) * HALF;
  f32x4 acc[HALF][2];
#pragma unroll
  for (int nb = 0; nb < HALF; ++nb) acc[nb][0] = acc[nb][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (slot < K.n) {
    const float* V = a.basis_k + (int64_t)kv * D * D + (8 * quarter) * D + G * pick4(K.grp, slot) + 8 * (col >> 2) + (col & 3);
    int64_t qoff[HALF];
#pragma unroll
    for (int nb = 0; nb < HALF; ++nb) {
      int tok, head;
      column(nb0 + nb, tok, head);
      qoff[nb] = (seq.first + tok0 + tok) * a.q_token_stride + (kv * a.n_qh + head) * a.q_head_stride + 8 * quarter;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      bf16x8 vp[2][3];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = V[(32 * k + e) * D + 4 * y];
        split8_pairs<3>(v, vp[y]);
      }
#pragma unroll
      for (int nb = 0; nb < HALF; ++nb) {
        bf16x8 qq[3];
        if (a.q_f32) {
          const f32x4* qp = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.q) + qoff[nb] + 32 * k);
          const f32x4 q0 = qp[0], q1 = qp[1];
          const float qv[8] = {q0[0], q0[1], q0[2], q0[3], q1[0], q1[1], q1[2], q1[3]};
          split8_pairs<3>(qv, qq);
        } else {
          qq[0] = as_bf16x8(*reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + qoff[nb] + 32 * k));
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
          for (int p = 0; p < 3; ++p) acc[nb][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[y][p], qq[0], acc[nb][y], 0, 0, 0);
          if (a.q_f32) {
            acc[nb][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[y][0], qq[1], acc[nb][y], 0, 0, 0);
            acc[nb][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[y][1], qq[1], acc[nb][y], 0, 0, 0);
            acc[nb][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[y][0], qq[2], acc[nb][y], 0, 0, 0);
          }
        }
      }
    }
  }
#pragma unroll
  for (int nb = 0; nb < HALF; ++nb) {
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, __builtin_fabsf(acc[nb][e >> 2][e & 3]));
    most = __builtin_fmaxf(most, __shfl_xor(most, 16));
    most = __builtin_fmaxf(most, other_half(most));
    if (quarter == 0) most_s[slot][16 * (nb0 + nb) + col] = most;
  }
  if constexpr (MODE == VALUES) {  // the heads' best over all chunks
    for (int c = tid; c < COLS; c += NT) {
      int tok = c >> a.pitch_log2, head = c & ((1 << a.pitch_log2) - 1);
      tok = tok < n_tok ? tok : 0;
      head = head < a.n_qh ? head : 0;
      const float* tops = a.tops + row_of(tok, head) * a.n_chunks;
      float top = -__builtin_inff();
#pragma unroll 16
      for (int i = 0; i < a.n_chunks; ++i) top = __builtin_fmaxf(top, tops[i]);
      top_s[0][c] = top;
    }
  }
  __syncthreads();
#pragma unroll
  for (int nb = 0; nb < HALF; ++nb) {
    const int row = 16 * (nb0 + nb) + col;
    const float most = __builtin_fmaxf(__builtin_fmaxf(most_s[0][row], most_s[1][row]), __builtin_fmaxf(most_s[2][row], most_s[3][row]));
    const float up = __builtin_ldexpf(1.0f, 9 - scale_exponent(most));
    if (slot == 0 && quarter == 0) un_s[row] = 1.0f / up;
    u32x4 r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 y = f32x2{acc[nb][j >> 1][2 * (j & 1)] * up, acc[nb][j >> 1][2 * (j & 1) + 1] * up};
      const f16x2 hi = __builtin_convertvector(y, f16x2);
      const uint32_t h = __builtin_bit_cast(uint32_t, hi);
      const uint32_t l = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{(y[0] - (float)hi[0]) * CA_LO, (y[1] - (float)hi[1]) * CA_LO}, f16x2));
      const uint32_t below = (y[0] < 0.0f ? 0xFFFFu : 0u) | (y[1] < 0.0f ? 0xFFFF0000u : 0u);
      r[0][j] = h & below;
      r[1][j] = l & below;
      r[2][j] = h & ~below;
      r[3][j] = l & ~below;
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) *reinterpret_cast<u32x4*>(q_s[slot][nb0 + nb][p] + 16 * lane) = r[p];
  }
  __syncthreads();

  float* out[NB];
  int lim[NB];  // blocks that the lane's row sees
  float un[NB], top[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    int tok, head;
    const bool live = column(nb, tok, head);
    out[nb] = nullptr;
    if (MODE == HEADS && live) out[nb] = a.scores + row_of(tok, head) * a.most_blocks;
    if ((MODE == VALUES || MODE == BOTH) && live && head == 0) out[nb] = a.scores + ((row0 + tok) * a.c.n_kv + kv) * a.most_blocks;
    const int64_t l = past + tok;
    lim[nb] = l > 0 ? (int)((l + TILE - 1) / TILE) : 0;
    un[nb] = un_s[16 * nb + col];
    top[nb] = MODE == VALUES ? top_s[0][16 * nb + col] : -__builtin_inff();
  }
  const int all_see = past > 0 ? (int)((past + TILE - 1) / TILE) : 0;  // blocks that the first token sees
  f32x4 hi[PAIR][NB], lo[PAIR][NB];
  auto multiply = [&](auto begins, const u32x4 (&y)[PAIR][2], int sl) __attribute__((always_inline)) {
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const f16x8 qh = as_f16x8(*reinterpret_cast<const u32x4*>(q_s[sl][nb][2 * side] + 16 * lane));
        const f16x8 ql = as_f16x8(*reinterpret_cast<const u32x4*>(q_s[sl][nb][2 * side + 1] + 16 * lane));
#pragma unroll
        for (int t = 0; t < PAIR; ++t) {
          const bool zero = decltype(begins)::value && side == 0;
          const f32x4 z = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
          hi[t][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(y[t][side]), qh, zero ? z : hi[t][nb], 0, 0, 0);
          lo[t][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(y[t][side]), ql, zero ? z : lo[t][nb], 0, 0, 0);
        }
      }
  };
  auto finish = [&](auto values, int step) __attribute__((always_inline)) {
    constexpr bool VALUE = decltype(values)::value;
#pragma unroll
    for (int t = 0; t < PAIR; ++t)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int blk = 16 * (PAIR * step + t) + 4 * quarter;
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_fmaf(lo[t][nb][i], 1.0f / CA_LO, hi[t][nb][i]) * un[nb];
        if (16 * PAIR * (step + 1) > all_see) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = blk + i < lim[nb] ? v[i] : -__builtin_inff();
        }
        if constexpr (VALUE) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float d = __builtin_fmaxf(v[i] - top[nb], -__builtin_inff());  // (NaN where the head has no number)
            if (a.pitch_log2 > 0) d = __builtin_fmaxf(d, dpp<0xB1, 0xF>(d, d));
            if (a.pitch_log2 > 1) d = __builtin_fmaxf(d, dpp<0x4E, 0xF>(d, d));
            if (a.pitch_log2 > 2) d = __builtin_fmaxf(d, dpp<0x141, 0xF>(d, d));
            if (a.pitch_log2 > 3) d = __builtin_fmaxf(d, dpp<0x128, 0xF>(d, d));
            v[i] = d;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) top[nb] = __builtin_fmaxf(top[nb], v[i]);
        }
        if ((VALUE || MODE == HEADS) && out[nb] != nullptr) *reinterpret_cast<f32x4*>(out[nb] + blk) = v;
      }
  };
  auto sweep = [&](auto values) __attribute__((always_inline)) {
    int sl = 0, step = begin + wave;
#pragma unroll 1
    for (int u = 0; u < n_units; u += DEEP) {
#pragma unroll
      for (int d = 0; d < DEEP; ++d) {
        if (u + d >= n_units) break;
        if (sl == 0)
          multiply(std::true_type{}, x[d], sl);
        else
          multiply(std::false_type{}, x[d], sl);
        load(x[d]);  // (past the last: empty boxes)
        if (++sl == n_sl) {
          finish(values, step);
          sl = 0;
          step += NW;
        }
      }
    }
  };
  if constexpr (MODE == VALUES) {
    sweep(std::true_type{});
  } else {
    sweep(std::false_type{});
    if constexpr (MODE == BOTH) {
      load_sl = n_sl;
      start();
#pragma unroll
      for (int d = 0; d < DEEP; ++d) load(x[d]);
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float t = __builtin_fmaxf(top[nb], __shfl_xor(top[nb], 16));
      t = __builtin_fmaxf(t, other_half(t));
      if (quarter == 0) top_s[wave][16 * nb + col] = t;
    }
    __syncthreads();
    auto best = [&](int c) {
      float t = top_s[0][c];
#pragma unroll
      for (int w = 1; w < NW; ++w) t = __builtin_fmaxf(t, top_s[w][c]);
      return t;
    };
    if constexpr (MODE == BOTH) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) top[nb] = best(16 * nb + col);
      sweep(std::true_type{});
    } else {
      for (int c = tid; c < COLS; c += NT) {
        const int tok = c >> a.pitch_log2, head = c & ((1 << a.pitch_log2) - 1);
        if (tok < n_tok && head < a.n_qh) a.tops[row_of(tok, head) * a.n_chunks + blockIdx.y] = best(c);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The best blocks of a (token, KV head), a workgroup each. A thread holds the values of four
// neighbouring blocks out of every 4 NT. They are counted in equal steps between the least and 0
// (rounding keeps the order, so a step's members stand between the steps beside it); the few values of the
// step that holds the n-th are ranked against each other, (value, then lowest index); should they be
// many, rounds of counts of 8 bits over value and index find the n-th instead. What stands at or before
// it is written in ascending order.
// A dozen barriers and one pass over the scores, whose first loads are on their way while the token's sequence is looked
// for: 13 us for 8 KV heads of four and 16384 blocks, by latency on the eight CUs that have work; 20 us for 4096 pairs of 1563
// values, the vector unit 65% busy.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

template <int NT>
struct PickScratch {
  static constexpr int STEPS = NT == 128 ? 512 : 2048, FEW = NT == 128 ? 256 : 1024;
  int32_t b;
  float top[16], least[NT / 64];
  int32_t count[STEPS], part[NT / 64];
  uint32_t sum[2][NT / 64];
  int32_t found[2], n;
  uint32_t key[FEW];
  int32_t at[FEW];
  uint32_t last_key;
  int32_t last_at;
};

// Inclusive sum over the workgroup.
template <int NT>
__device__ __forceinline__ int32_t sum_to(int32_t v, int32_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  if (lane == 63) part[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += part[w];
  return v;
}

// Of a round's counts (largest digits first): the digit at which `left` is reached, and what is left in it.
// PER counts a thread.
template <int NT, int N>
__device__ __forceinline__ void find_step(const int32_t* count, int left, int32_t* part, int32_t* found) {
  constexpr int PER = N / NT > 0 ? N / NT : 1;
  const int tid = threadIdx.x;
  int c[PER], mine = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int d = N - 1 - (tid * PER + i);
    c[i] = d >= 0 ? count[d] : 0;
    mine += c[i];
  }
  int before = sum_to<NT>(mine, part) - mine;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < left && before + c[i] >= left) {
      found[0] = N - 1 - (tid * PER + i);
      found[1] = left - before;
    }
    before += c[i];
  }
  __syncthreads();
}

// The heads' best over their chunks, also of one head: what is picked from counts down from 0 (raw scores, mostly positive,
// would all fall into one step: one token and one head to a KV head over 65k slots 306 us, so 16). Values: theirs is off already.
template <int NT>
__device__ __forceinline__ void best_of_heads(const PagedSelectArgs& a, int64_t at, int kv, int n_rows, float* top) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (a.by_values) {
    if (threadIdx.x == 0) top[0] = 0.0f;
    return;
  }
  for (int h = wave; h < n_rows; h += NT / 64) {
    const float* tops = a.tops + (at * a.n_q_heads + kv * a.n_qh + h) * a.n_chunks;
    float x = -__builtin_inff();
    for (int i = lane; i < a.n_chunks; i += 64) x = __builtin_fmaxf(x, tops[i]);
    x = wave_max(x);
    if (lane == 0) top[h] = x;
  }
}

template <int NT, int IT>
__global__ __launch_bounds__(NT, NT == 128 ? 4 : 1) void paged_pick_kernel(PagedSelectArgs a, int n_rows) {
  constexpr int STEPS = PickScratch<NT>::STEPS, FEW = PickScratch<NT>::FEW;
  __shared__ PickScratch<NT> s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int64_t at = blockIdx.x / (unsigned)a.c.n_kv, t = a.from + at;  // the token's place among the launch's, and the call's
  const float* rows = a.scores + (at * a.c.n_kv + kv) * (int64_t)n_rows * a.most_blocks;
  constexpr int HB = NT == 128 ? 1 : 16 / IT;  // rows at a time: 16 loads under way (values: one row)
  f32x4 x[HB][IT];
  auto load = [&](int h0) __attribute__((always_inline)) {  // (what lies behind the last block is not used)
#pragma unroll
    for (int h = 0; h < HB; ++h)
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int blk = 4 * (NT * i + tid);
        x[h][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (blk < a.most_blocks && h0 + h < n_rows) x[h][i] = *reinterpret_cast<const f32x4*>(rows + (int64_t)(h0 + h) * a.most_blocks + blk);
      }
  };
  load(0);  // while the token's sequence is looked for
  if (tid == 0) s.b = -1;
  __syncthreads();
  for (int b = tid; b < a.c.batch; b += NT) {
    const PagedSeq q = paged_seq(a.c, b);
    if (t >= q.first && t < q.first + q.n) atomicMax(&s.b, b);
  }
  for (int i = tid; i < STEPS; i += NT) s.count[i] = 0;
  if (tid == 0) s.n = 0;
  best_of_heads<NT>(a, at, kv, n_rows, s.top);
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(s.b);
  if (b < 0) return;
  const PagedSeq seq = paged_seq(a.c, b);
  if (seq.len > a.max_tokens) return;
  const int64_t see = seq.len - seq.n + (t - seq.first) + 1;
  const int have = see > 0 ? (int)((see + TILE - 1) / TILE) : 0, want = a.n_blocks;
  int32_t* out = a.blocks + (t * a.c.n_kv + kv) * want;
  if (have <= want) {
    for (int i = tid; i < want; i += NT) out[i] = i < have ? i : -1;
    return;
  }
  float v[IT][4], least = 0.0f;
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[i][e] = -__builtin_inff();
  for (int h0 = 0; h0 < n_rows; h0 += HB) {
    if (h0 > 0) load(h0);
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      if (h0 + h >= n_rows) break;
      const float top = s.top[h0 + h];
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = __builtin_fmaxf(v[i][e], x[h][i][e] - top);  // (NaN, where the head has no number, is passed over)
    }
  }
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * (NT * i + tid) + e < have && v[i][e] > -__builtin_inff()) least = __builtin_fminf(least, v[i][e]);
  least = -wave_max(-least);
  if (lane == 0) s.least[wave] = least;
  __syncthreads();
  for (int w = 0; w < NT / 64; ++w) least = __builtin_fminf(least, s.least[w]);
  // steps: -1 past the last block, STEPS for blocks that are in anyway
  const float per = least < 0.0f ? (STEPS - 1) / -least : 0.0f, off = (STEPS - 1);  // (values of -inf: the first step)
  const bool spread = least < 0.0f && per < __builtin_inff();
  int step_of[IT][4];
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int blk = 4 * (NT * i + tid) + e;
      const float y = spread ? __builtin_fmaf(v[i][e], per, off) : 0.0f;
      const int y0 = (int)__builtin_fminf(__builtin_fmaxf(y, 0.0f), off);
      step_of[i][e] = blk >= have ? -1 : blk < a.first || blk >= have - a.last ? STEPS : y0;
      if (step_of[i][e] >= 0 && step_of[i][e] < STEPS) atomicAdd(&s.count[y0], 1);
    }
  __syncthreads();
  const int others = want - a.first - a.last;  // (they do not meet: have > want)
  int step = STEPS - 1;
  if (others > 0) {
    find_step<NT, STEPS>(s.count, others, s.part, s.found);
    step = s.found[0];
    const int left = s.found[1], many = s.count[step];
    uint32_t last_key;
    int last_at;
    if (many <= FEW) {
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (step_of[i][e] == step) {
            const int n = atomicAdd(&s.n, 1);
            s.key[n] = order_of(v[i][e]);
            s.at[n] = 4 * (NT * i + tid) + e;
          }
      __syncthreads();
      for (int j = tid; j < many; j += NT) {  // their order does not depend on where they lie
        const uint32_t key = s.key[j];
        const int blk = s.at[j];
        int before = 0;
        for (int k = 0; k < many; ++k) before += s.key[k] > key || (s.key[k] == key && s.at[k] < blk) ? 1 : 0;
        if (before == left - 1) {
          s.last_key = key;
          s.last_at = blk;
        }
      }
      __syncthreads();
      last_key = s.last_key;
      last_at = s.last_at;
    } else {
      uint64_t prefix = 0u, mask = 0u;  // of (value, index counted down)
      int rest = left;
      for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = tid; i < 256; i += NT) s.count[i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint64_t key = (uint64_t)order_of(v[i][e]) << 32 | (uint32_t)~(4 * (NT * i + tid) + e);
            if (step_of[i][e] == step && (key & mask) == prefix) atomicAdd(&s.count[(int)(key >> shift) & 255], 1);
          }
        __syncthreads();
        find_step<NT, 256>(s.count, rest, s.part, s.found);
        prefix |= (uint64_t)s.found[0] << shift;
        mask |= (uint64_t)255 << shift;
        rest = s.found[1];
      }
      last_key = (uint32_t)(prefix >> 32);
      last_at = (int)~(uint32_t)prefix;
    }
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (step_of[i][e] == step) {
          const uint32_t key = order_of(v[i][e]);
          if (key > last_key || (key == last_key && 4 * (NT * i + tid) + e <= last_at)) step_of[i][e] = STEPS;
        }
  }
  // what stands above the step is taken; a thread's of each of four rounds in 16 bits
  int base = 0;
#pragma unroll
  for (int i0 = 0; i0 < IT; i0 += 4) {
    uint32_t mine[2] = {0u, 0u};
#pragma unroll
    for (int i = i0; i < IT && i < i0 + 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[(i - i0) >> 1] += step_of[i][e] > step ? 1u << (16 * (i & 1)) : 0u;
    uint32_t upto[2] = {mine[0], mine[1]};
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t u0 = __shfl_up(upto[0], o), u1 = __shfl_up(upto[1], o);
      upto[0] += lane >= o ? u0 : 0u;
      upto[1] += lane >= o ? u1 : 0u;
    }
    __syncthreads();
    if (lane == 63) {
      s.sum[0][wave] = upto[0];
      s.sum[1][wave] = upto[1];
    }
    __syncthreads();
    uint32_t all[2] = {0u, 0u};
    for (int w = 0; w < NT / 64; ++w)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        upto[k] += w < wave ? s.sum[k][w] : 0u;
        all[k] += s.sum[k][w];
      }
#pragma unroll
    for (int i = i0; i < IT && i < i0 + 4; ++i) {
      const int k = (i - i0) >> 1, at = 16 * (i & 1);
      int place = base + (int)((upto[k] - mine[k]) >> at & 0xFFFF);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (step_of[i][e] > step) out[place++] = 4 * (NT * i + tid) + e;
      base += (int)(all[k] >> at & 0xFFFF);
    }
  }
}

// The same for more blocks than registers hold: keys in the place of the first row's scores,
// the n-th by rounds of counts of 8 bits.
constexpr int PICK = 1024;
__global__ __launch_bounds__(PICK) void paged_pick_long_kernel(PagedSelectArgs a, int n_rows) {
  __shared__ int32_t b_s;
  __shared__ float top_s[16];
  __shared__ int32_t hist_s[256], part_s[PICK / 64], part2_s[PICK / 64], found_s[2];
  const int tid = threadIdx.x;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int64_t at = blockIdx.x / (unsigned)a.c.n_kv, t = a.from + at;
  if (tid == 0) b_s = -1;
  __syncthreads();
  for (int b = tid; b < a.c.batch; b += PICK) {
    const PagedSeq q = paged_seq(a.c, b);
    if (t >= q.first && t < q.first + q.n) atomicMax(&b_s, b);
  }
  best_of_heads<PICK>(a, at, kv, n_rows, top_s);
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
  float* rows = a.scores + (at * a.c.n_kv + kv) * (int64_t)n_rows * a.most_blocks;
  uint32_t* keys = reinterpret_cast<uint32_t*>(rows);
  for (int i = tid; i < have; i += PICK) {
    float v = -__builtin_inff();
    for (int h = 0; h < n_rows; ++h) {
      const float d = rows[(int64_t)h * a.most_blocks + i] - top_s[h];  // NaN where the head has no number
      v = __builtin_fmaxf(v, d == d ? d : -__builtin_inff());
    }
    keys[i] = i < a.first || i >= have - a.last ? 0xFFFFFFFFu : order_of(v);
  }
  uint32_t prefix = 0u, mask = 0u;
  int left = want;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist_s[tid] = 0;
    __syncthreads();
    for (int i = tid; i < have; i += PICK) {
      const uint32_t k = keys[i];
      if ((k & mask) == prefix) atomicAdd(&hist_s[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    find_step<PICK, 256>(hist_s, left, part_s, found_s);
    prefix |= (uint32_t)found_s[0] << shift;
    mask |= 255u << shift;
    left = found_s[1];
    __syncthreads();
  }
  // neighbouring blocks to a thread: how many above and equal, then their places
  const int each = (have + PICK - 1) / PICK;
  const int from = tid * each < have ? tid * each : have, to = from + each < have ? from + each : have;
  int above = 0, equal = 0;
  for (int i = from; i < to; ++i) {
    const uint32_t k = keys[i];
    above += k > prefix ? 1 : 0;
    equal += k == prefix ? 1 : 0;
  }
  const int va = sum_to<PICK>(above, part_s), ve = sum_to<PICK>(equal, part2_s);
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

size_t paged_select_bytes(int64_t n_new, int32_t n_q_heads, int32_t n_kv, int64_t max_tokens) {
  return (size_t)select_plan(n_new, n_q_heads, n_kv, max_tokens).floats * sizeof(float);
}

hipError_t launch_paged_select(const PagedSelectArgs& args, void* workspace, hipStream_t st) {
  PagedSelectArgs a = args;
  const int64_t n_kv = a.c.n_kv;
  const SelectPlan plan = select_plan(a.c.n_new, a.n_q_heads, a.c.n_kv, a.max_tokens);
  a.by_values = plan.many;
  a.most_blocks = (int32_t)plan.pitch;
  a.tops = static_cast<float*>(workspace);
  a.scores = a.tops + plan.scores_at;
  a.pitch_log2 = 0;
  while (1 << a.pitch_log2 < a.n_qh) ++a.pitch_log2;
  for (a.from = 0; a.from < a.c.n_new; a.from = a.to) {
    const int64_t left = a.c.n_new - a.from, tokens = left < plan.tokens ? left : plan.tokens;
    a.to = a.from + (int32_t)tokens;
    const SelectSlab slab = select_slab(plan, tokens, a.c.batch, a.c.n_kv, a.pitch_log2);
    a.n_chunks = (int32_t)slab.chunks;
    const dim3 grid((unsigned)(slab.units * n_kv), (unsigned)slab.chunks);
    if (slab.both) {
      hipLaunchKernelGGL((paged_block_scores_kernel<4, 8, BOTH>), grid, dim3(512), 0, st, a, (int)slab.steps);
    } else if (plan.many) {
      hipLaunchKernelGGL((paged_block_scores_kernel<4, 4, TOPS>), grid, dim3(256), 0, st, a, (int)slab.steps);
      hipLaunchKernelGGL((paged_block_scores_kernel<4, 4, VALUES>), grid, dim3(256), 0, st, a, (int)slab.steps);
    } else {
      hipLaunchKernelGGL((paged_block_scores_kernel<1, 4, HEADS>), grid, dim3(256), 0, st, a, (int)slab.steps);
    }
    const dim3 rows((unsigned)(tokens * n_kv));
    const int n_rows = plan.many ? 1 : a.n_qh;
    // (of 512 tokens and 1600 blocks in all 82 us, and 96 with 256 threads a pair)
    if (plan.many && a.most_blocks <= 2048)
      hipLaunchKernelGGL((paged_pick_kernel<128, 4>), rows, dim3(128), 0, st, a, n_rows);
    else if (a.most_blocks <= 1024)
      hipLaunchKernelGGL((paged_pick_kernel<256, 1>), rows, dim3(256), 0, st, a, n_rows);
    else if (a.most_blocks <= 4096)
      hipLaunchKernelGGL((paged_pick_kernel<256, 4>), rows, dim3(256), 0, st, a, n_rows);
    else if (a.most_blocks <= 16384)
      hipLaunchKernelGGL((paged_pick_kernel<1024, 4>), rows, dim3(1024), 0, st, a, n_rows);
    else
      hipLaunchKernelGGL(paged_pick_long_kernel, rows, dim3(PICK), 0, st, a, n_rows);
  }
  return hipGetLastError();
}

}  // namespace spectra
