// Attention of a few query rows over tiles of a paged packed cache: the drafted trees of sequences
// (rows = drafted tokens x query heads of a KV head, tiles = all of the sequence's) and tokens over
// listed blocks (rows = neighbouring tokens x query heads of a KV head, tiles = what their lists name together).
//
//   q'  = scale * log2(e) * q V_K
//   S   = q' . c_hat_K(t)                     (the constant q' . m_K cancels in the softmax)
//   p   = exp2(S - m), l = sum p, a = sum p c_hat_V(t)   in one pass, m the running maximum
//   out = (a / l + m_V) V_V^T
//
// A unit is NB blocks of 16 rows, a workgroup a chunk of the unit's tiles, a wavefront tiles of its
// own: it turns a kept group of 64 slots into fp16 coefficients in 4 KB of LDS, once for all rows of
// the unit, and multiplies them on 16 x 16 x 32 products whose columns are the rows. No barrier until
// the wavefronts' sums are merged. The chunks' partial sums meet in the combine kernels.
//
// Measured (8-word records): 48 tokens of 28 heads over 64 blocks 36 us (12300 tiles of 4 KB, 1.4 TB/s), with the join
// 39; 16 trees of up to 32 tokens of 32 heads over 8k slots 76 + 14 us; in fp32, 200 tokens over 32 blocks 85 + 12 (traced: a
// launch then counts from the end of the one before it). No unit is near its limit: a tile costs a wavefront
// about 10000 clocks of the 2000 that its instructions need alone, with three on a SIMD; while a CU holds work its vector unit is
// busy 47 to 62% of the time, its matrix cores 6 to 13, and a wavefront waits for memory, LDS or a barrier 36 to 50% of its
// time. Making the coefficients is half of a tile. With all records in the first cache 35 us for 37; with a
// second tile in LDS, filled while the first is multiplied, 38.
// With 16-bit outputs q', c and p are single fp16 numbers; with fp32 outputs (PRECISE) pairs of fp16 parts,
// every product three.
//
// What a row of a tree sees behind the history is a bit mask of at most 64 drafted slots: its own bit and
// its ancestors'.
#include <algorithm>

#include "encode_dev.hpp"
#include "paged_coef.hpp"
#include "paged_dev.hpp"
#include "splits.hpp"

namespace spectra_dev {

constexpr int RO_NW = 4, RO_NT = 64 * RO_NW;
constexpr int RO_PITCH = D + 4;

// LDS byte of 16-byte piece `piece` of slot `t` in a slot tile: eight neighbouring slots' equal pieces, and
// the two pieces of four slots that a transposed read takes, lie on distinct banks.
__device__ __forceinline__ int slot_piece(int t, int piece) { return t * 64 + ((piece ^ (t & 2) ^ ((t >> 2) & 1)) << 4); }

// One slot's group as fp16 coefficients z + s code into its LDS row, rounded once. PRECISE: and what the rounding
// left, 2^11 (z + s code) - 2^11 hi, in the tile `lo` bytes further (its fp32 product and sum are rounded to 2^-24).
template <int B, bool PRECISE>
__device__ __forceinline__ void write_slot(const uint32_t (&w)[8], uint32_t meta, uint8_t* tile, int t, int lo, uint32_t magic) {
  uint32_t Z[8];
  join_halves<B>(w, Z);
  const _Float16 s = __builtin_bit_cast(_Float16, (uint16_t)meta), z = __builtin_bit_cast(_Float16, (uint16_t)(meta >> 16));
  const float s2 = (float)s * CA_LO, z2 = (float)z * CA_LO;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f16x8 c = codes_f16<B, false>(Z, k, magic);
    u32x4 rh, rl;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f16x2 hi = __builtin_elementwise_fma(f16x2{s, s}, f16x2{c[2 * i], c[2 * i + 1]}, f16x2{z, z});
      rh[i] = __builtin_bit_cast(uint32_t, hi);
      if constexpr (PRECISE) {
        f16x2 rest;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          rest[e] = (_Float16)__builtin_fmaf((float)hi[e], -CA_LO, __builtin_fmaf(s2, (float)c[2 * i + e], z2));
        rl[i] = __builtin_bit_cast(uint32_t, rest);
      }
    }
    *reinterpret_cast<u32x4*>(tile + slot_piece(t, k)) = rh;
    if constexpr (PRECISE) *reinterpret_cast<u32x4*>(tile + lo + slot_piece(t, k)) = rl;
  }
}

// finite_meta with one test for all that is rare: z + s top is finite and within fp16 only where s and z are.
__device__ __forceinline__ uint32_t finite_slot(uint32_t m, int bits, float top) {
  const f16x2 sz = __builtin_bit_cast(f16x2, m);
  const float x = __builtin_fmaf((float)sz[0], top, (float)sz[1]);
  if (!(__builtin_fabsf(x) <= 65504.0f)) m = finite_meta(m, bits);
  return m;
}

// ---------------------------------------------------------------------------
// Where a workgroup's work lies
// ---------------------------------------------------------------------------
struct RowsPlace {
  int b;        // sequence; < 0: none
  int unit;     // of the sequence's units
  int chunk, n_chunks;
  int tiles;    // of a chunk
};
struct RowsScratch {
  int64_t part[2][RO_NW], total[2];
  int32_t b, at, n;
};

// Trees of few rows (the others are paged_chunk_kernel's): sequence b has ceil(n_b n_qh / rows) units, each cut into chunks of `tiles` tiles, the same
// for all, so that about p.want chunks come out; items are the chunks, the sequences' one after the
// other. The same in every thread.
__device__ __forceinline__ RowsPlace tree_place(const PagedRowsArgs& p, int rows, int item, RowsScratch& s) {
  const PagedCache& c = p.a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto look = [&](int b, int& units, int& tiles) {
    units = tiles = 0;
    if (b >= c.batch) return;
    const PagedSeq q = paged_seq(c, b);
    if (!scanned(p.a, q)) return;
    units = (int)((q.n * p.a.n_qh + rows - 1) / rows);
    tiles = units > 0 ? (int)((q.len + TILE - 1) / TILE) : 0;
  };
  // inclusive sums over the workgroup, their totals in s.total
  auto sum = [&](int64_t& u, int64_t& v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t x = __shfl_up(u, o), y = __shfl_up(v, o);
      if (lane >= o) {
        u += x;
        v += y;
      }
    }
    __syncthreads();
    if (lane == 63) {
      s.part[0][wave] = u;
      s.part[1][wave] = v;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
      u += s.part[0][w];
      v += s.part[1][w];
    }
    if (tid == RO_NT - 1) {
      s.total[0] = u;
      s.total[1] = v;
    }
    __syncthreads();
  };
  int units0, tiles0;  // of the first sequences, a thread each
  look(c.batch == 1 ? 0 : tid, units0, tiles0);
  int64_t n_units = units0, work = (int64_t)units0 * tiles0;
  if (c.batch > 1) {
    for (int b = tid + RO_NT; b < c.batch; b += RO_NT) {
      int u, t;
      look(b, u, t);
      n_units += u;
      work += (int64_t)u * t;
    }
    sum(n_units, work);
    n_units = s.total[0];
    work = s.total[1];
  }
  RowsPlace r;
  r.b = -1;
  r.unit = r.chunk = r.n_chunks = 0;
  // every unit ends in half a chunk on average: those count too
  const int64_t whole = p.want - (n_units < p.want ? n_units : p.want) / 2;
  int64_t each = (work + whole - 1) / whole;
  each = (each + RO_NW - 1) / RO_NW * RO_NW;
  constexpr int64_t most = (int64_t)1 << 24;  // tiles of the longest row
  r.tiles = (int)(each < RO_NW ? RO_NW : each < most ? each : most);
  auto chunks = [&](int tiles) { return (tiles + r.tiles - 1) / r.tiles; };
  if (c.batch == 1) {
    r.n_chunks = chunks(tiles0);
    if (r.n_chunks == 0 || item >= units0 * r.n_chunks) return r;
    r.b = 0;
    r.unit = item / r.n_chunks;
    r.chunk = item - r.unit * r.n_chunks;
    return r;
  }
  if (tid == 0) s.b = -1;
  int64_t base = 0;
  for (int b0 = 0; b0 < c.batch; b0 += RO_NT) {
    int u = units0, t = tiles0;
    if (b0 > 0) look(b0 + tid, u, t);
    const int n = chunks(t);
    int64_t v = (int64_t)u * n, none = 0;
    const int64_t mine = v;
    sum(v, none);
    const int64_t lo = base + v - mine;
    if (item >= lo && item < lo + mine) {
      s.b = b0 + tid;
      s.at = (int)(item - lo);
      s.n = n;
    }
    __syncthreads();
    if (s.b >= 0) break;
    base += s.total[0];
    __syncthreads();
  }
  r.b = __builtin_amdgcn_readfirstlane(s.b);
  if (r.b < 0) return r;
  r.n_chunks = __builtin_amdgcn_readfirstlane(s.n);
  r.unit = __builtin_amdgcn_readfirstlane(s.at) / r.n_chunks;
  r.chunk = __builtin_amdgcn_readfirstlane(s.at) - r.unit * r.n_chunks;
  return r;
}

// The place of a sequence's unit in the plan: units of two sequences never meet.
__device__ __forceinline__ int64_t plan_at(const PagedRowsArgs& p, int rows, const PagedSeq& seq, int b, int unit) {
  return seq.first * p.a.n_qh / rows + b + unit;
}

// Lists: a unit is p.tokens neighbouring new tokens of one sequence (sequence b's units begin at first_b /
// tokens + b, so those of two sequences never meet; with single tokens, at first_b). The last sequence that
// unit u belongs to, -1: none, and its first token. Every thread.
__device__ __forceinline__ int list_unit(const PagedRowsArgs& p, int64_t u, int32_t& b_s, int64_t& tok0) {
  const PagedCache& c = p.a.c;
  auto at = [&](int b, const PagedSeq& q) { return u - (p.tokens == 1 ? q.first : q.first / p.tokens + b); };
  auto has = [&](int b, const PagedSeq& q) {
    const int64_t x = at(b, q);
    return x >= 0 && x < (q.n + p.tokens - 1) / p.tokens;
  };
  int b = 0;
  if (c.batch > 1) {
    if (threadIdx.x == 0) b_s = -1;
    __syncthreads();
    for (int i = threadIdx.x; i < c.batch; i += RO_NT)
      if (has(i, paged_seq(c, i))) atomicMax(&b_s, i);
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(b_s);
    if (b < 0) return -1;
  }
  const PagedSeq q = paged_seq(c, b);
  if (!has(b, q)) return -1;
  tok0 = at(b, q) * p.tokens;
  return b;
}

// The chunk's entries of a list [from, to) that name blocks the token sees (below `blocks`) and are
// greater than all entries before them, packed into sel; returns how many.
struct ListScratch {
  int32_t top[RO_NW], count[RO_NW];
};
__device__ __forceinline__ int read_list(const int32_t* __restrict__ list, int from, int to, int blocks, int32_t* sel, ListScratch& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int before = -1, n = 0;
  for (int e0 = 0; e0 < to; e0 += RO_NT) {
    const int e = e0 + tid, x = e < to ? list[e] : -1;
    int top = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(top, o);
      if (lane >= o && u > top) top = u;
    }
    int prev = __shfl_up(top, 1);
    if (lane == 0) prev = -1;
    __syncthreads();
    if (lane == 63) s.top[wave] = top;
    __syncthreads();
    int all = before;
    for (int w = 0; w < RO_NW; ++w) {
      if (w < wave && s.top[w] > prev) prev = s.top[w];
      if (s.top[w] > all) all = s.top[w];
    }
    if (before > prev) prev = before;
    const bool take = e >= from && e < to && x > prev && x < blocks;
    const uint64_t m = __ballot(take);
    if (lane == 0) s.count[wave] = __popcll(m);
    __syncthreads();
    int at = n, total = n;
    for (int w = 0; w < RO_NW; ++w) {
      if (w < wave) at += s.count[w];
      total += s.count[w];
    }
    if (take) sel[at + __popcll(m & (((uint64_t)1 << lane) - 1))] = x;
    n = total;
    before = all;
  }
  __syncthreads();
  return n;
}

constexpr int LIST_CHUNK = 256;   // entries of a workgroup at most, where a unit is one token
constexpr int LIST_ALL = 256;     // entries of a unit's tokens at most, where it is several

// What the lists of n tokens name together, each block once, with the tokens that name it as bits. Lists as
// in read_list, token i's below blocks(i). A wavefront packs a token's list; then each of its entries is looked up in all
// (by halves, they ascend): the first token that names a block brings it in. packed, who: LIST_ALL entries. Returns how many.
struct UnionScratch {
  int32_t count[16], own[16];
};
template <typename Blocks>
__device__ __forceinline__ int read_lists(const int32_t* __restrict__ lists, int64_t stride, int n_blocks, int n, Blocks&& blocks,
                                          int32_t* packed, uint16_t* who, int32_t* sel, uint16_t* bits, UnionScratch& s) {
  constexpr int SEARCH = 4;  // lists searched side by side
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int i = wave; i < n; i += RO_NW) {
    const int32_t* list = lists + i * stride;
    const int end = blocks(i);
    int before = -1, at = 0;
    for (int e0 = 0; e0 < n_blocks; e0 += 64) {
      const int x = e0 + lane < n_blocks ? list[e0 + lane] : -1;
      int top = x;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(top, o);
        if (lane >= o && u > top) top = u;
      }
      int prev = __shfl_up(top, 1);
      prev = lane == 0 || before > prev ? before : prev;
      const bool take = x > prev && x < end;
      const uint64_t m = __ballot(take);
      if (take) packed[i * n_blocks + at + __popcll(m & below)] = x;
      at += __popcll(m);
      const int last = __shfl(top, 63);
      before = last > before ? last : before;
    }
    if (lane == 0) s.count[i] = at;
  }
  __syncthreads();
  int most = 1;  // the search's first step
  while (2 * most <= n_blocks) most *= 2;
  for (int i = wave; i < n; i += RO_NW) {
    int at = 0;
    for (int e0 = 0; e0 < s.count[i]; e0 += 64) {
      const int e = e0 + lane;
      const bool live = e < s.count[i];
      const int x = live ? packed[i * n_blocks + e] : 0;
      uint32_t by = 0u;
      for (int j0 = 0; j0 < n; j0 += SEARCH) {
        int pos[SEARCH], end[SEARCH];
#pragma unroll
        for (int k = 0; k < SEARCH; ++k) {
          pos[k] = 0;
          end[k] = j0 + k < n ? s.count[j0 + k] : 0;
        }
        for (int step = most; step > 0; step >>= 1) {
#pragma unroll
          for (int k = 0; k < SEARCH; ++k) {
            const int to = pos[k] + step;
            if (to <= end[k] && packed[(j0 + k) * n_blocks + to - 1] < x) pos[k] = to;
          }
        }
#pragma unroll
        for (int k = 0; k < SEARCH; ++k)
          if (pos[k] < end[k] && packed[(j0 + k) * n_blocks + pos[k]] == x) by |= 1u << (j0 + k);
      }
      const bool own = live && (by & ((1u << i) - 1)) == 0u;  // no token before names it
      if (live) who[i * n_blocks + e] = own ? (uint16_t)by : 0;
      at += __popcll(__ballot(own));
    }
    if (lane == 0) s.own[i] = at;
  }
  __syncthreads();
  for (int i = wave; i < n; i += RO_NW) {
    int at = 0;
    for (int j = 0; j < i; ++j) at += s.own[j];
    for (int e0 = 0; e0 < s.count[i]; e0 += 64) {
      const int e = e0 + lane;
      const uint16_t by = e < s.count[i] ? who[i * n_blocks + e] : 0;
      const uint64_t m = __ballot(by != 0);
      if (by != 0) {
        sel[at + __popcll(m & below)] = packed[i * n_blocks + e];
        bits[at + __popcll(m & below)] = by;
      }
      at += __popcll(m);
    }
  }
  __syncthreads();
  int total = 0;
  for (int i = 0; i < n; ++i) total += s.own[i];
  return total;
}

// u = scale V_K m_K of a KV head, by a workgroup: q . u is the part of the log-sum-exp that the softmax does not need.
__device__ __forceinline__ void lse_constants(const PagedAttnArgs& a, int kv) {
  const int ch = threadIdx.x >> 1, half = threadIdx.x & 1;
  const f32x4* v = reinterpret_cast<const f32x4*>(a.basis_k + ((int64_t)kv * D + ch) * D + 64 * half);
  const float* m = a.mean_k + kv * D + 64 * half;
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const f32x4 x = v[j];
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_fmaf(x[i], m[4 * j + i], s);
  }
  s += __shfl_xor(s, 1);
  if (half == 0) a.lse_u[kv * D + ch] = s * (a.scale_log2 * LN2);
}

// ---------------------------------------------------------------------------
// The sums of a unit over a chunk. A group's words are loaded while the one before is multiplied (a whole
// tile ahead, in registers, came to 45 us for 39: 48 tokens of seven heads over 64 blocks).
// ---------------------------------------------------------------------------
template <int NB, bool PRECISE, bool TREE>
__global__ __launch_bounds__(RO_NT, NB == 1 && !PRECISE ? 4 : 2) void paged_rows_kernel(PagedRowsArgs p) {
  constexpr int ROWS = 16 * NB, NP = PRECISE ? 2 : 1, QP = PRECISE ? 3 : 2;
  __shared__ RowsScratch place_s;
  __shared__ ListScratch list_s;
  __shared__ UnionScratch union_s;
  __shared__ int32_t sel_s[TREE ? 1 : LIST_ALL], b_s;
  __shared__ uint16_t who_s[TREE ? 1 : LIST_ALL];
  __shared__ uint64_t anc_s[TREE ? DRAFT : 1];
  __shared__ float m_s[RO_NW][ROWS], l_s[RO_NW][ROWS], un_s[PRECISE ? NG : 1][ROWS];
  __shared__ __attribute__((aligned(16))) float sums_s[RO_NW * 16 * RO_PITCH];  // the tiles while wavefronts walk
  __shared__ __attribute__((aligned(16))) uint8_t q_s[NG][NB][NP][64 * 16];      // q' as column operands, by lane
  static_assert(sizeof(sums_s) >= RO_NW * NP * CA_TILE, "the tiles lie where the sums do");
  static_assert(sizeof(sums_s) >= LIST_ALL * (sizeof(int32_t) + sizeof(uint16_t)), "and the packed lists before them");
  const PagedAttnArgs& a = p.a;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int64_t item = blockIdx.x / (unsigned)a.c.n_kv;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (a.lse != nullptr && item == 0) lse_constants(a, kv);
  int b, row0 = 0, begin = 0, count, chunk = 0;
  PagedSeq seq;
  int64_t tok0 = 0;  // lists: the unit's first token
  int n_tok = 1;
  uint32_t all = 1u;  // lists: the unit's tokens as bits
  if constexpr (TREE) {
    const RowsPlace at = tree_place(p, ROWS, (int)item, place_s);
    if (at.b < 0) return;
    b = at.b;
    seq = paged_seq(a.c, b);
    row0 = at.unit * ROWS;
    if (at.chunk == 0 && kv == 0 && tid == 0) {  // for the combine
      const int64_t u = plan_at(p, ROWS, seq, b, at.unit);
      p.plan[2 * u] = (int32_t)item;
      p.plan[2 * u + 1] = at.n_chunks;
    }
    const int n_tiles = (int)((seq.len + TILE - 1) / TILE);
    begin = at.chunk * at.tiles;
    count = n_tiles - begin < at.tiles ? n_tiles - begin : at.tiles;
  } else {
    const int64_t u = item / p.n_chunks;
    chunk = (int)(item - u * p.n_chunks);
    b = list_unit(p, u, b_s, tok0);
    if (b < 0) return;
    seq = paged_seq(a.c, b);
    n_tok = (int)(seq.n - tok0 < p.tokens ? seq.n - tok0 : p.tokens);
    auto blocks = [&](int i) {  // that token i of the unit sees
      const int64_t see = seq.len - seq.n + tok0 + i + 1;
      return see > 0 ? (int)((see + TILE - 1) / TILE) : 0;
    };
    const int32_t* list = p.blocks + ((seq.first + tok0) * a.c.n_kv + kv) * p.n_blocks;
    if (p.tokens == 1) {
      const int from = chunk * p.chunk, to = from + p.chunk < p.n_blocks ? from + p.chunk : p.n_blocks;
      count = read_list(list, from, to, blocks(0), sel_s, list_s);
    } else {
      all = (1u << n_tok) - 1;
      const int n = read_lists(list, (int64_t)a.c.n_kv * p.n_blocks, p.n_blocks, n_tok, blocks, reinterpret_cast<int32_t*>(sums_s),
                               reinterpret_cast<uint16_t*>(sums_s + LIST_ALL), sel_s, who_s, union_s);
      int each = (n + p.n_chunks - 1) / p.n_chunks;
      each = (each + RO_NW - 1) / RO_NW * RO_NW;
      begin = chunk * each < n ? chunk * each : n;
      count = n - begin < each ? n - begin : each;
    }
  }
  const int n_rows = TREE ? (int)(seq.n * a.n_qh) - row0 : n_tok * a.n_qh;  // of the unit, and those behind it
  Kept Kk = read_kept(a.bits_k + kv * NG), Kv = read_kept(a.bits_v + kv * NG);
  if (!Kk.ok || Kk.used > a.Wk) Kk.n = 0;  // width table inconsistent with the record
  if (!Kv.ok || Kv.used > a.Wv) Kv.n = 0;
  // the lane's row of block nb: token of the sequence, query head (rows past the last repeat the first)
  auto row_of = [&](int nb, int& tok, int& head) __attribute__((always_inline)) {
    const int r = row0 + (16 * nb + col < n_rows ? 16 * nb + col : 0);
    tok = r / a.n_qh;
    head = r - tok * a.n_qh;
    if (!TREE) tok += (int)tok0;
  };
  if constexpr (TREE) {
    if (wave == 0) anc_s[lane] = ancestors(a.parents, seq.first, (int)seq.n, lane);
  }

  const int tpp = a.c.page_tokens >> 6, n_keys = Kk.n, n_units = Kk.n + Kv.n;
  int unit_v = 0;  // lane u: kept group u of the keys, then of the values: bits, its place, its payload's first word
  {
    const int s = lane < n_keys ? lane : lane - n_keys;
    int bb = 0, pay = 0;
#pragma unroll
    for (int x = 0; x < NG; ++x) {
      bb = x == s ? (lane < n_keys ? Kk.bits[x] : Kv.bits[x]) : bb;
      pay = x == s ? (lane < n_keys ? Kk.pay[x] : Kv.pay[x]) : pay;
    }
    unit_v = bb | (s & 3) << 4 | pay << 6;
  }
  auto tile_of = [&](int x) __attribute__((always_inline)) { return TREE ? begin + x : __builtin_amdgcn_readfirstlane(sel_s[begin + x]); };
  // the tile whose words are loaded: `now` and its records; the one after it: `next`, its page, its place in that
  int load_x = wave, in_page = 0, page = -1, now = 0, next = 0;
  const uint32_t *kp = a.pool_k, *vp = a.pool_v;
  bool page_ok = false;
  uint32_t words[8], meta = 0u;
  auto look_up = [&]() __attribute__((always_inline)) {
    page = -1;
    if (load_x < count) {
      next = tile_of(load_x);
      const int idx = next / tpp;
      in_page = next - idx * tpp;
      page = a.c.table[(int64_t)seq.row * a.c.row_pages + idx];  // (not waited for until it is entered)
    }
  };
  auto enter = [&]() __attribute__((always_inline)) {  // the tile looked up; the walk goes on
    const int at = __builtin_amdgcn_readfirstlane(page);
    page_ok = at >= 0 && at < a.c.n_pages;
    now = next;
    const int64_t rec = ((int64_t)(page_ok ? at : 0) * a.c.n_kv + kv) * tpp + in_page;
    kp = a.pool_k + rec * (TILE * a.Wk) + lane;
    vp = a.pool_v + rec * (TILE * a.Wv) + lane;
    load_x += RO_NW;
    look_up();
  };
  int bits = 0;  // of the group whose words are loaded
  auto fetch = [&](int u) __attribute__((always_inline)) {
    const int d = __builtin_amdgcn_readlane(unit_v, u);
    const uint32_t* rec = u < n_keys ? kp : vp;
    bits = d & 15;
    meta = 0u;
    if (!page_ok) return;
    meta = rec[((d >> 4) & 3) * TILE];
    rec += (d >> 6) * TILE;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < bits) words[i] = rec[i * TILE];
  };
  look_up();
  if (n_units > 0) {
    enter();
    fetch(0);
  }
  // q': element e of quarter p is that of code 4 p + e / 2 + 16 (e % 2), as the tiles' places are; product y has
  // e = (i / 2) * 4 + i % 2 + 2 y, i < 4, so that a lane's codes of both products are neighbours. A wavefront takes
  // a group, or half of the row blocks of one where there are two at most, and cuts its basis into
  // parts once. PRECISE: a row's group is scaled by 2^E into [2^8, 2^9).
  {
    const bool halves = NB > 1 && Kk.n <= 2;
    const int sl = halves ? wave & 1 : wave, nb0 = halves && wave > 1 ? NB / 2 : 0, nb1 = halves && wave < 2 ? NB / 2 : NB;
    if (sl < Kk.n) {
      // KS of the four steps' loads at once (one by one they wait for memory four times), as registers allow
      constexpr int KS = NB == 2 || PRECISE ? 4 : 2;
      f32x4 acc[NB][2];
      u32x4 qr[NB][KS][2];
      f32x2 V[KS][8];
      int64_t qoff[NB];
      const float* v0 = a.basis_k + (int64_t)kv * D * D + (8 * quarter) * D + G * pick4(Kk.grp, sl) + 4 * (col >> 2) + (col & 2) + 16 * (col & 1);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        acc[nb][0] = acc[nb][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        int tok, head;
        row_of(nb, tok, head);
        qoff[nb] = (seq.first + tok) * a.q_token_stride + (kv * a.n_qh + head) * a.q_head_stride + 8 * quarter;
      }
#pragma unroll
      for (int k0 = 0; k0 < 4; k0 += KS) {
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) V[k][e] = *reinterpret_cast<const f32x2*>(v0 + (32 * (k0 + k) + e) * D);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          if (nb < nb0 || nb >= nb1) continue;
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            if (a.q_f32) {
              const u32x4* x = reinterpret_cast<const u32x4*>(reinterpret_cast<const float*>(a.q) + qoff[nb] + 32 * (k0 + k));
              qr[nb][k][0] = x[0];
              qr[nb][k][1] = x[1];
            } else {
              qr[nb][k][0] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + qoff[nb] + 32 * (k0 + k));
            }
          }
        }
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          float v[2][8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[0][e] = V[k][e][0];
            v[1][e] = V[k][e][1];
          }
          bf16x8 vp[2][QP];
          split8_pairs<QP>(v[0], vp[0]);
          split8_pairs<QP>(v[1], vp[1]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            if (nb < nb0 || nb >= nb1) continue;
            bf16x8 qq[QP];
            if (a.q_f32) {
              float qv[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) qv[e] = __uint_as_float(qr[nb][k][e >> 2][e & 3]);
              split8_pairs<QP>(qv, qq);
            } else {
              qq[0] = as_bf16x8(qr[nb][k][0]);
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
              for (int i = 0; i < QP; ++i) acc[nb][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[y][i], qq[0], acc[nb][y], 0, 0, 0);
              if (a.q_f32) {
#pragma unroll
                for (int i = 0; i < QP; ++i)
#pragma unroll
                  for (int j = 1; i + j < QP; ++j) acc[nb][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[y][i], qq[j], acc[nb][y], 0, 0, 0);
              }
            }
          }
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if (nb < nb0 || nb >= nb1) continue;
        float y[8], most = 0.0f, up = 1.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[e] = acc[nb][(e >> 1) & 1][2 * (e >> 2) + (e & 1)] * a.scale_log2;
          most = __builtin_fmaxf(most, __builtin_fabsf(y[e]));
        }
        if constexpr (PRECISE) {
          most = __builtin_fmaxf(most, __shfl_xor(most, 16));
          most = __builtin_fmaxf(most, other_half(most));
          up = __builtin_ldexpf(1.0f, 9 - scale_exponent(most));
          if (quarter == 0) un_s[sl][16 * nb + col] = 1.0f / up;
        }
        u32x4 rh, rl;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f32x2 x = f32x2{y[2 * j] * up, y[2 * j + 1] * up};
          if constexpr (!PRECISE) {  // NaN stays
#pragma unroll
            for (int e = 0; e < 2; ++e) x[e] = x[e] > 65504.0f ? 65504.0f : x[e] < -65504.0f ? -65504.0f : x[e];
          }
          const f16x2 hi = __builtin_convertvector(x, f16x2);
          rh[j] = __builtin_bit_cast(uint32_t, hi);
          rl[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{(x[0] - (float)hi[0]) * CA_LO, (x[1] - (float)hi[1]) * CA_LO}, f16x2));
        }
        *reinterpret_cast<u32x4*>(q_s[sl][nb][0] + 16 * lane) = rh;
        if constexpr (PRECISE) *reinterpret_cast<u32x4*>(q_s[sl][nb][1] + 16 * lane) = rl;
      }
    }
  }
  __syncthreads();  // q', ancestors
  uint8_t* tile = reinterpret_cast<uint8_t*>(sums_s) + wave * NP * CA_TILE;
  uint32_t magic = 0x64006400u;  // exponent of 1024 in both halves, in a VGPR
  asm volatile("" : "+v"(magic));
  // operands in the tile (the swizzle of slot_piece repeats every 8 slots)
  const uint8_t* key_at = tile + slot_piece(col, quarter);
  const uint8_t* val_at0 = tile + slot_piece(4 * quarter + (col >> 2), (lane & 3) >> 1) + 8 * (lane & 1);
  const uint8_t* val_at1 = tile + slot_piece(4 * quarter + (col >> 2), 2 + ((lane & 3) >> 1)) + 8 * (lane & 1);
  // group u's coefficients into the tile (its last readers are done: LDS serves a wavefront in
  // order), and the next group's words
  auto expand = [&](int u) __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const uint32_t m = finite_slot(meta, bits, (float)((1 << bits) - 1));
    with_bits(bits, [&](auto bc) __attribute__((always_inline)) {
      write_slot<decltype(bc)::value, PRECISE>(words, m, tile, lane, CA_TILE, magic);
    });
    if (u + 1 == n_units) enter();
    fetch(u + 1 == n_units ? 0 : u + 1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  // for NV value groups at most: the sums of four are 128 registers at four row blocks and spill, those of the
  // two or three that are kept mostly do not (16 trees of up to 32 tokens over 8k slots: 95 -> 81 us)
  auto walk = [&](auto groups) __attribute__((always_inline)) {
    constexpr int NV = decltype(groups)::value;
    const int64_t past = seq.len - seq.n;  // slots of the history
    const int64_t common = TREE ? past : past + tok0 + 1;  // slots that every row sees, as far as its list goes
    f32x4 acc[NV][2][NB];
    float ref[NB], l[NB];  // the reference less CA_LIFT (-inf: nothing seen yet)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      ref[nb] = -__builtin_inff();
      l[nb] = 0.0f;
#pragma unroll
      for (int sl = 0; sl < NV; ++sl) acc[sl][0][nb] = acc[sl][1][nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll 1
    for (int x = wave; x < count; x += RO_NW) {
      const int64_t t0 = (int64_t)(n_units > 0 ? now : tile_of(x)) * TILE;
      f32x4 S[NB][4];  // slot 16 s + 4 quarter + i
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int s = 0; s < 4; ++s) S[nb][s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
      for (int u = 0; u < n_keys; ++u) {
        expand(u);
        f16x8 qo[NB][NP];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int y = 0; y < NP; ++y) qo[nb][y] = as_f16x8(*reinterpret_cast<const u32x4*>(q_s[u][nb][y] + 16 * lane));
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const f16x8 kh = as_f16x8(*reinterpret_cast<const u32x4*>(key_at + 16 * 64 * s));
          if constexpr (!PRECISE) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) S[nb][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, qo[nb][0], S[nb][s], 0, 0, 0);
          } else {
            const f16x8 kl = as_f16x8(*reinterpret_cast<const u32x4*>(key_at + CA_TILE + 16 * 64 * s));
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const f32x4 z = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
              const f32x4 hi = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, qo[nb][0], z, 0, 0, 0);
              f32x4 lo = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, qo[nb][1], z, 0, 0, 0);
              lo = __builtin_amdgcn_mfma_f32_16x16x32_f16(kl, qo[nb][0], lo, 0, 0, 0);
              const float un = un_s[u][16 * nb + col];
#pragma unroll
              for (int i = 0; i < 4; ++i) S[nb][s][i] = __builtin_fmaf(__builtin_fmaf(lo[i], 1.0f / CA_LO, hi[i]), un, S[nb][s][i]);
            }
          }
        }
      }
      const uint32_t who = TREE || p.tokens == 1 ? all : (uint32_t)__builtin_amdgcn_readfirstlane(who_s[begin + x]);
      if (t0 + TILE > common || who != all) {  // some row does not see the whole tile
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          uint64_t own = 0u;  // of the slots at and behind `common`
          int tok, head;
          row_of(nb, tok, head);
          if constexpr (TREE)
            own = anc_s[tok];
          else
            own = ((uint64_t)1 << (tok - (int)tok0)) - 1;  // a token sees one slot more than the one before it
          uint64_t see = seen_slots(t0, common, own);
          if (!TREE && !(who >> (tok - (int)tok0) & 1u)) see = 0u;
          see >>= 4 * quarter;
          const uint32_t half[2] = {(uint32_t)see, (uint32_t)(see >> 32)};
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[nb][s][i] = half[s >> 1] & (1u << (16 * (s & 1) + i)) ? S[nb][s][i] : -__builtin_inff();
        }
      }
      float top[NB];
      bool moves = false;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        top[nb] = S[nb][0][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top[nb] = __builtin_fmaxf(top[nb], S[nb][i >> 2][i & 3]);
        top[nb] -= CA_LIFT + CA_SLACK;
        moves = moves || top[nb] > ref[nb];
      }
      if (__any(moves)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          top[nb] = __builtin_fmaxf(top[nb], __shfl_xor(top[nb], 16));
          top[nb] = __builtin_fmaxf(top[nb], other_half(top[nb]));
          const float next = top[nb] > ref[nb] ? top[nb] + CA_SLACK : ref[nb];
          const float f = ref[nb] == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(ref[nb] - next);  // 1: the sums are zeros (or NaN)
          ref[nb] = next;
          l[nb] *= f;
#pragma unroll
          for (int sl = 0; sl < NV; ++sl)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[sl][i >> 2][nb][i & 3] *= f;
        }
      }
      f16x8 w[NB][2][NP];  // weights of 32 slots: element e is slot 16 (e / 4) + 4 quarter + e % 4
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float base = ref[nb] == -__builtin_inff() ? 0.0f : ref[nb];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          u32x4 xh, xl;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x4 s = S[nb][2 * hf + (j >> 1)];
            const f32x2 e = f32x2{__builtin_amdgcn_exp2f(s[2 * (j & 1)] - base), __builtin_amdgcn_exp2f(s[2 * (j & 1) + 1] - base)};
            const f16x2 r = __builtin_convertvector(e, f16x2);
            xh[j] = __builtin_bit_cast(uint32_t, r);
            if constexpr (PRECISE) {
              l[nb] += e[0] + e[1];
              xl[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{(e[0] - (float)r[0]) * CA_LO, (e[1] - (float)r[1]) * CA_LO}, f16x2));
            } else {
              l[nb] = __builtin_amdgcn_fdot2(__builtin_bit_cast(h16x2, r), h16x2{(__fp16)1.0f, (__fp16)1.0f}, l[nb], false);
            }
          }
          w[nb][hf][0] = as_f16x8(xh);
          if constexpr (PRECISE) w[nb][hf][1] = as_f16x8(xl);
        }
      }
      // (one place that makes coefficients for all value groups: unrolled, twice the code for the same time)
#pragma unroll 1
      for (int g = 0; g < n_units - n_keys; ++g) {
        expand(n_keys + g);
        auto add = [&](f32x4 (&sum)[2][NB]) __attribute__((always_inline)) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            f32x4 lo[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) lo[nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const uint8_t* pt = (y ? val_at1 : val_at0) + 32 * 64 * hf;
              const u32x2 y0 = read_transposed(pt), y1 = read_transposed(pt + 16 * 64);
              const f16x8 vh = as_f16x8(u32x4{y0[0], y0[1], y1[0], y1[1]});
              f16x8 vl = vh;
              if constexpr (PRECISE) {
                const u32x2 z0 = read_transposed(pt + CA_TILE), z1 = read_transposed(pt + CA_TILE + 16 * 64);
                vl = as_f16x8(u32x4{z0[0], z0[1], z1[0], z1[1]});
              }
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) {
                sum[y][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, w[nb][hf][0], sum[y][nb], 0, 0, 0);
                if constexpr (PRECISE) {
                  lo[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vl, w[nb][hf][0], lo[nb], 0, 0, 0);
                  lo[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, w[nb][hf][NP - 1], lo[nb], 0, 0, 0);
                }
              }
            }
            if constexpr (PRECISE) {
#pragma unroll
              for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[y][nb][i] = __builtin_fmaf(lo[nb][i], 1.0f / CA_LO, sum[y][nb][i]);
            }
          }
        };
#pragma unroll
        for (int sl = 0; sl < NV; ++sl)
          if (sl == g) add(acc[sl]);
      }
    }
    // merge of the wavefronts, and the chunk's partial of every row, 16 rows at a time
    // (lists: [chunk][token][KV head][query head], trees: [item][KV head][row])
    float* part = p.partial + (item * a.c.n_kv + kv) * (int64_t)(ROWS * PART);
    const int64_t token_step = (int64_t)a.c.n_kv * a.n_qh * PART;
    if (!TREE) part = p.partial + ((chunk * a.c.n_new + seq.first + tok0) * a.c.n_kv + kv) * (int64_t)(a.n_qh * PART);
    float m[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float ll = l[nb] + __shfl_xor(l[nb], 16);
      ll += other_half(ll);
      m[nb] = ll == 0.0f ? -__builtin_inff() : ref[nb] == -__builtin_inff() ? 0.0f : ref[nb];
      if (quarter == 0) {
        m_s[wave][16 * nb + col] = m[nb];
        l_s[wave][16 * nb + col] = ll;
      }
    }
    __syncthreads();  // the maxima; the tiles have been read
    auto factor = [&](float mine, float top) __attribute__((always_inline)) { return mine == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(mine - top); };
    auto top_of = [&](int r) __attribute__((always_inline)) {
      float t = m_s[0][r];
#pragma unroll
      for (int v = 1; v < RO_NW; ++v) t = __builtin_fmaxf(t, m_s[v][r]);
      return t;
    };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (16 * nb >= n_rows) break;
      const float f = factor(m[nb], top_of(16 * nb + col));
#pragma unroll
      for (int sl = 0; sl < NV; ++sl)
        if (sl < Kv.n)
#pragma unroll
          for (int y = 0; y < 2; ++y)
            *reinterpret_cast<f32x4*>(sums_s + (wave * 16 + col) * RO_PITCH + G * sl + 16 * y + 4 * quarter) =
                f32x4{acc[sl][y][nb][0] * f, acc[sl][y][nb][1] * f, acc[sl][y][nb][2] * f, acc[sl][y][nb][3] * f};
      __syncthreads();
      const int here = n_rows - 16 * nb < 16 ? n_rows - 16 * nb : 16;
      auto out = [&](int r) __attribute__((always_inline)) {
        const int row = 16 * nb + r, tok = TREE ? 0 : row / a.n_qh;
        return part + tok * token_step + (row - tok * a.n_qh) * PART;
      };
      // sums as they lie: [kept group][place]
      for (int e = tid; e < here * (D / 4); e += RO_NT) {
        const int r = e / (D / 4), x = 4 * (e % (D / 4));
        if (x >= G * Kv.n) continue;
        f32x4 sum = *reinterpret_cast<const f32x4*>(sums_s + r * RO_PITCH + x);
#pragma unroll
        for (int v = 1; v < RO_NW; ++v) {
          const f32x4 y = *reinterpret_cast<const f32x4*>(sums_s + (v * 16 + r) * RO_PITCH + x);
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] += y[i];
        }
        *reinterpret_cast<f32x4*>(out(r) + 8 + x) = sum;
      }
      if (tid < here) {
        const int r = 16 * nb + tid;
        const float top = top_of(r);
        float total = 0.0f;
#pragma unroll
        for (int v = 0; v < RO_NW; ++v) total = __builtin_fmaf(factor(m_s[v][r], top), l_s[v][r], total);
        *reinterpret_cast<f32x2*>(out(tid)) = f32x2{top, total};
      }
      if (nb + 1 < NB) __syncthreads();  // the sums have been read
    }
  };
  if constexpr (NB < 4) {
    walk(std::integral_constant<int, NG>{});
  } else {
    switch (Kv.n) {
      case 4: walk(std::integral_constant<int, 4>{}); break;
      case 3: walk(std::integral_constant<int, 3>{}); break;
      default: walk(std::integral_constant<int, 2>{});
    }
  }
}

// ---------------------------------------------------------------------------
// Join of the chunks, the rotation back, and the outputs, for neighbouring rows (new token x query heads of a
// KV head, of all sequences) of one KV head.
// ---------------------------------------------------------------------------
struct RowParts {
  const float* first;  // the first chunk's
  int64_t step;        // to the next one's
  int n;               // chunks; 0: the row sees nothing
  bool live;
};
// Of row `row` (token x query heads) whose token's sequence is b (-1: none).
template <bool TREE>
__device__ __forceinline__ RowParts row_parts(const PagedRowsArgs& p, int rows, int64_t row, int b, int kv) {
  const PagedAttnArgs& a = p.a;
  RowParts r{p.partial, 0, 0, b >= 0};
  if (!r.live) return r;
  const int64_t tok = row / a.n_qh;
  const int head = (int)(row - tok * a.n_qh);
  if constexpr (TREE) {
    const PagedSeq seq = paged_seq(a.c, b);
    r.live = scanned(a, seq);
    r.step = (int64_t)a.c.n_kv * rows * PART;
    if (!r.live || seq.len <= 0) return r;
    const int64_t in_seq = (tok - seq.first) * a.n_qh + head, unit = in_seq / rows;
    const int64_t u = plan_at(p, rows, seq, b, (int)unit);
    const int item0 = p.plan[2 * u], most = p.plan[2 * u + 1];
    // (within the workspace whatever the lists of sequences hold)
    r.n = item0 < 0 || item0 >= p.items ? 0 : most < p.items - item0 ? most : p.items - item0;
    r.first += ((int64_t)(r.n > 0 ? item0 : 0) * a.c.n_kv + kv) * (rows * PART) + (in_seq - unit * rows) * PART;
  } else {
    r.n = p.n_chunks;
    r.step = a.c.n_new * a.n_q_heads * PART;
    r.first += ((tok * a.c.n_kv + kv) * a.n_qh + head) * PART;
  }
  return r;
}
// The sequences of the tokens t_lo .. t_lo + n - 1 into b_s. Every thread of NT.
template <int NT>
__device__ __forceinline__ void sequences_of(const PagedCache& c, int64_t t_lo, int n, int32_t* b_s) {
  for (int i = threadIdx.x; i < n; i += NT) b_s[i] = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < c.batch; b += NT) {
    const PagedSeq q = paged_seq(c, b);
    const int64_t lo = t_lo < q.first ? q.first : t_lo, hi = t_lo + n < q.first + q.n ? t_lo + n : q.first + q.n;
    for (int64_t t = lo; t < hi; ++t) atomicMax(&b_s[t - t_lo], b);
  }
  __syncthreads();
}

// Few rows: a workgroup each. Eight thread groups of 128 share the row's chunks; then a channel is 8 threads' dot
// product. Bound by latency (the sequence, the plan, the partials, one after the other): 5.8 us for 256 rows.
template <bool TREE>
__global__ __launch_bounds__(1024) void paged_row_combine_kernel(PagedRowsArgs p, int rows) {
  constexpr int SHARE = 8;
  __shared__ int32_t b_s[1];
  __shared__ float m_s[SHARE], l_s[SHARE], sums_s[SHARE][D], lse_s[2];
  __shared__ __attribute__((aligned(16))) float chat_s[D];
  const PagedAttnArgs& a = p.a;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int64_t row = blockIdx.x / (unsigned)a.c.n_kv, tok = row / a.n_qh;
  const int head = (int)(row - tok * a.n_qh);
  const int tid = threadIdx.x, j = tid & 127, share = tid >> 7;
  const int ri = tid >> 3, rpart = tid & 7;
  const f32x4* Vr = reinterpret_cast<const f32x4*>(a.basis_v + (int64_t)kv * D * D + (int64_t)ri * D + 16 * rpart);
  const f32x4 v0 = Vr[0], v1 = Vr[1], v2 = Vr[2], v3 = Vr[3];
  const float mv = a.mean_v[(int64_t)kv * D + j];
  Kept Kv = read_kept(a.bits_v + kv * NG);
  if (!Kv.ok || Kv.used > a.Wv) Kv.n = 0;
  int sl = -1;
#pragma unroll
  for (int x = 0; x < NG; ++x) sl = x < Kv.n && Kv.grp[x] == j >> 5 ? x : sl;
  const int at = sl < 0 ? 0 : 8 + G * sl + 8 * ((j & 15) >> 2) + 2 * (j & 3) + ((j >> 4) & 1);  // (none: m, not used)
  float u = 0.0f;
  if (a.lse != nullptr && share == 0) u = query_at(a, tok * a.q_token_stride + (kv * a.n_qh + head) * a.q_head_stride + j) * a.lse_u[kv * D + j];
  sequences_of<1024>(a.c, tok, 1, b_s);
  const RowParts r = row_parts<TREE>(p, rows, row, b_s[0], kv);
  if (!r.live) return;
  float M = -__builtin_inff(), L = 0.0f, A = 0.0f;
  constexpr int CB = 8;
  for (int c0 = share; c0 < r.n; c0 += CB * SHARE) {
    float m[CB], l[CB], x[CB];
#pragma unroll
    for (int k = 0; k < CB; ++k) {
      const int c = c0 + k * SHARE;
      const float* pc = r.first + (c < r.n ? c : c0) * r.step;
      m[k] = c < r.n ? pc[0] : -__builtin_inff();
      l[k] = pc[1];
      x[k] = pc[at];
    }
    float mb = M;
#pragma unroll
    for (int k = 0; k < CB; ++k) mb = __builtin_fmaxf(mb, m[k]);
    if (mb != -__builtin_inff()) {
      const float f = M == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(M - mb);
      L *= f;
      A *= f;
#pragma unroll
      for (int k = 0; k < CB; ++k) {
        const float w = m[k] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m[k] - mb);
        L = __builtin_fmaf(w, l[k], L);
        A = __builtin_fmaf(w, x[k], A);
      }
      M = mb;
    }
  }
  if (j == 0) {
    m_s[share] = M;
    l_s[share] = L;
  }
  sums_s[share][j] = A;
  if (a.lse != nullptr && share == 0) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) u += __shfl_xor(u, o);
    if ((tid & 63) == 0) lse_s[tid >> 6] = u;
  }
  __syncthreads();
  if (share == 0) {
    M = m_s[0];
#pragma unroll
    for (int k = 1; k < SHARE; ++k) M = __builtin_fmaxf(M, m_s[k]);
    L = A = 0.0f;
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      const float f = m_s[k] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m_s[k] - M);
      L = __builtin_fmaf(f, l_s[k], L);
      A = __builtin_fmaf(f, sums_s[k][j], A);
    }
    const bool seen = L > 0.0f || L != L;
    const float c = (sl >= 0 ? A / L : L != L ? L : 0.0f) + mv;
    chat_s[j] = seen ? c : 0.0f;
    if (a.lse != nullptr && j == 0)
      a.lse[tok * a.n_q_heads + kv * a.n_qh + head] = seen ? __builtin_fmaf(__builtin_amdgcn_logf(L) + M, LN2, lse_s[0] + lse_s[1]) : -__builtin_inff();
  }
  __syncthreads();
  const f32x4* c = reinterpret_cast<const f32x4*>(chat_s + 16 * rpart);
  const f32x4 c0 = c[0], c1 = c[1], c2 = c[2], c3 = c[3];
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = __builtin_fmaf(v0[i], c0[i], s);
    s = __builtin_fmaf(v1[i], c1[i], s);
    s = __builtin_fmaf(v2[i], c2[i], s);
    s = __builtin_fmaf(v3[i], c3[i], s);
  }
  s += __shfl_xor(s, 1);
  s += __shfl_xor(s, 2);
  s += __shfl_xor(s, 4);
  if (rpart == 0) {
    const int64_t o = (tok * a.n_q_heads + kv * a.n_qh + head) * D + ri;
    if (a.out_f32)
      reinterpret_cast<float*>(a.out)[o] = s;
    else
      reinterpret_cast<__bf16*>(a.out)[o] = (__bf16)s;
  }
}

// Many rows: 16 to a workgroup, 16 threads a row; then the rotation as 16 x 16 x 32 products of channels and rows, a
// wavefront 32 channels, both sides in NP bf16 parts. Bound by the same chain, then by the partials' bytes: 7.2 us for 1344
// rows of four chunks, 14 for 8200 rows of up to four chunks, 12 for 6400 fp32 rows of two.
constexpr int CO_ROWS = 16, CO_PITCH = D + 4;
template <bool TREE, int NP>
__global__ __launch_bounds__(256) void paged_rows_combine_kernel(PagedRowsArgs p, int rows) {
  __shared__ int32_t b_s[CO_ROWS + 1];
  __shared__ __attribute__((aligned(16))) float chat_s[CO_ROWS][CO_PITCH];
  const PagedAttnArgs& a = p.a;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int64_t row0 = (int64_t)(blockIdx.x / (unsigned)a.c.n_kv) * CO_ROWS, n_all = a.c.n_new * a.n_qh;
  const int tid = threadIdx.x, r = tid >> 4, part = tid & 15, lane = tid & 63, col = lane & 15, quarter = lane >> 4, wave = tid >> 6;
  // the basis: channel 32 wave + 16 t + col, coefficients 32 k + 8 quarter ..
  f32x4 v[2][4][2];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        v[t][k][i] = *reinterpret_cast<const f32x4*>(a.basis_v + ((int64_t)kv * D + 32 * wave + 16 * t + col) * D + 32 * k + 8 * quarter + 4 * i);
  Kept Kv = read_kept(a.bits_v + kv * NG);
  if (!Kv.ok || Kv.used > a.Wv) Kv.n = 0;
  const int64_t t_lo = row0 / a.n_qh, t_hi = (row0 + CO_ROWS - 1) / a.n_qh;
  sequences_of<256>(a.c, t_lo, (int)(t_hi - t_lo) + 1, b_s);
  const int64_t row = row0 + r, tok = row / a.n_qh;
  const int head = (int)(row - tok * a.n_qh);
  const RowParts parts = row_parts<TREE>(p, rows, row, row < n_all ? b_s[tok - t_lo] : -1, kv);
  float M = -__builtin_inff(), L = 0.0f;
  f32x4 A[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
  constexpr int CB = 4;
  for (int c0 = 0; c0 < parts.n; c0 += CB) {
    f32x2 ml[CB];
    f32x4 x[CB][2];
#pragma unroll
    for (int k = 0; k < CB; ++k) {
      const float* pc = parts.first + (c0 + k < parts.n ? c0 + k : c0) * parts.step;
      ml[k] = *reinterpret_cast<const f32x2*>(pc);
      if (c0 + k >= parts.n) ml[k][0] = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (4 * part + 64 * i < G * Kv.n) x[k][i] = *reinterpret_cast<const f32x4*>(pc + 8 + 4 * part + 64 * i);
    }
    float mb = M;
#pragma unroll
    for (int k = 0; k < CB; ++k) mb = __builtin_fmaxf(mb, ml[k][0]);
    if (mb == -__builtin_inff()) continue;
    const float f = M == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(M - mb);
    L *= f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) A[i][e] *= f;
#pragma unroll
    for (int k = 0; k < CB; ++k) {
      const float w = ml[k][0] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(ml[k][0] - mb);
      L = __builtin_fmaf(w, ml[k][1], L);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) A[i][e] = __builtin_fmaf(w, x[k][i][e], A[i][e]);
    }
    M = mb;
  }
  const bool seen = L > 0.0f || L != L;
  // coefficients: the means, then what the kept groups have on top (a row of a wavefront alone: its own order)
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = part + 16 * (4 * i + e);
      chat_s[r][j] = !seen ? 0.0f : L != L ? L : a.mean_v[(int64_t)kv * D + j];
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (seen) {
    const float inv = 1.0f / L;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int x = 4 * part + 64 * i, sl = x >> 5, place = x & 31;
      if (sl < Kv.n) {
        float* c = &chat_s[r][G * pick4(Kv.grp, sl) + 4 * (place >> 3) + ((place & 7) >> 1)];
        c[0] = __builtin_fmaf(A[i][0], inv, c[0]);
        c[16] = __builtin_fmaf(A[i][1], inv, c[16]);
        c[1] = __builtin_fmaf(A[i][2], inv, c[1]);
        c[17] = __builtin_fmaf(A[i][3], inv, c[17]);
      }
    }
  }
  if (a.lse != nullptr) {
    float u = 0.0f;
    if (parts.live) {
      const int64_t qo = tok * a.q_token_stride + (kv * a.n_qh + head) * a.q_head_stride;
#pragma unroll
      for (int e = 0; e < 8; ++e) u = __builtin_fmaf(query_at(a, qo + part + 16 * e), a.lse_u[kv * D + part + 16 * e], u);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) u += __shfl_xor(u, o);
    if (parts.live && part == 0)
      a.lse[tok * a.n_q_heads + kv * a.n_qh + head] = seen ? __builtin_fmaf(__builtin_amdgcn_logf(L) + M, LN2, u) : -__builtin_inff();
  }
  __syncthreads();
  f32x4 out[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f32x4 c0 = *reinterpret_cast<const f32x4*>(&chat_s[col][32 * k + 8 * quarter]), c1 = *reinterpret_cast<const f32x4*>(&chat_s[col][32 * k + 8 * quarter + 4]);
    const float cf[8] = {c0[0], c0[1], c0[2], c0[3], c1[0], c1[1], c1[2], c1[3]};
    bf16x8 cp[NP];
    split8_pairs<NP>(cf, cp);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const f32x4 x = v[t][k][0], y = v[t][k][1];
      const float vf[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      bf16x8 vp[NP];
      split8_pairs<NP>(vf, vp);
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; i + j < NP; ++j) out[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[i], cp[j], out[t], 0, 0, 0);
    }
  }
  // lane: row `col`, channels 32 wave + 16 t + 4 quarter ..
  const int64_t w = row0 + col, t = w / a.n_qh;
  if (w >= n_all) return;
  const int wb = b_s[t - t_lo];
  if (wb < 0 || (TREE && !scanned(a, paged_seq(a.c, wb)))) return;
  const int64_t o = (t * a.n_q_heads + kv * a.n_qh + (w - t * a.n_qh)) * D + 32 * wave + 4 * quarter;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (a.out_f32) {
      *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + o + 16 * i) = out[i];
    } else {
      const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{out[i][0], out[i][1]}, bf16x2));
      const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{out[i][2], out[i][3]}, bf16x2));
      *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(a.out) + o + 16 * i) = u32x2{lo, hi};
    }
  }
}

}  // namespace spectra_dev

namespace spectra {
using namespace spectra_dev;

namespace {

template <int NB, bool PRECISE, bool TREE>
void launch_rows(const PagedRowsArgs& p, dim3 grid, hipStream_t st) {
  hipLaunchKernelGGL((paged_rows_kernel<NB, PRECISE, TREE>), grid, dim3(RO_NT), 0, st, p);
}

template <bool TREE>
hipError_t launch_combine(const PagedRowsArgs& p, int rows, hipStream_t st) {
  const int64_t all = p.a.c.n_new * p.a.n_qh, n_kv = p.a.c.n_kv;
  const dim3 grid((unsigned)(ceil_div(all, CO_ROWS) * n_kv));
  // a row a CU (8 tokens of 32 heads over 4k slots 21 us in all, and 24 by sixteen rows; 16 tokens 31 and 29)
  if (all * n_kv <= N_CU)
    hipLaunchKernelGGL((paged_row_combine_kernel<TREE>), dim3((unsigned)(all * n_kv)), dim3(1024), 0, st, p, rows);
  else if (p.a.out_f32)
    hipLaunchKernelGGL((paged_rows_combine_kernel<TREE, 3>), grid, dim3(256), 0, st, p, rows);
  else
    hipLaunchKernelGGL((paged_rows_combine_kernel<TREE, 2>), grid, dim3(256), 0, st, p, rows);
  return hipGetLastError();
}

}  // namespace

static_assert(PART * sizeof(float) == SCAN_PART_BYTES, "workspace of a row");

size_t paged_tree_bytes(int32_t batch, int64_t n_new, int32_t n_q_heads, int32_t n_kv, int32_t max_new, int64_t max_tokens) {
  return tree_workspace_bytes(batch, n_new, n_q_heads / n_kv, n_kv, max_new, max_tokens);
}

hipError_t launch_paged_tree(const PagedRowsArgs& args, void* workspace, hipStream_t st) {
  PagedRowsArgs p = args;
  const int32_t n_kv = p.a.c.n_kv;
  const TreePlan plan = tree_plan(p.a.c.batch, p.a.c.n_new, p.a.n_qh, n_kv, p.a.max_new, p.a.max_tokens, p.a.out_f32);
  char* ws = static_cast<char*>(workspace);
  p.a.lse_u = reinterpret_cast<float*>(ws);
  p.plan = reinterpret_cast<int32_t*>(ws + plan.plan_at);
  p.partial = reinterpret_cast<float*>(ws + plan.rows_at);
  p.a.scan_tokens = plan.scan_tokens;
  if (plan.units > 0) {
    p.a.part_slots = plan.split.slots;
    p.a.parts = plan.split.parts;
    p.a.partial = reinterpret_cast<float*>(ws + plan.part_at);
    if (p.a.lse != nullptr) launch_paged_lse(p.a, st);
    const hipError_t e = launch_paged_tree_chunks(p.a, plan.units, st);
    if (e != hipSuccess || p.a.scan_tokens == 0) return e;
  }
  const int nb = plan.nb;
  p.want = plan.want;
  p.items = plan.items;
  const dim3 grid((unsigned)((int64_t)p.items * n_kv));
  if (p.a.out_f32) {
    if (nb == 1)
      launch_rows<1, true, true>(p, grid, st);
    else
      launch_rows<2, true, true>(p, grid, st);
  } else {
    if (nb == 1)
      launch_rows<1, false, true>(p, grid, st);
    else if (nb == 2)
      launch_rows<2, false, true>(p, grid, st);
    else
      launch_rows<4, false, true>(p, grid, st);
  }
  return launch_combine<true>(p, 16 * nb, st);
}

// New tokens of a unit: as many as its rows hold, where sequences have 1.25 on average, their lists fit and single
// tokens have a workgroup for each CU (lists of 32 blocks over 60k slots, 8 KV heads: 8 tokens 25 us together and 20 single,
// 24 tokens 30 both, 64 tokens 39 and 47, 200 tokens 57 and 110; 64 blocks, 48 sequences of one or two tokens 79 and 105).
static int32_t list_tokens(int32_t batch, int64_t n_new, int32_t n_qh, int32_t n_kv, int32_t n_blocks) {
  int32_t t = 16 / n_qh;
  if (t > LIST_ALL / n_blocks) t = LIST_ALL / n_blocks;
  return 4 * n_new >= 5 * (int64_t)batch && n_new * n_kv >= N_CU && n_blocks <= LIST_CHUNK && t > 1 ? t : 1;
}

size_t paged_sparse_bytes(int64_t n_new, int32_t n_q_heads, int32_t n_kv, int32_t n_blocks) {
  // chunks of all rows: what the card's workgroups hold, and each row's own (more where chunks are full)
  const int64_t rows = N_CU * ROWS_PER_CU * 16 + n_new * n_q_heads * (1 + ceil_div(n_blocks, LIST_CHUNK));
  return paged_round((size_t)n_kv * D * sizeof(float)) + (size_t)rows * PART * sizeof(float);
}

hipError_t launch_paged_sparse(const PagedRowsArgs& args, void* workspace, hipStream_t st) {
  PagedRowsArgs p = args;
  const int32_t n_kv = p.a.c.n_kv;
  char* ws = static_cast<char*>(workspace);
  p.a.lse_u = reinterpret_cast<float*>(ws);
  p.partial = reinterpret_cast<float*>(ws + paged_round((size_t)n_kv * D * sizeof(float)));
  p.tokens = list_tokens(p.a.c.batch, p.a.c.n_new, p.a.n_qh, n_kv, p.n_blocks);
  // about as many workgroups as the card holds, of four entries at least
  const int64_t units = p.tokens == 1 ? p.a.c.n_new : p.a.c.n_new / p.tokens + p.a.c.batch;
  const int64_t real = std::max(ceil_div(p.a.c.n_new, p.tokens), std::min<int64_t>(p.a.c.batch, p.a.c.n_new)) * n_kv;
  int64_t n = N_CU * ROWS_PER_CU / real;
  if (n < 1) n = 1;
  int64_t each = ceil_div(ceil_div(p.n_blocks, n), RO_NW) * RO_NW;
  if (p.tokens == 1 && each > LIST_CHUNK) each = LIST_CHUNK;
  p.chunk = (int32_t)each;
  p.n_chunks = (int32_t)ceil_div(p.n_blocks, p.chunk);
  const dim3 grid((unsigned)(units * p.n_chunks * n_kv));
  if (p.a.out_f32)
    launch_rows<1, true, false>(p, grid, st);
  else
    launch_rows<1, false, false>(p, grid, st);
  return launch_combine<false>(p, p.a.n_qh, st);
}

}  // namespace spectra
