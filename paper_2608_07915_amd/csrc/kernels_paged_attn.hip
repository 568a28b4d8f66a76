// Attention of new tokens over the pages of a packed cache, in the latent space (App. E).
//
//   row (i, h) of a sequence: new token i of n, query head h; it sees slots t <= L - n + i
//   q'  = scale * log2(e) * q V_K
//   S   = q' . c_hat_K(t)                     (the constant q' . m_K cancels in the softmax)
//   p   = exp2(S - m), l = sum p, a = sum p c_hat_V(t)   in one pass, m the running maximum
//   out = (a / l + m_V) V_V^T
//
// A workgroup takes 256 rows of one KV head (new tokens x query heads on it), a wavefront 32.
// Products are transposed, slots or coefficients as MFMA rows and the query rows as columns, so
// a lane keeps one query row from q to the output and every product's result registers are the
// next product's column operand as they stand: nothing of q', p or a passes through LDS, and
// the softmax needs one exchange between the halves of a wavefront. Which K index of a product
// stands for which coefficient or slot is free as long as both operands agree.
//
// Records are turned into fp16 coefficients once per workgroup: a lane holds one slot's words of
// a kept group, makes z + s code by packed fp16 multiply-adds (z, s and code are exact in fp16,
// so this rounds once) and writes the 32 values as four 16-byte pieces into LDS. Keys and values
// have one layout, [group][slot][32 places], pieces XOR-swizzled by the slot so that 16-byte
// reads of 16 neighbouring slots fall on distinct banks; values are read transposed
// (ds_read_b64_tr_b16: four slots of a coefficient per lane).
//
// With 16-bit outputs the operands are single fp16 numbers (p between 2^-26 and 8 of the
// running maximum in the normal range). A coefficient's rounding is at most 2^(b-11) of the step of
// its b-bit code where the codes' range holds 0, against half a step of the codec's own, and makes
// most of the error: a score is off by up to 2^-10 sum_j |q'_j c_j|. Two parts of q' alone would leave
// the larger half of that; of the keys too they would take three products for one in the scores.
// With fp32 outputs q', p and the coefficients are two fp16 parts each and a product is three
// (relative error about 2^-21).
#include "attn_common.hpp"
#include "code_operands.hpp"
#include "encode_dev.hpp"
#include "kernels.hpp"
#include "paged_coef.hpp"
#include "paged_dev.hpp"
#include "splits.hpp"

namespace spectra_dev {

constexpr int CA_NW = 8;               // wavefronts of a workgroup
constexpr int CA_ROWS = 32 * CA_NW;    // query rows of a workgroup

// Which sequence a unit of CA_ROWS rows belongs to: sequence b has ceil(n_b n_qh / CA_ROWS) of
// them, but none where the scan takes it or it is past the call's bounds. The same in every
// thread of a workgroup of NW wavefronts; false when there is none. s: LDS.
struct FindScratch {
  int64_t part[CA_NW];
  int64_t total;
  int32_t b, tile;
};
template <int NW>
__device__ __forceinline__ bool find_unit(const PagedAttnArgs& a, int64_t unit, FindScratch& s, int& b, int64_t& tile) {
  const PagedCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) s.b = -1;
  int64_t base = 0;
  for (int b0 = 0; b0 < c.batch; b0 += 64 * NW) {
    int64_t mine = 0;
    if (b0 + tid < c.batch) {
      const PagedSeq q = paged_seq(c, b0 + tid);
      if (attended(a, q) && !scanned(a, q)) mine = (q.n * a.n_qh + CA_ROWS - 1) / CA_ROWS;
    }
    int64_t v = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t u = __shfl_up(v, o);
      if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 63) s.part[wave] = v;
    __syncthreads();
    int64_t before = base;
    for (int w = 0; w < wave; ++w) before += s.part[w];
    const int64_t lo = before + v - mine;
    if (unit >= lo && unit < lo + mine) {
      s.b = b0 + tid;
      s.tile = (int32_t)(unit - lo);
    }
    if (tid == 64 * NW - 1) s.total = before + v;
    __syncthreads();
    if (s.b >= 0) break;
    base = s.total;
  }
  b = __builtin_amdgcn_readfirstlane(s.b);
  tile = __builtin_amdgcn_readfirstlane(s.tile);
  return b >= 0;
}

// Row block `block` of a unit: 32 rows, row = new token x query heads on the KV head + query head.
// Rows past the sequence's last repeat that one and are not stored.
struct Rows {
  int tok, head;  // of the lane's row
  bool live;
  int lim;        // slots that it sees
  int lim_first, lim_last, lim_unit;  // that the block's first row sees, its last, the unit's last
  int past;       // trees: slots of the history, which every row sees (lim_first; the others: all slots), and of
  uint64_t own;   // the slots behind it those that the row sees
};
template <bool TREE>
__device__ __forceinline__ Rows rows_of(const PagedAttnArgs& a, const PagedSeq& seq, int64_t tile, int block, int col) {
  const int n_rows = (int)(seq.n * a.n_qh), past = (int)(seq.len - seq.n) + 1;  // slots that token 0 sees
  const int row0 = (int)tile * CA_ROWS + 32 * block, row = row0 + col;
  auto limit = [&](int r) {
    if constexpr (TREE) return (int)seq.len;
    const int l = past + (r < n_rows ? r : n_rows - 1) / a.n_qh;
    return l < 0 ? 0 : l;
  };
  Rows x;
  x.live = row < n_rows;
  const int rc = x.live ? row : n_rows - 1;
  x.tok = rc / a.n_qh;
  x.head = rc - x.tok * a.n_qh;
  x.lim = TREE ? (int)seq.len : past + x.tok < 0 ? 0 : past + x.tok;
  x.past = past - 1;
  x.own = 0u;
  x.lim_first = __builtin_amdgcn_readfirstlane(limit(row0));
  x.lim_last = __builtin_amdgcn_readfirstlane(limit(row0 + 31));
  x.lim_unit = __builtin_amdgcn_readfirstlane(limit((int)tile * CA_ROWS + CA_ROWS - 1));
  if constexpr (TREE) {
    x.own = __shfl(ancestors(a.parents, seq.first, (int)seq.n, threadIdx.x & 63), x.tok);
    x.lim_first = x.past < 0 ? 0 : x.past;
  }
  return x;
}

// Parts that a unit seeing lim slots has, and where a row block's results of one lie: 16 floats
// per value group and lane, then m and l.
__device__ __forceinline__ int parts_of(const PagedAttnArgs& a, int lim) { return (int)((lim + a.part_slots - 1) / a.part_slots); }
__device__ __forceinline__ int64_t part_at(const PagedAttnArgs& a, int64_t unit, int kv, int part, int block) {
  return (((unit * a.c.n_kv + kv) * a.parts + part) * CA_NW + block) * ((16 * NG + 2) * 64);
}

// out = (a / l + m_V) V_V^T of a wavefront's 32 rows, the coefficients as column operand, and
// both sides in NP bf16 parts; stores the rows and their log-sum-exp. m, l: of the lane's row. NC of the four blocks of
// 32 channels, from cb0 on.
template <int NP, int N, int NC = 4>
__device__ __forceinline__ void finish_rows(const PagedAttnArgs& a, const PagedSeq& seq, const Rows& r, int kv, const Kept& Kv,
                                            const f32x16 (&acc)[N], float m, float l, int lane, int cb0 = 0) {
  const int h = lane >> 5, col = lane & 31;
  const bool seen = l > 0.0f || !(l == l);
  const float inv = 1.0f / l;
  const float* Vv = a.basis_v + (int64_t)kv * D * D;
  f32x16 out[NC];
#pragma unroll
  for (int cb = 0; cb < NC; ++cb) out[cb] = zero16();
  const int i0 = 4 * (col >> 3) + (col & 3), h0 = (col >> 2) & 1;
  const int chan = 16 * h0 + i0;  // MFMA row col of a 32-channel block: then a lane half has 16 neighbouring channels
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    int sl = -1;
#pragma unroll
    for (int x = 0; x < N; ++x) sl = (x < Kv.n && Kv.grp[x] == g) ? x : sl;
    f32x16 av = zero16();
#pragma unroll
    for (int x = 0; x < N; ++x)
      if (x == sl) av = acc[x];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float cf[8];
      int at[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int place = 16 * s + 8 * (e >> 2) + 4 * h + (e & 3);  // of register 8 s + e
        at[e] = G * g + 4 * (place >> 3) + ((place & 7) >> 1) + 16 * (place & 1);
        cf[e] = (sl >= 0 ? av[8 * s + e] * inv : 0.0f) + a.mean_v[kv * D + at[e]];
      }
      bf16x8 cp[NP];
      split8<NP>(cf, cp);
#pragma unroll
      for (int cb = 0; cb < NC; ++cb) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = Vv[(32 * (cb0 + cb) + chan) * D + at[e]];
        bf16x8 vp[NP];
        split8<NP>(v, vp);
#pragma unroll
        for (int x = 0; x < NP; ++x)
#pragma unroll
          for (int y = 0; x + y < NP; ++y)
            out[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vp[x], cp[y], out[cb], 0, 0, 0);
      }
    }
  }
  if (!r.live) return;
  const int64_t o = ((seq.first + r.tok) * a.n_q_heads + kv * a.n_qh + r.head) * D + 32 * cb0 + 16 * h;
#pragma unroll
  for (int cb = 0; cb < NC; ++cb) {
    if (a.out_f32) {
      float* op = reinterpret_cast<float*>(a.out) + o + 32 * cb;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(op + 4 * i) = seen ? f32x4{out[cb][4 * i], out[cb][4 * i + 1], out[cb][4 * i + 2], out[cb][4 * i + 3]}
                                                     : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    } else {
      uint32_t* op = reinterpret_cast<uint32_t*>(reinterpret_cast<uint16_t*>(a.out) + o + 32 * cb);
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        w[i] = seen ? __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{out[cb][2 * i], out[cb][2 * i + 1]}, bf16x2)) : 0u;
      *reinterpret_cast<u32x4*>(op) = u32x4{w[0], w[1], w[2], w[3]};
      *reinterpret_cast<u32x4*>(op + 4) = u32x4{w[4], w[5], w[6], w[7]};
    }
  }
  if (a.lse != nullptr && h == 0 && cb0 == 0) {
    const int64_t qo = (seq.first + r.tok) * a.q_token_stride + (kv * a.n_qh + r.head) * a.q_head_stride;
    float s = 0.0f;
    for (int c = 0; c < D; ++c) s = __builtin_fmaf(query_at(a, qo + c), a.lse_u[kv * D + c], s);
    a.lse[(seq.first + r.tok) * a.n_q_heads + kv * a.n_qh + r.head] =
        seen ? __builtin_fmaf(__builtin_amdgcn_logf(l) + m, LN2, s) : -__builtin_inff();
  }
}

// ---------------------------------------------------------------------------
// A workgroup's group tiles: 64 slots of a kept group each, KT slot tiles of NK key and NV value
// groups a step, shared out over the wavefronts. A lane has one slot's words in registers, loaded
// a step before they are written to LDS, its page read another step ahead. Key tiles begin KOFF
// slots later than value tiles (see chunk_steps).
// ---------------------------------------------------------------------------
template <int NK, int NV, int KT, int KOFF>
struct GroupTiles {
  static constexpr int NS = NK + NV, N = KT * NS, UNITS = (N + CA_NW - 1) / CA_NW;
  uint32_t words[UNITS][8], meta[UNITS];
  int page[UNITS], in_page[UNITS];  // of the slot to load next: its page, and its record's place in it
  int idx[UNITS], off[UNITS];       // of the slot to look up next: page index and slot in the page
  int bits[UNITS], pay[UNITS], slot[UNITS], first[UNITS];  // uniform; 0 bits: no such group, zeros
  bool val[UNITS];
  int64_t page_words[2];
  const uint32_t* base[2];

  __device__ __forceinline__ void init(const PagedAttnArgs& a, int kv, const Kept& Kk, const Kept& Kv, int wave) {
    base[0] = a.pool_k + (int64_t)kv * a.c.page_tokens * a.Wk;
    base[1] = a.pool_v + (int64_t)kv * a.c.page_tokens * a.Wv;
    page_words[0] = (int64_t)a.c.n_kv * a.c.page_tokens * a.Wk;
    page_words[1] = (int64_t)a.c.n_kv * a.c.page_tokens * a.Wv;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int x = wave + CA_NW * u, si = x % NS;
      val[u] = si >= NK;
      slot[u] = val[u] ? si - NK : si;
      first[u] = x / NS * TILE + (val[u] ? 0 : KOFF);
      bits[u] = val[u] ? pick4(Kv.bits, slot[u]) : pick4(Kk.bits, slot[u]);
      pay[u] = val[u] ? pick4(Kv.pay, slot[u]) : pick4(Kk.pay, slot[u]);
      if (x >= N || slot[u] >= (val[u] ? Kv.n : Kk.n)) bits[u] = 0;
      page[u] = -1;
      in_page[u] = 0;
    }
  }
  // The pages of the step whose slots begin at t0 (any t0, by division: where a walk begins).
  __device__ __forceinline__ void look_up_at(const PagedAttnArgs& a, int row, int t0, int from, int to, int lane) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int t = t0 + first[u] + lane;
      idx[u] = (t < 0 ? 0 : t) / a.c.page_tokens;
      off[u] = t - idx[u] * a.c.page_tokens;
    }
    look_up(a, row, t0, from, to, lane);
  }
  // The same, and the walk goes on by a step.
  __device__ __forceinline__ void look_up(const PagedAttnArgs& a, int row, int t0, int from, int to, int lane) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int t = t0 + first[u] + lane;
      page[u] = -1;
      if (bits[u] != 0 && t >= from && t < to) page[u] = a.c.table[(int64_t)row * a.c.row_pages + idx[u]];
      in_page[u] = (off[u] & -TILE) * (val[u] ? a.Wv : a.Wk) + (off[u] & (TILE - 1));
      off[u] += KT * TILE;
#pragma unroll
      for (int i = 0; i < KT; ++i) {  // a page has at least one tile
        const bool next = off[u] >= a.c.page_tokens;
        off[u] -= next ? a.c.page_tokens : 0;
        idx[u] += next ? 1 : 0;
      }
    }
  }
  // The words of the step looked up last; slots without a page of the pool: zeros (metadata 0).
  __device__ __forceinline__ void load(const PagedAttnArgs& a) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      meta[u] = 0u;
      if (page[u] < 0 || page[u] >= a.c.n_pages) continue;
      const uint32_t* rec = (val[u] ? base[1] : base[0]) + (int64_t)page[u] * (val[u] ? page_words[1] : page_words[0]) + in_page[u];
      meta[u] = rec[slot[u] * TILE];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < bits[u]) words[u][i] = rec[(pay[u] + i) * TILE];
    }
  }
  // The loaded step's coefficients into the buffer `buf` (low parts: lo bytes further).
  template <bool PRECISE>
  __device__ __forceinline__ void write(uint8_t* buf, int lo, int wave, int lane, uint32_t magic) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      if (wave + CA_NW * u >= N) continue;
      uint8_t* tile = buf + (wave + CA_NW * u) * CA_TILE;
      if (bits[u] == 0) {
        const u32x4 z = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int k = 0; k < (PRECISE ? 8 : 4); ++k) *reinterpret_cast<u32x4*>(tile + (k >> 2) * lo + piece_at(lane, k & 3)) = z;
      }
      const uint32_t m = finite_meta(meta[u], bits[u]);
      with_bits(bits[u], [&](auto bc) __attribute__((always_inline)) { write_coefficients<decltype(bc)::value, PRECISE>(words[u], m, tile, lane, lo, magic); });
    }
  }
};

// The slots [from, to) of a pass over a workgroup's rows; lim: the slots that the lane's row sees, and
// lim_first the wavefront's first row, none past `to`; lim_last: those of its last row.
struct Pass {
  int row;  // of the table
  int from, to, lim_first, lim_last;
  int past;      // trees: as in Rows
  uint64_t own;
};
// Trees: which of the 32 slots from t0 on the lane's row sees, no slot past the pass's last.
__device__ __forceinline__ uint32_t seen_block(const Pass& pass, int t0) {
  const uint32_t see = (uint32_t)seen_slots(t0, pass.past, pass.own);
  const int n = pass.to - t0;
  return n >= 32 ? see : n <= 0 ? 0u : see & ((1u << n) - 1);
}

// A lane's row in a row block: the result of a pass.
struct RowSum {
  float m, l;  // reference of the weights (log2; -inf: none), their sum over the lane's slots
};

__device__ __forceinline__ float max16(const f32x16& S) {
  float top = __builtin_fmaxf(S[0], S[1]);
#pragma unroll
  for (int i = 2; i < 16; ++i) top = __builtin_fmaxf(top, S[i]);
  return top;
}

// Value operand of 32 slots (block k of a slot tile), transposed: K element 8 h + e of product s is
// slot 16 s + 8 (e / 4) + 4 h + e % 4, as the weights' registers have them.
__device__ __forceinline__ f16x8 value_operand(const uint8_t* tile, int k, int s, int lane) {
  const int piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), t = 32 * k + 16 * s + 4 * (lane >> 5) + ((lane & 15) >> 2);
  const uint8_t* p = tile + 8 * (lane & 1);
  const u32x2 x0 = read_transposed(p + piece_at(t, piece)), x1 = read_transposed(p + piece_at(t + 8, piece));
  return as_f16x8(u32x4{x0[0], x0[1], x1[0], x1[1]});
}
__device__ __forceinline__ f16x8 key_operand(const uint8_t* tile, int k, int s, int h, int col) {
  return as_f16x8(*reinterpret_cast<const u32x4*>(tile + piece_at(32 * k + col, 2 * s + h)));
}

// ---------------------------------------------------------------------------
// 16-bit outputs. A wavefront has 32 rows and goes 32 slots at a time; all counts are compile-time,
// so a block is straight-line code (with the groups counted at run time a 4096-token chunk over 32k
// slots took 2.7 ms). Weights are exp2(S - ref); the reference moves only when a score passes it by
// CA_SLACK, in all rows at once, which after the first block is rare.
// The score products of the next block run among the exponentials and value products of this one;
// as keys are then wanted a block earlier than values, key tiles begin 32 slots later.
// Two buffers of tiles, one barrier a step of two slot tiles. Two wavefronts on a SIMD: three or
// four of them without the lead, so with fewer registers, came to the same rate a row.
// Bound by the vector unit and the matrix cores together: per 32 rows and 32 slots, 16 exponentials,
// 16 differences, 8 maxima, 8 conversions and 8 sums, and 8 to 16 matrix instructions; making the
// coefficients takes a fifth of the time (4096 rows of four heads a KV head over 32k slots, two
// groups: 1.47 ms, 1.17 without it).
// ---------------------------------------------------------------------------
template <int NK, int NV, bool TREE>
__device__ __forceinline__ void chunk_steps(const PagedAttnArgs& a, int kv, const Kept& Kk, const Kept& Kv, const Pass& pass, int lim,
                                            uint8_t* tiles, int wave, int lane, const f16x8 (&qb)[NK][2], f32x16 (&acc)[NV],
                                            RowSum& sum) {
  constexpr int KT = 2, NS = NK + NV, BUF = KT * NS * CA_TILE, STEP = KT * TILE;
  const int h = lane >> 5, col = lane & 31;
  uint32_t magic = 0x64006400u;  // exponent of 1024 in both halves, in a VGPR
  asm volatile("" : "+v"(magic));
  float ref = 0.0f, l = 0.0f;  // the reference less CA_LIFT
  const int n_steps = (pass.to - pass.from + STEP - 1) / STEP;
  auto scores = [&](const uint8_t* tile, int k) {
    f16x8 ko[NK][2];
#pragma unroll
    for (int sl = 0; sl < NK; ++sl)
#pragma unroll
      for (int s = 0; s < 2; ++s) ko[sl][s] = key_operand(tile + sl * CA_TILE, k, s, h, col);
    f32x16 S = zero16();
#pragma unroll
    for (int sl = 0; sl < NK; ++sl)
#pragma unroll
      for (int s = 0; s < 2; ++s) S = mfma_f16(ko[sl][s], qb[sl][s], S);
    return S;
  };
  // The scores of the block at slot t0 are there: what a row does not see weighs nothing; the
  // reference moves.
  auto settle = [&](f32x16& S, int t0, bool begin) {
    if (TREE && t0 + 32 > pass.lim_first) {
      uint32_t see = seen_block(pass, t0) >> (4 * h);
      asm volatile("" : "+v"(see));  // a branch, as below
#pragma unroll
      for (int i = 0; i < 16; ++i) S[i] = see >> (8 * (i >> 2) + (i & 3)) & 1u ? S[i] : -__builtin_inff();
    } else if (!TREE && t0 + 32 > pass.lim_first) {
      int left = lim - t0 - 4 * h;
      asm volatile("" : "+v"(left));  // a branch: as selects this took two instructions a score in every block
#pragma unroll
      for (int i = 0; i < 16; ++i) S[i] = 8 * (i >> 2) + (i & 3) < left ? S[i] : -__builtin_inff();
    }
    float top = max16(S) - (CA_LIFT + CA_SLACK);
    if (begin) {  // the row's largest score so far (none: left at 0)
      top = __builtin_fmaxf(top, other_half(top));
      // (a row of a tree may see later slots yet: far below all scores)
      ref = top == -__builtin_inff() ? (TREE ? -1e30f : 0.0f) : top + CA_SLACK;
    } else if (__any(top > ref)) {
      top = __builtin_fmaxf(top, other_half(top));
      const float d = top > ref ? top + CA_SLACK - ref : 0.0f, f = __builtin_amdgcn_exp2f(-d);
      l *= f;
      ref = TREE ? (top > ref ? top + CA_SLACK : ref) : ref + d;
#pragma unroll
      for (int sl = 0; sl < NV; ++sl)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[sl][i] *= f;
    }
  };
  auto values = [&](const f16x8 (&vo)[NV][2], const f32x16& S) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 w;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const f32x2 e = f32x2{__builtin_amdgcn_exp2f(S[8 * s + 2 * x] - ref), __builtin_amdgcn_exp2f(S[8 * s + 2 * x + 1] - ref)};
        const f16x2 r = __builtin_convertvector(e, f16x2);
        w[x] = __builtin_bit_cast(uint32_t, r);
        // the sum of the rounded weights, two a time
        l = __builtin_amdgcn_fdot2(__builtin_bit_cast(h16x2, r), h16x2{(__fp16)1.0f, (__fp16)1.0f}, l, false);
      }
#pragma unroll
      for (int sl = 0; sl < NV; ++sl) acc[sl] = mfma_f16(vo[sl][s], as_f16x8(w), acc[sl]);
    }
  };
  if (n_steps > 0) {
    GroupTiles<NK, NV, KT, 32> g;
    g.init(a, kv, Kk, Kv, wave);
    // step -1 holds the first 32 keys, in the last half of its last key tile
    g.look_up_at(a, pass.row, pass.from - STEP, pass.from, pass.to, lane);
    g.load(a);
    g.template write<false>(tiles + BUF, 0, wave, lane, magic);
    g.look_up_at(a, pass.row, pass.from, pass.from, pass.to, lane);
    g.load(a);
    g.look_up(a, pass.row, pass.from + STEP, pass.from, pass.to, lane);
    g.template write<false>(tiles, 0, wave, lane, magic);
    g.load(a);
    g.look_up(a, pass.row, pass.from + 2 * STEP, pass.from, pass.to, lane);
    __syncthreads();
    f32x16 S[2];
    S[0] = scores(tiles + BUF + (KT - 1) * NS * CA_TILE, 1);
    settle(S[0], pass.from, true);
    __syncthreads();
#pragma unroll 1
    for (int j = 0; j < n_steps; ++j) {
      const int t0 = pass.from + j * STEP;
      if (j + 1 < n_steps) {
        g.template write<false>(tiles + ((j + 1) & 1) * BUF, 0, wave, lane, magic);
        g.load(a);
        g.look_up(a, pass.row, t0 + 3 * STEP, pass.from, pass.to, lane);
      }
      if (t0 < pass.lim_last) {
        const uint8_t* buf = tiles + (j & 1) * BUF;
#pragma unroll
        for (int i = 0; i < 2 * KT; ++i) {
          const uint8_t* tile = buf + (i >> 1) * NS * CA_TILE;
          f16x8 vo[NV][2];
#pragma unroll
          for (int sl = 0; sl < NV; ++sl)
#pragma unroll
            for (int s = 0; s < 2; ++s) vo[sl][s] = value_operand(tile + (NK + sl) * CA_TILE, i & 1, s, lane);
          f32x16& next = S[(i + 1) & 1];
          next = scores(tile, i & 1);
          values(vo, S[i & 1]);
          settle(next, t0 + 32 * i + 32, false);
        }
      }
      __syncthreads();  // the next step's tiles are written, this one's are free
    }
  }
  sum = RowSum{l == 0.0f ? -__builtin_inff() : ref, l};
}

// ---------------------------------------------------------------------------
// fp32 outputs: every factor in two fp16 parts, every product three matrix instructions; scores
// carry the row's scale 2^E (unscale = 2^-E). Steps of 64 slots, the rest as above.
// ---------------------------------------------------------------------------
template <int NK, int NV>
__device__ __forceinline__ void chunk_steps_precise(const PagedAttnArgs& a, int kv, const Kept& Kk, const Kept& Kv, const Pass& pass,
                                                    int lim, float unscale, uint8_t* tiles, int wave, int lane,
                                                    const f16x8 (&qb)[NK][2], const f16x8 (&ql)[NK][2], f32x16 (&acc)[NV], RowSum& sum) {
  constexpr int NS = NK + NV, LO = NS * CA_TILE, BUF = 2 * LO;
  const int h = lane >> 5, col = lane & 31;
  uint32_t magic = 0x64006400u;
  asm volatile("" : "+v"(magic));
  float m_run = -__builtin_inff(), l_run = 0.0f;
  const int n_steps = (pass.to - pass.from + TILE - 1) / TILE;
  if (n_steps > 0) {
    GroupTiles<NK, NV, 1, 0> g;
    g.init(a, kv, Kk, Kv, wave);
    g.look_up_at(a, pass.row, pass.from, pass.from, pass.to, lane);
    g.load(a);
    g.look_up(a, pass.row, pass.from + TILE, pass.from, pass.to, lane);
    g.template write<true>(tiles, LO, wave, lane, magic);
    g.load(a);
    g.look_up(a, pass.row, pass.from + 2 * TILE, pass.from, pass.to, lane);
    __syncthreads();
#pragma unroll 1
    for (int j = 0; j < n_steps; ++j) {
      const int t0 = pass.from + j * TILE;
      if (j + 1 < n_steps) {
        g.template write<true>(tiles + ((j + 1) & 1) * BUF, LO, wave, lane, magic);
        g.load(a);
        g.look_up(a, pass.row, t0 + 3 * TILE, pass.from, pass.to, lane);
      }
      if (t0 < pass.lim_last) {
        const uint8_t* buf = tiles + (j & 1) * BUF;
        f32x16 S[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          S[k] = zero16();
          f32x16 lo = zero16();
#pragma unroll
          for (int sl = 0; sl < NK; ++sl)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const f16x8 kh = key_operand(buf + sl * CA_TILE, k, s, h, col), kl = key_operand(buf + LO + sl * CA_TILE, k, s, h, col);
              S[k] = mfma_f16(kh, qb[sl][s], S[k]);
              lo = mfma_f16(kh, ql[sl][s], lo);
              lo = mfma_f16(kl, qb[sl][s], lo);
            }
#pragma unroll
          for (int i = 0; i < 16; ++i) S[k][i] = __builtin_fmaf(lo[i], 1.0f / CA_LO, S[k][i]);
        }
        if (t0 + TILE > pass.lim_first) {  // some row of the wavefront does not see the whole step
          int left = lim - t0 - 4 * h;
          asm volatile("" : "+v"(left));
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) S[k][i] = 32 * k + 8 * (i >> 2) + (i & 3) < left ? S[k][i] : -__builtin_inff();
        }
        float top = __builtin_fmaxf(max16(S[0]), max16(S[1]));
        top = __builtin_fmaxf(top, other_half(top)) * unscale;
        if (__any(top > m_run + CA_SLACK)) {
          const float mn = __builtin_fmaxf(m_run, top);
          const float f = m_run == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m_run - mn);
          l_run *= f;
#pragma unroll
          for (int sl = 0; sl < NV; ++sl)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[sl][i] *= f;
          m_run = mn;
        }
        const float lift = CA_LIFT - (m_run == -__builtin_inff() ? 0.0f : m_run);
        f32x16 lo[NV];
#pragma unroll
        for (int sl = 0; sl < NV; ++sl) lo[sl] = zero16();
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            u32x4 rh, rl;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x2 p = f32x2{__builtin_amdgcn_exp2f(__builtin_fmaf(S[k][8 * s + 2 * i], unscale, lift)),
                                    __builtin_amdgcn_exp2f(__builtin_fmaf(S[k][8 * s + 2 * i + 1], unscale, lift))};
              l_run += p[0] + p[1];
              const f16x2 hi = __builtin_convertvector(p, f16x2);
              rh[i] = __builtin_bit_cast(uint32_t, hi);
              rl[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                                                       f32x2{(p[0] - (float)hi[0]) * CA_LO, (p[1] - (float)hi[1]) * CA_LO}, f16x2));
            }
#pragma unroll
            for (int sl = 0; sl < NV; ++sl) {
              const uint8_t* vt = buf + (NK + sl) * CA_TILE;
              const f16x8 vh = value_operand(vt, k, s, lane), vl = value_operand(vt + LO, k, s, lane);
              acc[sl] = mfma_f16(vh, as_f16x8(rh), acc[sl]);
              lo[sl] = mfma_f16(vl, as_f16x8(rh), lo[sl]);
              lo[sl] = mfma_f16(vh, as_f16x8(rl), lo[sl]);
            }
          }
#pragma unroll
        for (int sl = 0; sl < NV; ++sl)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[sl][i] = __builtin_fmaf(lo[sl][i], 1.0f / CA_LO, acc[sl][i]);
      }
      __syncthreads();  // the next step's tiles are written, this one's are free
    }
  }
  sum = RowSum{m_run == -__builtin_inff() ? m_run : m_run - CA_LIFT, l_run};
}

// q' of a row block as column operands: element e of piece 2s + h of slot sl is the lane's row's
// q' of code 4 (2s + h) + e / 2 + 16 (e % 2). With parts, scaled by 2^E into [2^8, 2^9) and the low
// parts in ql; returns 2^-E.
template <bool PRECISE, int N>
__device__ __forceinline__ float rotate_queries(const PagedAttnArgs& a, const PagedSeq& seq, const Rows& rows, int kv, const Kept& Kk,
                                                int lane, f16x8 (&qb)[N][2], f16x8 (&ql)[PRECISE ? N : 1][2]) {
  constexpr int NP = PRECISE ? 3 : 2;  // bf16 parts of the basis (and of fp32 queries)
  const int h = lane >> 5, col = lane & 31;
  const int64_t qoff = (seq.first + rows.tok) * a.q_token_stride + (kv * a.n_qh + rows.head) * a.q_head_stride + 8 * h;
  f32x16 acc[N];
  float most = 0.0f;
  const int i = 4 * (col >> 3) + (col & 3), hh = (col >> 2) & 1;  // MFMA row col is register i of lane half hh
  const int code = 4 * (2 * (i >> 3) + hh) + ((i & 7) >> 1) + 16 * (i & 1);
#pragma unroll
  for (int sl = 0; sl < N; ++sl) {
    acc[sl] = zero16();
    if (sl >= Kk.n) continue;
    const float* V = a.basis_k + (int64_t)kv * D * D + (8 * h) * D + G * Kk.grp[sl] + code;
#pragma unroll 1
    for (int k = 0; k < 8; ++k) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = V[(16 * k + e) * D];
      bf16x8 vp[NP];
      split8<NP>(v, vp);
      if (a.q_f32) {
        const f32x4* qp = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.q) + qoff + 16 * k);
        const f32x4 q0 = qp[0], q1 = qp[1];
        const float qv[8] = {q0[0], q0[1], q0[2], q0[3], q1[0], q1[1], q1[2], q1[3]};
        bf16x8 qq[NP];
        split8<NP>(qv, qq);
#pragma unroll
        for (int x = 0; x < NP; ++x)
#pragma unroll
          for (int y = 0; x + y < NP; ++y)
            acc[sl] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vp[x], qq[y], acc[sl], 0, 0, 0);
      } else {
        const bf16x8 qq = as_bf16x8(*reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + qoff + 16 * k));
#pragma unroll
        for (int x = 0; x < NP; ++x) acc[sl] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vp[x], qq, acc[sl], 0, 0, 0);
      }
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      acc[sl][j] *= a.scale_log2;
      most = __builtin_fmaxf(most, __builtin_fabsf(acc[sl][j]));
    }
  }
  float up = 1.0f;
  if constexpr (PRECISE) {
    most = __builtin_fmaxf(most, other_half(most));
    up = __builtin_ldexpf(1.0f, 9 - scale_exponent(most));
  }
#pragma unroll
  for (int sl = 0; sl < N; ++sl)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 rh, rl;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f32x2 x = f32x2{acc[sl][8 * s + 2 * j] * up, acc[sl][8 * s + 2 * j + 1] * up};
        if constexpr (!PRECISE) {  // NaN stays
#pragma unroll
          for (int e = 0; e < 2; ++e) x[e] = x[e] > 65504.0f ? 65504.0f : x[e] < -65504.0f ? -65504.0f : x[e];
        }
        const f16x2 hi = __builtin_convertvector(x, f16x2);
        rh[j] = __builtin_bit_cast(uint32_t, hi);
        rl[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{(x[0] - (float)hi[0]) * CA_LO, (x[1] - (float)hi[1]) * CA_LO}, f16x2));
      }
      qb[sl][s] = as_f16x8(rh);
      if constexpr (PRECISE) ql[sl][s] = as_f16x8(rl);
    }
  return 1.0f / up;
}

// What a wavefront does, for N groups of each kind (missing ones are zeros).
template <bool PRECISE, bool TREE, int N>
__device__ __forceinline__ void chunk_rows(const PagedAttnArgs& a, const PagedSeq& seq, int kv, const Kept& Kk, const Kept& Kv,
                                           int64_t unit, int64_t tile, int part, int wave, int lane, uint8_t* tiles) {
  const Rows rows = rows_of<TREE>(a, seq, tile, wave, lane & 31);
  // the part's slots: those of a unit end at its last row's
  const int n_parts = parts_of(a, rows.lim_unit);
  if (part > 0 && part >= n_parts) return;
  Pass pass;
  pass.row = seq.row;
  pass.from = (int)(part * a.part_slots);
  pass.to = rows.lim_unit < pass.from + a.part_slots ? rows.lim_unit : (int)(pass.from + a.part_slots);
  // No row sees past the part: the block that the 16-bit form scores ahead of a part's last one lies
  // there, on tiles of zeros, whose scores of 0 would pass for its largest.
  const int lim = rows.lim < pass.to ? rows.lim : pass.to;
  pass.lim_first = rows.lim_first < pass.to ? rows.lim_first : pass.to;
  pass.lim_last = rows.lim_last;
  pass.past = rows.past;
  pass.own = rows.own;

  f16x8 qb[N][2], ql[PRECISE ? N : 1][2];
  const float unscale = rotate_queries<PRECISE, N>(a, seq, rows, kv, Kk, lane, qb, ql);
  f32x16 acc[N];
#pragma unroll
  for (int sl = 0; sl < N; ++sl) acc[sl] = zero16();
  RowSum sum;
  if constexpr (PRECISE)
    chunk_steps_precise<N, N>(a, kv, Kk, Kv, pass, lim, unscale, tiles, wave, lane, qb, ql, acc, sum);
  else
    chunk_steps<N, N, TREE>(a, kv, Kk, Kv, pass, lim, tiles, wave, lane, qb, acc, sum);
  const float m = __builtin_fmaxf(sum.m, other_half(sum.m)), l = sum.l + other_half(sum.l);
  if (n_parts > 1) {
    float* p = a.partial + part_at(a, unit, kv, part, wave) + lane;
#pragma unroll
    for (int sl = 0; sl < N; ++sl)
      if (sl < Kv.n)
#pragma unroll
        for (int i = 0; i < 16; ++i) p[(16 * sl + i) * 64] = acc[sl][i];
    p[16 * NG * 64] = l == 0.0f ? -__builtin_inff() : m;
    p[(16 * NG + 1) * 64] = l;
    return;
  }
  finish_rows<PRECISE ? 3 : 2, N>(a, seq, rows, kv, Kv, acc, m, l, lane);
}

// Workgroup = (unit of 256 rows, KV head; part of the slots). The counts of kept groups lie on the
// device and differ from head to head: their cases share nothing but the scalars, so that each
// has its own registers (with preparation and output outside the switch, the products of two
// groups ran at the widest case's; as kernels of their own, the heads of one waited for the others').
template <bool PRECISE, bool TREE>
__global__ __launch_bounds__(64 * CA_NW, 2) void paged_chunk_kernel(PagedAttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t tiles[];
  __shared__ FindScratch find_s;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = blockIdx.x / (unsigned)a.c.n_kv;
  int b;
  int64_t tile;
  if (!find_unit<CA_NW>(a, unit, find_s, b, tile)) return;
  const PagedSeq seq = paged_seq(a.c, b);
  Kept Kk = read_kept(a.bits_k + kv * NG), Kv = read_kept(a.bits_v + kv * NG);
  if (!Kk.ok || Kk.used > a.Wk) Kk.n = 0;  // width table inconsistent with the record
  if (!Kv.ok || Kv.used > a.Wv) Kv.n = 0;
  switch (Kk.n > Kv.n ? Kk.n : Kv.n) {
    case 4: chunk_rows<PRECISE, TREE, 4>(a, seq, kv, Kk, Kv, unit, tile, blockIdx.y, wave, lane, tiles); break;
    case 3: chunk_rows<PRECISE, TREE, 3>(a, seq, kv, Kk, Kv, unit, tile, blockIdx.y, wave, lane, tiles); break;
    default: chunk_rows<PRECISE, TREE, 2>(a, seq, kv, Kk, Kv, unit, tile, blockIdx.y, wave, lane, tiles);
  }
}

// ---------------------------------------------------------------------------
// Join of a unit's parts: a wavefront per 32 rows, on registers as the parts left them.
// ---------------------------------------------------------------------------
template <bool PRECISE>
__global__ __launch_bounds__(64) void paged_join_kernel(PagedAttnArgs a) {
  __shared__ FindScratch find_s;
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv), block = blockIdx.y, lane = threadIdx.x;
  const int64_t unit = blockIdx.x / (unsigned)a.c.n_kv;
  int b;
  int64_t tile;
  if (!find_unit<1>(a, unit, find_s, b, tile)) return;
  const PagedSeq seq = paged_seq(a.c, b);
  const Rows rows = rows_of<false>(a, seq, tile, block, lane & 31);
  const int n_parts = parts_of(a, rows.lim_unit);
  if (n_parts <= 1) return;  // done by the part itself
  Kept Kv = read_kept(a.bits_v + kv * NG);
  if (!Kv.ok || Kv.used > a.Wv) Kv.n = 0;
  float m = -__builtin_inff(), l = 0.0f;
  const int ml = 16 * NG * 64 + lane;
  for (int i = 0; i < n_parts; ++i) m = __builtin_fmaxf(m, a.partial[part_at(a, unit, kv, i, block) + ml]);
  f32x16 acc[NG];
#pragma unroll
  for (int sl = 0; sl < NG; ++sl) acc[sl] = zero16();
  for (int i = 0; i < n_parts; ++i) {
    const float* p = a.partial + part_at(a, unit, kv, i, block);
    const float mi = p[ml], f = mi == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(mi - m);
    l = __builtin_fmaf(f, p[ml + 64], l);
#pragma unroll
    for (int sl = 0; sl < NG; ++sl)
      if (sl < Kv.n)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[sl][j] = __builtin_fmaf(f, p[(16 * sl + j) * 64 + lane], acc[sl][j]);
  }
  finish_rows<PRECISE ? 3 : 2, NG>(a, seq, rows, kv, Kv, acc, m, l, lane);
}

// The same for trees: four wavefronts share a unit's parts, which are many where a sequence is alone, then each takes a
// block of 32 channels (64 tokens of seven heads over 131k slots, 256 parts: 20 us, 22 with one that does all channels;
// eight wavefronts the same: a chain of latencies).
__global__ __launch_bounds__(256) void paged_tree_join_kernel(PagedAttnArgs a) {
  constexpr int NW = 4, SIZE = (16 * NG + 2) * 64;
  __shared__ FindScratch find_s;
  __shared__ float sums_s[NW * SIZE];
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv), block = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t unit = blockIdx.x / (unsigned)a.c.n_kv;
  int b;
  int64_t tile;
  if (!find_unit<NW>(a, unit, find_s, b, tile)) return;
  const PagedSeq seq = paged_seq(a.c, b);
  const Rows rows = rows_of<true>(a, seq, tile, block, lane & 31);
  const int n_parts = parts_of(a, rows.lim_unit);
  if (n_parts <= 1) return;  // done by the part itself
  Kept Kv = read_kept(a.bits_v + kv * NG);
  if (!Kv.ok || Kv.used > a.Wv) Kv.n = 0;
  float m = -__builtin_inff(), l = 0.0f;
  f32x16 acc[NG];
#pragma unroll
  for (int sl = 0; sl < NG; ++sl) acc[sl] = zero16();
  auto add = [&](const float* p) __attribute__((always_inline)) {
    const float mi = p[16 * NG * 64], li = p[(16 * NG + 1) * 64], top = __builtin_fmaxf(m, mi);
    f32x16 x[NG];
#pragma unroll
    for (int sl = 0; sl < NG; ++sl)
      if (sl < Kv.n)
#pragma unroll
        for (int j = 0; j < 16; ++j) x[sl][j] = p[(16 * sl + j) * 64];
    const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - top), fi = mi == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(mi - top);
    l = __builtin_fmaf(fi, li, f * l);
#pragma unroll
    for (int sl = 0; sl < NG; ++sl)
      if (sl < Kv.n)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[sl][j] = __builtin_fmaf(fi, x[sl][j], f * acc[sl][j]);
    m = top;
  };
#pragma unroll 1
  for (int i = wave; i < n_parts; i += NW) add(a.partial + part_at(a, unit, kv, i, block) + lane);
  float* mine = sums_s + wave * SIZE + lane;
#pragma unroll
  for (int sl = 0; sl < NG; ++sl)
    if (sl < Kv.n)
#pragma unroll
      for (int j = 0; j < 16; ++j) mine[(16 * sl + j) * 64] = acc[sl][j];
  mine[16 * NG * 64] = m;
  mine[(16 * NG + 1) * 64] = l;
  __syncthreads();
  m = -__builtin_inff();
  l = 0.0f;
#pragma unroll
  for (int sl = 0; sl < NG; ++sl) acc[sl] = zero16();
#pragma unroll 1
  for (int w = 0; w < NW; ++w) add(sums_s + w * SIZE + lane);
  finish_rows<2, NG, 1>(a, seq, rows, kv, Kv, acc, m, l, lane, wave);
}

// ---------------------------------------------------------------------------
// Few rows (a decode step's single tokens, a few speculative ones), 16-bit outputs: a sequence's
// rows on a KV head, at most 16, are the columns of 16 x 16 products, and a chunk of its slots a
// workgroup's (scan_place). Each wavefront walks tiles of its own, a kept group at a time through
// one 4 KB tile of LDS, the group's words loaded while the one before is multiplied; no barrier
// until the wavefronts' sums are merged, and 16 wavefronts on a CU hide each other's chains.
// 635 vector instructions a tile of seven heads (about 75 a group to make coefficients), where the
// latent scan, whose products take bit fields and whose sums hold for fp32 outputs, has 1000: 48
// sequences of 8k slots 53 us and 76. Bound by the chain of a group through LDS: all groups of a tile
// loaded a tile ahead (three wavefronts a SIMD by registers) came to the same 54, with the next
// group's coefficients made among the products to 62 (spills).
// ---------------------------------------------------------------------------
constexpr int FEW_NW = 4, FEW_ROWS = 16, FEW_PITCH = D + 4;
__global__ __launch_bounds__(64 * FEW_NW, 4) void paged_few_kernel(PagedAttnArgs a, float* __restrict__ partial) {
  __shared__ ScanScratch place_s;
  __shared__ float m_s[FEW_NW][FEW_ROWS], l_s[FEW_NW][FEW_ROWS];
  __shared__ int32_t unit_s[2 * NG];
  __shared__ __attribute__((aligned(16))) float sums_s[FEW_NW * FEW_ROWS * FEW_PITCH];  // the tiles while wavefronts walk
  __shared__ __attribute__((aligned(16))) uint8_t q_s[NG][64 * 16];                      // q' as column operands, by lane
  const int kv = (int)(blockIdx.x % (unsigned)a.c.n_kv), item = (int)(blockIdx.x / (unsigned)a.c.n_kv);
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const ScanPlace at = scan_place(a, item, place_s);
  if (at.b < 0) return;
  if (at.chunk == 0 && kv == 0 && tid == 0) {  // for the combine
    a.scan_plan[2 * at.b] = item;
    a.scan_plan[2 * at.b + 1] = at.n_chunks;
  }
  const PagedSeq seq = paged_seq(a.c, at.b);
  const int n_rows = (int)seq.n * a.n_qh;
  Kept Kk = read_kept(a.bits_k + kv * NG), Kv = read_kept(a.bits_v + kv * NG);
  if (!Kk.ok || Kk.used > a.Wk) Kk.n = 0;  // width table inconsistent with the record
  if (!Kv.ok || Kv.used > a.Wv) Kv.n = 0;
  const int row = col < n_rows ? col : 0;  // columns past the rows repeat the first
  const int tok = row / a.n_qh, head = row - tok * a.n_qh;
  const int64_t past = seq.len - seq.n + 1;  // slots that token 0 sees
  const int lim = past + tok < 0 ? 0 : (int)(past + tok), lim_first = past < 0 ? 0 : (int)past;

  // q' of kept group `wave`: element e of quarter p is that of code 4 p + e / 2 + 16 (e % 2), as
  // the tiles' places are; product x has e = 4 x .. 4 x + 3
  if (wave < Kk.n) {
    const int64_t qoff = (seq.first + tok) * a.q_token_stride + (kv * a.n_qh + head) * a.q_head_stride + 8 * quarter;
    const float* V = a.basis_k + (int64_t)kv * D * D + (8 * quarter) * D + G * pick4(Kk.grp, wave) + 4 * (col >> 2) +
                     ((col & 3) >> 1) + 16 * (col & 1);
    f32x4 acc[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float v[2][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[0][e] = V[(32 * k + e) * D];
        v[1][e] = V[(32 * k + e) * D + 2];
      }
      bf16x8 qq[2];
      if (a.q_f32) {
        const f32x4* qp = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.q) + qoff + 32 * k);
        const f32x4 q0 = qp[0], q1 = qp[1];
        const float qv[8] = {q0[0], q0[1], q0[2], q0[3], q1[0], q1[1], q1[2], q1[3]};
        split8<2>(qv, qq);
      } else {
        qq[0] = as_bf16x8(*reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + qoff + 32 * k));
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        bf16x8 vp[2];
        split8<2>(v[x], vp);
        acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[0], qq[0], acc[x], 0, 0, 0);
        acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[1], qq[0], acc[x], 0, 0, 0);
        if (a.q_f32) acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[0], qq[1], acc[x], 0, 0, 0);
      }
    }
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x2 x = f32x2{acc[j >> 1][2 * (j & 1)] * a.scale_log2, acc[j >> 1][2 * (j & 1) + 1] * a.scale_log2};
#pragma unroll
      for (int e = 0; e < 2; ++e) x[e] = x[e] > 65504.0f ? 65504.0f : x[e] < -65504.0f ? -65504.0f : x[e];
      r[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
    }
    *reinterpret_cast<u32x4*>(q_s[wave] + 16 * lane) = r;
  }

  const int n_tiles = (int)((seq.len + TILE - 1) / TILE), tpp = a.c.page_tokens >> 6;
  const int begin = at.chunk * at.tiles_per_chunk;
  const int end = n_tiles - begin < at.tiles_per_chunk ? n_tiles : begin + at.tiles_per_chunk;
  const int n_keys = Kk.n, n_units = Kk.n + Kv.n;
  if (tid < 2 * NG) {  // a unit: a kept group of the keys, then of the values
    const int s = tid < n_keys ? tid : tid - n_keys;
    int b = 0, pay = 0;
#pragma unroll
    for (int x = 0; x < NG; ++x) {
      b = x == s ? (tid < n_keys ? Kk.bits[x] : Kv.bits[x]) : b;
      pay = x == s ? (tid < n_keys ? Kk.pay[x] : Kv.pay[x]) : pay;
    }
    unit_s[tid] = b | (s & 3) << 4 | pay << 6;
  }
  __syncthreads();  // q' and units
  uint8_t* tile = reinterpret_cast<uint8_t*>(sums_s) + wave * CA_TILE;
  uint32_t magic = 0x64006400u;  // exponent of 1024 in both halves, in a VGPR
  asm volatile("" : "+v"(magic));
  // the tile whose words are loaded: its page's place in the table, its own in the page, its records
  int load_tt = begin + wave, idx = load_tt / tpp, in_page = load_tt - idx * tpp, page = -1;
  const uint32_t *kp = a.pool_k, *vp = a.pool_v;
  bool page_ok = false;
  uint32_t words[8], meta = 0u;
  auto look_up = [&]() __attribute__((always_inline)) {
    page = load_tt < end ? __builtin_amdgcn_readfirstlane(a.c.table[(int64_t)seq.row * a.c.row_pages + idx]) : -1;
  };
  auto enter = [&]() __attribute__((always_inline)) {  // the tile looked up; the walk goes on
    page_ok = page >= 0 && page < a.c.n_pages;
    const int64_t rec = ((int64_t)(page_ok ? page : 0) * a.c.n_kv + kv) * tpp + in_page;
    kp = a.pool_k + rec * (TILE * a.Wk) + lane;
    vp = a.pool_v + rec * (TILE * a.Wv) + lane;
    load_tt += FEW_NW;
    in_page += FEW_NW;
    while (in_page >= tpp) {
      in_page -= tpp;
      ++idx;
    }
    look_up();
  };
  // operands in the tile (the swizzle of piece_at repeats every 16 slots)
  const uint8_t* key_at = tile + piece_at(col, quarter);
  const uint8_t* val_at0 = tile + piece_at(4 * quarter + (col >> 2), (lane & 3) >> 1) + 8 * (lane & 1);
  const uint8_t* val_at1 = tile + piece_at(4 * quarter + (col >> 2), 2 + ((lane & 3) >> 1)) + 8 * (lane & 1);
  int bits = 0;  // of the unit whose words are loaded: kept group u of the keys, or u - Kk.n of the values
  auto fetch = [&](int u) __attribute__((always_inline)) {
    const int d = __builtin_amdgcn_readfirstlane(unit_s[u]);
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
  // unit u's coefficients into the tile (its last readers are done: LDS serves a wavefront in
  // order), and the next unit's words
  auto expand = [&](int u) __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const uint32_t m = finite_meta(meta, bits);
    with_bits(bits, [&](auto bc) __attribute__((always_inline)) { write_coefficients<decltype(bc)::value, false>(words, m, tile, lane, 0, magic); });
    if (u + 1 == n_units) enter();
    fetch(u + 1 == n_units ? 0 : u + 1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  look_up();
  if (n_units > 0) {
    enter();
    fetch(0);
  }
  f32x4 acc[NG][2];
#pragma unroll
  for (int sl = 0; sl < NG; ++sl) acc[sl][0] = acc[sl][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float ref = 0.0f, l = 0.0f;  // the reference less CA_LIFT
#pragma unroll 1
  for (int tt = begin + wave; tt < end; tt += FEW_NW) {
    f32x4 S[4];  // slot 16 b + 4 quarter + i
#pragma unroll
    for (int b = 0; b < 4; ++b) S[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int u = 0; u < n_keys; ++u) {
      expand(u);
      const f16x8 qo = as_f16x8(*reinterpret_cast<const u32x4*>(q_s[u] + 16 * lane));
#pragma unroll
      for (int b = 0; b < 4; ++b)
        S[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(*reinterpret_cast<const u32x4*>(key_at + 16 * 64 * b)), qo, S[b], 0, 0, 0);
    }
    const int t0 = tt * TILE;
    if (t0 + TILE > lim_first) {
      const int left = lim - t0 - 4 * quarter;
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) S[b][i] = 16 * b + i < left ? S[b][i] : -__builtin_inff();
    }
    float top = S[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = __builtin_fmaxf(top, S[i >> 2][i & 3]);
    top -= CA_LIFT + CA_SLACK;
    const bool first = tt == begin + wave;
    if (first || __any(top > ref)) {
      top = __builtin_fmaxf(top, __shfl_xor(top, 16));
      top = __builtin_fmaxf(top, other_half(top));
      // a row that sees nothing in the first tile sees nothing later
      const float d = first ? (top == -__builtin_inff() ? 0.0f : top + CA_SLACK) : top > ref ? top + CA_SLACK - ref : 0.0f;
      const float f = __builtin_amdgcn_exp2f(-d);
      ref += d;
      if (!first) {
        l *= f;
#pragma unroll
        for (int sl = 0; sl < NG; ++sl)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[sl][i >> 2][i & 3] *= f;
      }
    }
    f16x8 w[2];  // weights of 32 slots: element e is slot 16 (e / 4) + 4 quarter + e % 4
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      u32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 s = S[2 * hf + (j >> 1)];
        const f32x2 e = f32x2{__builtin_amdgcn_exp2f(s[2 * (j & 1)] - ref), __builtin_amdgcn_exp2f(s[2 * (j & 1) + 1] - ref)};
        const f16x2 r = __builtin_convertvector(e, f16x2);
        x[j] = __builtin_bit_cast(uint32_t, r);
        l = __builtin_amdgcn_fdot2(__builtin_bit_cast(h16x2, r), h16x2{(__fp16)1.0f, (__fp16)1.0f}, l, false);
      }
      w[hf] = as_f16x8(x);
    }
#pragma unroll
    for (int sl = 0; sl < NG; ++sl) {
      if (sl < n_units - n_keys) {
        expand(n_keys + sl);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const uint8_t* p = (x ? val_at1 : val_at0) + 32 * 64 * hf;
            const u32x2 y0 = read_transposed(p), y1 = read_transposed(p + 16 * 64);
            acc[sl][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(u32x4{y0[0], y0[1], y1[0], y1[1]}), w[hf], acc[sl][x], 0, 0, 0);
          }
      }
    }
  }
  // merge of the wavefronts, and the chunk's partial of every row
  l += __shfl_xor(l, 16);
  l += other_half(l);
  __syncthreads();  // the tiles have been read
  if (quarter == 0) {
    m_s[wave][col] = l == 0.0f ? -__builtin_inff() : ref;
    l_s[wave][col] = l;
  }
#pragma unroll
  for (int sl = 0; sl < NG; ++sl)
    if (sl < Kv.n)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        *reinterpret_cast<f32x4*>(sums_s + (wave * FEW_ROWS + col) * FEW_PITCH + G * sl + 16 * x + 4 * quarter) = acc[sl][x];
  __syncthreads();
  float* part = partial + ((int64_t)item * a.c.n_kv + kv) * (a.scan_tokens * a.n_qh) * PART;
  for (int e = tid; e < n_rows * D; e += 64 * FEW_NW) {
    const int r = e >> 7, j = e & 127, g = j >> 5, c = j & 31;
    const int place = 8 * ((c & 15) >> 2) + 2 * (c & 3) + (c >> 4);
    int sl = -1;
#pragma unroll
    for (int x = 0; x < NG; ++x) sl = (x < Kv.n && Kv.grp[x] == g) ? x : sl;
    float m = -__builtin_inff(), sum = 0.0f, total = 0.0f;
#pragma unroll
    for (int w = 0; w < FEW_NW; ++w) m = __builtin_fmaxf(m, m_s[w][r]);
#pragma unroll
    for (int w = 0; w < FEW_NW; ++w) {
      const float f = m_s[w][r] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m_s[w][r] - m);
      if (sl >= 0) sum = __builtin_fmaf(f, sums_s[(w * FEW_ROWS + r) * FEW_PITCH + G * sl + place], sum);
      total = __builtin_fmaf(f, l_s[w][r], total);
    }
    part[r * PART + 8 + j] = sum;
    if (j < NG) part[r * PART + 2 + j] = 0.0f;
    if (j == 0) {
      part[r * PART] = m;
      part[r * PART + 1] = total;
    }
  }
}

// ---------------------------------------------------------------------------
// u = scale V_K m_K of each KV head: q . u is the part of the log-sum-exp that the softmax does
// not need.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void paged_lse_kernel(PagedAttnArgs a) {
  const int kv = blockIdx.x, ch = threadIdx.x >> 1, half = threadIdx.x & 1;
  const float* v = a.basis_k + ((int64_t)kv * D + ch) * D + 64 * half;
  const float* m = a.mean_k + kv * D + 64 * half;
  float s = 0.0f;
#pragma unroll 16
  for (int j = 0; j < 64; ++j) s = __builtin_fmaf(v[j], m[j], s);
  s += __shfl_xor(s, 1);
  if (half == 0) a.lse_u[kv * D + ch] = s * (a.scale_log2 * LN2);
}

}  // namespace spectra_dev

namespace spectra {
using namespace spectra_dev;

static_assert(PAGED_STEP % (2 * TILE) == 0, "whole steps in a part");

static_assert(CA_ROWS == PAGED_ROWS && CA_NW * (16 * NG + 2) * 64 * sizeof(float) == PAGED_PART_BYTES, "workspace of a part");

// A kept group takes two words at least; two buffers of two slot tiles, or of one in two parts.
static int chunk_lds(const PagedAttnArgs& a) {
  auto groups = [](int W) { return W < 6 ? 2 : W / 2 < NG ? W / 2 : NG; };
  return 2 * 2 * 2 * (groups(a.Wk) > groups(a.Wv) ? groups(a.Wk) : groups(a.Wv)) * CA_TILE;
}

hipError_t launch_paged_tree_chunks(const PagedAttnArgs& a, int64_t units, hipStream_t st) {
  const unsigned groups = (unsigned)(units * a.c.n_kv);
  hipLaunchKernelGGL((paged_chunk_kernel<false, true>), dim3(groups, (unsigned)a.parts), dim3(64 * CA_NW), chunk_lds(a), st, a);
  if (a.parts > 1) hipLaunchKernelGGL(paged_tree_join_kernel, dim3(groups, CA_NW), dim3(256), 0, st, a);
  return hipGetLastError();
}

void launch_paged_lse(const PagedAttnArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(paged_lse_kernel, dim3(a.c.n_kv), dim3(256), 0, st, a);
}

hipError_t launch_paged_attention(const PagedAttnArgs& args, void* workspace, hipStream_t st) {
  PagedAttnArgs a = args;
  const PagedPlan p = paged_plan(a.c.batch, a.c.n_new, a.n_q_heads, a.c.n_kv, a.max_new, a.max_tokens,
                                 a.out_f32 ? scan_rows(a.Wk, a.Wv) : FEW_ROWS);
  char* ws = static_cast<char*>(workspace);
  a.lse_u = reinterpret_cast<float*>(ws);
  a.scan_tokens = p.scan_tokens;
  a.part_slots = p.split.slots;
  a.parts = p.split.parts;
  a.partial = reinterpret_cast<float*>(ws + p.part_at);
  if (a.lse != nullptr) launch_paged_lse(a, st);
  hipError_t e = hipSuccess;
  if (p.units > 0) {
    const int lds = chunk_lds(a);
    const dim3 grid((unsigned)(p.units * a.c.n_kv), (unsigned)p.split.parts), join((unsigned)(p.units * a.c.n_kv), CA_NW);
    if (a.out_f32)
      hipLaunchKernelGGL((paged_chunk_kernel<true, false>), grid, dim3(64 * CA_NW), lds, st, a);
    else
      hipLaunchKernelGGL((paged_chunk_kernel<false, false>), grid, dim3(64 * CA_NW), lds, st, a);
    if (p.split.parts > 1) {
      if (a.out_f32)
        hipLaunchKernelGGL((paged_join_kernel<true>), join, dim3(64), 0, st, a);
      else
        hipLaunchKernelGGL((paged_join_kernel<false>), join, dim3(64), 0, st, a);
    }
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.scan_tokens == 0) return e;
  a.scan_least = PAGED_SCAN_LEAST;
  a.scan_plan = reinterpret_cast<int32_t*>(ws + p.plan_at);
  float* partial = reinterpret_cast<float*>(ws + p.scan_at);
  // Also for 16-bit outputs the latent scan where it has one quad of rows and records of 8 words (no
  // clamped loads, three workgroups on a CU), sequences may be long and there may be work for many
  // tiles a wavefront. Scan and paged_few_kernel, four heads on each of eight KV heads, lengths between a
  // quarter of the bound and the bound: 100 sequences of up to 8192 slots 173 and 196 us, 64 of 16384 200
  // and 206, 256 of 8192 357 and 427, one of 2^20 225 and 250; below the border 64 of 8192 116 and 109,
  // 48 of 8192 91 and 90, one of 2^18 78 and 78 (though with equal lengths, which paged_few_kernel cuts
  // badly, 64 of 8192 are 141 and 170). Other records, equal lengths: 5 words, 256 sequences of 4096 211
  // and 203; 4 and 12 words 229 and 216; 12 words 369 and 297; 30 words 1717 and 431. The host knows the
  // bound of the lengths only: many short sequences under a long one pay the difference (256 of 128
  // slots 72 and 61).
  const bool long_quad = p.scan_tokens * a.n_qh <= 4 && a.Wk == 8 && a.Wv == 8 && a.max_tokens > 2048 &&
                         a.c.batch * a.max_tokens * a.c.n_kv > (int64_t)1 << 22;
  if (a.out_f32 || long_quad) {
    launch_paged_scan(a, partial, st);
  } else {
    a.scan_items = (int32_t)paged_scan_items(a.c.n_kv, PAGED_SCAN_PER_CU);
    hipLaunchKernelGGL(paged_few_kernel, dim3((unsigned)((a.scan_items + a.c.batch) * a.c.n_kv)), dim3(64 * FEW_NW), 0, st, a, partial);
  }
  return launch_paged_combine(a, partial, st);
}

}  // namespace spectra
