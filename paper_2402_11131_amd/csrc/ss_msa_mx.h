// n5, a2 over a cache in microscaling formats: what the two kernels share (ss_msa_mx.hip: every wave its own keys; ss_msa_mx_rows.hip:
// the waves of a group share keys).
//
// Scores, S^T = K Q^T with v_mfma_scale_f32_16x16x128_f8f6f4: the cached elements and scale bytes are operands as they are.  A
// query row is the sum of two e4m3 rows, the second with a scale 2^-4 of the first's: four and four of a bf16 value's eight
// significant bits (features below 2^-17 of the row's largest lose bits, none more than 2^-22 of it).  Lane (lq, lg) = (lane &
// 15, lane >> 4) supplies, of a 4-bit operand, elements 32 lg .. +31 of row lq, of an 8-bit one elements 16 lg .. +15 and 64 +
// 16 lg .. +15; the scale of elements 32 g .. +31 comes from lane group g.  Heads of 128 take two instructions (one per part)
// for 16 keys and 16 queries; heads of 64 one, with the first part against elements 0..63 and the second against a repetition.
//
// O^T += V^T P^T with v_mfma_f32_16x16x32_bf16.  A scale belongs to one token, and the sum runs over tokens, so values are
// multiplied by their scales first: both formats are exact in bf16.  A lane turns half a block of a token into bf16 and puts it
// into an LDS tile of 32 tokens x 32 features (token-major, swizzled); the transposing read hands out four consecutive tokens
// of a feature.  A lane's scores are those of keys 4 lg .. +3 of either half of 32 keys, which is what it must supply of P.
#pragma once

#include <type_traits>

#include "ss_msa_mfma.h"
#include "ss_mx.h"

namespace ss {

struct MsaMxArgs {
  const uint16_t *q, *k_new, *v_new;
  uint16_t* out;
  MxCache c;
  const int32_t *seq_lens, *parent, *n_nodes;
  // Splits' results, divided by their own sums, as pieces of 1 KB: 64 lanes' four features of a 16-row tile.  Unit: what one
  // wave merges (P pieces, U units per workgroup).
  float* part_o;         // [items, n_splits, U, P, 64, 4]
  float* part_lse;       // [items, n_splits, tiles, 16]: log2-domain log-sum-exp of a row
  unsigned int* arrive;  // [items, U]: splits that have arrived; zero before the call, zero again after it
  int B, T, gamma, R, H, g, n_splits, n_qc;
  float scale_log2;
  // Running maximum before the first score: below every score whose product with scale_log2 an fp32 number holds, and its own
  // product with it is one too (rows that see nothing of a block keep it, and -inf * scale_log2 - (-inf) would be NaN).
  float no_max;
  uint32_t flags;
};

constexpr float kMxLazyLog2 = 16.0f;

// Tokens per split of a sequence of L in a call that was planned with up to n_splits: a share of L, but no fewer than are worth
// it.  One row, 8 KV heads: 128 tokens of a split take 1 us, merging two splits 2 us and each further one a quarter more, so the
// least worthwhile length grows with the root of L.  Two splits from 410 tokens on: few rows lose or gain little there, many rows
// gain (512 tokens, unsplit / halves, us: one row 8.8 / 8.9, in 8 bits 9.3 / 9.0, heads of 64 7.4 / 7.7; 320 rows 22.9 / 20.3).
// Later (one row): 1024 tokens 12.5 and, in quarters, 9.1; 4096 in splits of 256 / 512 / 1024 / 2048 tokens 12.5 / 12.5 / 15.7 / 23.
SS_HD int mx_split_len(int L, int n_splits) {
  const float root = 5.f * sqrtf((float)L);
  const int least = root < 256.f ? 256 : (int)root & ~127;
  if (5 * (long)L < 8 * (long)least) n_splits = 1;
  const int even = (L - 1) / n_splits + 1, up = (even + 127) & ~127;  // (L + n_splits may pass 32 bits)
  return n_splits > 1 && up < least ? least : up < 128 ? 128 : up;
}

template <int D, bool FP8>
struct MxBlock {
  static constexpr int DT = D / 16, NB = D / kMxBlock;
  static constexpr int ROWB = FP8 ? D : D / 2;               // bytes of a cached row
  static constexpr int PR = ROWB / 16;                       // 16-byte pieces of a row
  static constexpr int HALF = 16 * ROWB;                     // bytes of 16 rows: they share a page and are contiguous there
  static constexpr int HL = HALF / 1024;                     // loads of a half; 0 (rows of 32 bytes): one load takes both halves
  static constexpr int LOADS = (HL ? 2 * HL : 1) + 1;        // loads of a block's keys, or values: rows, scales
  static constexpr int SLOT = 32 * ROWB + 32 * NB;
  static constexpr int QW = D / 32;                          // 16-byte pieces of a lane's part of a bf16 query row
};

// Piece of a raw row that lies at piece position p of row t is p ^ raw_swz(t): 16 rows' pieces of one index meet all banks.
template <int PR>
SS_DEV int raw_swz(int t) { return (t / (16 / PR)) & (PR - 1); }
// 16-byte chunk of a row of the value tile where chunk c lies is c ^ tile_swz(row).  A write takes one chunk of 16 rows, or two
// (c, c + 2) of eight; the transposing read takes two neighbouring chunks of eight rows: all meet every bank once.
SS_DEV int tile_swz(int row) { return ((row >> 2) & 1) * 3 ^ ((row >> 3) & 1); }
// 4 bytes per lane straight into LDS, lane l's at lds_addr + 4*l.
SS_DEV void dma4(const void* p, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(p), "s"(lds_addr) : "memory", "m0");
}
SS_DEV void dma4(const void* sbase, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, %0" ::"s"(sbase), "v"(voff), "s"(lds_addr) : "memory", "m0");
}
// Loads that are coherent at device scope (the sc1 bit, see st16_device), known to the compiler as loads.
SS_DEV floatx4 ld16_device(const float* base, uint32_t byte) {
  const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0xffffffff, 0x00027000);
  return __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(r, byte, 0, 16));
}
SS_DEV float ld4_device(const float* base, uint32_t byte) {
  const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0xffffffff, 0x00027000);
  return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, byte, 0, 16));
}
// Maximum of three as one instruction; a NaN wins.
SS_DEV float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
SS_DEV float max8(const floatx4 (&S)[2]) {
  return max3(max3(max3(S[0][0], S[0][1], S[0][2]), S[0][3], S[1][0]), max3(S[1][1], S[1][2], S[1][3]), S[1][3]);
}
// Keeps the compiler from holding what is derived from x in registers across a loop.
SS_DEV uint32_t fresh(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}
// The wave's own LDS accesses stay in this order (they complete in it).
SS_DEV void in_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ------------------------------------------------------------------ a workgroup's piece of work
struct MxItem {
  int b, hk, s, qc;            // sequence, KV head, split, chunk of query rows
  int n_kept, R_kept, F, f0;   // kept nodes and rows of the sequence; folded rows of the KV head, the chunk's first
  int k0, k1, n_active;        // cached tokens of the split; splits of the sequence
};
// False: nothing to do.  The row chunks of one (sequence, KV head, split) get workgroup ids that are equal mod 8: ids go round
// robin over the XCDs, so they share an L2.
SS_DEV bool mx_item(const MsaMxArgs& a, int chunk_rows, MxItem& m) {
  const int G = a.B * a.c.Hkv * a.n_splits;
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const int group = (slot / a.n_qc) * 8 + xcd;
  m.qc = slot % a.n_qc;
  if (group >= G) return false;
  const int head = group / a.n_splits;
  m.s = group % a.n_splits;
  m.b = head / a.c.Hkv;
  m.hk = head - m.b * a.c.Hkv;
  const int L = min(max(a.seq_lens[m.b], 0), a.c.max_pages * a.c.page);
  m.n_kept = a.n_nodes ? min(max(a.n_nodes[m.b], 1), a.T) : a.T;
  m.R_kept = m.n_kept * (1 + a.gamma);
  m.F = a.g * m.R_kept;
  m.f0 = m.qc * chunk_rows;
  if (m.f0 >= m.F) return false;
  const int split = mx_split_len(L, a.n_splits);
  m.n_active = L <= split ? 1 : (L + split - 1) / split;
  if (m.s >= m.n_active) return false;
  m.k0 = m.s * split;
  m.k1 = min(L, m.k0 + split);
  return true;
}
// Query row r and head h of folded row f0 + at (clamped to the last); whether there is such a row.
SS_DEV bool mx_row_of(const MsaMxArgs& a, const MxItem& m, int at, int& r, int& h) {
  const int f = min(m.f0 + at, m.F - 1);
  const int fh = fast_div(f, m.R_kept), fr = f - fh * m.R_kept;
  r = fr < m.n_kept ? fr : a.T + (fr - m.n_kept);
  h = m.hk * a.g + fh;
  return m.f0 + at < m.F;
}
// This lane's features of that row, 16 lg .. and 64 + 16 lg ..
template <int D>
SS_DEV void mx_load_query(const MsaMxArgs& a, const MxItem& m, int at, int lg, uintx4 (&raw)[D / 32]) {
  int r, h;
  mx_row_of(a, m, at, r, h);
  const uint16_t* qp = a.q + (((size_t)m.b * a.R + r) * a.H + h) * D + 16 * lg;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) raw[i] = ld16(qp + 64 * (i >> 1) + 8 * (i & 1));
}
// ... as two e4m3 rows and their scale bytes.
template <int D>
SS_DEV int split_query(const uintx4 (&raw)[D / 32], uint32_t (&hi)[D / 16], uint32_t (&lo)[D / 16], int lg) {
  typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;
  u16x2 m2 = {0, 0};
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, raw[i][e] & 0x7fff7fffu));
  uint32_t m = max((uint32_t)m2[0], (uint32_t)m2[1]);
  m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
  m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
  const int sh = mx_scale_code<true>(m << 16), sl = sh == 255 ? 255 : max(sh - 4, 0);
  const float fh = mx_scale(sh), fl = mx_scale(sl);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    shortx2 ph = {0, 0}, pl = {0, 0};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const bf16x2 x = __builtin_bit_cast(bf16x2, sh == 255 ? 0u : raw[i >> 1][2 * (i & 1) + e]);
      ph = e ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(ph, x, fh, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(ph, x, fh, false);
      const uint32_t pw = __builtin_bit_cast(uint32_t, ph);
      const floatx2 back = e ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(pw, fh, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(pw, fh, false);
      const float r0 = (float)x[0] - back[0], r1 = (float)x[1] - back[1];
      pl = e ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(pl, r0, r1, fl, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(pl, r0, r1, fl, false);
    }
    hi[i] = __builtin_bit_cast(uint32_t, ph);
    lo[i] = sh == 255 ? 0u : __builtin_bit_cast(uint32_t, pl);
  }
  return D == 128 ? sh | (sl << 8) : (lg < 2 ? sh : sl);
}
// Operands: heads of 128 both parts; heads of 64 all in the first.
template <int D>
SS_DEV void mx_query_operands(const uint32_t (&hi)[D / 16], const uint32_t (&lo)[D / 16], intx8& Qh, intx8& Ql) {
  if constexpr (D == 128) {
    Qh = intx8{(int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3], (int)hi[4], (int)hi[5], (int)hi[6], (int)hi[7]};
    Ql = intx8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)lo[4], (int)lo[5], (int)lo[6], (int)lo[7]};
  } else {
    Qh = intx8{(int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3], (int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3]};
    Ql = Qh;
  }
}

// ------------------------------------------------------------------ from memory to LDS
// Blocks first, first + stride, ... of a split's 32-token blocks; lane i of a wave holds the ids of iteration jbase + i's pages
// (of both 16-token halves: a page may be that small).
template <int D, bool FP8>
struct MxMover {
  using Bk = MxBlock<D, FP8>;
  const MxCache& c;
  const int32_t* table;
  int hk, first_tok, stride_tok;  // KV head; first token of iteration 0, tokens between iterations
  uint32_t page_rows, raw_voff, raw_voff1, sc_off, tab_a, tab_b;
  int sc_tok;
  SS_DEV MxMover(const MxCache& cache, int b, int head, int tok0, int tok_stride, int lane)
      : c(cache), table(cache.block_table + (size_t)b * cache.max_pages), hk(head), first_tok(tok0), stride_tok(tok_stride), tab_a(0), tab_b(0) {
    page_rows = (uint32_t)(c.Hkv * c.page);  // rows of a page, all heads
    // bytes of this lane's piece from the base of 1024 bytes of rows; of the second load of a half, where there are two
    auto piece_off = [&](int t) { return (uint32_t)(t * Bk::ROWB + (((lane % Bk::PR) ^ raw_swz<Bk::PR>(t)) * 16)); };
    raw_voff = piece_off(lane / Bk::PR);
    raw_voff1 = piece_off(64 / Bk::PR + lane / Bk::PR);
    sc_tok = (lane % (8 * Bk::NB)) * (4 / Bk::NB);  // lane l's dword of scales is that of token (4 / NB) * l of the block
    sc_off = (uint32_t)((hk * c.page + (sc_tok & 15)) * Bk::NB);
  }
  SS_DEV void load_pages(int jbase, int lane) {
    const int kb = first_tok + (jbase + lane) * stride_tok;
    tab_a = (uint32_t)min(max(table[min(kb >> c.page_shift, c.max_pages - 1)], 0), c.num_pages - 1);
    tab_b = (uint32_t)min(max(table[min((kb + 16) >> c.page_shift, c.max_pages - 1)], 0), c.num_pages - 1);
  }
  // Block `it`'s keys (values: kv = 1) to the slot at LDS address `at`.
  SS_DEV void issue(int kv, int it, uint32_t at, int lane) const {
    const uint32_t pa = __builtin_amdgcn_readlane(tab_a, it & 63), pb = __builtin_amdgcn_readlane(tab_b, it & 63);
    const int kb = first_tok + it * stride_tok;
    const uint32_t sa = (uint32_t)(kb & (c.page - 1)), sb = (uint32_t)((kb + 16) & (c.page - 1));
    const size_t ra = (size_t)pa * page_rows + (uint32_t)hk * c.page + sa, rb = (size_t)pb * page_rows + (uint32_t)hk * c.page + sb;
    const uint8_t* base = kv ? c.v : c.k;
    if constexpr (Bk::HL > 0) {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < Bk::HL; ++i) dma16<true>(base + (half ? rb : ra) * Bk::ROWB, i ? raw_voff1 : raw_voff, at + half * Bk::HALF + i * 1024);
    } else {  // 32 rows of 32 bytes in one load: lanes 32.. take the second half
      const uint8_t* p = base + (lane < 32 ? ra : rb) * Bk::ROWB + (raw_voff & (Bk::HALF - 1));
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(p), "s"(at) : "memory", "m0");
    }
    const uint32_t pg = sc_tok < 16 ? pa : pb, row = sc_tok < 16 ? sa : sb;
    const uint8_t* sp = (kv ? c.vs : c.ks) + ((size_t)pg * page_rows + row) * Bk::NB + sc_off;
    if (lane < 8 * Bk::NB) dma4(sp, at + 32 * Bk::ROWB);
  }
};

// A quarter of every block: the keys or the values (kv) of its first or second 16 tokens, which share a page.  Lane i of a wave
// holds the cache row (of all heads and pages; fewer than 2^32, checked on the host) at which that of iteration jbase + i begins.
template <int D, bool FP8, bool STREAM>
struct MxQuarter {
  using Bk = MxBlock<D, FP8>;
  static constexpr int LOADS = (Bk::HL ? Bk::HL : 1) + 1;
  const uint8_t *rows, *scales;
  uint32_t voff, voff1, at, sc_at, tab;
  SS_DEV void init(const MxCache& c, int kv, int half, int lane) {
    rows = kv ? c.v : c.k;
    scales = kv ? c.vs : c.ks;
    tab = 0;
    auto piece_off = [&](int t) { return (uint32_t)(t * Bk::ROWB + (((lane % Bk::PR) ^ raw_swz<Bk::PR>(t)) * 16)); };
    voff = piece_off((lane / Bk::PR) & 15);
    voff1 = piece_off((64 / Bk::PR + lane / Bk::PR) & 15);
    at = kv * Bk::SLOT + half * Bk::HALF;
    sc_at = kv * Bk::SLOT + 32 * Bk::ROWB + half * 16 * Bk::NB;
  }
  // tok: the quarter's first token in iteration jbase + lane
  SS_DEV void load_rows(const MxCache& c, int b, int hk, int tok) {
    const int page = min(max(c.block_table[(size_t)b * c.max_pages + min(tok >> c.page_shift, c.max_pages - 1)], 0), c.num_pages - 1);
    tab = (uint32_t)page * (uint32_t)(c.Hkv * c.page) + (uint32_t)(hk * c.page + (tok & (c.page - 1)));
  }
  // Iteration `it`'s to the block at LDS address `to`.
  SS_DEV void issue(int it, uint32_t to, int lane) const {
    const uint32_t row = __builtin_amdgcn_readlane(tab, it & 63);
    const uint8_t* const from = rows + mx_row_at(row, Bk::ROWB);
    if constexpr (Bk::HL > 0) {
#pragma unroll
      for (int i = 0; i < Bk::HL; ++i) dma16<STREAM>(from, i ? voff1 : voff, to + at + i * 1024);
    } else {
      if (lane < 32) dma16<STREAM>(from, voff, to + at);
    }
    if (lane < 4 * Bk::NB) dma4(scales + mx_row_at(row, Bk::NB), (uint32_t)(4 * lane), to + sc_at);
  }
};

// ------------------------------------------------------------------ from LDS to operands
template <int D, bool FP8>
struct MxReader {
  using Bk = MxBlock<D, FP8>;
  typedef std::conditional_t<FP8, uintx4, uintx2> Raw;  // half a block
  uint32_t k_rd, sk_rd, raw_rd, tile_wr, tr_rd;
  int vt;  // token whose values the lane turns into bf16, of block halves `vh`: with 8-byte halves neighbouring lanes share a piece
  SS_DEV explicit MxReader(int lane) {
    const int lq = lane & 15, lg = lane >> 4, vh = FP8 ? lane >> 5 : lane & 1;
    vt = FP8 ? lane & 31 : lane >> 1;
    k_rd = lq * Bk::ROWB + (((FP8 ? lg : lg % Bk::NB) ^ raw_swz<Bk::PR>(lq)) * 16);  // 16 rows further: the same swizzle
    sk_rd = 32 * Bk::ROWB + lq * Bk::NB + lg % Bk::NB;
    raw_rd = vt * Bk::ROWB + ((FP8 ? vh : 0) ^ raw_swz<Bk::PR>(vt & 15)) * 16 + (FP8 ? 0 : 8 * vh);
    tile_wr = vt * 64 + (((2 * vh) ^ tile_swz(vt)) * 16);
    const int tr_row = 4 * lg + (lq >> 2);  // 16 rows further: the same swizzle
    tr_rd = tr_row * 64 + ((((lq & 3) >> 1) ^ tile_swz(tr_row)) * 16) + (lq & 1) * 8;
  }
  SS_DEV void keys(const unsigned char* st, intx8 (&K)[2], int (&sk)[2]) const {
    const uint32_t kr = fresh(k_rd);
#pragma unroll
    for (int X = 0; X < 2; ++X) {
      sk[X] = st[sk_rd + 16 * Bk::NB * X];
      const uintx4 p0 = *reinterpret_cast<const uintx4*>(st + kr + X * Bk::HALF);
      uintx4 p1 = FP8 ? p0 : uintx4{0u, 0u, 0u, 0u};
      if constexpr (FP8 && D == 128) p1 = *reinterpret_cast<const uintx4*>(st + (kr ^ 64) + X * Bk::HALF);
      K[X] = intx8{(int)p0[0], (int)p0[1], (int)p0[2], (int)p0[3], (int)p1[0], (int)p1[1], (int)p1[2], (int)p1[3]};
    }
  }
  SS_DEV uint32_t scales(const unsigned char* st) const {
    if constexpr (Bk::NB == 4) return *reinterpret_cast<const uint32_t*>(st + 32 * Bk::ROWB + vt * 4);
    else return *reinterpret_cast<const uint16_t*>(st + 32 * Bk::ROWB + vt * 2);
  }
  SS_DEV Raw raw(int np, const unsigned char* st) const {
    return *reinterpret_cast<const Raw*>(st + (fresh(raw_rd) ^ (uint32_t)((FP8 ? 32 : 16) * np)));
  }
  // Half a block of values as bf16 into the tile.
  SS_DEV void put(int np, unsigned char* tile, Raw raw, uint32_t scales) const {
    const uint32_t wr = fresh(tile_wr);
    const float scale = mx_scale((scales >> (8 * np)) & 255u);
#pragma unroll
    for (int ch = 0; ch < 2; ++ch) {
      uintx4 o;
      if constexpr (FP8) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          o[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[2 * ch + e], scale, false));
          o[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[2 * ch + e], scale, true));
        }
      } else {
        o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[ch], scale, 0));
        o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[ch], scale, 1));
        o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[ch], scale, 2));
        o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[ch], scale, 3));
      }
      *reinterpret_cast<uintx4*>(tile + (wr ^ (16 * ch))) = o;
    }
  }
  // V^T operand of 16 features: tile's first or second.
  SS_DEV bf16x8 values(const unsigned char* tile, uint32_t rd, int dp) const {
    uintx2 half[2];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) half[hh] = lds_read_tr16(tile + 1024 * hh + (rd ^ (uint32_t)(32 * dp)));
    return as_bf16x8(uintx4{half[0][0], half[0][1], half[1][0], half[1][1]});
  }
  // Scores of 32 keys against 16 queries.
  SS_DEV void scores(const intx8 (&K)[2], const int (&sk)[2], const intx8& Qh, const intx8& Ql, int sq, floatx4 (&S)[2]) const {
#pragma unroll
    for (int X = 0; X < 2; ++X)
      S[X] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(K[X], Qh, floatx4{0.f, 0.f, 0.f, 0.f}, FP8 ? 0 : 4, 0, 0, sk[X], 0, sq);
    if constexpr (D == 128) {
#pragma unroll
      for (int X = 0; X < 2; ++X) S[X] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(K[X], Ql, S[X], FP8 ? 0 : 4, 0, 0, sk[X], 1, sq);
    }
  }
};

// Scores to probabilities, rounded to bf16; the sum takes the rounded ones.  The product with V takes bf16 operands.  A result's
// error in the 2-norm grows from 1.6e-3 to 1.7e-3, which its own rounding to bf16 makes of it, to 1.8e-3 to 2.3e-3; probabilities in
// two parts, which would leave it there, cost as many matrix instructions again as the values take, 8 of 12 per 16 rows and 32 keys.
SS_DEV bf16x8 mx_softmax(const floatx4 (&S)[2], float c, float m_run, float& l_run) {
  const float nmc = -(m_run * c);
  uintx4 P;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 p = {(__bf16)__builtin_amdgcn_exp2f(fmaf(S[i >> 1][2 * (i & 1)], c, nmc)),
                      (__bf16)__builtin_amdgcn_exp2f(fmaf(S[i >> 1][2 * (i & 1) + 1], c, nmc))};
    P[i] = __builtin_bit_cast(uint32_t, p);
    l_run = __builtin_amdgcn_fdot2_f32_bf16(p, bf16x2{(__bf16)1.f, (__bf16)1.f}, l_run, false);
  }
  return as_bf16x8(P);
}
// Running maxima: a query row's moves, and its outputs are scaled, only when one of its scores passes it by 2^16, and by its
// own scores alone.  FIRST: outputs and sums are zero.
template <int NT, int DT, bool FIRST = false>
SS_DEV void mx_raise(const floatx4 (&S)[NT][2], float c, float lazy_thr, float pinf, float (&m_run)[NT], float (&l_run)[NT], floatx4 (&O)[NT][DT]) {
  float mx[NT];
  bool any = false;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    mx[t] = max8(S[t]);
    any |= mx[t] > m_run[t] + lazy_thr;
  }
  if (__any(any)) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float of_row = max_over_lane_groups(mx[t], pinf);
      const float m_new = of_row > m_run[t] + lazy_thr ? of_row : m_run[t];
      if constexpr (!FIRST) {
        const float alpha = __builtin_amdgcn_exp2f((m_run[t] - m_new) * c);
        l_run[t] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) O[t][dt] *= alpha;
      }
      m_run[t] = m_new;
    }
  }
}
// Keys from `seen` on of a block's 32 are not there.
template <int NT>
SS_DEV void mx_mask_tail(floatx4 (&S)[NT][2], int lg, int seen) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int X = 0; X < 2; ++X)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float sv = S[t][X][i];
        S[t][X][i] = 16 * X + 4 * lg + i < seen ? sv : -INFINITY;
      }
}

// ------------------------------------------------------------------ the step's own rows
// Ancestors-or-self of node `lane`: the set doubles its reach until every path has met the root.
SS_DEV uint64_t mx_ancestors(const MsaMxArgs& a, int b, int lane) {
  const int par = a.parent[(size_t)b * a.T + min(lane, a.T - 1)];
  uint64_t anc = lane < a.T ? 1ull << lane : 1ull;
  int up = lane < a.T && lane > 0 ? clamp_parent(par, lane) : 0;
  for (bool last = false; !last;) {
    last = !__any(up > 0);
    const uint32_t lo = __shfl((uint32_t)anc, up, 64), hi = __shfl((uint32_t)(anc >> 32), up, 64);
    anc |= ((uint64_t)hi << 32) | lo;
    up = __shfl(up, up, 64);
  }
  return anc;
}
// Scores of own rows c0 .. c0 + 31 (keys in kf, features in the queries' order) against a tile's queries, masked.
template <int D>
SS_DEV void mx_own_scores(const MsaMxArgs& a, const MxItem& m, int at, int lane, uint64_t anc, int c0, const uintx4 (&kf)[2][D / 32],
                          const uintx4 (&qv)[D / 32], floatx4 (&S)[2]) {
  int r, h;
  mx_row_of(a, m, at, r, h);
  const int stream_row = r - a.T, node = stream_row < 0 ? r : fast_div(stream_row, max(a.gamma, 1));
  const uint32_t lo = __shfl((uint32_t)anc, node, 64), hi = __shfl((uint32_t)(anc >> 32), node, 64);
  const RowVis vis = make_row_vis(node, stream_row < 0 ? 0 : stream_row - node * a.gamma + 1, ((uint64_t)hi << 32) | lo, a.T, a.gamma,
                                  (a.flags & SS_STREAM_EXCLUDE_SELF) != 0);
  // bit i: the row sees key c0 + i, a main row (bits of nodes, all below T) or one of the at most 8 stream rows lo .. hi - 1
  const int s_lo = min(max(vis.lo - c0, 0), 32), s_hi = min(max(vis.hi - c0, 0), 32);
  const uint32_t bits = (c0 < 64 ? (uint32_t)(vis.anc >> c0) : 0u) | (s_lo < s_hi ? ((1u << (s_hi - s_lo)) - 1u) << s_lo : 0u);
  const int mine = (int)(bits >> (4 * (lane >> 4)));
#pragma unroll
  for (int X = 0; X < 2; ++X) {
    S[X] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) S[X] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[X][i]), as_bf16x8(qv[i]), S[X], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int seen = mine << (31 - 16 * X - i) >> 31;  // all ones or none
      S[X][i] = __int_as_float((seen & __float_as_int(S[X][i])) | (~seen & (int)0xff800000));
    }
  }
}
template <int D>
SS_DEV void mx_load_own_keys(const MsaMxArgs& a, const MxItem& m, int c0, int lane, uintx4 (&kf)[2][D / 32]) {
  const uint16_t* kn = a.k_new + ((size_t)m.b * a.R * a.c.Hkv + m.hk) * D + 16 * (lane >> 4);
#pragma unroll
  for (int X = 0; X < 2; ++X)
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      kf[X][i] = ld16(kn + min(c0 + 16 * X + (lane & 15), a.R - 1) * ((size_t)a.c.Hkv * D) + 64 * (i >> 1) + 8 * (i & 1));
}
// Values of 32 own rows, feature block np: 16 bytes of rows lane / 4 and 16 + lane / 4.
template <int D>
SS_DEV void mx_load_own_values(const MsaMxArgs& a, const MxItem& m, int c0, int np, int lane, uintx4 (&vf)[2]) {
  const uint16_t* vn = a.v_new + ((size_t)m.b * a.R * a.c.Hkv + m.hk) * D + 32 * np + 8 * (lane & 3);
#pragma unroll
  for (int i = 0; i < 2; ++i) vf[i] = ld16(vn + min(c0 + 16 * i + (lane >> 2), a.R - 1) * ((size_t)a.c.Hkv * D));
}
// Rows past the last and those of pruned nodes, which nobody has filled, become zeros: a NaN there would not be hidden by
// probabilities of zero.
SS_DEV void mx_put_own_values(const MsaMxArgs& a, const MxItem& m, int c0, int lane, unsigned char* tile, const uintx4 (&vf)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 16 * i + (lane >> 2), r = c0 + row;
    const bool kept = (r < m.n_kept) | ((r >= a.T) & (r < a.T + m.n_kept * a.gamma));
    *reinterpret_cast<uintx4*>(tile + row * 64 + (((lane & 3) ^ tile_swz(row)) * 16)) = kept ? vf[i] : uintx4{0u, 0u, 0u, 0u};
  }
}

// ------------------------------------------------------------------ results
// What one wave (unit `u` of U) holds of NT query tiles, K pieces of each (tile(t): which of the workgroup's n_tiles; dt(k): which
// 16 features), to the output or, where the sequence has several splits, to the workspace.  The wave of a unit's splits that comes
// last merges them, in index order whichever came last.  The splits run on different XCDs: partial results are stored and loaded
// coherently at device scope, and a wave announces itself only when its stores have completed.  l, mx: sum and maximum of the
// lane's query row.
template <int D, int NT, int K, class Tile, class Dt>
SS_DEV void mx_finish(const MsaMxArgs& a, const MxItem& m, int u, int U, int n_tiles, int lane, const floatx4 (&res)[NT][K], const float (&l)[NT],
                      const float (&mx)[NT], Tile tile, Dt dt) {
  const int lq = lane & 15, lg = lane >> 4;
  auto store = [&](int t, const floatx4 (&v)[K], float w) {
    int r, h;
    if (!mx_row_of(a, m, 16 * tile(t) + lq, r, h)) return;
    uint16_t* const o = a.out + (((size_t)m.b * a.R + r) * a.H + h) * D + 4 * lg;
#pragma unroll
    for (int k = 0; k < K; ++k)
      *reinterpret_cast<uintx2*>(o + 16 * dt(k)) = uintx2{pack_bf16x2(v[k][0] * w, v[k][1] * w), pack_bf16x2(v[k][2] * w, v[k][3] * w)};
  };
  float inv[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) inv[t] = l[t] > 0.f ? 1.f / l[t] : 0.f;
  if (m.n_active == 1) {
#pragma unroll
    for (int t = 0; t < NT; ++t) store(t, res[t], inv[t]);
    return;
  }
  const size_t item = ((size_t)m.b * a.c.Hkv + m.hk) * a.n_qc + m.qc;
  const int stride = U * (NT * K * 256);  // floats of a split
  float* const part = a.part_o + item * a.n_splits * stride + u * (NT * K * 256);  // [split][NT][K][64][4]
  float* const plse = a.part_lse + item * a.n_splits * (n_tiles * 16);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const bool has = m.f0 + 16 * tile(t) + lq < m.F;  // (nobody reads the others' results)
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (has) st16_device(part + (size_t)m.s * stride + (t * K + k) * 256 + lane * 4, res[t][k] * inv[t]);
    if (lg == 0 && has) st4_device(plse + m.s * (n_tiles * 16) + 16 * tile(t) + lq, mx[t] * a.scale_log2 + __log2f(l[t]));  // (waves of one tile write the same)
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  unsigned int* const ctr = a.arrive + item * U + u;
  unsigned int seen = 0;
  if (lane == 0) seen = atomicAdd(ctr, 1u);
  if (__builtin_amdgcn_readfirstlane(seen) + 1 != (unsigned)m.n_active) return;
  constexpr int AHEAD = K == 8 ? 2 : 4;  // splits whose results are asked for at once, its own (kept they cost too many registers) among them
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    floatx4 acc[K];
    float M = -INFINITY, wsum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) acc[k] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int sp = 0; sp < m.n_active; sp += AHEAD) {
      floatx4 o[AHEAD][K];
      float lo[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int from = sp + i;
        if (from >= m.n_active) break;
        lo[i] = ld4_device(plse, (uint32_t)((from * n_tiles + tile(t)) * 64 + lq * 4));
#pragma unroll
        for (int k = 0; k < K; ++k) o[i][k] = ld16_device(part + (size_t)from * stride, (uint32_t)((t * K + k) * 1024 + lane * 16));
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (sp + i >= m.n_active) break;
        const bool use = lo[i] != -INFINITY;  // (a NaN counts)
        const float m_new = use ? fmaxf(M, lo[i]) : M;
        const float keep = use ? exp2f(M - m_new) : 1.f, wt = use ? exp2f(lo[i] - m_new) : 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[k][e] = use ? __builtin_fmaf(o[i][k][e], wt, acc[k][e] * keep) : acc[k][e];
        wsum = __builtin_fmaf(wsum, keep, wt);
        M = m_new;
      }
    }
    store(t, acc, wsum > 0.f ? 1.f / wsum : 0.f);
  }
  if (lane == 0) st_counter_device(ctr, 0u);  // the next call finds the counters zero again
}

// Launches; the plan's shape: query tiles per wave, waves that share keys (1: none).
struct MxKernel {
  int nt, nw;
};
int launch_msa_mx(const MsaMxArgs& a, MxKernel k, bool fp8, long wgs, hipStream_t st);
int launch_msa_mx_rows(const MsaMxArgs& a, MxKernel k, bool fp8, long wgs, hipStream_t st);

}  // namespace ss
