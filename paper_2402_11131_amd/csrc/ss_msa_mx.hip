// n5, a2 over a cache in microscaling formats: multi-stream attention (Eq. 1 / Eq. 2) on the gfx950 matrix cores.
//
// Work split.  A workgroup of four wavefronts owns one (sequence, KV head, split of the cached tokens, chunk of up to 16 NT
// query rows; the query heads of a group are folded into the rows).  Every wave holds ALL of the chunk's rows (queries, running
// maximum and sum, outputs in registers) and walks blocks of 32 keys of its own: what is done once per key, above all turning
// values into bf16, is then done by one wave only, and the waves need nothing from each other until their results are merged.
//
// Memory pipeline.  Every wave has a ring of stages in LDS, each a block's raw bytes: keys, values, scales.  Direct
// global-to-LDS loads fill them; a wave waits for its own loads by count and nobody waits at a barrier.  Rows lie in a stage as
// in the page, their 16-byte pieces XOR-swizzled by the lane -> address mapping so that operand reads meet every bank once.
//
// Scores, S^T = K Q^T with v_mfma_scale_f32_16x16x128_f8f6f4: the cached elements and scale bytes are operands as they are.  A
// query row is the sum of two e4m3 rows, the second with a scale 2^-4 of the first's: four and four of a bf16 value's eight
// significant bits (features below 2^-17 of the row's largest lose bits, none more than 2^-22 of it).  Lane (lq, lg) = (lane &
// 15, lane >> 4) supplies, of a 4-bit operand, elements 32 lg .. +31 of row lq, of an 8-bit one elements 16 lg .. +15 and 64 +
// 16 lg .. +15; the scale of elements 32 g .. +31 comes from lane group g.  Heads of 128 take two instructions (one per part)
// for 16 keys and 16 queries; heads of 64 one, with the first part against elements 0..63 and the second against a repetition.
//
// O^T += V^T P^T with v_mfma_f32_16x16x32_bf16.  A scale belongs to one token, and the sum runs over tokens, so values are
// multiplied by their scales first: both formats are exact in bf16.  FB features at a time, a lane turns a piece of one token's
// row into bf16 and puts it into the wave's LDS tile (token-major, swizzled); the transposing read hands out four consecutive
// tokens of a feature.
#include <math.h>

#include <type_traits>

#include "ss_msa_mfma.h"
#include "ss_mx.h"

namespace ss {

struct MsaMxArgs {
  const uint16_t *q, *k_new, *v_new;
  uint16_t* out;
  MxCache c;
  const int32_t *seq_lens, *parent, *n_nodes;
  float* part_o;    // [items, n_splits, rows, D]: a split's outputs divided by its own sum
  float* part_lse;  // [items, n_splits, rows]: log2-domain log-sum-exp
  unsigned int* arrive;  // [items]: splits that have arrived; zero before the call, zero again after it
  int B, T, gamma, R, H, g, n_splits, n_qc;
  float scale_log2;
  uint32_t flags;
};

constexpr int kMxWaves = 4;
constexpr int kMxMinSplit = 256;  // cached tokens of the shortest split
constexpr float kMxLazyLog2 = 16.0f;

// Tokens per split of a sequence of L.
SS_HD int mx_split_len(int L, int n_splits) {
  const int even = (L + n_splits - 1) / n_splits, up = (even + 127) & ~127;
  return up < kMxMinSplit ? kMxMinSplit : up;
}

// Sizes of one instance.
template <int D, bool FP8, int NT>
struct MxShape {
  static constexpr int DT = D / 16, KS = D / 32, NB = D / kMxBlock;
  static constexpr int ROWB = FP8 ? D : D / 2;               // bytes of a cached row
  static constexpr int PR = ROWB / 16;                       // 16-byte pieces of a row
  static constexpr int HALF = 16 * ROWB;                     // bytes of 16 rows: they share a page and are contiguous there
  static constexpr int HL = HALF / 1024 ? HALF / 1024 : 1;   // loads of a half (32-byte rows: one load takes both halves)
  static constexpr int ROWS_LOADS = HALF / 1024 ? 2 * HL : 1;  // loads of 32 rows
  static constexpr int LPU = 2 * ROWS_LOADS + 1;             // loads of a block: keys, values, scales
  static constexpr int STAGE = 2 * 32 * ROWB + 256;
  static constexpr int FB = FP8 ? 32 : 64;                   // features of a value tile: two pieces of a row
  static constexpr int TILE = 32 * FB * 2;
  // three workgroups per compute unit with one query tile and 4-bit rows, else two
  static constexpr int BUDGET = (NT == 1 && !(FP8 && D == 128) ? 53 : 79) * 1024 / kMxWaves;
  static constexpr int DEPTH = (BUDGET - TILE) / STAGE > 6 ? 6 : (BUDGET - TILE) / STAGE;
  static constexpr int WAVE_LDS = TILE + DEPTH * STAGE;
  static constexpr int MERGE = NT * DT * 1024;               // bytes of a wave's outputs
  static constexpr int LDS = kMxWaves * WAVE_LDS > 2 * MERGE ? kMxWaves * WAVE_LDS : 2 * MERGE;
  static constexpr int WAVES_PER_SIMD = NT == 1 && !(FP8 && D == 128) ? 3 : 2;
  static_assert(DEPTH >= 2, "a block in flight while another is computed");
};

// Piece of a raw row that lies at piece position p of row t is p ^ raw_swz(t): 16 rows' pieces of one index meet all banks.
template <int PR>
SS_DEV int raw_swz(int t) { return (t / (16 / PR)) & (PR - 1); }
// 16-byte chunk of a row of the value tile where chunk c lies is c ^ tile_swz(row).  Writes take one chunk of 16 consecutive
// rows, transposing reads pieces of two neighbouring chunks of eight rows: both meet every bank once.
template <int FB>
SS_DEV int tile_swz(int row) {
  return FB == 64 ? ((((row >> 1) & 3) << 1) | ((row >> 3) & 1)) : ((((row >> 2) & 1) << 1) | ((row >> 3) & 1));
}
// 4 bytes per lane straight into LDS, lane l's at lds_addr + 4*l.
SS_DEV void dma4(const void* p, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(p), "s"(lds_addr) : "memory", "m0");
}
// Maximum of three as one instruction; a NaN wins.
SS_DEV float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

template <int D, bool FP8, int NT>
__global__ __launch_bounds__(64 * kMxWaves, (MxShape<D, FP8, NT>::WAVES_PER_SIMD)) void msa_mx_kernel(MsaMxArgs a) {
  using Sh = MxShape<D, FP8, NT>;
  constexpr int DT = Sh::DT, KS = Sh::KS, NB = Sh::NB, ROWB = Sh::ROWB, PR = Sh::PR, FB = Sh::FB, STAGE = Sh::STAGE, DEPTH = Sh::DEPTH;
  constexpr int NP = D / FB, DTP = FB / 16;        // passes over the features, feature tiles of a pass
  __shared__ __attribute__((aligned(1024))) unsigned char smem[Sh::LDS];
  __shared__ float ml[kMxWaves][NT][2][16];
  __shared__ unsigned int seen_s;

  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // XCD-aware order: the row chunks of one (sequence, KV head, split) get workgroup ids that are equal mod 8 and share an L2
  const int G = a.B * a.c.Hkv * a.n_splits;
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const int qc = slot % a.n_qc, group = (slot / a.n_qc) * 8 + xcd;
  if (group >= G) return;
  const int s = group % a.n_splits, head = group / a.n_splits, b = head / a.c.Hkv, hk = head - b * a.c.Hkv;
  const int cap = a.c.max_pages * a.c.page;
  const int L = min(max(a.seq_lens[b], 0), cap);
  const int n_kept = a.n_nodes ? min(max(a.n_nodes[b], 1), a.T) : a.T;
  const int R_kept = n_kept * (1 + a.gamma), F = a.g * R_kept, f0 = qc * 16 * NT;
  if (f0 >= F) return;
  const int split = mx_split_len(L, a.n_splits), n_active = L <= split ? 1 : (L + split - 1) / split;
  if (s >= n_active) return;
  const int k0 = s * split, k1 = min(L, k0 + split);

  // ---- blocks of this wave: w, w + 4, ... of the split's; the ids of their pages (of both 16-token halves: a page may be that
  // small), lane i those of iteration jbase + i
  const int n_full = (k1 - k0) >> 5, n_units = (k1 - k0 + 31) >> 5;
  const int n_mine = w < n_units ? (n_units - w + kMxWaves - 1) / kMxWaves : 0;
  const int32_t* my_table = a.c.block_table + (size_t)b * a.c.max_pages;
  uint32_t tab_a = 0, tab_b = 0;
  auto load_pages = [&](int jbase) {
    const int kb = k0 + 32 * (w + (jbase + lane) * kMxWaves);
    tab_a = (uint32_t)min(max(my_table[min(kb >> a.c.page_shift, a.c.max_pages - 1)], 0), a.c.num_pages - 1);
    tab_b = (uint32_t)min(max(my_table[min((kb + 16) >> a.c.page_shift, a.c.max_pages - 1)], 0), a.c.num_pages - 1);
  };
  load_pages(0);

  unsigned char* const mine = smem + w * Sh::WAVE_LDS;  // tile, then stages
  unsigned char* const tile = mine;
  const uint32_t lds_stage0 = (uint32_t)(uintptr_t)mine + Sh::TILE;
  const uint32_t page_rows = (uint32_t)(a.c.Hkv * a.c.page);  // rows of a page, all heads
  const uint32_t raw_voff = [&]() {  // bytes of this lane's piece from the base of 1024 bytes of rows
    const int t = lane / PR, p = lane % PR;
    return (uint32_t)(t * ROWB + ((p ^ raw_swz<PR>(t)) * 16));
  }();
  // second load of a half, where there are two: other rows, another swizzle
  const uint32_t raw_voff1 = [&]() {
    const int t = 64 / PR + lane / PR, p = lane % PR;
    return (uint32_t)(t * ROWB + ((p ^ raw_swz<PR>(t)) * 16));
  }();
  // the scales: lane l's dword is that of token (4 / NB) * (l mod n) of the block, keys' first, then values'
  constexpr int SN = 32 * NB / 4;  // dwords of the keys' scales
  const int sc_tok = (lane % SN) * (4 / NB);
  const uint8_t* const sc_base = (((lane / SN) & 1) ? a.c.vs : a.c.ks) + ((size_t)hk * a.c.page + (sc_tok & 15)) * NB;

  auto issue = [&](int it, int stage) {
    const int j = it & 63;
    const uint32_t pa = __builtin_amdgcn_readlane(tab_a, j), pb = __builtin_amdgcn_readlane(tab_b, j);
    const int kb = k0 + 32 * (w + it * kMxWaves);
    const uint32_t sa = (uint32_t)(kb & (a.c.page - 1)), sb = (uint32_t)((kb + 16) & (a.c.page - 1));
    const size_t ra = (size_t)pa * page_rows + (uint32_t)hk * a.c.page + sa, rb = (size_t)pb * page_rows + (uint32_t)hk * a.c.page + sb;
    const uint32_t at = lds_stage0 + (uint32_t)stage * STAGE;
    if constexpr (Sh::HALF >= 1024) {
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const uint8_t* base = kv ? a.c.v : a.c.k;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < Sh::HL; ++i)
            dma16<true>(base + (half ? rb : ra) * ROWB, i ? raw_voff1 : raw_voff, at + (kv * 2 + half) * Sh::HALF + i * 1024);
      }
    } else {  // 32 rows of 32 bytes in one load: lanes 32.. take the second half
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const uint8_t* base = kv ? a.c.v : a.c.k;
        const size_t r = lane < 32 ? ra : rb;
        const uint8_t* p = base + r * ROWB + (raw_voff & (Sh::HALF - 1));
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(p), "s"(at + kv * 1024) : "memory", "m0");
      }
    }
    const uint32_t pg = sc_tok < 16 ? pa : pb, off = (sc_tok < 16 ? sa : sb) * NB;
    dma4(sc_base + ((size_t)pg * page_rows * NB + off), at + 2 * 32 * ROWB);
  };

  // query row of tile t that this lane's column lq is
  auto row_of = [&](int t, int& r, int& h) {
    const int f = min(f0 + 16 * t + lq, F - 1);
    const int fh = fast_div(f, R_kept), fr = f - fh * R_kept;
    r = fr < n_kept ? fr : a.T + (fr - n_kept);
    h = hk * a.g + fh;
    return f0 + 16 * t + lq < F;
  };

#pragma unroll
  for (int i = 0; i < DEPTH; ++i)
    if (i < n_mine) issue(i, i);

  floatx4 O[NT][DT];
  float m_run[NT], l_run[NT];  // maximum of the query row, sum of this lane's probabilities
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m_run[t] = -1e30f;
    l_run[t] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[t][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const float c = a.scale_log2, lazy_thr = kMxLazyLog2 / c;
  float pinf = INFINITY;  // see vmax2
  asm volatile("" : "+s"(pinf));

  // Running maxima: a query row's moves, and its outputs are scaled, only when one of its scores passes it by 2^16, and by its
  // own scores alone.  Tiles t0 .. t1 - 1.
  auto raise = [&](int t0, int t1, const floatx4 (&S)[NT][2]) {
    float mx[NT];
    bool any = false;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t < t0 || t >= t1) continue;
      mx[t] = max3(max3(max3(S[t][0][0], S[t][0][1], S[t][0][2]), S[t][0][3], S[t][1][0]), max3(S[t][1][1], S[t][1][2], S[t][1][3]), S[t][1][3]);
      any |= mx[t] > m_run[t] + lazy_thr;
    }
    if (__any(any)) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (t < t0 || t >= t1) continue;
        const float of_row = max_over_lane_groups(mx[t], pinf);
        const float m_new = of_row > m_run[t] + lazy_thr ? of_row : m_run[t];
        const float alpha = __builtin_amdgcn_exp2f((m_run[t] - m_new) * c);
        l_run[t] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) O[t][dt] *= alpha;
        m_run[t] = m_new;
      }
    }
  };
  // scores to probabilities, rounded to bf16; the sum takes the rounded ones
  auto softmax = [&](int t, const floatx4 (&S)[2]) {
    const float nmc = -(m_run[t] * c);
    uintx4 P;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 p = {(__bf16)__builtin_amdgcn_exp2f(fmaf(S[i >> 1][2 * (i & 1)], c, nmc)),
                        (__bf16)__builtin_amdgcn_exp2f(fmaf(S[i >> 1][2 * (i & 1) + 1], c, nmc))};
      P[i] = __builtin_bit_cast(uint32_t, p);
      l_run[t] = __builtin_amdgcn_fdot2_f32_bf16(p, bf16x2{(__bf16)1.f, (__bf16)1.f}, l_run[t], false);
    }
    return as_bf16x8(P);
  };
  // O += P V for the features of pass `np`, whose values are in the tile.  A lane's probabilities are those of tokens 4 lg .. +3
  // of either half of the block.
  const int tr_row = 4 * lg + (lq >> 2);  // 16 rows further: the same swizzle
  const uint32_t tr_rd = tr_row * (2 * FB) + ((((lq & 3) >> 1) ^ tile_swz<FB>(tr_row)) * 16) + (lq & 1) * 8;
  auto add_values = [&](int np, const bf16x8 (&P)[NT]) {
    uint32_t rd = tr_rd;
    asm volatile("" : "+v"(rd));  // the addresses are formed here and not kept in registers across the loop
#pragma unroll
    for (int dp = 0; dp < DTP; ++dp) {
      uintx2 half[2];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) half[hh] = lds_read_tr16(tile + 32 * FB * hh + (rd ^ (32 * dp)));
      const bf16x8 vv = as_bf16x8(uintx4{half[0][0], half[0][1], half[1][0], half[1][1]});
#pragma unroll
      for (int t = 0; t < NT; ++t) O[t][np * DTP + dp] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, P[t], O[t][np * DTP + dp], 0, 0, 0);
    }
  };
  // the wave's own LDS accesses stay in this order (they complete in it)
  auto in_order = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };

  // ---- the step's own rows (split 0, which every sequence has), while the first blocks are on their way
  if (s == 0) {
    const int par = a.parent[(size_t)b * a.T + min(lane, a.T - 1)], par_c = lane < a.T ? clamp_parent(par, lane) : -1;
    for (int c0 = 32 * w; c0 < a.R; c0 += 32 * kMxWaves) {
      const size_t own0 = ((size_t)b * a.R * a.c.Hkv + hk) * D;  // row 0 of this head
      const size_t stride = (size_t)a.c.Hkv * D;
      uintx4 kf[2][KS];
#pragma unroll
      for (int X = 0; X < 2; ++X)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          kf[X][ks] = ld16(a.k_new + own0 + min(c0 + 16 * X + lq, a.R - 1) * stride + 32 * ks + 8 * lg);
      bf16x8 P[NT];
      floatx4 S[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        int r, h;
        row_of(t, r, h);
        const int node = r < a.T ? r : (r - a.T) / max(a.gamma, 1), strm = r < a.T ? 0 : (r - a.T) % max(a.gamma, 1) + 1;
        const RowVis vis = make_row_vis(node, strm, ancestors_of(node, par_c), a.T, a.gamma, (a.flags & SS_STREAM_EXCLUDE_SELF) != 0);
        const uint16_t* qp = a.q + (((size_t)b * a.R + r) * a.H + h) * D + 8 * lg;
#pragma unroll
        for (int X = 0; X < 2; ++X) S[t][X] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 qv = as_bf16x8(ld16(qp + 32 * ks));
#pragma unroll
          for (int X = 0; X < 2; ++X) S[t][X] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[X][ks]), qv, S[t][X], 0, 0, 0);
        }
#pragma unroll
        for (int X = 0; X < 2; ++X)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = c0 + 16 * X + 4 * lg + i;
            const float sv = S[t][X][i];
            S[t][X][i] = (key < a.R) & row_sees(vis, key, a.T) ? sv : -INFINITY;
          }
        raise(t, t + 1, S);
        P[t] = softmax(t, S[t]);
      }
      constexpr int CPR = FB / 8, RPL = 64 / CPR;  // chunks per row of the tile, rows per load
#pragma unroll
      for (int np = 0; np < NP; ++np) {
        in_order();
#pragma unroll
        for (int i = 0; i < 32 / RPL; ++i) {
          const int row = RPL * i + lane / CPR, ch = lane % CPR;
          const uintx4 v = ld16(a.v_new + own0 + min(c0 + row, a.R - 1) * stride + FB * np + 8 * ch);
          *reinterpret_cast<uintx4*>(tile + row * (2 * FB) + ((ch ^ tile_swz<FB>(row)) * 16)) = c0 + row < a.R ? v : uintx4{0u, 0u, 0u, 0u};
        }
        in_order();
        add_values(np, P);
      }
    }
  }

  // ---- queries as two e4m3 rows each
  intx8 Qh[NT], Ql[D == 128 ? NT : 1];
  int sq[NT];  // scale bytes: of the first part, then of the second (heads of 64: this lane's)
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    int r, h;
    row_of(t, r, h);
    const uint16_t* qp = a.q + (((size_t)b * a.R + r) * a.H + h) * D + 16 * lg;
    constexpr int N = D == 128 ? 2 : 1;  // runs of 16 features
    uintx4 raw[2 * N];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) {
      raw[i] = ld16(qp + 64 * (i >> 1) + 8 * (i & 1));
#pragma unroll
      for (int e = 0; e < 4; ++e) m = max(max(m, raw[i][e] & 0x7fffu), (raw[i][e] >> 16) & 0x7fffu);
    }
    m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
    const int sh = mx_scale_code<true>(m << 16), sl = sh == 255 ? 255 : max(sh - 4, 0);
    const float fh = mx_scale(sh), fl = mx_scale(sl);
    uint32_t hi[4 * N], lo[4 * N];
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
      shortx2 ph = {0, 0}, pl = {0, 0};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t two = raw[i >> 1][2 * (i & 1) + e];
        const bf16x2 x = __builtin_bit_cast(bf16x2, sh == 255 ? 0u : two);
        ph = e ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(ph, x, fh, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(ph, x, fh, false);
        const uint32_t pw = __builtin_bit_cast(uint32_t, ph);
        const floatx2 back = e ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(pw, fh, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(pw, fh, false);
        const float r0 = (float)x[0] - back[0], r1 = (float)x[1] - back[1];
        pl = e ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(pl, r0, r1, fl, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(pl, r0, r1, fl, false);
      }
      hi[i] = __builtin_bit_cast(uint32_t, ph);
      lo[i] = sh == 255 ? 0u : __builtin_bit_cast(uint32_t, pl);
    }
    if constexpr (D == 128) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        Qh[t][i] = (int)hi[i];
        Ql[t][i] = (int)lo[i];
      }
      sq[t] = sh | (sl << 8);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        Qh[t][i] = (int)hi[i];
        Qh[t][4 + i] = (int)lo[i];
      }
      sq[t] = lg < 2 ? sh : sl;
    }
  }

  // ---- the cached tokens
  const int k_rd = lq * ROWB, k_sw = raw_swz<PR>(lq);  // 16 rows further: the same swizzle
  const int vt = lane & 31, vp = lane >> 5;            // token, and which of a pass' pieces, of the lane's values
  constexpr int VCH = FP8 ? 2 : 4;                     // chunks of the tile that a piece gives
  const uint32_t tile_wr = vt * (2 * FB) + (((vp * VCH) ^ tile_swz<FB>(vt)) * 16);
  auto block = [&](auto full, int nv, const unsigned char* st) {
    constexpr bool FULL = decltype(full)::value;
    const unsigned char* sc = st + 2 * 32 * ROWB;
    floatx4 S[NT][2];
#pragma unroll
    for (int X = 0; X < 2; ++X) {
      const unsigned char* kr = st + X * Sh::HALF + k_rd;
      const int sk = sc[(16 * X + lq) * NB + lg % NB];
      const uintx4 p0 = *reinterpret_cast<const uintx4*>(kr + (((FP8 ? lg : lg % NB) ^ k_sw) * 16));
      uintx4 p1 = FP8 ? p0 : uintx4{0u, 0u, 0u, 0u};
      if constexpr (FP8 && D == 128) p1 = *reinterpret_cast<const uintx4*>(kr + (((4 + lg) ^ k_sw) * 16));
      const intx8 K = {(int)p0[0], (int)p0[1], (int)p0[2], (int)p0[3], (int)p1[0], (int)p1[1], (int)p1[2], (int)p1[3]};
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        floatx4 acc = floatx4{0.f, 0.f, 0.f, 0.f};
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(K, Qh[t], acc, FP8 ? 0 : 4, 0, 0, sk, 0, sq[t]);
        if constexpr (D == 128) acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(K, Ql[t], acc, FP8 ? 0 : 4, 0, 0, sk, 1, sq[t]);
        S[t][X] = acc;
      }
    }
    // values of pass np into the tile
    auto put_values = [&](int np) {
      const int piece = (FB / 16) / (FP8 ? 1 : 2) * np + vp;  // of the row
      const int blk = FP8 ? piece >> 1 : piece;
      uint32_t wr = tile_wr;
      asm volatile("" : "+v"(wr));
      uintx4 raw = *reinterpret_cast<const uintx4*>(st + 32 * ROWB + vt * ROWB + ((piece ^ raw_swz<PR>(vt & 15)) * 16));
      uint32_t code = sc[32 * NB + vt * NB + blk];
      if (!FULL) {  // what lies behind the sequence must not be NaN
        const bool ok = vt < nv;
        raw = ok ? raw : uintx4{0u, 0u, 0u, 0u};
        code = ok ? code : 127u;
      }
      const float scale = mx_scale((int)code);
#pragma unroll
      for (int ch = 0; ch < VCH; ++ch) {
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
    };
    in_order();
    put_values(0);
    bf16x8 P[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (!FULL) {
#pragma unroll
        for (int X = 0; X < 2; ++X)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float sv = S[t][X][i];
            S[t][X][i] = 16 * X + 4 * lg + i < nv ? sv : -INFINITY;
          }
      }
    }
    raise(0, NT, S);
#pragma unroll
    for (int t = 0; t < NT; ++t) P[t] = softmax(t, S[t]);
    in_order();
    add_values(0, P);
#pragma unroll
    for (int np = 1; np < NP; ++np) {
      in_order();
      put_values(np);
      in_order();
      add_values(np, P);
    }
  };

  {
    const int n_whole = w < n_full ? (n_full - w + kMxWaves - 1) / kMxWaves : 0;  // n_mine, or one less: the ragged block is the last
    int stage = 0;
    for (int it = 0; it < n_whole; ++it) {
      wait_vm_units<Sh::LPU>(min(n_mine - 1 - it, DEPTH - 1));
      block(std::true_type{}, 32, mine + Sh::TILE + stage * STAGE);
      if (it + DEPTH < n_mine) {
        if (((it + DEPTH) & 63) == 0) load_pages(it + DEPTH);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage has been read
        issue(it + DEPTH, stage);
      }
      stage = stage + 1 == DEPTH ? 0 : stage + 1;
    }
    if (n_whole < n_mine) {
      wait_vmcnt<0>();
      block(std::false_type{}, (k1 - k0) & 31, mine + Sh::TILE + stage * STAGE);
    }
  }

  // ---- merge the waves: to a common maximum, then pairs of waves through LDS
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    l_run[t] += __shfl_xor(l_run[t], 16, 64);
    l_run[t] += __shfl_xor(l_run[t], 32, 64);
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
    if (lg == 0) {
      ml[w][t][0][lq] = m_run[t];
      ml[w][t][1][lq] = l_run[t];
    }
  __syncthreads();
  float l_tot[NT], m_tot[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float mm = ml[0][t][0][lq];
#pragma unroll
    for (int i = 1; i < kMxWaves; ++i) mm = fmaxf(mm, ml[i][t][0][lq]);
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < kMxWaves; ++i) l = fmaf(ml[i][t][1][lq], __builtin_amdgcn_exp2f((ml[i][t][0][lq] - mm) * c), l);
    const float fac = __builtin_amdgcn_exp2f((m_run[t] - mm) * c);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[t][dt] *= fac;
    l_tot[t] = l;
    m_tot[t] = mm;
  }
  floatx4* buf = reinterpret_cast<floatx4*>(smem);
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    __syncthreads();
    if (w >= half && w < 2 * half) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) buf[((w - half) * NT * DT + t * DT + dt) * 64 + lane] = O[t][dt];
    }
    __syncthreads();
    if (w < half) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) O[t][dt] += buf[(w * NT * DT + t * DT + dt) * 64 + lane];
    }
  }

  // ---- normalise and store: a lane holds features 16 dt + 4 lg .. +3 of its query rows
  const int item = (b * a.c.Hkv + hk) * a.n_qc + qc;
  if (w == 0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      int r, h;
      const bool ok = row_of(t, r, h);
      const float inv = l_tot[t] > 0.f ? 1.f / l_tot[t] : 0.f;
      if (n_active == 1) {
        uint16_t* op = a.out + (((size_t)b * a.R + r) * a.H + h) * D + 4 * lg;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const floatx4 v = O[t][dt] * inv;
          if (ok) *reinterpret_cast<uintx2*>(op + 16 * dt) = uintx2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        }
      } else {
        const size_t pr = ((size_t)item * a.n_splits + s) * (16 * NT) + 16 * t + lq;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) st16_device(a.part_o + pr * D + 16 * dt + 4 * lg, O[t][dt] * inv);
        if (lg == 0) st4_device(a.part_lse + pr, m_tot[t] * c + __log2f(l_tot[t]));
      }
    }
  }
  if (n_active == 1) return;

  // ---- the workgroup of the sequence's splits that comes last merges them, in index order whichever came last.  The splits run
  // on different XCDs: partial rows are stored and loaded coherently at device scope, and a workgroup announces itself only
  // when its stores have completed.
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __syncthreads();
  if (tid == 0) seen_s = atomicAdd(a.arrive + item, 1u);
  __syncthreads();
  if (seen_s + 1 != (unsigned)n_active) return;
  constexpr int DQ = D / 4;
  for (int i = tid; i < 16 * NT * DQ; i += 64 * kMxWaves) {
    const int row = i / DQ, d0 = (i % DQ) * 4, f = f0 + row;
    if (f >= F) continue;
    float M = -INFINITY, wsum = 0.f;
    floatx4 acc = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int sp = 0; sp < n_active; ++sp) {
      const size_t pr = ((size_t)item * a.n_splits + sp) * (16 * NT) + row;
      float l;
      floatx4 o[1];
      ld_row_device<1>(a.part_lse + pr, a.part_o + pr * D + d0, l, o);
      if (l == -INFINITY) continue;
      const float m_new = fmaxf(M, l), keep = exp2f(M - m_new), wt = exp2f(l - m_new);
      acc = merge_step(acc, keep, o[0], wt);
      wsum = __builtin_fmaf(wsum, keep, wt);
      M = m_new;
    }
    const int fh = fast_div(f, R_kept), fr = f - fh * R_kept, r = fr < n_kept ? fr : a.T + (fr - n_kept);
    const float inv = wsum > 0.f ? 1.f / wsum : 0.f;
    const floatx4 v = acc * inv;
    *reinterpret_cast<uintx2*>(a.out + (((size_t)b * a.R + r) * a.H + hk * a.g + fh) * D + d0) = uintx2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  }
  if (tid == 0) st_counter_device(a.arrive + item, 0u);  // the next call finds the counters zero again
}

// ------------------------------------------------------------------ planning (host)
struct MxPlan {
  int nt, n_qc, n_splits;
  size_t part_o_at, part_lse_at, total_bytes;
};

static MxPlan mx_plan(int B, int R, int H, int Hkv, int D, int max_len) {
  MxPlan p;
  const int F = (H / Hkv) * R, tiles = ceil_div(F, 16);
  p.n_qc = ceil_div(tiles, 3);
  p.nt = ceil_div(tiles, p.n_qc);
  const long items = (long)B * Hkv * p.n_qc;
  const int len = max_len < 1 ? 1 : max_len;
  const int resident = p.nt == 1 ? 768 : 512;  // workgroups that the chip holds
  long n = (resident + items - 1) / (items < 1 ? 1 : items);
  const int most = ceil_div(len, kMxMinSplit);
  if (n > most) n = most;
  if (n < 1 || items * sizeof(unsigned int) > kArriveRegionBytes) n = 1;
  p.n_splits = (int)n;
  p.part_o_at = p.part_lse_at = 0;
  p.total_bytes = 256;  // to align the start
  if (p.n_splits > 1) {
    const size_t rows = (size_t)items * p.n_splits * 16 * p.nt;
    p.part_o_at = kArriveRegionBytes;
    p.part_lse_at = p.part_o_at + align_up(rows * D * sizeof(float), 256);
    p.total_bytes += p.part_lse_at + align_up(rows * sizeof(float), 256);
  }
  return p;
}

static int mx_check_shape(const char* fn, int B, int T, int gamma, int H, int Hkv, int D) {
  SS_REQUIRE(B >= 0 && B <= 65535, SS_ERR_INVALID_ARG, "%s: B=%d", fn, B);
  SS_REQUIRE(T >= 1 && T <= SS_MAX_T, SS_ERR_UNSUPPORTED, "%s: T=%d outside [1,%d]", fn, T, SS_MAX_T);
  SS_REQUIRE(gamma >= 0 && gamma <= SS_MAX_GAMMA, SS_ERR_UNSUPPORTED, "%s: gamma=%d outside [0,%d]", fn, gamma, SS_MAX_GAMMA);
  SS_REQUIRE(H >= 1 && Hkv >= 1 && H % Hkv == 0, SS_ERR_INVALID_ARG, "%s: H=%d must be a multiple of Hkv=%d", fn, H, Hkv);
  SS_REQUIRE(D == 64 || D == 128, SS_ERR_UNSUPPORTED, "%s: head dim %d not in {64,128}", fn, D);
  SS_REQUIRE(H / Hkv <= 4096, SS_ERR_UNSUPPORTED, "%s: %d query heads per KV head", fn, H / Hkv);
  return SS_OK;
}

template <int D, bool FP8>
static void launch_nt(int nt, unsigned wgs, hipStream_t st, const MsaMxArgs& a) {
  auto kern = nt == 1 ? msa_mx_kernel<D, FP8, 1> : nt == 2 ? msa_mx_kernel<D, FP8, 2> : msa_mx_kernel<D, FP8, 3>;
  hipLaunchKernelGGL(kern, dim3(wgs), dim3(64 * kMxWaves), 0, st, a);
}

}  // namespace ss

extern "C" {

size_t ss_msa_mx_workspace_bytes(int B, int T, int gamma, int H, int Hkv, int D, int max_seq_len) {
  ss::clear_error();
  if (ss::mx_check_shape("ss_msa_mx_workspace_bytes", B, T, gamma, H, Hkv, D) != SS_OK) return 0;
  return ss::mx_plan(B, T * (1 + gamma), H, Hkv, D, max_seq_len).total_bytes;
}

int ss_msa_mx_plan(int B, int T, int gamma, int H, int Hkv, int D, int max_seq_len, int* n_splits, int* rows_per_workgroup) {
  ss::clear_error();
  if (int rc = ss::mx_check_shape("ss_msa_mx_plan", B, T, gamma, H, Hkv, D)) return rc;
  const ss::MxPlan p = ss::mx_plan(B, T * (1 + gamma), H, Hkv, D, max_seq_len);
  if (n_splits) *n_splits = p.n_splits;
  if (rows_per_workgroup) *rows_per_workgroup = 16 * p.nt;
  return SS_OK;
}

int ss_msa_attention_mx(const void* q, const void* k_new, const void* v_new, const void* k_cache, const void* k_scale,
                        const void* v_cache, const void* v_scale, const int32_t* block_table, int max_pages_per_seq, int num_pages,
                        const int32_t* seq_lens, const int32_t* parent, const int32_t* n_nodes, int B, int T, int gamma, int H, int Hkv,
                        int D, int page_size, float scale, int format, uint32_t flags, void* out, void* workspace, size_t workspace_bytes,
                        void* stream) {
  using namespace ss;
  clear_error();
  const char* fn = "ss_msa_attention_mx";
  if (int rc = mx_check_shape(fn, B, T, gamma, H, Hkv, D)) return rc;
  if (int rc = mx_check(fn, Hkv, D, page_size, max_pages_per_seq, num_pages, format, k_cache, k_scale, v_cache, v_scale, block_table, B > 0)) return rc;
  SS_REQUIRE(scale > 0.f && isfinite(scale), SS_ERR_INVALID_ARG, "%s: scale must be positive and finite", fn);
  SS_REQUIRE((flags & ~SS_STREAM_EXCLUDE_SELF) == 0, SS_ERR_INVALID_ARG, "%s: unknown flags 0x%x", fn, flags);
  if (B == 0) return SS_OK;
  SS_REQUIRE(q && k_new && v_new && seq_lens && parent && out, SS_ERR_INVALID_ARG, "%s: NULL tensor argument", fn);
  SS_REQUIRE((((uintptr_t)q | (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)out) & 15) == 0, SS_ERR_INVALID_ARG,
             "%s: q, k_new, v_new or out not aligned to 16 bytes", fn);
  const int R = T * (1 + gamma);
  const MxPlan plan = mx_plan(B, R, H, Hkv, D, max_pages_per_seq * page_size);
  SS_REQUIRE(plan.n_splits == 1 || (workspace != nullptr && workspace_bytes >= plan.total_bytes), SS_ERR_WORKSPACE,
             "%s: workspace of %zu bytes needed, %zu given", fn, plan.total_bytes, workspace_bytes);
  const long wgs = ((long)B * Hkv * plan.n_splits + 7) / 8 * 8 * plan.n_qc;
  SS_REQUIRE(wgs <= 0x7fffffffL && (long)B * Hkv * plan.n_qc <= 0x7fffffffL, SS_ERR_UNSUPPORTED, "%s: grid too large", fn);
  MsaMxArgs a;
  a.q = (const uint16_t*)q; a.k_new = (const uint16_t*)k_new; a.v_new = (const uint16_t*)v_new; a.out = (uint16_t*)out;
  a.c.k = (uint8_t*)k_cache; a.c.ks = (uint8_t*)k_scale; a.c.v = (uint8_t*)v_cache; a.c.vs = (uint8_t*)v_scale;
  a.c.block_table = block_table; a.c.Hkv = Hkv; a.c.D = D; a.c.page = page_size;
  a.c.page_shift = page_size == 16 ? 4 : (page_size == 32 ? 5 : 6);
  a.c.max_pages = max_pages_per_seq; a.c.num_pages = num_pages;
  a.seq_lens = seq_lens; a.parent = parent; a.n_nodes = n_nodes;
  char* ws = (char*)(((uintptr_t)workspace + 255) & ~(uintptr_t)255);
  a.arrive = (unsigned int*)ws;
  a.part_o = (float*)(ws + plan.part_o_at);
  a.part_lse = (float*)(ws + plan.part_lse_at);
  a.B = B; a.T = T; a.gamma = gamma; a.R = R; a.H = H; a.g = H / Hkv; a.n_splits = plan.n_splits; a.n_qc = plan.n_qc;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.flags = flags;
  hipStream_t st = (hipStream_t)stream;
  const bool fp8 = format == SS_KV_MXFP8;
  if (D == 128) fp8 ? launch_nt<128, true>(plan.nt, (unsigned)wgs, st, a) : launch_nt<128, false>(plan.nt, (unsigned)wgs, st, a);
  else fp8 ? launch_nt<64, true>(plan.nt, (unsigned)wgs, st, a) : launch_nt<64, false>(plan.nt, (unsigned)wgs, st, a);
  return check_launch(fn);
}

}  // extern "C"
