// n5, a2 over a cache in microscaling formats, few query rows: every wave walks keys of its own.  This file also holds the entry
// points and the plan.
//
// A workgroup of four wavefronts owns one (sequence, KV head, split of the cached tokens); the query heads of a group are folded
// into the rows, of which there are 16 NT, NT = 1 or 2.  Every wave holds ALL rows (queries, running maximum and sum, outputs in
// registers) and walks blocks of 32 keys of its own, so what is done once per key, above all turning values into bf16, is done
// by one wave only, and the waves need nothing from each other until their results are merged.  Bound by the bytes of the cache:
// one row, 32 sequences of 16384 tokens, 8 KV heads of 128 in 4 bits (570 MB) 101 us, 5.7 TB/s; with sequences of 1001 to 8003
// (157 MB) 36.5 us, of which 6 before the first block and 3 for merging.  One sequence of 411 tokens: 8.8 us, eight dependent
// trips to memory.
//
// Memory pipeline.  Every wave has two rings of raw blocks in LDS, keys and values each with their scales.  Direct global-to-LDS
// loads fill them; a wave waits for its own loads by count and nobody waits at a barrier.  Rows lie there as in the page, their
// 16-byte pieces XOR-swizzled by the lane -> address mapping so that operand reads meet every bank once.  A pass of the loop
// turns one block's scores into probabilities while the next block's scores are computed, then adds the block's values.
#include <math.h>

#include "ss_msa_mx.h"

namespace ss {

constexpr int kMxWaves = 4;

// Sizes of one instance.
template <int D, bool FP8, int NT>
struct MxShape : MxBlock<D, FP8> {
  using Bk = MxBlock<D, FP8>;
  static constexpr int WGS = NT == 1 && !(FP8 && D == 128) ? 3 : 2;  // workgroups per compute unit
  static constexpr int TILES = FP8 ? 1 : 2;                  // value tiles of a wave, 2 KB each
  static constexpr int FIT = (160 * 1024 / WGS / kMxWaves - TILES * 2048) / (2 * Bk::SLOT);
  static constexpr int DEPTH = FIT > 4 ? 4 : FIT;            // slots of a ring
  static constexpr int WAVE = TILES * 2048 + 2 * DEPTH * Bk::SLOT;
  static constexpr int NF = NT * Bk::DT, PW = NF / kMxWaves;  // 1 KB pieces of the workgroup's outputs, of a wave's share
  static constexpr int OUT = kMxWaves * NF * 1024 + kMxWaves * NT * 32 * 4;
  static constexpr int LDS = kMxWaves * WAVE > OUT ? kMxWaves * WAVE : OUT;
  static_assert(DEPTH >= 2 && LDS * WGS <= 160 * 1024, "a block in flight while another is computed");
};

template <int D, bool FP8, int NT>
__global__ __launch_bounds__(64 * kMxWaves, (MxShape<D, FP8, NT>::WGS)) void msa_mx_kernel(MsaMxArgs a) {
  using Sh = MxShape<D, FP8, NT>;
  constexpr int DT = Sh::DT, NB = Sh::NB, SLOT = Sh::SLOT, DEPTH = Sh::DEPTH, TL = Sh::TILES, LD = Sh::LOADS;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[Sh::LDS];  // the waves' tiles and rings; at the end outputs, maxima, sums

  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  MxItem m;
  if (!mx_item(a, 16 * NT, m)) return;
  const int n_units = (m.k1 - m.k0 + 31) >> 5, tail = (m.k1 - m.k0) & 31;
  const int n_mine = w < n_units ? (n_units - w + kMxWaves - 1) / kMxWaves : 0;  // this wave's blocks: w, w + 4, ...
  const bool ragged = tail != 0 && n_mine > 0 && w + (n_mine - 1) * kMxWaves == n_units - 1;  // its last is the split's ragged one
  MxMover<D, FP8> mv(a.c, m.b, m.hk, m.k0 + 32 * w, 32 * kMxWaves, lane);
  mv.load_pages(0, lane);
  uintx4 q_raw[NT][D / 32];
#pragma unroll
  for (int t = 0; t < NT; ++t) mx_load_query<D>(a, m, 16 * t + lq, lg, q_raw[t]);
  // blocks of 32 of the step's own rows go to the waves of all splits in turn; their loads go out with the first trip
  const int own0 = 32 * (m.s * kMxWaves + w), own_step = 32 * kMxWaves * m.n_active;
  const bool own = own0 < a.R;
  uintx4 kf[2][D / 32], vf[NB][2];
  uint64_t anc = 0;
  if (own) {
    mx_load_own_keys<D>(a, m, own0, lane, kf);
#pragma unroll
    for (int np = 0; np < NB; ++np) mx_load_own_values<D>(a, m, own0, np, lane, vf[np]);
  }

  unsigned char* const tiles = smem + w * Sh::WAVE;
  unsigned char* const rings = tiles + TL * 2048;  // keys' slots, then values'
  const uint32_t lds_rings = (uint32_t)(uintptr_t)rings;
  auto issue = [&](int kv, int it, int slot) { mv.issue(kv, it, lds_rings + (uint32_t)(kv * DEPTH + slot) * SLOT, lane); };
  // Order of the loads: keys of block 0, then in turn values of block i and keys of block i + 1, as far as the rings have slots.
  if (n_mine > 0) {
    issue(0, 0, 0);
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      if (i < n_mine) issue(1, i, i);
      if (i + 1 < n_mine && i + 1 < DEPTH) issue(0, i + 1, i + 1);
    }
  }

  const float c = a.scale_log2, lazy_thr = kMxLazyLog2 / c;
  floatx4 O[NT][DT], S[NT][2];
  float m_run[NT], l_run[NT];  // maximum of the query row, sum of this lane's probabilities
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m_run[t] = a.no_max;
    l_run[t] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[t][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  float pinf = INFINITY;  // see vmax2
  asm volatile("" : "+s"(pinf));
  const MxReader<D, FP8> rd(lane);
  auto add_values = [&](int np, const bf16x8 (&P)[NT]) {
    const uint32_t tr = fresh(rd.tr_rd);
#pragma unroll
    for (int dp = 0; dp < 2; ++dp) {
      const bf16x8 vv = rd.values(tiles + (np % TL) * 2048, tr, dp);
#pragma unroll
      for (int t = 0; t < NT; ++t) O[t][2 * np + dp] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, P[t], O[t][2 * np + dp], 0, 0, 0);
    }
  };

  // ---- the step's own rows, while the first blocks are on their way
  if (own) {
    anc = mx_ancestors(a, m.b, lane);
    for (int c0 = own0;;) {
      bf16x8 P[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) mx_own_scores<D>(a, m, 16 * t + lq, lane, anc, c0, kf, q_raw[t], S[t]);
      if (c0 == own0) mx_raise<NT, DT, true>(S, c, lazy_thr, pinf, m_run, l_run, O);
      else mx_raise<NT, DT>(S, c, lazy_thr, pinf, m_run, l_run, O);
#pragma unroll
      for (int t = 0; t < NT; ++t) P[t] = mx_softmax(S[t], c, m_run[t], l_run[t]);
#pragma unroll
      for (int np = 0; np < NB; ++np) {
        in_order();
        mx_put_own_values(a, m, c0, lane, tiles + (np % TL) * 2048, vf[np]);
        in_order();
        add_values(np, P);
      }
      c0 += own_step;
      if (c0 >= a.R) break;
      mx_load_own_keys<D>(a, m, c0, lane, kf);
#pragma unroll
      for (int np = 0; np < NB; ++np) mx_load_own_values<D>(a, m, c0, np, lane, vf[np]);
    }
  }

  intx8 Qh[NT], Ql[NT];
  int sq[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    uint32_t hi[D / 16], lo[D / 16];
    sq[t] = split_query<D>(q_raw[t], hi, lo, lg);
    mx_query_operands<D>(hi, lo, Qh[t], Ql[t]);
  }

  // ---- the cached tokens
  // What lies behind the sequence in the values' slot becomes zeros: a NaN there would not be hidden by probabilities of zero.
  auto clean_tail = [&](int v_slot) {
    unsigned char* st = rings + (DEPTH + v_slot) * SLOT;
    for (int i = lane; i < 32 * Sh::PR; i += 64)
      if (i / Sh::PR >= tail) *reinterpret_cast<uintx4*>(st + 16 * i) = uintx4{0u, 0u, 0u, 0u};
    for (int i = lane; i < 32 * NB; i += 64)
      if (i / NB >= tail) st[32 * Sh::ROWB + i] = 0;
  };
  // One block: its probabilities and the next block's scores (after the last block those of whatever the slot holds, for
  // nobody: a second copy of the code without them costs more registers than there are), then its values.
  auto pass = [&](int v_slot, int k_slot) {
    const unsigned char* st = rings + (DEPTH + v_slot) * SLOT;
    const uint32_t scales = rd.scales(st);
    intx8 K[2];
    int sk[2];
    typename MxReader<D, FP8>::Raw raw[NB];
    rd.keys(rings + k_slot * SLOT, K, sk);
#pragma unroll
    for (int np = 0; np < (FP8 ? TL : NB); ++np) raw[np] = rd.raw(np, st);
#pragma unroll
    for (int np = 0; np < TL; ++np) rd.put(np, tiles + np * 2048, raw[np], scales);
    bf16x8 P[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      P[t] = mx_softmax(S[t], c, m_run[t], l_run[t]);
      rd.scores(K, sk, Qh[t], Ql[t], sq[t], S[t]);
    }
#pragma unroll
    for (int np = 0; np < NB; ++np) {
      if (FP8 && np + TL < NB) raw[np + TL] = rd.raw(np + TL, st);
      in_order();
      add_values(np, P);
      in_order();
      if (np + TL < NB) rd.put(np + TL, tiles + (np % TL) * 2048, raw[np + TL], scales);
    }
  };
  if (n_mine > 0) {
    wait_vmcnt<0>();
    {
      intx8 K[2];
      int sk[2];
      rd.keys(rings, K, sk);
#pragma unroll
      for (int t = 0; t < NT; ++t) rd.scores(K, sk, Qh[t], Ql[t], sq[t], S[t]);
    }
    if (ragged && n_mine == 1) mx_mask_tail<NT>(S, lg, tail);
    mx_raise<NT, DT>(S, c, lazy_thr, pinf, m_run, l_run, O);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // keys 0 have been read
    if (DEPTH < n_mine) issue(0, DEPTH, 0);
    int v_slot = 0, it = 0;
    do {
      const int k_slot = v_slot + 1 == DEPTH ? 0 : v_slot + 1, more = n_mine - 1 - it;  // blocks after this one
      // values of this block and keys of the next have landed; what was asked for after them may still be under way
      if (more >= DEPTH) wait_vmcnt<2 * (DEPTH - 1) * LD>();
      else if (DEPTH > 2 && more == 2) wait_vmcnt<3 * LD>();
      else if (more == 1) wait_vmcnt<LD>();
      else wait_vmcnt<0>();  // (also three blocks before the end with a ring of four)
      if (ragged && more == 0) clean_tail(v_slot);
      in_order();
      pass(v_slot, k_slot);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // both slots have been read
      if (more >= DEPTH) issue(1, it + DEPTH, v_slot);
      if (more > DEPTH) {
        if (((it + DEPTH + 1) & 63) == 0) mv.load_pages(it + DEPTH + 1, lane);
        issue(0, it + DEPTH + 1, k_slot);
      }
      // (not left out after the last block: what is skipped there is moved there by the compiler, scores and all)
      const int seen = more == 0 ? 0 : ragged && more == 1 ? tail : 32;
      if (seen < 32) mx_mask_tail<NT>(S, lg, seen);
      mx_raise<NT, DT>(S, c, lazy_thr, pinf, m_run, l_run, O);
      v_slot = k_slot;
    } while (++it < n_mine);
  }

  // ---- merge the waves: to a common maximum, then piece by piece, a wave taking a quarter
  __syncthreads();  // nobody reads a ring any more
  float* const ml = reinterpret_cast<float*>(smem + kMxWaves * Sh::NF * 1024);  // [wave][NT][max, sum][16]
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    l_run[t] += __shfl_xor(l_run[t], 16, 64);
    l_run[t] += __shfl_xor(l_run[t], 32, 64);
    if (lg == 0) {
      ml[(w * NT + t) * 32 + lq] = m_run[t];
      ml[(w * NT + t) * 32 + 16 + lq] = l_run[t];
    }
  }
  floatx4* buf = reinterpret_cast<floatx4*>(smem);  // [wave][NF][64]
#pragma unroll
  for (int k = 0; k < Sh::NF; ++k) buf[(w * Sh::NF + k) * 64 + lane] = O[k / DT][k % DT];
  __syncthreads();
  constexpr int PW = Sh::PW;
  static_assert(DT % PW == 0, "a wave's pieces belong to one tile");
  const int t = w * PW / DT;
  floatx4 res[1][PW];
  float l[1] = {0.f}, mx[1] = {ml[t * 32 + lq]};
#pragma unroll
  for (int i = 1; i < kMxWaves; ++i) mx[0] = fmaxf(mx[0], ml[(i * NT + t) * 32 + lq]);
#pragma unroll
  for (int k = 0; k < PW; ++k) res[0][k] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kMxWaves; ++i) {
    const float fac = __builtin_amdgcn_exp2f((ml[(i * NT + t) * 32 + lq] - mx[0]) * c);
    l[0] = fmaf(ml[(i * NT + t) * 32 + 16 + lq], fac, l[0]);
#pragma unroll
    for (int k = 0; k < PW; ++k) res[0][k] += buf[(i * Sh::NF + w * PW + k) * 64 + lane] * fac;
  }
  mx_finish<D, 1, PW>(a, m, w, kMxWaves, NT, lane, res, l, mx, [&](int) { return t; }, [&](int k) { return w * PW % DT + k; });
}

template <int D, bool FP8>
static int launch_mx(const MsaMxArgs& a, int nt, long wgs, hipStream_t st) {
  SS_REQUIRE(wgs <= kMxMaxThreads / (64 * kMxWaves), SS_ERR_UNSUPPORTED, "ss_msa_attention_mx: grid too large");
  auto kern = nt == 1 ? msa_mx_kernel<D, FP8, 1> : msa_mx_kernel<D, FP8, 2>;
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(64 * kMxWaves), 0, st, a);
  return check_launch("ss_msa_attention_mx");
}
int launch_msa_mx(const MsaMxArgs& a, MxKernel k, bool fp8, long wgs, hipStream_t st) {
  if (a.c.D == 128) return fp8 ? launch_mx<128, true>(a, k.nt, wgs, st) : launch_mx<128, false>(a, k.nt, wgs, st);
  return fp8 ? launch_mx<64, true>(a, k.nt, wgs, st) : launch_mx<64, false>(a, k.nt, wgs, st);
}

// ------------------------------------------------------------------ planning (host)
struct MxPlan {
  MxKernel kernel;
  int n_qc, n_splits;
  size_t part_o_at, part_lse_at, total_bytes;
};

// Workgroups of the kernel for few rows that the chip holds: two or three per compute unit.  Single tokens of heads of 128 in 8
// bits, counted with three / with the two that fit, us: 256 items of 8192 tokens 102 / 92, 128 items 57 /
// 50, 512 items of 4096 99 / 88, 1024 items 191 / 174; where that splits and the other count did not, 640 items 121 / 124, 768
// items 130 / 139 (a last round that does not fill the chip goes faster than the rule counts).  Two tiles of heads of 64 in 4 bits
// are counted with two per compute unit though three fit: 512 items of 4096 tokens 46 us, 50 with three, 1024 items 82 / 90, 640
// items 61 / 57, 768 items 66 / 60.
static int mx_resident(int tiles, int D, bool fp8) {
  if (D == 128) return 256 * (tiles == 2 ? fp8 ? MxShape<128, true, 2>::WGS : MxShape<128, false, 2>::WGS
                                         : fp8 ? MxShape<128, true, 1>::WGS : MxShape<128, false, 1>::WGS);
  return 256 * (tiles == 2 ? fp8 ? MxShape<64, true, 2>::WGS : MxShape<64, false, 2>::WGS
                           : fp8 ? MxShape<64, true, 1>::WGS : MxShape<64, false, 1>::WGS);
}
static MxPlan mx_plan(int B, int R, int H, int Hkv, int D, int max_len, bool fp8) {
  MxPlan p;
  const int F = (H / Hkv) * R, tiles = ceil_div(F, 16);
  int units, resident;  // waves of a workgroup that merge; workgroups that the chip holds
  // One or two query tiles: keys of their own, us against keys shared by three waves: four sequences of 4096 tokens, 32 heads, 16
  // rows 22.5 / 24.5, 32 rows 27.2 / 27.2; one of 2000, 8 heads, 11.2 / 14.1 and 14.3 / 15.4; heads of 64, 17.5 / 18.5 and 19.7 /
  // 21.5; sixteen in 8 bits 69.4 / 66.4 and 67.7 / 70.5.
  if (tiles <= 2) {
    p.kernel = MxKernel{tiles, 1};
    p.n_qc = 1;
    units = kMxWaves;
    resident = mx_resident(tiles, D, fp8);
  } else {
    // Up to five: a wave each, and two to four groups.  More: two per wave and as few chunks as there can be of up to eight (five
    // tiles that way: 51 us, 41 the other; four sequences of 4096 tokens, 32 heads).
    const int per_wg = tiles <= 5 ? 5 : 8;
    p.n_qc = ceil_div(tiles, per_wg);
    const int per = ceil_div(tiles, p.n_qc), nt = per <= 5 ? 1 : 2, nw = ceil_div(per, nt);
    p.kernel = MxKernel{nt, nw};
    units = nw;
    resident = nt == 1 ? 256 : 512;
  }
  const long items = (long)B * Hkv * p.n_qc;
  const int len = min(max(max_len, 1), kMxMaxLen);
  // Splits: as if all sequences were as long as they may get, rounds of the chip times what a workgroup takes, its tokens and,
  // for what it does once, some 512 more (128 and 2048 choose almost the same); and merging them (see mx_split_len).  Four
  // sequences of 4096 tokens and 32 heads, 80 rows: 2 splits 43 us, 4 splits 61.  Eight of 32768 and 8 heads, 640 rows: 2 splits
  // 931 us, 3 splits 756.
  long n = 1, best = 0;
  const int most = items * units * (long)sizeof(unsigned int) <= (long)kArriveRegionBytes ? min(ceil_div(len, mx_split_len(len, len)), 256) : 1;
  for (int i = 1; i <= most; ++i) {
    const long cost = (items * i + resident - 1) / resident * (ceil_div(len, i) + 512) + (i > 1 ? 128 + 50 * i : 0);
    if (i == 1 || cost < best) {
      best = cost;
      n = i;
    }
  }
  p.n_splits = (int)n;
  p.part_o_at = p.part_lse_at = 0;
  p.total_bytes = 256;  // to align the start
  if (p.n_splits > 1) {
    const size_t rows = (size_t)items * p.n_splits * 16 * p.kernel.nt * p.kernel.nw;
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

}  // namespace ss

extern "C" {

size_t ss_msa_mx_workspace_bytes(int B, int T, int gamma, int H, int Hkv, int D, int max_seq_len) {
  ss::clear_error();
  if (ss::mx_check_shape("ss_msa_mx_workspace_bytes", B, T, gamma, H, Hkv, D) != SS_OK) return 0;
  return max(ss::mx_plan(B, T * (1 + gamma), H, Hkv, D, max_seq_len, false).total_bytes,
             ss::mx_plan(B, T * (1 + gamma), H, Hkv, D, max_seq_len, true).total_bytes);
}

int ss_msa_mx_plan(int B, int T, int gamma, int H, int Hkv, int D, int max_seq_len, int* n_splits, int* rows_per_workgroup) {
  ss::clear_error();
  if (int rc = ss::mx_check_shape("ss_msa_mx_plan", B, T, gamma, H, Hkv, D)) return rc;
  const ss::MxPlan p = ss::mx_plan(B, T * (1 + gamma), H, Hkv, D, max_seq_len, false);
  if (n_splits) *n_splits = max(p.n_splits, ss::mx_plan(B, T * (1 + gamma), H, Hkv, D, max_seq_len, true).n_splits);
  if (rows_per_workgroup) *rows_per_workgroup = 16 * p.kernel.nt * p.kernel.nw;
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
  SS_REQUIRE(scale > 0.f && isfinite(scale * 1.4426950408889634f), SS_ERR_INVALID_ARG, "%s: scale must be positive and finite, and so its product with log2(e)", fn);
  SS_REQUIRE((flags & ~SS_STREAM_EXCLUDE_SELF) == 0, SS_ERR_INVALID_ARG, "%s: unknown flags 0x%x", fn, flags);
  SS_REQUIRE((long)num_pages * Hkv <= (1L << 32) / page_size, SS_ERR_UNSUPPORTED, "%s: a cache of more than 2^32 rows", fn);
  if (B == 0) return SS_OK;
  SS_REQUIRE(q && k_new && v_new && seq_lens && parent && out, SS_ERR_INVALID_ARG, "%s: NULL tensor argument", fn);
  SS_REQUIRE((((uintptr_t)q | (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)out) & 15) == 0, SS_ERR_INVALID_ARG,
             "%s: q, k_new, v_new or out not aligned to 16 bytes", fn);
  const int R = T * (1 + gamma);
  const bool fp8 = format == SS_KV_MXFP8;
  const MxPlan plan = mx_plan(B, R, H, Hkv, D, max_pages_per_seq * page_size, fp8);
  SS_REQUIRE(plan.n_splits == 1 || (workspace != nullptr && workspace_bytes >= plan.total_bytes), SS_ERR_WORKSPACE,
             "%s: workspace of %zu bytes needed, %zu given", fn, plan.total_bytes, workspace_bytes);
  const long wgs = ((long)B * Hkv * plan.n_splits + 7) / 8 * 8 * plan.n_qc;
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
  a.no_max = -3e38f / fmaxf(a.scale_log2, 1.f);
  a.flags = flags;
  hipStream_t st = (hipStream_t)stream;
  return plan.kernel.nw == 1 ? launch_msa_mx(a, plan.kernel, fp8, wgs, st) : launch_msa_mx_rows(a, plan.kernel, fp8, wgs, st);
}

}  // extern "C"
