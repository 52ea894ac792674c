// n5, a2 over a cache in microscaling formats, many query rows: the waves of a group share keys.
//
// A workgroup owns one (sequence, KV head, split of the cached tokens, chunk of 16 NW NT query rows); the query heads of a group
// are folded into the rows.  It consists of G groups of NW waves.  Inside a group every wave owns NT 16-row query tiles and all
// walk the same blocks of 32 keys; the groups take the split's blocks in turn and are merged through LDS at the end.  Scores
// come from the raw keys in LDS; of the values every wave turns a feature block or two into bf16 for all (double-buffered
// tiles), one block of keys ahead.  One barrier per block: it tells that the next raw block has landed, the next values are in
// their tiles and the last ones have been read.  Between two barriers a wave turns its scores into probabilities, computes the
// next block's scores, makes its share of the next block's values and adds this block's: matrix and vector instructions that do
// not depend on each other, of two to four waves per SIMD.
//
// A block's raw bytes are moved in quarters (keys or values of 16 tokens), one or two per wave: a wave that moved all of them came
// last to every barrier (NT = 2, eight of up to 32768 tokens, 640 rows: 1354 us, 1017 with quarters).  What a wave takes of a raw
// block is read before the barrier and used behind it (939 us).
//
// Per 16 rows and 32 keys (D 128, 4 bits) 12 matrix instructions, 256 cycles of a SIMD, and 62 (NT = 1) or 48 (NT = 2) vector
// instructions; 10 or 6 KB read from LDS.  NT = 2, eight sequences of 32768 tokens, 640 rows: 637 us, 1080 TFLOP/s; in a run with
// counters (685 us, 2.15 GHz) the matrix pipe is busy 45 % and vector instructions are active 51 % of the cycles, which overlap
// little.  NT = 1, four of 4096, 32 heads, 80 rows: 40 us, 535 TFLOP/s; with counters (43.9 us, 2.03 GHz) 24 % and 40 %, and waves
// wait a third of their time: ten waves lie on the four SIMDs as 3, 3, 2 and 2, and the barrier every 0.9 us waits for the threes.
#include "ss_msa_mx.h"

#include <mutex>

namespace ss {

template <int D, bool FP8, int NW, int NT, int G>
struct MxRowsShape : MxBlock<D, FP8> {
  using Bk = MxBlock<D, FP8>;
  static constexpr int WAVES = NW * G;
  static constexpr int TILES = 2 * Bk::NB * 2048;            // bytes of a group's value tiles
  static constexpr int UNIT = 2 * Bk::SLOT;                  // bytes of a raw block
  static constexpr int PER_SIMD = NT == 2 ? 2 : WAVES > 12 ? 4 : 3;  // wavefronts of a SIMD
  static constexpr int WGS = 4 * PER_SIMD / WAVES > 0 ? 4 * PER_SIMD / WAVES : 1;  // workgroups of a compute unit
  static constexpr int FIT = (156 * 1024 / WGS / G - TILES) / UNIT;
  static constexpr int DEPTH = FIT > 5 ? 5 : FIT;            // raw blocks of a group's ring
  static constexpr int GROUP = TILES + DEPTH * UNIT;
  static constexpr int NF = NT * Bk::DT;                     // 1 KB pieces of a wave's outputs
  static constexpr int OUT = (G - 1) * NW * (NF * 1024 + NT * 128);  // the other groups' outputs, maxima and sums
  static constexpr int LDS = G * GROUP > OUT ? G * GROUP : OUT;
  static constexpr int QS = (3 + NW) / NW;                   // quarters of a block that a wave moves (the last ones may move none)
  static_assert(DEPTH >= 3 && LDS <= 160 * 1024, "two blocks in flight");
};

template <int D, bool FP8, int NW, int NT, int G>
__global__ __launch_bounds__(64 * NW * G, (MxRowsShape<D, FP8, NW, NT, G>::PER_SIMD)) void msa_mx_rows_kernel(MsaMxArgs a) {
  using Sh = MxRowsShape<D, FP8, NW, NT, G>;
  constexpr int DT = Sh::DT, NB = Sh::NB, SLOT = Sh::SLOT, UNIT = Sh::UNIT, DEPTH = Sh::DEPTH, NF = Sh::NF, QS = Sh::QS;
  using Quarter = MxQuarter<D, FP8, NT == 1>;  // (several chunks of rows read the same blocks)
  constexpr int LPW = QS * Quarter::LOADS;  // a wave's loads of a block
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // groups' tiles and rings; at the end outputs, maxima, sums

  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = w / NW, wt = w % NW;
  MxItem m;
  if (!mx_item(a, 16 * NW * NT, m)) return;
  const int at0 = 16 * NT * wt;                  // this wave's first row in the chunk
  const bool live = m.f0 + at0 < m.F;            // it has any
  const bool loader = wt * QS < 4;               // moves quarters of the group's blocks
  const int n_units = (m.k1 - m.k0 + 31) >> 5, tail = (m.k1 - m.k0) & 31;
  const int n_iter = (n_units + G - 1) / G;      // of the first group, for all
  const int n_mine = grp < n_units ? (n_units - grp + G - 1) / G : 0;
  const bool ragged = tail != 0 && n_mine > 0 && grp + (n_mine - 1) * G == n_units - 1;  // the group's last block is the ragged one

  unsigned char* const tiles = smem + grp * Sh::GROUP;
  unsigned char* const ring = tiles + Sh::TILES;
  const uint32_t lds_ring = (uint32_t)(uintptr_t)ring;
  const int qn = min(wt * QS, 4 - QS);  // its first quarter: keys' halves, values' halves
  Quarter quarter[QS];
#pragma unroll
  for (int i = 0; i < QS; ++i) quarter[i].init(a.c, qn >> 1, (qn + i) & 1, lane);
  auto load_rows = [&](int jbase) {
#pragma unroll
    for (int i = 0; i < QS; ++i) quarter[i].load_rows(a.c, m.b, m.hk, m.k0 + 32 * (grp + (jbase + lane) * G) + 16 * ((qn + i) & 1));
  };
  if (loader) load_rows(0);
  uintx4 q_raw[NT][D / 32];
#pragma unroll
  for (int t = 0; t < NT; ++t) mx_load_query<D>(a, m, at0 + 16 * t + lq, lg, q_raw[t]);
  // blocks of 32 of the step's own rows go to the groups of all splits in turn
  const int own_all = (a.R + 31) >> 5, own_step = m.n_active * G;
  const int n_own = m.s * G < own_all ? (own_all - m.s * G + own_step - 1) / own_step : 0;  // rounds
  const int own_at = m.s * G + grp;
  uintx4 kf[2][D / 32], vf[(NB + NW - 1) / NW][2];
  auto load_own = [&](int c0) {
    mx_load_own_keys<D>(a, m, c0, lane, kf);
#pragma unroll
    for (int i = 0; i < (NB + NW - 1) / NW; ++i) mx_load_own_values<D>(a, m, c0, min(wt + i * NW, NB - 1), lane, vf[i]);
  };
  if (own_at < own_all) load_own(32 * own_at);
  auto issue = [&](int it, int slot) {
#pragma unroll
    for (int i = 0; i < QS; ++i) quarter[i].issue(it, lds_ring + (uint32_t)slot * UNIT, lane);
  };
  if (loader) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
      if (i < n_mine) issue(i, i);
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
  auto add_values = [&](const unsigned char* set, const bf16x8 (&P)[NT]) {
    const uint32_t tr = fresh(rd.tr_rd);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const bf16x8 vv = rd.values(set + (dt >> 1) * 2048, tr, dt & 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) O[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, P[t], O[t][dt], 0, 0, 0);
    }
  };

  // ---- the step's own rows, while the first blocks are on their way
  if (n_own > 0) {
    const uint64_t anc = mx_ancestors(a, m.b, lane);
    for (int j = 0; j < n_own; ++j) {
      const int c0 = 32 * (own_at + j * own_step);
      const bool mine = c0 < a.R;
      if (j > 0) {
        if (mine) load_own(c0);
        __syncthreads();  // the tiles have been read
      }
      if (mine) {
#pragma unroll
        for (int i = 0; i < (NB + NW - 1) / NW; ++i)
          if (wt + i * NW < NB) mx_put_own_values(a, m, c0, lane, tiles + (wt + i * NW) * 2048, vf[i]);
      }
      __syncthreads();
      if (mine && live) {
        bf16x8 P[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) mx_own_scores<D>(a, m, at0 + 16 * t + lq, lane, anc, c0, kf, q_raw[t], S[t]);
        if (j == 0) mx_raise<NT, DT, true>(S, c, lazy_thr, pinf, m_run, l_run, O);
        else mx_raise<NT, DT>(S, c, lazy_thr, pinf, m_run, l_run, O);
#pragma unroll
        for (int t = 0; t < NT; ++t) P[t] = mx_softmax(S[t], c, m_run[t], l_run[t]);
        add_values(tiles, P);
      }
    }
    __syncthreads();  // the tiles have been read
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
  // What a wave takes from a raw block: the keys, and its share of the values (feature blocks wt, wt + NW, ..).
  constexpr int SHARE = (NB + NW - 1) / NW;
  typedef typename MxReader<D, FP8>::Raw Raw;
  intx8 K[2];
  int sk[2];
  Raw raw[SHARE];
  uint32_t scales = 0;
  auto take = [&](const unsigned char* st, auto with_rows, auto with_share) {
    if constexpr (decltype(with_rows)::value) rd.keys(st, K, sk);
    if constexpr (decltype(with_share)::value) {
      scales = rd.scales(st + SLOT);
#pragma unroll
      for (int i = 0; i < SHARE; ++i) raw[i] = rd.raw(min(wt + i * NW, NB - 1), st + SLOT);
    }
  };
  // The share as bf16 into a set of tiles.
  auto put_values = [&](unsigned char* set) {
#pragma unroll
    for (int i = 0; i < SHARE; ++i)
      if (i + 1 < SHARE || NB % NW == 0 || wt + i * NW < NB) rd.put(wt + i * NW, set + (wt + i * NW) * 2048, raw[i], scales);
  };
  // The same of a block of which `seen` tokens are there: the others become zeros, for a NaN there would not be hidden by
  // probabilities of zero.
  auto put_tail = [&](unsigned char* set, int seen) {
#pragma unroll
    for (int i = 0; i < SHARE; ++i) raw[i] = rd.vt < seen ? raw[i] : Raw{};
    scales = rd.vt < seen ? scales : 0u;
#pragma unroll
    for (int i = 0; i < SHARE; ++i)
      if (wt + i * NW < NB) rd.put(wt + i * NW, set + (wt + i * NW) * 2048, raw[i], scales);
  };
  if (n_iter > 0) {
    if (loader) {  // the first three blocks have landed
      if (n_mine >= DEPTH) wait_vmcnt<(DEPTH - 3) * LPW>();
      else wait_vmcnt<0>();
    }
    __syncthreads();
    // A wave without rows moves blocks and makes its share of the values, no more.
    auto walk = [&](auto with_rows, auto with_share) {
      if (n_mine > 0) {
        take(ring, with_rows, with_share);
        const int seen = ragged && n_mine == 1 ? tail : 32;
        if constexpr (decltype(with_rows)::value) {
#pragma unroll
          for (int t = 0; t < NT; ++t) rd.scores(K, sk, Qh[t], Ql[t], sq[t], S[t]);
          if (seen < 32) mx_mask_tail<NT>(S, lg, seen);
          mx_raise<NT, DT>(S, c, lazy_thr, pinf, m_run, l_run, O);
        }
        if constexpr (decltype(with_share)::value) put_tail(tiles, seen);
        take(ring + UNIT, with_rows, with_share);  // (after the last block of whatever a slot holds, for nobody; also below)
      }
      __syncthreads();
      if (loader && DEPTH < n_mine) issue(DEPTH, 0);
      int slot = 1;  // of block it + 1
      // STEADY: more than DEPTH blocks follow, so nothing has to be asked.  A loop of its own (us without and with it: 640 rows,
      // eight sequences of 32768 tokens, 667 and 647; 80 rows, four of 4096, 41.0 and 40.2) where registers allow two.
      constexpr bool TWO_LOOPS = NT == 2 || D == 64 || !FP8;
      auto pass = [&](int it, auto steady) {
        constexpr bool STEADY = decltype(steady)::value;
        const int next = slot + 1 == DEPTH ? 0 : slot + 1, more = n_mine - 1 - it;  // blocks of the group after this one
        if (loader && (STEADY || more > DEPTH)) {  // block it + 1 has been read before the barrier
          if (((it + 1 + DEPTH) & 63) == 0) load_rows(it + 1 + DEPTH);
          issue(it + 1 + DEPTH, slot);
        }
        unsigned char* const set = tiles + (it & 1) * (NB * 2048);
        unsigned char* const set_next = tiles + ((it & 1) ^ 1) * (NB * 2048);
        const int seen = STEADY ? 32 : more == 0 ? 0 : ragged && more == 1 ? tail : 32;  // of the next block's keys
        if constexpr (decltype(with_rows)::value) {
          // Values are asked for LEAD feature tiles ahead, the first before all else: read where they are used, every matrix
          // instruction waits for LDS, and the compiler would put them there (NT = 2, 640 rows: 757 us, 667 with two tiles ahead, 700
          // with three).
          constexpr int LEAD = NT == 1 ? 4 : 2;
          const uint32_t tr = fresh(rd.tr_rd);
          auto value = [&](int dt) { return rd.values(set + (dt >> 1) * 2048, tr, dt & 1); };
          bf16x8 P[NT], V[LEAD];
          // With three waves per SIMD those that still make probabilities go before those that add values: 42.3 -> 41.0 us (four
          // sequences of 4096 tokens, 80 rows), 100.7 -> 97.9 (sixteen, 8 bits).  With two it costs nothing and gives nothing.
          if constexpr (NT == 1) __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int dt = 0; dt < LEAD; ++dt) V[dt] = value(dt);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            P[t] = mx_softmax(S[t], c, m_run[t], l_run[t]);
            rd.scores(K, sk, Qh[t], Ql[t], sq[t], S[t]);
          }
          if constexpr (decltype(with_share)::value) put_values(set_next);
          // matrix and vector instructions in turn
#pragma unroll
          for (int i = 0; i < (D == 128 ? 4 : 2) * NT; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x2, D == 128 ? 8 : 16, 0);
          }
          if constexpr (NT == 1) __builtin_amdgcn_s_setprio(0);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
            for (int t = 0; t < NT; ++t) O[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(V[dt % LEAD], P[t], O[t][dt], 0, 0, 0);
            if (dt + LEAD < DT) V[dt % LEAD] = value(dt + LEAD);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (!STEADY && seen < 32) {
            if constexpr (decltype(with_share)::value)
              if (more == 1) put_tail(set_next, seen);
            mx_mask_tail<NT>(S, lg, seen);
          }
          take(ring + next * UNIT, with_rows, with_share);
          mx_raise<NT, DT>(S, c, lazy_thr, pinf, m_run, l_run, O);
        } else if constexpr (decltype(with_share)::value) {
          put_tail(set_next, more == 0 ? 32 : seen);
          take(ring + next * UNIT, with_rows, with_share);
        }
        if (loader) {  // block it + 3 has landed; those after it, up to it + 1 + DEPTH, may still be under way
          if (STEADY || more > DEPTH) wait_vmcnt<(DEPTH - 2) * LPW>();
          else if (DEPTH > 4 && more == 5) wait_vmcnt<2 * LPW>();
          else if (DEPTH > 3 && more == 4) wait_vmcnt<LPW>();
          else wait_vmcnt<0>();
        }
        __syncthreads();
        slot = next;
      };
      int it = 0;
      if constexpr (TWO_LOOPS)
        for (; it + DEPTH + 1 < n_mine; ++it) pass(it, std::true_type{});
      for (; it < n_mine; ++it) pass(it, std::false_type{});
    };
    if (live) {
      if (NW <= NB || wt < NB) walk(std::true_type{}, std::true_type{});
      else walk(std::true_type{}, std::false_type{});
    } else {
      if (NW <= NB || wt < NB) walk(std::false_type{}, std::true_type{});
      else walk(std::false_type{}, std::false_type{});
    }
    if (n_mine < n_iter) __syncthreads();  // one block less than the first group
  }

  // ---- merge the groups into the first: to a common maximum, then piece by piece
  __syncthreads();
  float* const ml = reinterpret_cast<float*>(smem + (G - 1) * NW * NF * 1024);  // [(group - 1)*NW + wave][NT][max, sum][16]
  floatx4* const buf = reinterpret_cast<floatx4*>(smem);                        // [(group - 1)*NW + wave][NF][64]
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    l_run[t] += __shfl_xor(l_run[t], 16, 64);
    l_run[t] += __shfl_xor(l_run[t], 32, 64);
  }
  if (grp > 0) {
    const int at = (grp - 1) * NW + wt;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (lg == 0) {
        ml[(at * NT + t) * 32 + lq] = m_run[t];
        ml[(at * NT + t) * 32 + 16 + lq] = l_run[t];
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) buf[(at * NF + t * DT + dt) * 64 + lane] = O[t][dt];
    }
  }
  __syncthreads();
  if (grp > 0 || !live) return;
  floatx4 res[NT][DT];
  float l[NT], mx[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    mx[t] = m_run[t];
#pragma unroll
    for (int i = 0; i < G - 1; ++i) mx[t] = fmaxf(mx[t], ml[((i * NW + wt) * NT + t) * 32 + lq]);
    float fac = __builtin_amdgcn_exp2f((m_run[t] - mx[t]) * c);
    l[t] = l_run[t] * fac;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) res[t][dt] = O[t][dt] * fac;
#pragma unroll
    for (int i = 0; i < G - 1; ++i) {
      fac = __builtin_amdgcn_exp2f((ml[((i * NW + wt) * NT + t) * 32 + lq] - mx[t]) * c);
      l[t] = fmaf(ml[((i * NW + wt) * NT + t) * 32 + 16 + lq], fac, l[t]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) res[t][dt] += buf[((i * NW + wt) * NF + t * DT + dt) * 64 + lane] * fac;
    }
  }
  mx_finish<D, NT, DT>(a, m, wt, NW, NW * NT, lane, res, l, mx, [&](int t) { return wt * NT + t; }, [&](int k) { return k; });
}

template <int D, bool FP8, int NW, int NT, int G>
static int launch_rows(const MsaMxArgs& a, long wgs, hipStream_t st) {
  using Sh = MxRowsShape<D, FP8, NW, NT, G>;
  SS_REQUIRE(wgs <= kMxMaxThreads / (64 * NW * G), SS_ERR_UNSUPPORTED, "ss_msa_attention_mx: grid too large");
  auto kern = msa_mx_rows_kernel<D, FP8, NW, NT, G>;
  static std::once_flag attr_once;
  static hipError_t attr_err = hipSuccess;
  std::call_once(attr_once, [&]() {
    attr_err = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
  });
  if (attr_err != hipSuccess) SS_FAIL(SS_ERR_HIP, "ss_msa_attention_mx: hipFuncSetAttribute: %s", hipGetErrorString(attr_err));
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(64 * NW * G), Sh::LDS, st, a);
  return check_launch("ss_msa_attention_mx");
}
template <int D, bool FP8>
static int launch_rows_d(const MsaMxArgs& a, MxKernel k, long wgs, hipStream_t st) {
  if (k.nt == 1) {
    if (k.nw == 3) return launch_rows<D, FP8, 3, 1, FP8 && D == 128 ? 3 : 4>(a, wgs, st);
    if (k.nw == 4) return launch_rows<D, FP8, 4, 1, 3>(a, wgs, st);
    // heads of 64 have registers for fifteen waves: sixteen sequences, 80 rows 63.5 -> 58.6 us (three or four waves per group: no gain)
    return launch_rows<D, FP8, 5, 1, D == 64 ? 3 : 2>(a, wgs, st);
  }
  if (k.nw == 3) return launch_rows<D, FP8, 3, 2, 1>(a, wgs, st);
  return launch_rows<D, FP8, 4, 2, 1>(a, wgs, st);
}
int launch_msa_mx_rows(const MsaMxArgs& a, MxKernel k, bool fp8, long wgs, hipStream_t st) {
  if (a.c.D == 128) return fp8 ? launch_rows_d<128, true>(a, k, wgs, st) : launch_rows_d<128, false>(a, k, wgs, st);
  return fp8 ? launch_rows_d<64, true>(a, k, wgs, st) : launch_rows_d<64, false>(a, k, wgs, st);
}

}  // namespace ss
