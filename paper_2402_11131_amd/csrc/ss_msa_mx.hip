// n5, a2 over a cache in microscaling formats: multi-stream attention (Eq. 1 / Eq. 2) on the gfx950 matrix cores.
//
// Work split.  A workgroup of four wavefronts owns one (sequence, KV head, split of the cached tokens, chunk of up to 16 NT
// query rows; the query heads of a group are folded into the rows).  Every wave holds ALL of the chunk's rows (queries, running
// maximum and sum, outputs in registers) and walks blocks of 32 keys of its own: what is done once per key, above all turning
// values into bf16, is then done by one wave only, and the waves need nothing from each other until their results are merged.
//
// Scores, S^T = K Q^T with v_mfma_scale_f32_16x16x128_f8f6f4: the cached elements and scale bytes are operands as they are.  A
// query row is the sum of two e4m3 rows, the second with a scale 2^-4 of the first's: four and four of a bf16 value's eight
// significant bits (features below 2^-17 of the row's largest lose bits, none more than 2^-22 of it).  Lane (lq, lg) = (lane &
// 15, lane >> 4) supplies, of a 4-bit operand, elements 32 lg .. +31 of row lq, of an 8-bit one elements 16 lg .. +15 and 64 +
// 16 lg .. +15; the scale of elements 32 g .. +31 comes from lane group g.  Heads of 128 take two instructions (one per part)
// for 16 keys and 16 queries; heads of 64 one, with the first part against elements 0..63 and the second against a repetition.
//
// O^T += V^T P^T with v_mfma_f32_16x16x32_bf16.  A scale belongs to one token, and the sum runs over tokens, so values are
// multiplied by their scales first: both formats are exact in bf16.  A lane turns a block of one token's features into bf16 and
// puts it into the wave's LDS tile (token-major, 16-byte chunks XOR-swizzled), the transposing read hands out four consecutive
// tokens of a feature.  Row sums are a further row of ones times P^T.
#include <math.h>

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

// 16-byte chunk of a row of the value tile where chunk c lies.  Writes take one chunk of 16 consecutive rows, transposing reads
// pieces of two neighbouring chunks of eight rows: both meet every bank once.
template <int D>
SS_DEV int v_swz(int row) {
  return D == 128 ? (((row & 7) << 1) | ((row >> 3) & 1)) : ((((row >> 1) & 3) << 1) | ((row >> 3) & 1));
}

template <int D, bool FP8, int NT>
__global__ __launch_bounds__(64 * kMxWaves) void msa_mx_kernel(MsaMxArgs a) {
  constexpr int DT = D / 16, KS = D / 32, NB = D / kMxBlock;
  constexpr int ROWB = FP8 ? D : D / 2;            // bytes of a cached row
  constexpr int TPL = 64 / NB, VL = 32 / TPL;      // tokens per load of values, loads per 32 tokens
  constexpr int VPIECES = FP8 ? 2 : 1;             // 16-byte pieces of a block
  constexpr int TILE = 32 * D * 2;                 // bytes of a wave's value tile
  constexpr int MERGE = NT * DT * 1024;            // bytes of a wave's outputs
  __shared__ __attribute__((aligned(16))) unsigned char smem[kMxWaves * TILE > 2 * MERGE ? kMxWaves * TILE : 2 * MERGE];
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
  const int par = a.parent[(size_t)b * a.T + min(lane, a.T - 1)];

  // query row of tile t that this lane's column lq is
  auto row_of = [&](int t, int& r, int& h) {
    const int f = min(f0 + 16 * t + lq, F - 1);
    const int fh = fast_div(f, R_kept), fr = f - fh * R_kept;
    r = fr < n_kept ? fr : a.T + (fr - n_kept);
    h = hk * a.g + fh;
    return f0 + 16 * t + lq < F;
  };

  // ---- queries as two e4m3 rows each
  intx8 Qh[NT], Ql[D == 128 ? NT : 1];
  int sq_h[NT], sq_l[D == 128 ? NT : 1];
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
      sq_h[t] = sh;
      sq_l[t] = sl;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        Qh[t][i] = (int)hi[i];
        Qh[t][4 + i] = (int)lo[i];
      }
      sq_h[t] = lg < 2 ? sh : sl;
    }
  }

  floatx4 O[NT][DT], Ls[NT];
  float m_run[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m_run[t] = -1e30f;
    Ls[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[t][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const float c = a.scale_log2, lazy_thr = kMxLazyLog2 / c;
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
  float pinf = INFINITY;  // see vmax2
  asm volatile("" : "+s"(pinf));

  unsigned char* tile = smem + w * TILE;
  // O += P V for 32 tokens in the tile, of which the lane's query row of tile t has the scores S
  auto attend = [&](int t, floatx4 (&S)[2]) {
    const float mx8 = vmax2(vmax2(vmax2(S[0][0], S[0][1], pinf), vmax2(S[0][2], S[0][3], pinf), pinf),
                            vmax2(vmax2(S[1][0], S[1][1], pinf), vmax2(S[1][2], S[1][3], pinf), pinf), pinf);
    if (__any(mx8 > m_run[t] + lazy_thr)) {
      const float mx = max_over_lane_groups(mx8, pinf);  // of the query row: a row's maximum moves by its own scores alone
      const float m_new = mx > m_run[t] + lazy_thr ? mx : m_run[t];
      const float alpha = __builtin_amdgcn_exp2f((m_run[t] - m_new) * c);
      Ls[t] *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[t][dt] *= alpha;
      m_run[t] = m_new;
    }
    const float nmc = -(m_run[t] * c);
    bf16x8 P;
#pragma unroll
    for (int X = 0; X < 2; ++X)
#pragma unroll
      for (int i = 0; i < 4; ++i) P[4 * X + i] = (__bf16)__builtin_amdgcn_exp2f(fmaf(S[X][i], c, nmc));
    Ls[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, P, Ls[t], 0, 0, 0);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      uintx2 half[2];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int row = 16 * hh + 4 * lg + (lq >> 2), ch = 2 * dt + ((lq & 3) >> 1);
        half[hh] = lds_read_tr16(tile + row * (2 * D) + ((ch ^ v_swz<D>(row)) * 16) + (lq & 1) * 8);
      }
      const uintx4 vv = uintx4{half[0][0], half[0][1], half[1][0], half[1][1]};
      O[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vv), P, O[t][dt], 0, 0, 0);
    }
  };
  // the wave's own LDS writes are done, and not moved over
  auto tile_ready = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };

  // ---- the step's own rows (split 0, which every sequence has)
  if (s == 0) {
    const int par_c = lane < a.T ? clamp_parent(par, lane) : -1;
    for (int c0 = 32 * w; c0 < a.R; c0 += 32 * kMxWaves) {
      const size_t own0 = ((size_t)b * a.R * a.c.Hkv + hk) * D;  // row 0 of this head
      const size_t stride = (size_t)a.c.Hkv * D;
      uintx4 kf[2][KS];
#pragma unroll
      for (int X = 0; X < 2; ++X)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          kf[X][ks] = ld16(a.k_new + own0 + min(c0 + 16 * X + lq, a.R - 1) * stride + 32 * ks + 8 * lg);
      constexpr int CPR = D / 8, RPL = 64 / CPR;  // chunks per row, rows per load
      tile_ready();
#pragma unroll
      for (int i = 0; i < 32 / RPL; ++i) {
        const int row = RPL * i + lane / CPR, ch = lane % CPR;
        const uintx4 v = ld16(a.v_new + own0 + min(c0 + row, a.R - 1) * stride + 8 * ch);
        *reinterpret_cast<uintx4*>(tile + row * (2 * D) + ((ch ^ v_swz<D>(row)) * 16)) = c0 + row < a.R ? v : uintx4{0u, 0u, 0u, 0u};
      }
      tile_ready();
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        int r, h;
        row_of(t, r, h);
        const int node = r < a.T ? r : (r - a.T) / max(a.gamma, 1), strm = r < a.T ? 0 : (r - a.T) % max(a.gamma, 1) + 1;
        const RowVis vis = make_row_vis(node, strm, ancestors_of(node, par_c), a.T, a.gamma, (a.flags & SS_STREAM_EXCLUDE_SELF) != 0);
        const uint16_t* qp = a.q + (((size_t)b * a.R + r) * a.H + h) * D + 8 * lg;
        floatx4 S[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 qv = as_bf16x8(ld16(qp + 32 * ks));
#pragma unroll
          for (int X = 0; X < 2; ++X) S[X] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[X][ks]), qv, S[X], 0, 0, 0);
        }
#pragma unroll
        for (int X = 0; X < 2; ++X)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = c0 + 16 * X + 4 * lg + i;
            const float sv = S[X][i];
            S[X][i] = (key < a.R) & row_sees(vis, key, a.T) ? sv : -INFINITY;
          }
        attend(t, S);
      }
    }
  }

  // ---- the cached tokens, 32 at a time
  for (int kb = k0 + 32 * w; kb < k1; kb += 32 * kMxWaves) {
    const int nv = min(k1 - kb, 32);
    intx8 K[2];
    int sk[2];
#pragma unroll
    for (int X = 0; X < 2; ++X) {
      const int pos = min(kb + 16 * X + lq, k1 - 1);
      const size_t row = mx_row(a.c, mx_page(a.c, b, pos), hk, pos);
      const uint8_t* kp = a.c.k + row * ROWB;
      sk[X] = a.c.ks[row * NB + lg % NB];
      uintx4 p0, p1 = uintx4{0u, 0u, 0u, 0u};
      if constexpr (FP8) {
        p0 = *reinterpret_cast<const uintx4*>(kp + 16 * lg);
        p1 = D == 128 ? *reinterpret_cast<const uintx4*>(kp + D / 2 + 16 * lg) : p0;
      } else {
        p0 = *reinterpret_cast<const uintx4*>(kp + 16 * (lg % NB));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        K[X][i] = (int)p0[i];
        K[X][4 + i] = (int)p1[i];
      }
    }
    tile_ready();  // the tile has been read
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int trow = TPL * i + lane % TPL, blk = lane / TPL;
      const int pos = min(kb + trow, k1 - 1);
      const size_t row = mx_row(a.c, mx_page(a.c, b, pos), hk, pos);
      const bool ok = trow < nv;
      const float scale = mx_scale(ok ? a.c.vs[row * NB + blk] : 127);
#pragma unroll
      for (int p = 0; p < VPIECES; ++p) {
        uintx4 raw = *reinterpret_cast<const uintx4*>(a.c.v + row * ROWB + blk * (16 * VPIECES) + 16 * p);
        if (!ok) raw = uintx4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int ch = 0; ch < 4 / VPIECES; ++ch) {
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
          const int chunk = 4 * blk + (4 / VPIECES) * p + ch;
          *reinterpret_cast<uintx4*>(tile + trow * (2 * D) + ((chunk ^ v_swz<D>(trow)) * 16)) = o;
        }
      }
    }
    tile_ready();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      floatx4 S[2];
#pragma unroll
      for (int X = 0; X < 2; ++X) {
        floatx4 acc = floatx4{0.f, 0.f, 0.f, 0.f};
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(K[X], Qh[t], acc, FP8 ? 0 : 4, 0, 0, sk[X], 0, sq_h[t]);
        if constexpr (D == 128) acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(K[X], Ql[t], acc, FP8 ? 0 : 4, 0, 0, sk[X], 0, sq_l[t]);
        S[X] = acc;
      }
      if (nv < 32) {
#pragma unroll
        for (int X = 0; X < 2; ++X)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float sv = S[X][i];
            S[X][i] = 16 * X + 4 * lg + i < nv ? sv : -INFINITY;
          }
      }
      attend(t, S);
    }
  }

  // ---- merge the waves: to a common maximum, then pairs of waves through LDS
#pragma unroll
  for (int t = 0; t < NT; ++t)
    if (lg == 0) {
      ml[w][t][0][lq] = m_run[t];
      ml[w][t][1][lq] = Ls[t][0];
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
  p.n_qc = ceil_div(tiles, 5);
  p.nt = ceil_div(tiles, p.n_qc);
  const long items = (long)B * Hkv * p.n_qc;
  const int len = max_len < 1 ? 1 : max_len;
  long n = (256 + items - 1) / (items < 1 ? 1 : items);
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
  auto kern = nt == 1 ? msa_mx_kernel<D, FP8, 1> : nt == 2 ? msa_mx_kernel<D, FP8, 2> : nt == 3 ? msa_mx_kernel<D, FP8, 3>
            : nt == 4 ? msa_mx_kernel<D, FP8, 4> : msa_mx_kernel<D, FP8, 5>;
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
