// n5: the paged cache in microscaling formats: rows quantised as they are written (a prompt's or a step's accepted path), and
// read back.  Each kernel reads and writes every value once, a few operations each: bytes and launches are what it costs.  Alone:
// a step's accepted path 3 us to write and 3 to read; 8192 rows of 32 heads of 128 from bf16 to 4 bits (170 MB) 26 us, 6.5 TB/s;
// 257 MB of bf16 rows from 4 bits 47 us, 6.9 TB/s.
#include <type_traits>

#include "ss_mx.h"

namespace ss {

int mx_check(const char* fn, int Hkv, int D, int page_size, int max_pages_per_seq, int num_pages, int format, const void* k_cache,
             const void* k_scale, const void* v_cache, const void* v_scale, const void* block_table, bool tensors) {
  SS_REQUIRE(Hkv >= 1 && Hkv <= 65535, SS_ERR_INVALID_ARG, "%s: Hkv=%d", fn, Hkv);
  SS_REQUIRE(D == 64 || D == 128, SS_ERR_UNSUPPORTED, "%s: head dim %d not in {64,128}", fn, D);
  SS_REQUIRE(format == SS_KV_MXFP8 || format == SS_KV_MXFP4, SS_ERR_UNSUPPORTED, "%s: format %d", fn, format);
  SS_REQUIRE(page_size == 16 || page_size == 32 || page_size == 64, SS_ERR_UNSUPPORTED, "%s: page_size %d not in {16,32,64}", fn,
             page_size);
  SS_REQUIRE(max_pages_per_seq >= 1 && num_pages >= 1, SS_ERR_INVALID_ARG, "%s: max_pages_per_seq=%d num_pages=%d", fn,
             max_pages_per_seq, num_pages);
  SS_REQUIRE((long)max_pages_per_seq * page_size <= kMxMaxLen, SS_ERR_UNSUPPORTED, "%s: sequence capacity too large", fn);
  if (!tensors) return SS_OK;
  SS_REQUIRE(k_cache && k_scale && v_cache && v_scale && block_table, SS_ERR_INVALID_ARG, "%s: NULL tensor argument", fn);
  SS_REQUIRE((((uintptr_t)k_cache | (uintptr_t)v_cache) & 15) == 0 && (((uintptr_t)k_scale | (uintptr_t)v_scale) & 3) == 0,
             SS_ERR_INVALID_ARG, "%s: a cache not aligned to 16 bytes, or scales not to 4", fn);
  return SS_OK;
}

// ------------------------------------------------------------------ writing
struct MxWriteArgs {
  MxCache c;
  const void *k_rows, *v_rows;  // [B,S,Hkv,D]
  const int32_t* seq_lens;      // position of the first row that is written
  const int32_t* path;          // [B,n_path] row of S that is written j-th, or NULL: row j
  const int32_t* count;         // rows of the sequence; with a path: its last entry's index
  int32_t* new_seq_lens;
  int S, n_path, T;  // rows per sequence in k_rows; entries of a path; rows a path may name
};

// Four lanes hold a block, eight features each; a workgroup takes rows of one head, so that what it writes is contiguous in the
// page.  E: the rows' type.
template <typename E>
struct MxIn;
template <>
struct MxIn<uint16_t> {
  uintx4 v;
  SS_DEV void load(const void* p, size_t at) { v = *reinterpret_cast<const uintx4*>((const uint16_t*)p + at); }
  SS_DEV uint32_t amax() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(max(m, v[i] & 0x7fffu), (v[i] >> 16) & 0x7fffu);
    return m << 16;
  }
  template <bool FP8>
  SS_DEV uintx2 codes(float scale) const {
    uint32_t out[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 x = __builtin_bit_cast(bf16x2, (uint32_t)v[i]);
      if constexpr (FP8) {
        const shortx2 old = __builtin_bit_cast(shortx2, out[i >> 1]);
        out[i >> 1] = __builtin_bit_cast(uint32_t, (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, x, scale, true)
                                                           : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, x, scale, false));
      } else {
        if (i == 0) out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out[0], x, scale, 0);
        if (i == 1) out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out[0], x, scale, 1);
        if (i == 2) out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out[0], x, scale, 2);
        if (i == 3) out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out[0], x, scale, 3);
      }
    }
    return uintx2{out[0], out[1]};
  }
};
template <>
struct MxIn<float> {
  floatx4 v[2];
  SS_DEV void load(const void* p, size_t at) {
    v[0] = reinterpret_cast<const floatx4*>((const float*)p + at)[0];
    v[1] = reinterpret_cast<const floatx4*>((const float*)p + at)[1];
  }
  SS_DEV uint32_t amax() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i >> 2][i & 3]) & 0x7fffffffu);
    return m;
  }
  template <bool FP8>
  SS_DEV uintx2 codes(float scale) const {
    uint32_t out[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = v[i >> 1][2 * (i & 1)], y = v[i >> 1][2 * (i & 1) + 1];
      if constexpr (FP8) {
        const shortx2 old = __builtin_bit_cast(shortx2, out[i >> 1]);
        out[i >> 1] = __builtin_bit_cast(uint32_t, (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, x, y, scale, true)
                                                           : __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, x, y, scale, false));
      } else {
        if (i == 0) out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out[0], x, y, scale, 0);
        if (i == 1) out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out[0], x, y, scale, 1);
        if (i == 2) out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out[0], x, y, scale, 2);
        if (i == 3) out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out[0], x, y, scale, 3);
      }
    }
    return uintx2{out[0], out[1]};
  }
};

constexpr int kMxThreads = 256;
// Rows of a thread, all of whose loads go out first.  Four prompts of 2048 rows (32 heads of 128, bf16 to 4 bits) and reading
// back 3500 to 4096: 105 us with one row, 88 with two, 101 with four; with one, the writer waits for its page id and its row alone.
constexpr int kMxRows = 2;

template <typename E, bool FP8>
__global__ __launch_bounds__(kMxThreads) void kv_write_mx_kernel(MxWriteArgs a) {
  const int shift = a.c.D == 128 ? 4 : 3, per_pass = kMxThreads >> shift;  // lanes of a row (log 2), rows of a pass
  const unsigned chunk = blockIdx.x / (unsigned)a.c.Hkv;  // heads first: neighbouring workgroups share rows
  const int b = blockIdx.z, h = blockIdx.x - chunk * a.c.Hkv;
  const int j0 = (int)chunk * per_pass * kMxRows + (threadIdx.x >> shift), d0 = (threadIdx.x & ((1 << shift) - 1)) * 8;
  const int cap = a.c.max_pages * a.c.page;
  const int L = min(max(a.seq_lens[b], 0), cap);
  const int n = a.path ? min(max(a.count[b], -1), a.n_path - 1) + 1 : min(max(a.count[b], 0), a.S);
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.new_seq_lens) a.new_seq_lens[b] = L + min(n, cap - L);
  const int end = min(n, cap - L);
  if (j0 >= end) return;
  MxIn<E> x[kMxRows][2];
  size_t at[kMxRows];
#pragma unroll
  for (int r = 0; r < kMxRows; ++r) {
    const int j = min(j0 + r * per_pass, end - 1);  // (rows past the end: the last one again, not written)
    const int row = a.path ? min(max(a.path[(size_t)b * a.n_path + j], 0), a.T - 1) : j;
    const size_t src = (((size_t)b * a.S + row) * a.c.Hkv + h) * a.c.D + d0;
    x[r][0].load(a.k_rows, src);
    x[r][1].load(a.v_rows, src);
    at[r] = mx_row(a.c, mx_page(a.c, b, L + j), h, L + j);
  }
#pragma unroll
  for (int r = 0; r < kMxRows; ++r) {
    if (j0 + r * per_pass >= end) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t m = x[r][i].amax();  // of the block: over its four lanes
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0xB1, 0xf, 0xf, false));
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0x4E, 0xf, 0xf, false));
      const int s = mx_scale_code<FP8>(m);
      uintx2 code = x[r][i].template codes<FP8>(mx_scale(s));
      if (s == 255) code = uintx2{0u, 0u};
      uint8_t* to = (i ? a.c.v : a.c.k) + at[r] * mx_row_bytes(a.c.D, FP8);
      if constexpr (FP8) *reinterpret_cast<uintx2*>(to + d0) = code;
      else *reinterpret_cast<uint32_t*>(to + d0 / 2) = code[0];
      if ((threadIdx.x & 3) == 0) (i ? a.c.vs : a.c.ks)[at[r] * (a.c.D / kMxBlock) + d0 / kMxBlock] = (uint8_t)s;
    }
  }
}

static int launch_write(const char* fn, const MxWriteArgs& a, int B, int rows, int dtype, int format, hipStream_t st) {
  const int per_wg = kMxThreads / (a.c.D >> 3) * kMxRows;
  SS_REQUIRE((long)ceil_div(rows, per_wg) * a.c.Hkv <= kMxMaxThreads / kMxThreads, SS_ERR_UNSUPPORTED, "%s: grid too large", fn);
  const dim3 grid((unsigned)(ceil_div(rows, per_wg) * a.c.Hkv), 1, (unsigned)B);
  auto kern = dtype == SS_F32 ? (format == SS_KV_MXFP8 ? kv_write_mx_kernel<float, true> : kv_write_mx_kernel<float, false>)
                              : (format == SS_KV_MXFP8 ? kv_write_mx_kernel<uint16_t, true> : kv_write_mx_kernel<uint16_t, false>);
  hipLaunchKernelGGL(kern, grid, dim3(kMxThreads), 0, st, a);
  return check_launch(fn);
}

// ------------------------------------------------------------------ reading
struct MxReadArgs {
  MxCache c;
  const int32_t *first, *seq_lens;
  void *k_rows, *v_rows;  // [B,S,Hkv,D]
  int S;
};

// STREAM: rows are stored past the caches.  Two sequences of 32768 tokens, 8 heads of 128 (257 MB of rows): 48 us, 6.8 TB/s,
// against 66.  Rows that the caches can hold stay there for who reads them next.
constexpr size_t kMxStreamBytes = 32u << 20;  // the L2 caches of the chip
template <typename E, bool FP8, bool STREAM>
__global__ __launch_bounds__(kMxThreads) void kv_read_mx_kernel(MxReadArgs a) {
  auto put = [](auto* p, auto v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
  };
  const int shift = a.c.D == 128 ? 4 : 3, per_pass = kMxThreads >> shift;
  const unsigned chunk = blockIdx.x / (unsigned)a.c.Hkv;  // heads first: neighbouring workgroups share rows
  const int b = blockIdx.z, h = blockIdx.x - chunk * a.c.Hkv;
  const int j0 = (int)chunk * per_pass * kMxRows + (threadIdx.x >> shift), d0 = (threadIdx.x & ((1 << shift) - 1)) * 8;
  const int L = min(max(a.seq_lens[b], 0), a.c.max_pages * a.c.page);
  const int first = a.first ? max(a.first[b], 0) : 0;
  const int end = first >= L ? 0 : min(a.S, L - first);
  if (j0 >= end) return;
  typedef std::conditional_t<FP8, uintx2, uint32_t> Raw;
  Raw w[kMxRows][2];
  uint32_t code[kMxRows][2];
#pragma unroll
  for (int r = 0; r < kMxRows; ++r) {
    const int pos = first + min(j0 + r * per_pass, end - 1);  // (rows past the end: the last one again, not written)
    const size_t at = mx_row(a.c, mx_page(a.c, b, pos), h, pos);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[r][i] = *reinterpret_cast<const Raw*>((i ? a.c.v : a.c.k) + at * mx_row_bytes(a.c.D, FP8) + (FP8 ? d0 : d0 / 2));
      code[r][i] = (i ? a.c.vs : a.c.ks)[at * (a.c.D / kMxBlock) + d0 / kMxBlock];
    }
  }
#pragma unroll
  for (int r = 0; r < kMxRows; ++r) {
    const int j = j0 + r * per_pass;
    if (j >= end) return;
    const size_t to = (((size_t)b * a.S + j) * a.c.Hkv + h) * a.c.D + d0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float scale = mx_scale((int)code[r][i]);
      floatx2 x[4];
      if constexpr (FP8) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[2 * e] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[r][i][e], scale, false);
          x[2 * e + 1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[r][i][e], scale, true);
        }
      } else {
        x[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[r][i], scale, 0);
        x[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[r][i], scale, 1);
        x[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[r][i], scale, 2);
        x[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[r][i], scale, 3);
      }
      void* out = i ? a.v_rows : a.k_rows;
      if constexpr (sizeof(E) == 4) {
        floatx4* o = reinterpret_cast<floatx4*>((float*)out + to);
        put(&o[0], floatx4{x[0][0], x[0][1], x[1][0], x[1][1]});
        put(&o[1], floatx4{x[2][0], x[2][1], x[3][0], x[3][1]});
      } else {  // exact but for e4m3 values below 2^-133, which are rounded to nearest even
        uintx4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bf16x2 v = {(__bf16)x[e][0], (__bf16)x[e][1]};
          o[e] = __builtin_bit_cast(uint32_t, v);
        }
        put(reinterpret_cast<uintx4*>((uint16_t*)out + to), o);
      }
    }
  }
}

template <typename E>
static auto read_kernel(int format, bool stream) {
  if (format == SS_KV_MXFP8) return stream ? kv_read_mx_kernel<E, true, true> : kv_read_mx_kernel<E, true, false>;
  return stream ? kv_read_mx_kernel<E, false, true> : kv_read_mx_kernel<E, false, false>;
}

static MxCache mx_cache(void* k, void* ks, void* v, void* vs, const int32_t* block_table, int max_pages, int num_pages, int Hkv, int D,
                        int page) {
  MxCache c;
  c.k = (uint8_t*)k; c.ks = (uint8_t*)ks; c.v = (uint8_t*)v; c.vs = (uint8_t*)vs;
  c.block_table = block_table; c.Hkv = Hkv; c.D = D; c.page = page;
  c.page_shift = page == 16 ? 4 : (page == 32 ? 5 : 6);
  c.max_pages = max_pages; c.num_pages = num_pages;
  return c;
}
static int check_rows(const char* fn, int B, int dtype, const void* k_rows, const void* v_rows) {
  SS_REQUIRE(B <= 65535, SS_ERR_UNSUPPORTED, "%s: B=%d", fn, B);
  SS_REQUIRE(k_rows && v_rows, SS_ERR_INVALID_ARG, "%s: NULL tensor argument", fn);
  SS_REQUIRE((((uintptr_t)k_rows | (uintptr_t)v_rows) & 15) == 0, SS_ERR_INVALID_ARG, "%s: rows not aligned to 16 bytes", fn);
  return SS_OK;
}
// New lengths are written while other workgroups still read what the call was given.
static bool shares(const int32_t* out, long n_out, const int32_t* in, long n_in) {
  return out != nullptr && (uintptr_t)out < (uintptr_t)(in + n_in) && (uintptr_t)in < (uintptr_t)(out + n_out);
}

}  // namespace ss

extern "C" {

int ss_kv_append_mx(const void* k_rows, const void* v_rows, void* k_cache, void* k_scale, void* v_cache, void* v_scale,
                    const int32_t* block_table, int max_pages_per_seq, int num_pages, const int32_t* seq_lens, const int32_t* n_rows,
                    int B, int S, int Hkv, int D, int page_size, int dtype, int format, int32_t* new_seq_lens, void* stream) {
  using namespace ss;
  clear_error();
  const char* fn = "ss_kv_append_mx";
  SS_REQUIRE(B >= 0 && S >= 0, SS_ERR_INVALID_ARG, "%s: B=%d S=%d", fn, B, S);
  SS_REQUIRE(S <= (1 << 30), SS_ERR_UNSUPPORTED, "%s: S=%d", fn, S);
  SS_REQUIRE(dtype == SS_F32 || dtype == SS_BF16, SS_ERR_UNSUPPORTED, "%s: dtype %d", fn, dtype);
  if (int rc = mx_check(fn, Hkv, D, page_size, max_pages_per_seq, num_pages, format, k_cache, k_scale, v_cache, v_scale, block_table, B > 0)) return rc;
  if (B == 0) return SS_OK;
  if (S > 0)
    if (int rc = check_rows(fn, B, dtype, k_rows, v_rows)) return rc;
  SS_REQUIRE(B <= 65535, SS_ERR_UNSUPPORTED, "%s: B=%d", fn, B);
  SS_REQUIRE(seq_lens && n_rows, SS_ERR_INVALID_ARG, "%s: NULL seq_lens or n_rows", fn);
  SS_REQUIRE(!shares(new_seq_lens, B, seq_lens, B) && !shares(new_seq_lens, B, n_rows, B) &&
                 !shares(new_seq_lens, B, block_table, (long)B * max_pages_per_seq),
             SS_ERR_INVALID_ARG, "%s: new_seq_lens shares memory with seq_lens, n_rows or block_table", fn);
  MxWriteArgs a;
  a.c = mx_cache(k_cache, k_scale, v_cache, v_scale, block_table, max_pages_per_seq, num_pages, Hkv, D, page_size);
  a.k_rows = k_rows; a.v_rows = v_rows; a.seq_lens = seq_lens; a.path = nullptr; a.count = n_rows; a.new_seq_lens = new_seq_lens;
  a.S = S; a.n_path = 0; a.T = S;
  return launch_write(fn, a, B, S < 1 ? 1 : S, dtype, format, (hipStream_t)stream);
}

int ss_kv_commit_mx(const void* k_new, const void* v_new, void* k_cache, void* k_scale, void* v_cache, void* v_scale,
                    const int32_t* block_table, int max_pages_per_seq, int num_pages, const int32_t* seq_lens, const int32_t* path,
                    const int32_t* n_accept, int B, int T, int gamma, int Hkv, int D, int page_size, int max_depth, int dtype, int format,
                    int32_t* new_seq_lens, void* stream) {
  using namespace ss;
  clear_error();
  const char* fn = "ss_kv_commit_mx";
  SS_REQUIRE(B >= 0, SS_ERR_INVALID_ARG, "%s: B=%d", fn, B);
  SS_REQUIRE(T >= 1 && T <= SS_MAX_T, SS_ERR_UNSUPPORTED, "%s: T=%d outside [1,%d]", fn, T, SS_MAX_T);
  SS_REQUIRE(gamma >= 0 && gamma <= SS_MAX_GAMMA, SS_ERR_UNSUPPORTED, "%s: gamma=%d outside [0,%d]", fn, gamma, SS_MAX_GAMMA);
  SS_REQUIRE(dtype == SS_F32 || dtype == SS_BF16, SS_ERR_UNSUPPORTED, "%s: dtype %d", fn, dtype);
  SS_REQUIRE(max_depth >= 0 && max_depth < SS_MAX_T, SS_ERR_INVALID_ARG, "%s: max_depth=%d", fn, max_depth);
  if (int rc = mx_check(fn, Hkv, D, page_size, max_pages_per_seq, num_pages, format, k_cache, k_scale, v_cache, v_scale, block_table, B > 0)) return rc;
  if (B == 0) return SS_OK;
  if (int rc = check_rows(fn, B, dtype, k_new, v_new)) return rc;
  SS_REQUIRE(seq_lens && path && n_accept, SS_ERR_INVALID_ARG, "%s: NULL tensor argument", fn);
  SS_REQUIRE(!shares(new_seq_lens, B, seq_lens, B) && !shares(new_seq_lens, B, n_accept, B) &&
                 !shares(new_seq_lens, B, path, (long)B * (max_depth + 1)) && !shares(new_seq_lens, B, block_table, (long)B * max_pages_per_seq),
             SS_ERR_INVALID_ARG, "%s: new_seq_lens shares memory with seq_lens, path, n_accept or block_table", fn);
  MxWriteArgs a;
  a.c = mx_cache(k_cache, k_scale, v_cache, v_scale, block_table, max_pages_per_seq, num_pages, Hkv, D, page_size);
  a.k_rows = k_new; a.v_rows = v_new; a.seq_lens = seq_lens; a.path = path; a.count = n_accept; a.new_seq_lens = new_seq_lens;
  a.S = T * (1 + gamma); a.n_path = max_depth + 1; a.T = T;
  return launch_write(fn, a, B, max_depth + 1, dtype, format, (hipStream_t)stream);
}

int ss_kv_read_mx(const void* k_cache, const void* k_scale, const void* v_cache, const void* v_scale, const int32_t* block_table,
                  int max_pages_per_seq, int num_pages, const int32_t* first, const int32_t* seq_lens, int B, int S, int Hkv, int D,
                  int page_size, int dtype, int format, void* k_rows, void* v_rows, void* stream) {
  using namespace ss;
  clear_error();
  const char* fn = "ss_kv_read_mx";
  SS_REQUIRE(B >= 0 && S >= 0, SS_ERR_INVALID_ARG, "%s: B=%d S=%d", fn, B, S);
  SS_REQUIRE(S <= (1 << 30), SS_ERR_UNSUPPORTED, "%s: S=%d", fn, S);
  SS_REQUIRE(dtype == SS_F32 || dtype == SS_BF16, SS_ERR_UNSUPPORTED, "%s: dtype %d", fn, dtype);
  if (int rc = mx_check(fn, Hkv, D, page_size, max_pages_per_seq, num_pages, format, k_cache, k_scale, v_cache, v_scale, block_table, B > 0 && S > 0)) return rc;
  if (B == 0 || S == 0) return SS_OK;
  if (int rc = check_rows(fn, B, dtype, k_rows, v_rows)) return rc;
  SS_REQUIRE(seq_lens, SS_ERR_INVALID_ARG, "%s: NULL seq_lens", fn);
  MxReadArgs a;
  a.c = mx_cache((void*)k_cache, (void*)k_scale, (void*)v_cache, (void*)v_scale, block_table, max_pages_per_seq, num_pages, Hkv, D, page_size);
  a.first = first; a.seq_lens = seq_lens; a.k_rows = k_rows; a.v_rows = v_rows; a.S = S;
  const int per_wg = kMxThreads / (D >> 3) * kMxRows;
  SS_REQUIRE((long)ceil_div(S, per_wg) * Hkv <= kMxMaxThreads / kMxThreads, SS_ERR_UNSUPPORTED, "%s: grid too large", fn);
  const dim3 grid((unsigned)(ceil_div(S, per_wg) * Hkv), 1, (unsigned)B);
  const bool stream_out = 2 * (size_t)B * S * Hkv * D * (dtype == SS_F32 ? 4 : 2) > kMxStreamBytes;
  auto kern = dtype == SS_F32 ? read_kernel<float>(format, stream_out) : read_kernel<uint16_t>(format, stream_out);
  hipLaunchKernelGGL(kern, grid, dim3(kMxThreads), 0, (hipStream_t)stream, a);
  return check_launch(fn);
}

}  // extern "C"
