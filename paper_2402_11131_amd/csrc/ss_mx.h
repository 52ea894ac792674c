// The cache in microscaling formats: blocks of 32 features of one (token, KV head), elements of 8 bits (e4m3) or 4 bits (e2m1,
// the even feature in a byte's low half) and a scale byte s that stands for 2^(s-127), 255 for NaN.  Rows are token-major for
// keys and values alike: a value in 4 bits shares its byte with the neighbouring feature of its own token, so that tokens are
// written independently of each other.
#pragma once

#include "ss_common.h"

namespace ss {

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(2 * sizeof(short)))) short shortx2;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float floatx2;
typedef __attribute__((__vector_size__(8 * sizeof(int)))) int intx8;

constexpr int kMxBlock = 32;
constexpr long kMxMaxThreads = 0xffffffffL;  // of a launch, as the runtime counts them
constexpr int kMxMaxLen = 1 << 30;  // tokens that a row of a block table may hold
SS_HD int mx_row_bytes(int D, bool fp8) { return fp8 ? D : D / 2; }

// A cache as the kernels see it: keys and values have the same shape.
struct MxCache {
  uint8_t *k, *ks, *v, *vs;  // [num_pages,Hkv,page,row_bytes] and [num_pages,Hkv,page,D/32]
  const int32_t* block_table;
  int Hkv, D, page, page_shift, max_pages, num_pages;
};
SS_DEV int mx_page(const MxCache& c, int b, int pos) {
  return min(max(c.block_table[(size_t)b * c.max_pages + (pos >> c.page_shift)], 0), c.num_pages - 1);
}
// Where row `row` of a cache lies, `bytes` each.  Row indices take all 32 bits: as an int, which is what a lane's register is read
// as, one from 2^31 on would be widened to an address far in front of the cache.
SS_HD constexpr size_t mx_row_at(uint32_t row, int bytes) { return (size_t)row * (uint32_t)bytes; }
// Row of a position inside the cache, in tokens of one head.
SS_DEV size_t mx_row(const MxCache& c, int page, int h, int pos) {
  return ((size_t)page * c.Hkv + h) * c.page + (pos & (c.page - 1));
}

// Scale byte of a block whose largest magnitude has these fp32 bits: the smallest power of two that brings it to the largest
// element, 1.75 * 2^8 (e4m3) or 1.5 * 2^2 (e2m1), or below, so no element is clamped.  A NaN or an infinity gives 255.
template <bool FP8>
SS_DEV int mx_scale_code(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23);
  const int s = e - (FP8 ? 8 : 2) + ((amax_bits & 0x7fffffu) > (FP8 ? 0x600000u : 0x400000u) ? 1 : 0);
  return e == 255 ? 255 : max(s, 0);
}
// The scale as the conversion instructions take it: they look at a float's exponent alone, and 0 is 2^-127 to them.
SS_DEV float mx_scale(int code) { return __uint_as_float((uint32_t)code << 23); }

// What every call on such a cache requires; `tensors`: the pointers are looked at too (a call with nothing to do needs none).
int mx_check(const char* fn, int Hkv, int D, int page_size, int max_pages_per_seq, int num_pages, int format, const void* k_cache,
             const void* k_scale, const void* v_cache, const void* v_scale, const void* block_table, bool tensors);

}  // namespace ss
