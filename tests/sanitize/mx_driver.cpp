// Calls the host side of the calls on a cache in a microscaling format: the plan and workspace queries over their whole ranges, and
// the refusals, none of which enqueues anything.  Built with the host pass under -fsanitize=address,undefined by
// tests/test_mx_sanitizers.py; exits 0 if nothing was reported.
#include <limits.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "ss.h"

int main() {
  const int lens[] = {INT_MIN, -1, 0, 1, 127, 128, 129, 409, 410, 4096, 32768, 1 << 20, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, INT_MAX};
  const int shapes[][6] = {{0, 1, 0, 1, 1, 64},        {1, 1, 0, 1, 1, 64},        {1, 64, 8, 4096, 1, 128}, {4, 16, 4, 32, 32, 128},
                           {8, 32, 4, 32, 8, 128},     {64, 1, 0, 32, 4, 128},     {65535, 1, 0, 8, 8, 64},  {65535, 64, 8, 65536, 64, 128},
                           {3, 20, 3, 40, 8, 64},      {512, 1, 0, 1, 1, 128},     {1, 1, 8, 65535, 65535, 128}};
  for (const auto& s : shapes)
    for (int len : lens) {
      int n = 0, rows = 0;
      if (ss_msa_mx_plan(s[0], s[1], s[2], s[3], s[4], s[5], len, &n, &rows) != SS_OK || n < 1 || n > 256 || rows < 16 || rows > 128) return 2;
      if (ss_msa_mx_workspace_bytes(s[0], s[1], s[2], s[3], s[4], s[5], len) < 256) return 3;
      if (ss_msa_mx_plan(s[0], s[1], s[2], s[3], s[4], s[5], len, nullptr, nullptr) != SS_OK) return 4;
    }
  if (ss_msa_mx_workspace_bytes(1, 1, 0, 1, 1, 96, 64) != 0 || ss_msa_mx_workspace_bytes(-1, 1, 0, 1, 1, 64, 64) != 0) return 5;
  // refusals at the ends of the ranges; pointers are never dereferenced
  void* const p = (void*)4096;
  int32_t* const i = (int32_t*)4096;
  int32_t* const out = (int32_t*)(1 << 30);
  if (ss_kv_append_mx(p, p, p, p, p, p, i, INT_MAX, INT_MAX, i, i, 65535, 1 << 30, 65535, 128, 64, SS_F32, SS_KV_MXFP8, out, nullptr) != SS_ERR_UNSUPPORTED) return 6;
  if (ss_kv_append_mx(p, p, p, p, p, p, i, 1 << 24, INT_MAX, i, i, 65535, 1 << 30, 65535, 128, 64, SS_F32, SS_KV_MXFP8, out, nullptr) == SS_OK) return 7;
  if (ss_kv_read_mx(p, p, p, p, i, 1 << 24, INT_MAX, nullptr, i, 65535, 1 << 30, 65535, 64, 64, SS_BF16, SS_KV_MXFP4, p, p, nullptr) == SS_OK) return 8;
  if (ss_kv_commit_mx(p, p, p, p, p, p, i, 1 << 24, INT_MAX, i, i, i, 65535, 64, 8, 65535, 128, 64, 63, SS_BF16, SS_KV_MXFP4, i + 1, nullptr) != SS_ERR_INVALID_ARG)
    return 9;
  if (ss_msa_attention_mx(p, p, p, p, p, p, p, i, 1 << 24, INT_MAX, i, i, nullptr, 65535, 64, 8, 65535, 65535, 128, 64, 1.f, SS_KV_MXFP4, 0, p, p, SIZE_MAX,
                          nullptr) != SS_ERR_UNSUPPORTED)
    return 10;
  if (ss_msa_attention_mx(p, p, p, p, p, p, p, i, 1 << 24, 1, i, i, nullptr, 65535, 64, 8, 65535, 65535, 128, 64, 1.f, SS_KV_MXFP4, 0, p, p, SIZE_MAX,
                          nullptr) != SS_ERR_UNSUPPORTED)
    return 11;
  printf("mx driver done\n");
  return 0;
}
