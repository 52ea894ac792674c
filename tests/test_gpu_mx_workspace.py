"""One workspace, zeroed once, serves the attention over a cache in a microscaling format and ss_msa_attention in turn."""
import pytest
import torch

import mx_device as dev
import test_gpu_workspace as bf16
from paper_2402_11131_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FP8, FP4 = api.SS_KV_MXFP8, api.SS_KV_MXFP4
# B, T, gamma, H, Hkv, D, lengths, format: several splits of up to 32 rows, of 80, of 120; one split
MX = {"few_rows": (2, 4, 1, 4, 4, 64, (3000, 1777), FP4), "shared_keys": (2, 16, 4, 4, 2, 128, (2500, 900), FP8),
      "two_tiles_per_wave": (1, 24, 4, 2, 2, 128, (4000,), FP4), "one_split": (3, 1, 0, 4, 4, 128, (40, 200, 7), FP8)}


def test_calls_of_both_kinds_alternate_in_one_workspace():
    calls, want, need = {}, {}, 0
    for i, (name, (B, T, gamma, H, Hkv, D, lens, fmt)) in enumerate(MX.items()):
        d = dev.problem(400 + i, B, T, gamma, H, Hkv, D, 16, lens, fmt, max(lens))
        cap = d["table"].shape[1] * 16
        assert (api.ss_msa_mx_plan(B, T, gamma, H, Hkv, D, cap)[0] > 1) == (name != "one_split")
        need = max(need, api.ss_msa_mx_workspace_bytes(B, T, gamma, H, Hkv, D, cap))
        calls[name] = lambda ws, d=d, g=gamma: dev.call(d, g, 0.1, workspace=ws, out=torch.full_like(d["q"], 3.0))
        want[name] = dev.call(d, gamma, 0.1)                       # a fresh workspace each
        for b in range(B):
            dev.check(d, want[name], fmt, gamma, 0.1, 16, b, Hkv - 1)
    for name in ("two_splits_large", "two_splits_batch_5", "merge_kernel", "cut_on_the_device"):
        shape, args = bf16._args(name)
        assert api.ss_msa_plan(*shape)[0] > 1
        need = max(need, api.ss_msa_workspace_bytes(*shape))
        calls[name] = lambda ws, args=args: api.ss_msa_attention(*args, out=torch.full_like(args[0], 3.0), workspace=ws)
        want[name] = api.ss_msa_attention(*args)
    ws = api.ss_msa_workspace_init(torch.empty(need, dtype=torch.uint8, device=DEV))
    order = ["few_rows", "two_splits_large", "few_rows", "shared_keys", "cut_on_the_device", "shared_keys", "two_splits_batch_5", "two_tiles_per_wave",
             "merge_kernel", "few_rows", "one_split", "two_splits_large", "two_tiles_per_wave", "shared_keys"]
    assert set(order) == set(calls)
    for name in order:
        assert torch.equal(calls[name](ws), want[name]), name
