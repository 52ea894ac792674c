"""The calls on a cache in a microscaling format with their outputs, caches and workspaces inside guard bytes, at ragged shapes: the
guards stay as they were (what is written is checked by the parity tests)."""
import pytest
import torch

import mx_device as dev
from paper_2402_11131_amd import api
from test_gpu_canaries import Guarded, _check_all

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FMTS = [api.SS_KV_MXFP8, api.SS_KV_MXFP4]
I32 = torch.int32


def _cache(num, Hkv, page, D, fmt):
    row = D if fmt == api.SS_KV_MXFP8 else D // 2
    return [Guarded((num, Hkv, page, n), torch.uint8) for n in (row, D // 32, row, D // 32)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,page,Hkv", [(64, 16, 3), (128, 64, 1), (128, 16, 2)])
@pytest.mark.parametrize("fmt", FMTS)
def test_append_commit_and_read(fmt, D, page, Hkv, dtype):
    B, cols, S, T, gamma, depth = 3, 3, 37, 5, 2, 4
    cap = cols * page
    cache = _cache(B * cols, Hkv, page, D, fmt)
    mem = [c.t for c in cache]
    table = torch.arange(B * cols, dtype=I32, device=DEV).view(B, cols)          # the last page of the pool is used to its end
    rows = [torch.randn((B, S, Hkv, D), device=DEV).to(dtype) for _ in range(2)]
    new = Guarded((B,), I32)
    lens = torch.tensor([0, 11, cap - 20], dtype=I32, device=DEV)
    api.ss_kv_append_mx(*rows, *mem, table, lens, torch.tensor([S, 1, S], dtype=I32, device=DEV), new.t)
    _check_all(cache + [new], "ss_kv_append_mx")
    assert new.t.tolist() == [S, 12, cap]
    step = [torch.randn((B, T * (1 + gamma), Hkv, D), device=DEV).to(dtype) for _ in range(2)]
    path = torch.zeros((B, depth + 1), dtype=I32, device=DEV)
    lens = torch.tensor([0, 11, cap - 2], dtype=I32, device=DEV)
    api.ss_kv_commit_mx(*step, *mem, table, lens, path, torch.tensor([depth, -1, depth], dtype=I32, device=DEV), gamma, new.t)
    _check_all(cache + [new], "ss_kv_commit_mx")
    assert new.t.tolist() == [depth + 1, 11, cap]
    for n in (1, 37, cap, cap + 5):
        out = [Guarded((B, n, Hkv, D), dtype) for _ in range(2)]
        api.ss_kv_read_mx(*mem, table, torch.tensor([cap, 12, cap], dtype=I32, device=DEV), out[0].t, out[1].t)
        _check_all(out, "ss_kv_read_mx")
    _check_all(cache, "ss_kv_read_mx")


# one tile, two; three, four and five, a wave each; six and eight, two per wave; several chunks
@pytest.mark.parametrize("T,gamma,H", [(1, 0, 2), (7, 1, 4), (7, 4, 2), (7, 7, 2), (11, 3, 4), (7, 5, 4), (13, 4, 4), (33, 4, 4)])
@pytest.mark.parametrize("D,page,fmt", [(64, 16, FMTS[0]), (64, 64, FMTS[1]), (128, 16, FMTS[1]), (128, 32, FMTS[0])])
def test_attention(T, gamma, H, D, page, fmt):
    for lens in ((0, 5, 64), (1100, 333, 1)):
        d = dev.problem(7 * T + D, 3, T, gamma, H, 2, D, page, lens, fmt, max(lens))
        cap = d["table"].shape[1] * page
        ws = Guarded((api.ss_msa_mx_workspace_bytes(3, T, gamma, H, 2, D, cap),), torch.uint8)
        api.ss_msa_workspace_init(ws.t)
        out = Guarded(tuple(d["q"].shape), torch.bfloat16)
        for kept in (None, torch.tensor([T, 1, max(T // 2, 1)], dtype=I32, device=DEV)):
            dev.call(d, gamma, 0.1, out=out.t, workspace=ws.t, n_nodes=kept)
            _check_all([out, ws], "ss_msa_attention_mx")


@pytest.mark.parametrize("T,gamma", [(3, 1), (16, 4), (20, 4)])
@pytest.mark.parametrize("fmt", FMTS)
def test_entries_behind_a_table_of_one_page_are_not_read(T, gamma, fmt):
    d = dev.problem(9, 2, T, gamma, 2, 2, 64, 16, (16, 15), fmt, 16)
    assert d["table"].shape == (2, 1)
    tab = Guarded((2, 1), I32)
    tab.buf.view(I32)[:] = 0x7fffffff
    tab.t.copy_(d["table"])
    assert torch.equal(dev.call(dict(d, table=tab.t), gamma, 0.1), dev.call(d, gamma, 0.1))
