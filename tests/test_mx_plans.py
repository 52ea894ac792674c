"""Host logic of the plans of the attention over a cache in a microscaling format (no GPU)."""
import ctypes

import pytest

from paper_2402_11131_amd import api

SHAPES = [(1, 1, 0, 1, 1, 64), (4, 16, 4, 32, 32, 128), (8, 32, 4, 32, 8, 128), (64, 1, 0, 32, 4, 128), (1, 1, 0, 8, 8, 128)]


@pytest.mark.parametrize("shape", SHAPES)
def test_lengths_beyond_what_a_table_may_hold(shape):
    want = api.ss_msa_mx_plan(*shape, 1 << 30), api.ss_msa_mx_workspace_bytes(*shape, 1 << 30)
    assert want[0][0] > 1
    for n in ((1 << 30) + 1, (1 << 31) - 4096, (1 << 31) - 1):
        assert (api.ss_msa_mx_plan(*shape, n), api.ss_msa_mx_workspace_bytes(*shape, n)) == want


def test_slots_of_heads_of_128_in_8_bits():
    """Two workgroups of that instance fit a compute unit, three of the others with one query tile: 640 single tokens are more
    than one round of the chip, and are split; in 4 bits and heads of 64 they are not."""
    P = ctypes.c_void_p(4096)      # never dereferenced: the call is refused for want of a workspace
    rc = api.load_library().ss_msa_attention_mx(P, P, P, P, P, P, P, P, 256, 16, P, P, None, 20, 1, 0, 32, 32, 128, 16, ctypes.c_float(0.1),
                                                api.SS_KV_MXFP8, 0, P, None, 0, None)
    assert rc == 4 and b"workspace" in api.load_library().ss_last_error()
    # the queries answer for whichever format needs more
    n, rows = api.ss_msa_mx_plan(20, 1, 0, 32, 32, 128, 4096)
    assert n > 1 and rows == 16 and api.ss_msa_mx_workspace_bytes(20, 1, 0, 32, 32, 128, 4096) > 640 * n * 128 * 4 * 16
    assert api.ss_msa_mx_plan(20, 1, 0, 32, 32, 64, 4096) == (1, 16)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [api.SS_KV_MXFP8, api.SS_KV_MXFP4])
@pytest.mark.parametrize("B", [16, 20, 24])
def test_calls_around_a_round_of_the_chip(fmt, B):
    """512, 640 and 768 single tokens of heads of 128, with the workspace that the query asks for."""
    import mx_device as dev
    d = dev.problem(90 + B, B, 1, 0, 32, 32, 128, 16, [700 - 29 * i for i in range(B)], fmt, 4096)
    out = dev.call(d, 0, 0.1)
    for b, head in ((0, 0), (1, 31), (B // 2, 7), (B - 1, 20)):
        dev.check(d, out, fmt, 0, 0.1, 16, b, head)


@pytest.mark.gpu
def test_one_round_of_the_chip_needs_no_workspace():
    """512 single tokens of heads of 128 in 8 bits are one round, unsplit."""
    import torch
    import mx_device as dev
    d = dev.problem(95, 16, 1, 0, 32, 32, 128, 64, [4096] + [33] * 15, api.SS_KV_MXFP8, 4096)
    out = dev.call(d, 0, 0.1, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda:0"))
    assert torch.equal(out, dev.call(d, 0, 0.1))
    dev.check(d, out, api.SS_KV_MXFP8, 0, 0.1, 64, 0, 5)
