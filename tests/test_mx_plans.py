"""Host logic of the plans of the attention over a cache in a microscaling format (no GPU)."""
import pytest

from paper_2402_11131_amd import api

SHAPES = [(1, 1, 0, 1, 1, 64), (4, 16, 4, 32, 32, 128), (8, 32, 4, 32, 8, 128), (64, 1, 0, 32, 4, 128), (1, 1, 0, 8, 8, 128)]


@pytest.mark.parametrize("shape", SHAPES)
def test_lengths_beyond_what_a_table_may_hold(shape):
    want = api.ss_msa_mx_plan(*shape, 1 << 30), api.ss_msa_mx_workspace_bytes(*shape, 1 << 30)
    assert want[0][0] > 1
    for n in ((1 << 30) + 1, (1 << 31) - 4096, (1 << 31) - 1):
        assert (api.ss_msa_mx_plan(*shape, n), api.ss_msa_mx_workspace_bytes(*shape, n)) == want
