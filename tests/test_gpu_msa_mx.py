"""GPU parity of the attention over a cache in a microscaling format (n5) against 64 bits; tests/mx_reference.py derives the
tolerance."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import oracle
from helpers import to_np_f32
from paper_2402_11131_amd import api, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FP8, FP4 = api.SS_KV_MXFP8, api.SS_KV_MXFP4


def _call(d, gamma, scale, **kw):
    return api.ss_msa_attention_mx(d["q"], d["k_new"], d["v_new"], *d["cache"], d["table"], d["lens"], d["parent"], gamma, scale, **kw)


def _check(host, out, fmt, gamma, scale, page, exclude_self=False, kept=None, before=None):
    got = to_np_f32(out)
    B, R, H, D = got.shape
    T = R // (1 + gamma)
    for b in range(B):
        K, V = ref.rows_of_cache(host["cache"], fmt, host["table"][b], int(host["lens"][b]), page)
        want, tol = ref.attention(to_np_f32(host["q"][b]), to_np_f32(host["k_new"][b]), to_np_f32(host["v_new"][b]), K, V, host["parent"][b],
                                  gamma, scale, exclude_self, device=DEV)
        rows = np.ones(R, bool)
        if kept is not None:
            node = np.where(np.arange(R) < T, np.arange(R), (np.arange(R) - T) // max(gamma, 1))
            rows = node < kept[b]
            assert np.array_equal(got[b][~rows], before[b][~rows])
        assert np.all(np.isfinite(got[b][rows]))
        off = np.abs(got[b] - want)[rows] / tol[rows]
        assert off.max() <= 1.0, (b, float(off.max()))


SHAPES = [
    # B, T, gamma, H, Hkv, D, page, lens, room
    (1, 1, 0, 4, 4, 64, 16, (1,), 1.0),
    (2, 1, 0, 8, 2, 128, 16, (0, 33), 1.0),
    (3, 1, 4, 4, 4, 64, 16, (5, 31, 32), 3.0),
    (2, 16, 4, 4, 4, 128, 16, (300, 517), 1.0),       # 80 rows, two splits and more
    (2, 7, 2, 6, 2, 128, 32, (63, 700), 2.0),         # 63 folded rows
    (1, 64, 8, 2, 1, 64, 64, (129,), 1.0),            # the largest tree: 1152 folded rows
    (2, 5, 0, 40, 8, 64, 64, (1000, 95), 1.0),
    (1, 3, 1, 2, 2, 128, 64, (4097,), 1.0),           # many splits, one key in the last
    (5, 2, 3, 8, 4, 128, 16, (16, 15, 17, 255, 257), 4.0),
]


@pytest.mark.parametrize("fmt", [FP8, FP4])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_shapes(case, fmt):
    B, T, gamma, H, Hkv, D, page, lens, room = SHAPES[case]
    host, d = ref.problem(100 + case, B, T, gamma, H, Hkv, D, page, lens, fmt, room, wide=case % 2 == 1)
    scale = D ** -0.5
    _check(host, _call(d, gamma, scale), fmt, gamma, scale, page)


@pytest.mark.parametrize("rows", [1, 16, 17, 32, 33, 48, 49, 64, 65, 80, 81, 96, 161])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_per_kv_head(rows, D):
    """gamma = 0, one query head per KV head or several: every number of query tiles, full and with one row more."""
    H = next(h for h in (1, 2, 3, 4, 5, 7, 9) if rows % h == 0 and rows // h <= 64)
    fmt = FP4 if rows % 2 else FP8
    host, d = ref.problem(rows, 2, rows // H, 0, 2 * H, 2, D, 16, (700, 129), fmt)
    _check(host, _call(d, 0, D ** -0.5), fmt, 0, D ** -0.5, 16)


@pytest.mark.parametrize("L", [0, 1, 2, 31, 32, 33, 127, 128, 129, 255, 256, 257, 383, 511, 512, 513, 1023, 1025])
def test_lengths(L):
    for D, page, fmt in ((128, 16, FP4), (64, 64, FP8)):
        host, d = ref.problem(L + 7, 2, 2, 2, 4, 2, D, page, (L, max(L - 1, 0)), fmt, room=2.0)
        _check(host, _call(d, 2, 0.2), fmt, 2, 0.2, page)


def test_exclude_self():
    host, d = ref.problem(3, 2, 6, 3, 4, 4, 64, 16, (40, 200), FP4)
    _check(host, _call(d, 3, 0.125, flags=api.SS_STREAM_EXCLUDE_SELF), FP4, 3, 0.125, 16, exclude_self=True)


@pytest.mark.parametrize("fmt", [FP8, FP4])
def test_pruned(fmt):
    B, T, gamma, page = 4, 20, 3, 16
    host, d = ref.problem(8, B, T, gamma, 8, 2, 128, page, (600, 31, 1200, 0), fmt)
    kept = np.array([20, 1, 7, 13], np.int32)
    for b in range(B):                                   # the form ss_tree_prune leaves: padding hangs off the root
        host["parent"][b, kept[b]:] = 0
        host["parent"][b, 0] = -1
    d["parent"] = torch.from_numpy(host["parent"]).to(DEV)
    out = torch.full_like(d["q"], 5.0)
    _call(d, gamma, 0.1, n_nodes=torch.from_numpy(kept).to(DEV), out=out)
    _check(host, out, fmt, gamma, 0.1, page, kept=kept, before=np.full(tuple(out.shape), 5.0, np.float32))


def test_equals_the_oracle_on_the_values_that_the_cache_holds():
    """The oracle's own attention on the dequantised cache: the same numbers as the 64-bit reference of these tests."""
    host, d = ref.problem(9, 2, 8, 3, 4, 2, 64, 16, (70, 128), FP4)
    kc, ks, vc, vs = host["cache"]
    K = oracle.mx_values(kc, ks, FP4).astype(np.float32)
    V = np.ascontiguousarray(oracle.mx_values(vc, vs, FP4).astype(np.float32).transpose(0, 1, 3, 2))
    want = oracle.msa_attention(to_np_f32(host["q"]), to_np_f32(host["k_new"]), to_np_f32(host["v_new"]), K, V, host["table"], host["lens"],
                                host["parent"], 3, 0.125)
    for b in range(2):
        Kb, Vb = ref.rows_of_cache(host["cache"], FP4, host["table"][b], int(host["lens"][b]), 16)
        mine, _ = ref.attention(to_np_f32(host["q"][b]), to_np_f32(host["k_new"][b]), to_np_f32(host["v_new"][b]), Kb, Vb, host["parent"][b], 3, 0.125)
        assert np.abs(mine - want[b]).max() < 1e-12
    _check(host, _call(d, 3, 0.125), FP4, 3, 0.125, 16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fmt", [FP8, FP4])
def test_scores_are_exact(D, fmt):
    """A key wins by a part of 2^-10 of the scores: scale 4096 turns that into certainty, so queries that were rounded to
    anything less than their 8 bits, or features paired with another block's scale, pick another value.  Values are one-hot."""
    page, L, T = 16, 64, 16
    host, d = ref.problem(31, 1, T, 0, 1, 1, D, page, (L,), fmt, wide=True)
    K, V = ref.rows_of_cache(host["cache"], fmt, host["table"][0], L, page)
    q = to_np_f32(host["q"][0])[:, 0].astype(np.float64)
    z = q @ np.concatenate((K[:, 0], to_np_f32(host["k_new"][0])[:, 0])).T
    vis = np.concatenate((np.ones((T, L), bool), np.array([[c in s for c in range(T)] for s in ref.visible_new_keys(host["parent"][0].tolist(), 0)])), 1)
    z = np.where(vis, z, -np.inf)
    order = np.sort(z, 1)
    sure = (order[:, -1] - order[:, -2]) > 2.0 ** -10 * np.abs(order[:, -1])
    assert sure.sum() >= T // 2
    got = to_np_f32(_call(d, 0, 4096.0))[0, :, 0]
    Vall = np.concatenate((V[:, 0], to_np_f32(host["v_new"][0])[:, 0]))
    assert np.array_equal(got[sure], Vall[z.argmax(1)][sure].astype(np.float32))


def test_what_lies_behind_a_sequence_is_not_seen():
    """NaN scales and codes in the unused slots of the last page, in unused pages and behind a table's used entries."""
    for fmt, D in ((FP4, 128), (FP8, 64)):
        host, d = ref.problem(17, 3, 3, 2, 4, 2, D, 16, (5, 0, 300), fmt, room=2.0)
        used = [np.zeros(host["cache"][1].shape[0] * 16, bool) for _ in range(1)][0].reshape(-1, 16)
        for b in range(3):
            for pos in range(int(host["lens"][b])):
                used[host["table"][b, pos // 16], pos % 16] = True
        for c in host["cache"]:
            c[np.broadcast_to(~used[:, None, :], c.shape[:3])] = 255
        d["cache"] = [torch.from_numpy(c).to(DEV) for c in host["cache"]]
        _check(host, _call(d, 2, 0.1), fmt, 2, 0.1, 16)


def test_nan_and_infinity():
    """A NaN query row gives NaN in its own row alone; a NaN block of a key in every row of its head; a NaN block of a value in
    its 32 features."""
    host, d = ref.problem(19, 1, 2, 0, 4, 2, 128, 16, (600,), FP4)
    q = d["q"].clone()
    q[0, 1, 2, 5] = float("nan")
    q[0, 0, 0, 3] = float("inf")
    got = _call(dict(d, q=q), 0, 0.1)
    clean = _call(d, 0, 0.1)
    bad = torch.zeros(2, 4, dtype=torch.bool, device=DEV)
    bad[1, 2] = bad[0, 0] = True
    assert torch.isnan(got[0][bad]).all() and torch.equal(got[0][~bad], clean[0][~bad])
    pg, slot = int(host["table"][0, 20]), 7
    c = [x.clone() for x in d["cache"]]
    c[3][pg, 1, slot, 2] = 255
    got = _call(dict(d, cache=c), 0, 0.1)
    assert torch.isnan(got[0, :, 2:, 64:96]).all() and torch.isfinite(got[0, :, 2:, :64]).all() and torch.equal(got[0, :, :2], clean[0, :, :2])
    c = [x.clone() for x in d["cache"]]
    c[1][pg, 0, slot, 3] = 255
    got = _call(dict(d, cache=c), 0, 0.1)
    assert torch.isnan(got[0, :, :2]).all() and torch.equal(got[0, :, 2:], clean[0, :, 2:])


def test_large_and_small_scores():
    """Scores far apart (one key takes all) and all alike (the mean), queries of zero, and scales at the ends of the format."""
    host, d = ref.problem(23, 1, 4, 1, 2, 2, 128, 16, (400,), FP8)
    host["q"][0, 0] = 0
    host["q"][0, 1] *= 64
    host["q"][0, 2] *= 2.0 ** -60
    d["q"] = host["q"].to(DEV)
    _check(host, _call(d, 1, 1.0), FP8, 1, 1.0, 16)
    for s, f in ((10, 1.0), (200, 2.0 ** -70)):
        host["cache"][1][:] = s
        d["cache"] = [torch.from_numpy(c).to(DEV) for c in host["cache"]]
        _check(host, _call(d, 1, f), FP8, 1, f, 16)


def test_workspace_is_left_as_it_was_and_results_do_not_depend_on_the_order_of_the_splits():
    host, d = ref.problem(29, 2, 4, 1, 4, 4, 64, 16, (3000, 1777), FP4)
    n, _ = api.ss_msa_mx_plan(2, 4, 1, 4, 4, 64, d["table"].shape[1] * 16)
    assert n >= 4
    ws = api.ss_msa_mx_workspace(2, 4, 1, 4, 4, 64, d["table"].shape[1] * 16, DEV)
    outs = [_call(d, 1, 0.1, workspace=ws) for _ in range(20)]
    assert all(torch.equal(o, outs[0]) for o in outs[1:])
    # a smaller problem and ss_msa_attention in the same workspace, then this one again
    h2, d2 = ref.problem(30, 1, 1, 0, 4, 4, 64, 16, (900,), FP8)
    _check(h2, _call(d2, 0, 0.1, workspace=ws), FP8, 0, 0.1, 16)
    assert torch.equal(_call(d, 1, 0.1, workspace=ws), outs[0])
    _check(host, outs[0], FP4, 1, 0.1, 16)


def test_a_sequence_alone_gives_the_same_bits_as_in_a_batch():
    """Its splits follow from its own length and the number of splits, so the same table width and split number give the same
    bits whatever the other sequences hold."""
    host, d = ref.problem(37, 3, 2, 1, 4, 4, 128, 16, (2000, 700, 90), FP4)
    whole = _call(d, 1, 0.1)
    lens = d["lens"].clone()
    lens[1:] = torch.tensor([3, 64], dtype=torch.int32, device=DEV)
    assert torch.equal(_call(dict(d, lens=lens), 1, 0.1)[0], whole[0])


def test_captured_graph_replays():
    """Several replays, with other work and other lengths between them, equal the eager results."""
    host, d = ref.problem(41, 2, 4, 2, 8, 4, 128, 16, (1500, 800), FP4, room=1.5)
    ws = api.ss_msa_mx_workspace(2, 4, 2, 8, 4, 128, d["table"].shape[1] * 16, DEV)
    out, lens = torch.zeros_like(d["q"]), d["lens"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _call(dict(d, lens=lens), 2, 0.1, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _call(dict(d, lens=lens), 2, 0.1, out=out, workspace=ws)
    for step in range(5):
        lens.copy_(torch.tensor([1500 - 300 * step, 800 - 190 * step], dtype=torch.int32))
        out.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        want = _call(dict(d, lens=lens), 2, 0.1)
        torch.cuda.synchronize()
        assert torch.equal(out, want), step


def test_a_cache_beyond_four_gib():
    """Pages past the 32-bit offset of a tensor."""
    Hkv, D, page = 8, 128, 64
    row = D * page * Hkv
    num = (1 << 32) // row + 40
    kc = torch.zeros((num, Hkv, page, D), dtype=torch.uint8, device=DEV)
    vc = torch.zeros((num, Hkv, page, D), dtype=torch.uint8, device=DEV)
    ks, vs = (torch.zeros((num, Hkv, page, D // 32), dtype=torch.uint8, device=DEV) for _ in range(2))
    L = 1000
    table = torch.arange(num - 20, num - 4, dtype=torch.int32, device=DEV)[None].contiguous()
    rng = synth.rng_for(3)
    x = torch.from_numpy(rng.standard_normal((2, 1, L, Hkv, D), np.float32)).to(torch.bfloat16)
    lens = torch.zeros(1, dtype=torch.int32, device=DEV)
    new = api.ss_kv_append_mx(x[0].to(DEV), x[1].to(DEV), kc, ks, vc, vs, table, lens, lens + L)
    kr, vr = (torch.zeros((1, L, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    api.ss_kv_read_mx(kc, ks, vc, vs, table, new, kr, vr)
    for got, src in ((kr, x[0]), (vr, x[1])):
        assert np.array_equal(to_np_f32(got), oracle.mx_values(*oracle.mx_quantise(to_np_f32(src), FP8), FP8))
    q, kn, vn = (torch.from_numpy(rng.standard_normal((1, 2, h, D), np.float32)).to(torch.bfloat16) for h in (16, Hkv, Hkv))
    parent = torch.tensor([[-1, 0]], dtype=torch.int32, device=DEV)
    out = api.ss_msa_attention_mx(q.to(DEV), kn.to(DEV), vn.to(DEV), kc, ks, vc, vs, table, new, parent, 0, 0.1)
    want, tol = ref.attention(to_np_f32(q[0]), to_np_f32(kn[0]), to_np_f32(vn[0]), to_np_f32(kr[0]), to_np_f32(vr[0]), [-1, 0], 0, 0.1, device=DEV)
    assert np.all(np.abs(to_np_f32(out[0]) - want) <= tol)
