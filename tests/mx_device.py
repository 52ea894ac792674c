"""Caches in microscaling formats made on the GPU from random bytes, for problems that are too large to quantise on the host, and
their attention in 64 bits for some sequences and heads."""
import numpy as np
import torch

import mx_reference as ref
from helpers import to_np_f32
from paper_2402_11131_amd import api, synth

DEV = "cuda:0"


def problem(seed, B, T, gamma, H, Hkv, D, page, lens, fmt, capacity):
    """A call's tensors.  Elements are any of the format's, scales 2^-9 .. 2^-6 (8 bits) or 2^-3 .. 1 (4 bits), so that blocks reach
    up to 0.875 .. 7 or 0.75 .. 6; pages are shuffled, unused entries of the table name pages of others."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    need = [-(-n // page) for n in lens]
    num = sum(need) + 3
    order = torch.randperm(num, generator=g, device=DEV).to(torch.int32)
    table = torch.randint(0, num, (B, -(-capacity // page)), generator=g, device=DEV, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    cache = []
    for _ in range(2):
        code = torch.randint(0, 256, (num, Hkv, page, D if fmt == api.SS_KV_MXFP8 else D // 2), generator=g, device=DEV, dtype=torch.uint8)
        if fmt == api.SS_KV_MXFP8:
            code[(code & 127) == 127] = 0      # no NaN
        first = 118 if fmt == api.SS_KV_MXFP8 else 124
        cache += [code, torch.randint(first, first + 4, (num, Hkv, page, D // 32), generator=g, device=DEV, dtype=torch.uint8)]
    rng = synth.rng_for(seed)
    bf = lambda *s: torch.randn(s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    parent = torch.from_numpy(np.stack([synth.make_tree(rng, T, (64,) * 8, 6) for _ in range(B)]).astype(np.int32)).to(DEV)
    R = T * (1 + gamma)
    return dict(q=bf(B, R, H, D), k_new=bf(B, R, Hkv, D), v_new=bf(B, R, Hkv, D), cache=cache, table=table,
                lens=torch.tensor(lens, dtype=torch.int32, device=DEV), parent=parent)


def call(d, gamma, scale, **kw):
    return api.ss_msa_attention_mx(d["q"], d["k_new"], d["v_new"], *d["cache"], d["table"], d["lens"], d["parent"], gamma, scale, **kw)


def check(d, out, fmt, gamma, scale, page, b, head):
    """One sequence's results of one KV head against 64 bits."""
    L = int(d["lens"][b])
    pages = d["table"][b, :-(-L // page)].long()
    host = [c[pages, head:head + 1].cpu().numpy() for c in d["cache"]]
    K, V = ref.rows_of_cache(host, fmt, np.arange(len(pages)), L, page)
    g = d["q"].shape[2] // d["k_new"].shape[2]
    mine = slice(head * g, (head + 1) * g)
    want, tol = ref.attention(to_np_f32(d["q"][b, :, mine]), to_np_f32(d["k_new"][b, :, head:head + 1]), to_np_f32(d["v_new"][b, :, head:head + 1]),
                              K, V, d["parent"][b].tolist(), gamma, scale, device=DEV)
    got = to_np_f32(out[b, :, mine])
    assert np.all(np.isfinite(got))
    off = np.abs(got - want) / tol
    assert off.max() <= 1.0, (b, head, float(off.max()))
