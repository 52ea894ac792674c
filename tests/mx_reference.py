"""Caches in microscaling formats for the tests: made by the oracle's quantisation, and attention over them in 64 bits."""
import math

import numpy as np
import torch

import oracle
from helpers import visible_new_keys
from paper_2402_11131_amd import synth


def random_cache(rng, num_pages, Hkv, page, D, fmt, wide=False):
    """(k_cache, k_scale, v_cache, v_scale) as uint8 arrays: N(0,1) rows as the oracle quantises them; wide: every block has a
    scale of its own over a dozen powers of two."""
    out = []
    for _ in range(2):
        x = rng.standard_normal((num_pages, Hkv, page, D), np.float32)
        if wide:
            x = x.reshape(num_pages, Hkv, page, D // 32, 32)
            x = (x * np.exp2(rng.integers(-9, 4, x.shape[:-1] + (1,))).astype(np.float32)).reshape(num_pages, Hkv, page, D)
        out += oracle.mx_quantise(x, fmt)
    return out


def rows_of_cache(cache, fmt, table, L, page):
    """K, V [L,Hkv,D] float64 of one sequence (table: its row)."""
    kc, ks, vc, vs = cache
    npg = -(-L // page)
    pages = np.asarray(table[:npg])
    out = []
    for c, s in ((kc, ks), (vc, vs)):
        v = oracle.mx_values(c[pages], s[pages], fmt)          # [npg,Hkv,page,D]
        out.append(v.transpose(0, 2, 1, 3).reshape(npg * page, v.shape[1], v.shape[3])[:L])
    return out


def attention(q, k_new, v_new, K, V, parent, gamma, scale, exclude_self=False, device="cpu"):
    """One sequence in 64 bits.  q [R,H,D], k_new, v_new [R,Hkv,D], K, V [L,Hkv,D] float64 -> (out [R,H,D], tol [R,H,D]).

    tol is how far a bf16 result may be off.  Three kinds of roundings enter (half a bf16 step is e = 2^-8 of a value):
      - the result's own: e |out|;
      - the probabilities', as they enter the product with V and, rounded alike, the row sum: out' = sum p(1+d)v / sum p(1+d)
        with independent d, |d| <= e: off by sum p d (v - out), which 8 times e sqrt(sum p^2 (v - out)^2) bounds but for a
        chance of 1e-13 (Hoeffding), and by 2 e sum p |v - out| without chance where that is less;
      - everything in fp32 (scores of a few hundred at most, exponentials, sums, merges): 2^-14 sum p |v|.
    """
    t = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.float64, device=device)  # noqa: E731
    q, kk, vv = t(q), torch.cat((t(K), t(k_new))), torch.cat((t(V), t(v_new)))
    R, H, D = q.shape
    L, g, e = len(K), H // kk.shape[1], 2.0 ** -8
    see = torch.zeros((R, L + R), dtype=torch.bool, device=device)
    see[:, :L] = True
    for r, cols in enumerate(visible_new_keys([int(p) for p in parent], gamma, exclude_self)):
        see[r, [L + c for c in cols]] = True
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    for h in range(H):
        k, v = kk[:, h // g], vv[:, h // g].contiguous()
        z = torch.where(see, (q[:, h] @ k.T.contiguous()) * scale, torch.tensor(-math.inf, dtype=torch.float64, device=device))
        p = torch.softmax(z, -1)
        o = p @ v
        # sum p^2 (v-o)^2 and sum p |v-o| <= sqrt(sum p (v-o)^2), without forming v - o per row
        p2 = p * p
        var2 = (p2 @ (v * v) - 2 * o * (p2 @ v) + o * o * p2.sum(-1, keepdim=True)).clamp(min=0)
        var1 = (p @ (v * v) - o * o).clamp(min=0)
        out[:, h] = o
        tol[:, h] = e * o.abs() + torch.minimum(8 * e * var2.sqrt(), 2 * e * var1.sqrt()) + 2.0 ** -14 * (p @ v.abs())
    return out.cpu().numpy(), tol.cpu().numpy()


def problem(seed, B, T, gamma, H, Hkv, D, page, lens, fmt, room=1.0, wide=False, device="cuda:0"):
    """A whole call's inputs: `np` (host arrays) and `dev` (the same as tensors), with the unused slots of pages and the pages of
    no sequence holding values of their own."""
    rng = synth.rng_for(seed)
    table, num = synth.make_page_table(seed, np.array(lens, np.int32), page, 1.3)
    cols = max(table.shape[1], -(-int(math.ceil(max(max(lens), 1) * room)) // page))
    wide_table = np.zeros((B, cols), np.int32)
    wide_table[:, :table.shape[1]] = table
    cache = random_cache(rng, num, Hkv, page, D, fmt, wide)
    R = T * (1 + gamma)
    bf = lambda *s: torch.from_numpy(rng.standard_normal(s, np.float32)).to(torch.bfloat16)  # noqa: E731
    parent = np.stack([synth.make_tree(rng, T, (64,) * 8, 6) for _ in range(B)]).astype(np.int32)
    host = dict(q=bf(B, R, H, D), k_new=bf(B, R, Hkv, D), v_new=bf(B, R, Hkv, D), table=wide_table, lens=np.array(lens, np.int32),
                parent=parent, cache=cache)
    dev = dict(q=host["q"].to(device), k_new=host["k_new"].to(device), v_new=host["v_new"].to(device),
               cache=[torch.from_numpy(c).to(device) for c in cache], table=torch.from_numpy(wide_table).to(device),
               lens=torch.from_numpy(host["lens"]).to(device), parent=torch.from_numpy(parent).to(device))
    return host, dev
