"""The key/value cache in microscaling formats and the attention that reads it, as cases that can be timed and compared.

A cache holds, for every token and KV head, blocks of 32 features: a scale byte s per block, which stands for 2^(s-127), and
elements of 8 bits (e4m3, "mxfp8") or 4 bits (e2m1, "mxfp4", the even feature in a byte's low half).  The scale is the
smallest power of two with which no element of the block is out of range; elements are rounded to nearest, ties to even.

Kinds of cases, each one pass on inputs that are already on the GPU:

  attn    multi-stream attention of one layer over the cache: t tree nodes with gamma streams each, h query heads on hkv.
          t = 1, gamma = 0 is the decoding of single tokens.  keep < 1: pruned trees.
  prompt  a chunk of every sequence's prompt is quantised into the cache and the sequences are read back whole, as the
          chunk's own attention in a prompt pass needs them.
  read    sequences are read back.
  commit  the accepted path of a step is quantised into the caches of some layers, and what was written is read back.

Sequences have lengths from l_min to l_max; `room` is the capacity of the block table over the longest sequence.
`own` false: plain torch in 32 bits (64 where values lie next to a border); true: the framework's calls.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of e2m1 by code


def listed():
    return [
        # One token of one sequence, grouped query heads: latency.
        dict(name="attn_token_b1", kind="attn", fmt="mxfp4", b=1, h=32, hkv=8, d=128, l_min=411, l_max=411, room=2.0, page=16,
             t=1, gamma=0, keep=1.0),
        # The step right after a prompt: the tree is its root, four streams make the first draft.
        dict(name="attn_root_b2", kind="attn", fmt="mxfp8", b=2, h=32, hkv=32, d=64, l_min=411, l_max=777, room=4.0, page=16,
             t=1, gamma=4, keep=1.0),
        # The headline step's attention: 4 sequences of 4096 tokens, 16-node trees, 4 streams.
        dict(name="attn_b4", kind="attn", fmt="mxfp4", b=4, h=32, hkv=32, d=128, l_min=4096, l_max=4096, room=1.0, page=16,
             t=16, gamma=4, keep=1.0),
        # Batched decode with 16 sequences of uneven length, 8 bits.
        dict(name="attn_b16", kind="attn", fmt="mxfp8", b=16, h=32, hkv=32, d=128, l_min=1024, l_max=4096, room=1.0, page=16,
             t=16, gamma=4, keep=1.0),
        # Single tokens of 32 sequences with grouped query heads: plain serving, a table with room to grow.
        dict(name="attn_token_b32", kind="attn", fmt="mxfp4", b=32, h=32, hkv=8, d=128, l_min=1001, l_max=8003, room=1.5, page=64,
             t=1, gamma=0, keep=1.0),
        # Grouped query heads after pruning: half of every 32-node tree kept.
        dict(name="attn_pruned_b8", kind="attn", fmt="mxfp4", b=8, h=32, hkv=8, d=128, l_min=2000, l_max=8192, room=1.0, page=64,
             t=32, gamma=4, keep=0.5),
        # Long context: 8 sequences of 32768 tokens, 640 query rows per KV head.
        dict(name="attn_gqa_32k", kind="attn", fmt="mxfp4", b=8, h=32, hkv=8, d=128, l_min=32768, l_max=32768, room=1.0, page=64,
             t=32, gamma=4, keep=1.0),
        # A short fp32 prompt behind 21 tokens: latency, ragged pages.
        dict(name="prompt_b1", kind="prompt", fmt="mxfp8", dtype="f32", b=1, hkv=4, d=64, l_min=128, l_max=128, chunk=107, room=1.0,
             page=16),
        # Prompt chunks of four sequences behind what is cached of them.
        dict(name="prompt_b4", kind="prompt", fmt="mxfp4", dtype="bf16", b=4, hkv=32, d=128, l_min=3500, l_max=4096, chunk=2048,
             room=1.1, page=16),
        # Long sequences read back.
        dict(name="read_32k", kind="read", fmt="mxfp4", dtype="bf16", b=2, hkv=8, d=128, l_min=30011, l_max=32768, room=1.0, page=64),
        # The accepted tokens of one sequence into the cache of one layer.
        dict(name="commit_b1", kind="commit", fmt="mxfp8", dtype="bf16", b=1, hkv=8, d=128, l_min=2048, l_max=2048, room=1.1, page=16,
             t=16, gamma=4, depth=4, layers=1),
        # Those of 16 sequences into the caches of four layers.
        dict(name="commit_b16", kind="commit", fmt="mxfp4", dtype="bf16", b=16, hkv=32, d=128, l_min=101, l_max=509, room=1.1, page=16,
             t=16, gamma=4, depth=4, layers=4),
    ]


# ------------------------------------------------------------------ more cases of the same ranges

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["attn", "attn", "attn", "tokens", "tokens", "prompt", "read", "commit"])
    h, hkv, d = rng.choice([(32, 32, 128), (32, 8, 128), (32, 32, 64), (32, 4, 128), (16, 16, 128), (40, 8, 64)])
    case = dict(fmt=rng.choice(["mxfp4", "mxfp8"]), b=_log_int(rng, 1, 16), page=rng.choice([16, 16, 32, 64]),
                room=rng.choice([1.0, 1.0, 1.5, 2.0, 4.0]))
    longest = _log_int(rng, 64, 32768 if kind in ("attn", "tokens") else 8192)
    case.update(l_max=longest, l_min=rng.randint(longest // 3, longest))
    if kind == "tokens":
        case["b"] = _log_int(rng, 1, 64)
        return dict(kind="attn", h=h, hkv=hkv, d=d, t=1, gamma=0, keep=1.0, **case)
    if kind == "attn":
        t = rng.randint(1, 32)
        return dict(kind="attn", h=h, hkv=hkv, d=d, t=t, gamma=rng.randint(2, 5),
                    keep=rng.choice([1.0, 1.0, 1.0, rng.uniform(0.3, 0.8)]) if t >= 8 else 1.0, **case)
    case["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "prompt":
        return dict(kind="prompt", hkv=hkv, d=d, chunk=_log_int(rng, 1, max(1, case["l_min"])), **case)
    if kind == "read":
        return dict(kind="read", hkv=hkv, d=d, **case)
    gamma = rng.randint(2, 5)
    case["room"] = max(case["room"], 1.5)
    return dict(kind="commit", hkv=hkv, d=d, t=rng.randint(2, 32), gamma=gamma, depth=min(gamma, rng.randint(2, 4)),
                layers=rng.randint(1, 4), **case)


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / 1e15)


def draw(rng):
    most = 0.8 * max(_cost(c) for c in listed())
    while True:
        case = _draw_once(rng)
        if _cost(case) <= most:
            return case


# ------------------------------------------------------------------ sizes

def _lengths(case):
    """The batch's cached tokens after the pass' writes (attn, read: as they are), evenly from l_max to l_min."""
    return [int(v) for v in np.rint(np.linspace(case["l_max"], case["l_min"], case["b"]))]


def _capacity(case):
    return -(-int(math.ceil(case["l_max"] * case["room"])) // case["page"]) * case["page"]


def _chunks(case):
    """Rows of the chunk that each sequence appends: the longest sequence all of `chunk`, others what they have of it."""
    c = min(case["chunk"], case["l_min"])
    return [max(1, c - (i % 3)) for i in range(case["b"])]


def _accepted(case, seed):
    rng = np.random.default_rng(seed + 17)
    return rng.integers(0, min(case["depth"], case["t"] - 1) + 1, case["b"])


def _kept(case):
    """Nodes that pruning keeps of each tree: around keep * t."""
    return [max(1, min(case["t"], round(case["t"] * case["keep"] * (0.7 + 0.6 * i / max(1, case["b"] - 1))))) for i in range(case["b"])]


def work(case):
    hkv, d = case["hkv"], case["d"]
    token = 2 * hkv * d * ((1.0 if case["fmt"] == "mxfp8" else 0.5) + 1.0 / 32)  # bytes of a cached token, keys and values
    lens = _lengths(case)
    if case["kind"] == "attn":
        nodes = _kept(case) if case["keep"] < 1 else [case["t"]] * case["b"]
        rows = [n * (1 + case["gamma"]) for n in nodes]
        flops = sum(4.0 * d * case["h"] * r * n for r, n in zip(rows, lens))
        flops += sum(4.0 * d * case["h"] * r * min(r, 1 + case["gamma"]) for r in rows)  # at least the own keys
        return {"bytes": sum(lens) * token + sum(rows) * d * 2 * (2 * case["h"] + 2 * hkv), "flops": flops}
    row = 2 * hkv * d * (4 if case["dtype"] == "f32" else 2)  # bytes of a token as the caller has it
    if case["kind"] == "commit":
        n = case["b"] * (1 + min(case["depth"], case["t"] - 1) / 2.0) * case["layers"]
        return {"bytes": n * (2 * row + token), "flops": 2.0 * n * hkv * d * 2}
    read = sum(lens) * (token + row)
    if case["kind"] == "read":
        return {"bytes": read, "flops": 2.0 * sum(lens) * hkv * d}
    n = sum(_chunks(case))
    return {"bytes": n * (row + token) + read, "flops": 2.0 * (2 * n + sum(lens)) * hkv * d}


# ------------------------------------------------------------------ the formats, plainly

def _quantise(x, fmt):
    """x [...,d] -> (element bytes [...,d or d/2], scale bytes [...,d/32])."""
    shape = x.shape
    x = x.float().reshape(*shape[:-1], shape[-1] // 32, 32)
    bits = x.abs().amax(-1).view(torch.int32)
    bad = ~torch.isfinite(x).all(-1)
    # amax = 1.m * 2^(E-127) over max = 1.75 * 2^8 (e4m3) or 1.5 * 2^2 (e2m1)
    top, m = (8, 0x600000) if fmt == "mxfp8" else (2, 0x400000)
    s = ((bits >> 23) - top + ((bits & 0x7FFFFF) > m).int()).clamp(0, 254)
    s = torch.where(bad, torch.full_like(s, 255), s)
    y = torch.where(bad.unsqueeze(-1), torch.zeros_like(x), x).double() * torch.exp2(127.0 - s.double()).unsqueeze(-1)
    if fmt == "mxfp8":
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6).float())).double() - 3)
        code = ((y / step).round() * step).float().to(torch.float8_e4m3fn).view(torch.uint8).reshape(shape)
    else:
        a = y.abs()
        code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int()
                + (a > 5.0).int() + 8 * torch.signbit(y).int()).reshape(shape)
        code = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
    return code, s.to(torch.uint8)


def _values(code, scale, fmt):
    """Element and scale bytes -> the values they stand for, fp32."""
    if fmt == "mxfp8":
        e = code.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(GRID + tuple(-v for v in GRID), device=code.device)
        e = torch.stack((table[(code & 15).int()], table[(code >> 4).int()]), -1).flatten(-2)
    s = torch.exp2(scale.double() - 127.0).float()
    s = torch.where(scale == 255, torch.full_like(s, math.nan), s)
    return (e.unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


# ------------------------------------------------------------------ inputs

def _rows(gen, shape, dtype, keys):
    """Keys or values as a projection gives them: N(0,1), of the keys' features one in sixteen eight times as large."""
    x = torch.randn(shape, generator=gen, device=DEVICE)
    if keys:
        x[..., 5::16] *= 8.0
    return x.to(dtype)


def _pages(case, gen, lens):
    """A page table in a pool with a quarter to spare; entries past a sequence's pages are unused (0)."""
    page, cols = case["page"], _capacity(case) // case["page"]
    need = torch.tensor([-(-n // page) for n in lens], device=DEVICE)
    total = int(need.sum())
    num = max(1, -(-total * 5 // 4))
    table = torch.zeros((case["b"], cols), dtype=torch.int32, device=DEVICE)
    used = torch.arange(cols, device=DEVICE)[None] < need[:, None]
    table[used] = torch.randperm(num, generator=gen, device=DEVICE)[:total].int()
    return table, num


def _cache(case, gen, num):
    """What a pool of pages holds: quantised rows, made some pages at a time."""
    hkv, page, d, out = case["hkv"], case["page"], case["d"], []
    per = max(1, (1 << 27) // (hkv * page * d))
    for keys in (True, False):
        parts = [_quantise(_rows(gen, (min(per, num - at), hkv, page, d), torch.float32, keys), case["fmt"]) for at in range(0, num, per)]
        out += [torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])]
    return dict(zip(("k_cache", "k_scale", "v_cache", "v_scale"), out))


def _parents(case, seed, depth):
    """Trees in level order: every node's parent is an earlier node that is not too deep."""
    rng = np.random.default_rng(seed + 5)
    out = np.full((case["b"], case["t"]), -1, np.int32)
    for b in range(case["b"]):
        deep = [0]
        for i in range(1, case["t"]):
            p = int(rng.choice([j for j in range(i) if deep[j] < depth]))
            out[b, i] = p
            deep.append(deep[p] + 1)
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    lens = _lengths(case)
    table, num = _pages(case, gen, lens)
    s = dict(case=case, table=table)
    b, hkv, d = case["b"], case["hkv"], case["d"]
    dt = DTYPES[case.get("dtype", "bf16")]
    ints = lambda v: torch.tensor([int(x) for x in v], dtype=torch.int32, device=DEVICE)  # noqa: E731
    if case["kind"] == "commit":
        r = case["t"] * (1 + case["gamma"])
        acc, parent = _accepted(case, seed), _parents(case, seed, case["depth"])
        path = np.full((b, case["depth"] + 1), -1, np.int32)
        for i in range(b):  # the path to the last node that is deep enough for the accepted tokens, or as deep as there is one
            depth_of = [0]
            for p in parent[i, 1:]:
                depth_of.append(depth_of[p] + 1)
            acc[i] = min(acc[i], max(depth_of))
            node = max(j for j in range(case["t"]) if depth_of[j] == acc[i])
            for j in range(int(acc[i]), -1, -1):
                path[i, j] = node
                node = parent[i, node]
        s.update(path=torch.from_numpy(path).to(DEVICE), n_accept=ints(acc), lens=ints([n - int(a) - 1 for n, a in zip(lens, acc)]))
        s["layers"] = [dict(_cache(case, gen, num), k_new=_rows(gen, (b, r, hkv, d), dt, True), v_new=_rows(gen, (b, r, hkv, d), dt, False),
                            k_rows=torch.zeros((b, case["depth"] + 1, hkv, d), dtype=dt, device=DEVICE),
                            v_rows=torch.zeros((b, case["depth"] + 1, hkv, d), dtype=dt, device=DEVICE)) for _ in range(case["layers"])]
        return s
    s.update(_cache(case, gen, num))
    if case["kind"] == "attn":
        t, r = case["t"], case["t"] * (1 + case["gamma"])
        s.update(lens=ints(lens), parent=torch.from_numpy(_parents(case, seed, 4)).to(DEVICE), scale=1.0 / math.sqrt(d),
                 q=torch.randn((b, r, case["h"], d), generator=gen, device=DEVICE).to(dt), k_new=_rows(gen, (b, r, hkv, d), dt, True),
                 v_new=_rows(gen, (b, r, hkv, d), dt, False), out=torch.zeros((b, r, case["h"], d), dtype=dt, device=DEVICE))
        s["n_nodes"] = ints(_kept(case)) if case["keep"] < 1 else None
        if s["n_nodes"] is not None:  # a pruned tree: the kept nodes first, padding hangs off the root
            i = torch.arange(t, device=DEVICE)[None]
            s["parent"] = torch.where(i < s["n_nodes"][:, None], s["parent"], 0).masked_fill(i == 0, -1).int()
        return s
    s["k_rows"], s["v_rows"] = (torch.zeros((b, max(lens), hkv, d), dtype=dt, device=DEVICE) for _ in range(2))
    s["lens"] = ints(lens)
    if case["kind"] == "prompt":
        n = _chunks(case)
        s.update(n_rows=ints(n), start=ints([a - c for a, c in zip(lens, n)]), k_in=_rows(gen, (b, max(n), hkv, d), dt, True),
                 v_in=_rows(gen, (b, max(n), hkv, d), dt, False))
    return s


# ------------------------------------------------------------------ one pass

def _plain_write(c, fmt, table, page, k, v, at, ok):
    """Rows k, v [b,n,hkv,d] to the positions at [b,n] where ok."""
    at = at.long()
    pg = table.long().gather(1, (at // page).clamp(0, table.shape[1] - 1))
    pg, slot = pg[ok], (at % page)[ok]
    for x, name in ((k, "k"), (v, "v")):
        code, s = _quantise(x[ok], fmt)
        c[name + "_cache"][pg, :, slot] = code
        c[name + "_scale"][pg, :, slot] = s


def _plain_read(c, fmt, table, page, at, ok):
    """The rows at the positions at [b,n], fp32 [b,n,hkv,d]; zeros where not ok."""
    at = at.long()
    pg = table.long().gather(1, (at // page).clamp(0, table.shape[1] - 1))
    slot, keep = at % page, ok[:, :, None, None]
    return [torch.where(keep, _values(c[n + "_cache"][pg, :, slot], c[n + "_scale"][pg, :, slot], fmt), 0.0) for n in ("k", "v")]


def _own_keys(parent, gamma):
    """Which of the step's own rows each of them sees, [b,r,r]: main rows the main rows of the nodes on their path; stream j
    of a node those and streams 1..j of its node."""
    b, t = parent.shape
    i = torch.arange(t, device=parent.device)
    step = (parent[:, :, None] == i).float() + torch.eye(t, device=parent.device)
    anc = torch.linalg.matrix_power(step.double(), 64) > 0  # trees have at most 64 nodes
    r = torch.arange(t * (1 + gamma), device=parent.device)
    node = torch.where(r < t, r, (r - t) // max(gamma, 1))
    strm = torch.where(r < t, 0, (r - t) % max(gamma, 1) + 1)
    main = anc[:, node][:, :, node] & (strm == 0)[None, None, :]
    mine = (node[:, None] == node) & (strm[:, None] > 0) & (strm > 0) & (strm <= strm[:, None])
    return main | mine[None]


def _plain_attention(s):
    case = s["case"]
    b, r, h, d = s["q"].shape
    hkv, lens = case["hkv"], s["lens"].long()
    pos = torch.arange(case["l_max"], device=DEVICE)[None].expand(b, -1)
    ok = pos < lens[:, None]
    kc, vc = _plain_read(s, case["fmt"], s["table"], case["page"], pos, ok)
    k = torch.cat((kc, s["k_new"].float()), 1).permute(0, 2, 3, 1).contiguous()
    v = torch.cat((vc, s["v_new"].float()), 1).permute(0, 2, 1, 3).contiguous()
    g = h // hkv
    q = s["q"].float().view(b, r, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, g * r, d)
    see = torch.cat((ok[:, None, :].expand(b, r, -1), _own_keys(s["parent"], case["gamma"])), 2)
    z = (torch.matmul(q, k) * s["scale"]).view(b, hkv, g, r, -1).masked_fill(~see[:, None, None], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hkv, g * r, -1), v).view(b, hkv, g, r, d).permute(0, 3, 1, 2, 4).reshape(b, r, h, d)
    if s["n_nodes"] is not None:  # rows of pruned nodes stay as they were
        row = torch.arange(r, device=DEVICE)
        node = torch.where(row < case["t"], row, (row - case["t"]) // max(case["gamma"], 1))
        return torch.where((node[None] < s["n_nodes"][:, None])[:, :, None, None], o.to(s["out"].dtype), s["out"])
    return o.to(s["out"].dtype)


def _plain(s):
    case = s["case"]
    fmt, page, table = case["fmt"], case["page"], s["table"]
    if case["kind"] == "attn":
        return _plain_attention(s)
    if case["kind"] == "commit":
        j = torch.arange(case["depth"] + 1, device=DEVICE)[None]
        at, ok = s["lens"][:, None] + j, j <= s["n_accept"][:, None]
        node = s["path"].clamp(min=0).long()[:, :, None, None]
        out = []
        for c in s["layers"]:
            take = lambda x: x.gather(1, node.expand(-1, -1, x.shape[2], x.shape[3]))  # noqa: E731
            _plain_write(c, fmt, table, page, take(c["k_new"]), take(c["v_new"]), at, ok)
            out += [x.to(c["k_rows"].dtype) for x in _plain_read(c, fmt, table, page, at, ok)]
        return out + [s["lens"] + s["n_accept"] + 1]
    out = []
    if case["kind"] == "prompt":
        j = torch.arange(s["k_in"].shape[1], device=DEVICE)[None]
        _plain_write(s, fmt, table, page, s["k_in"], s["v_in"], s["start"][:, None] + j, j < s["n_rows"][:, None])
        out.append(s["start"] + s["n_rows"])
    at = torch.arange(s["k_rows"].shape[1], device=DEVICE)[None].expand(case["b"], -1)
    return [x.to(s["k_rows"].dtype) for x in _plain_read(s, fmt, table, page, at, at < s["lens"][:, None])] + out


def _own(s):
    from paper_2402_11131_amd import api
    case = s["case"]
    names = ("k_cache", "k_scale", "v_cache", "v_scale")
    if case["kind"] == "attn":
        b, _, h, d = s["q"].shape
        if "workspace" not in s:  # kept from step to step
            s["workspace"] = api.ss_msa_mx_workspace(b, case["t"], case["gamma"], h, case["hkv"], d, s["table"].shape[1] * case["page"], DEVICE)
        return api.ss_msa_attention_mx(s["q"], s["k_new"], s["v_new"], *(s[n] for n in names), s["table"], s["lens"], s["parent"], case["gamma"],
                                       s["scale"], out=s["out"], workspace=s["workspace"], n_nodes=s["n_nodes"])
    if case["kind"] == "commit":
        out = []
        for c in s["layers"]:
            cache = [c[n] for n in names]
            new = api.ss_kv_commit_mx(c["k_new"], c["v_new"], *cache, s["table"], s["lens"], s["path"], s["n_accept"], case["gamma"])
            out += api.ss_kv_read_mx(*cache, s["table"], new, c["k_rows"], c["v_rows"], first=s["lens"])
        return out + [new]
    cache, out = [s[n] for n in names], []
    if case["kind"] == "prompt":
        out.append(api.ss_kv_append_mx(s["k_in"], s["v_in"], *cache, s["table"], s["start"], s["n_rows"]))
    return list(api.ss_kv_read_mx(*cache, s["table"], out[0] if out else s["lens"], s["k_rows"], s["v_rows"])) + out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ in 64 bits, from the definitions

def _exact_grid(fmt):
    """All element values by code, and the largest."""
    if fmt == "mxfp4":
        mag = [0.0, 0.5] + [(1 + m / 2) * 2.0 ** e for e in range(3) for m in range(2)]
    else:
        mag = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1]
    return torch.tensor(mag, dtype=torch.float64, device=DEVICE)


def _exact_quantised(x, fmt):
    """The values that rows x are held as: the nearest of the grid times the block's power of two; of two as near the even code."""
    mag = _exact_grid(fmt)
    x = x.double().unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True) / mag[-1])  # amax / max = m * 2^e, m in [1/2, 1)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=-127)
    y = torch.ldexp(x, -e)
    hi = torch.bucketize(y.abs().contiguous(), mag).clamp(1, mag.numel() - 1)
    lo = hi - 1
    up, down = mag[hi] - y.abs(), y.abs() - mag[lo]
    near = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.ldexp(mag[near] * torch.sign(y), e).flatten(-2)


def _exact_rows(c, case, table, b, n):
    """The first n cached keys and values of sequence b as the values they stand for, [n,hkv,d] each."""
    mag, out = _exact_grid(case["fmt"]), []
    pages = table[b, :-(-n // case["page"])].long()
    for name in ("k", "v"):
        code = c[name + "_cache"][pages].transpose(1, 2).flatten(0, 1)[:n].long()
        if case["fmt"] == "mxfp4":
            code = torch.stack((code % 16, code // 16), -1).flatten(-2)
        half = 8 if case["fmt"] == "mxfp4" else 128
        e = mag[(code % half).clamp(max=mag.numel() - 1)] * (1 - 2 * (code // half)).double()
        s = c[name + "_scale"][pages].transpose(1, 2).flatten(0, 1)[:n].double() - 127
        out.append((e.unflatten(-1, (-1, 32)) * torch.pow(torch.full_like(s, 2.0), s).unsqueeze(-1)).flatten(-2))
    return out


def _exact_sees(parent, gamma):
    t = len(parent)
    rows = [(i, 0) for i in range(t)] + [(i, j) for i in range(t) for j in range(1, gamma + 1)]
    above = []
    for i in range(t):
        above.append({i} | (above[parent[i]] if i else set()))
    return [[(j2 == 0 and i2 in above[i]) or (j > 0 and i2 == i and 0 < j2 <= j) for i2, j2 in rows] for i, j in rows]


def exact(case, seed):
    s = prepare(case, seed)
    b = case["b"]
    if case["kind"] == "attn":
        r, h, d = s["q"].shape[1:]
        g, out = h // case["hkv"], torch.zeros((b, r, h, d), dtype=torch.float64, device=DEVICE)
        for i, n in enumerate(_lengths(case)):
            k, v = _exact_rows(s, case, s["table"], i, n)
            k, v = torch.cat((k, s["k_new"][i].double())), torch.cat((v, s["v_new"][i].double()))
            see = torch.tensor(_exact_sees(s["parent"][i].tolist(), case["gamma"]), device=DEVICE)
            see = torch.cat((torch.ones((r, n), dtype=torch.bool, device=DEVICE), see), 1).repeat(g, 1)
            for hk in range(case["hkv"]):
                q = s["q"][i, :, hk * g:(hk + 1) * g].double().transpose(0, 1).reshape(g * r, d)
                z = torch.where(see, (q @ k[:, hk].T.contiguous()) / math.sqrt(d), -math.inf)
                out[i, :, hk * g:(hk + 1) * g] = (torch.softmax(z, -1) @ v[:, hk].contiguous()).view(g, r, d).transpose(0, 1)
            if s["n_nodes"] is not None:
                n_kept = int(s["n_nodes"][i])
                out[i, n_kept:case["t"]] = 0
                out[i, case["t"] + n_kept * case["gamma"]:] = 0
        return out
    if case["kind"] == "commit":
        out = []
        for c in s["layers"]:
            for name in ("k", "v"):
                rows = torch.zeros(c["k_rows"].shape, dtype=torch.float64, device=DEVICE)
                for i in range(b):
                    n = int(s["n_accept"][i]) + 1
                    rows[i, :n] = _exact_quantised(c[name + "_new"][i, s["path"][i, :n].long()], case["fmt"])
                out.append(rows)
        return out + [None]
    shape = s["k_rows"].shape
    out = [torch.zeros(shape, dtype=torch.float64, device=DEVICE) for _ in range(2)]
    for i, n in enumerate(_lengths(case)):
        for o, rows in zip(out, _exact_rows(s, case, s["table"], i, n)):
            o[i, :n] = rows
        if case["kind"] == "prompt":
            m = int(s["n_rows"][i])
            for o, x in zip(out, (s["k_in"], s["v_in"])):
                o[i, n - m:n] = _exact_quantised(x[i, :m], case["fmt"])
    return out + ([None] if case["kind"] == "prompt" else [])
