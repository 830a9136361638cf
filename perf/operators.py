"""A step of speculative decoding, operator by operator: what a serving program calls and how its time is watched.

A draft proposes, for every sequence, a tree of tokens behind the last token that stands (node 0; a node's parent comes
before it).  The target scores all nodes at once over the cache (kind ``tree``: ``fa_decode_tree``), its probabilities
decide which of them stand and what follows (``verify``: ``fa_spec_verify``), the cache rows of the accepted path move
together (``compact``: ``fa_cache_compact``), and pages are reserved, given back (``resize``: ``fa_pages_resize``) and
shared between sequences that go on from the same prompt (``fork``: ``fa_pages_fork``).

``own`` false computes each operator in plain torch operations in 32 bits, ``own`` true calls the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one user, a small tree behind a short prompt, grouped heads: the latency of a single step
        dict(name="tree_one", kind="tree", B=1, T=8, Hq=32, Hkv=8, len_lo=512, len_hi=512, lens=1, page=0, d=128, dtype="fp16",
             shape="tree", ragged=False),
        # a chat batch on small pages, trees of different sizes
        dict(name="tree_chat", kind="tree", B=16, T=26, Hq=32, Hkv=8, len_lo=100, len_hi=8000, lens=5, page=16, d=128, dtype="bf16",
             shape="tree", ragged=True),
        # wide trees over long prompts: the largest
        dict(name="tree_wide", kind="tree", B=32, T=64, Hq=32, Hkv=8, len_lo=1024, len_hi=16384, lens=7, page=0, d=128,
             dtype="bf16", shape="tree", ragged=False),
        # head dimension 64, eight query heads to a kv head, sizes that are multiples of nothing
        dict(name="tree_d64", kind="tree", B=3, T=61, Hq=40, Hkv=5, len_lo=999, len_hi=7951, lens=3, page=64, d=64, dtype="fp16",
             shape="tree", ragged=False),
        # a chain of four drafted tokens for one user, a vocabulary of 32000
        dict(name="verify_one", kind="verify", B=1, T=5, V=32000, dtype="fp32", draft=True, shape="chain", lens=1, ragged=False),
        # trees for a batch over a large vocabulary
        dict(name="verify_batch", kind="verify", B=32, T=32, V=131072, dtype="fp32", draft=True, shape="tree", lens=2, ragged=False),
        # one user's accepted path in the caches of 32 layers
        dict(name="compact_one", kind="compact", B=1, T=8, L=32, Hkv=8, len_lo=256, len_hi=256, lens=1, page=0, d=128, dtype="fp16",
             shape="tree", ragged=False),
        # the same for a batch on small pages
        dict(name="compact_batch", kind="compact", B=64, T=26, L=32, Hkv=8, len_lo=40, len_hi=120, lens=4, page=16, d=128,
             dtype="bf16", shape="tree", ragged=True),
        # two samples of one prompt
        dict(name="fork_pair", kind="fork", n=2, L=32, Hkv=8, len_lo=301, len_hi=301, lens=1, pages=64, page=16, d=128,
             dtype="fp16"),
        # parallel sampling of a batch: 64 new sequences that share 16 prompts
        dict(name="fork_batch", kind="fork", n=64, L=32, Hkv=8, len_lo=100, len_hi=500, lens=3, pages=240, page=64, d=128,
             dtype="bf16"),
        # a few sequences on a small pool: room for the next trees, and what the last ones did not use
        dict(name="resize_few", kind="resize", B=4, len_hi=2000, grow=27, pages=1024, page=16),
        # a full server: 512 sequences on a pool of 128K pages
        dict(name="resize_full", kind="resize", B=512, len_hi=6000, grow=65, pages=131072, page=16),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        m = most.setdefault(c["kind"], {"bytes": 0.0, "flops": 0.0})
        m["bytes"], m["flops"] = max(m["bytes"], w["bytes"]), max(m["flops"], w["flops"])
    while True:
        case = _draw(rng)
        w, m = work(case), most[case["kind"]]
        if w["bytes"] <= m["bytes"] and w["flops"] <= max(m["flops"], 1.0) and _room(case) <= 6e9:
            return case


def _room(case):
    """About the bytes that the largest tensors of a case's plain form take."""
    if case["kind"] == "tree":
        return 4.0 * case["B"] * case["len_hi"] * (case["Hq"] * case["T"] + 2 * case["Hkv"] * case["d"])
    if case["kind"] == "verify":
        return 8.0 * case["B"] * case["T"] * case["V"]
    return 0.0


def _draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "verify", "verify", "compact", "fork", "resize"])
    page = rng.choice([0, 16, 64, 256])
    d = rng.choice([128, 128, 64])
    dtype = rng.choice(["fp16", "bf16"])
    shape = rng.choice(["tree", "tree", "chain"])
    lens = rng.randrange(1 << 20)
    ragged = rng.random() < 0.4
    if kind == "tree":
        hq, hkv = rng.choice([(32, 32), (32, 8), (64, 8), (8, 8), (5, 5), (8, 1)])
        hi = _log_int(rng, 256, 16384)
        return dict(kind=kind, B=_log_int(rng, 1, 48), T=_log_int(rng, 2, 80), Hq=hq, Hkv=hkv, len_lo=max(96, hi // 16), len_hi=hi,
                    lens=lens, page=page, d=d, dtype=dtype, shape=shape, ragged=ragged)
    if kind == "verify":
        return dict(kind=kind, B=_log_int(rng, 1, 48), T=_log_int(rng, 2, 64), V=_log_int(rng, 5000, 160000),
                    dtype=rng.choice(["fp32", "fp32", "bf16"]), draft=rng.random() < 0.7, shape=shape, lens=lens, ragged=ragged)
    if kind == "compact":
        return dict(kind=kind, B=_log_int(rng, 1, 96), T=_log_int(rng, 2, 64), L=_log_int(rng, 8, 32), Hkv=rng.choice([1, 5, 8]),
                    len_lo=70, len_hi=_log_int(rng, 72, 140), lens=lens, page=rng.choice([0, 16, 64]), d=d, dtype=dtype, shape=shape,
                    ragged=ragged)
    if kind == "fork":
        n, page = _log_int(rng, 1, 64), rng.choice([16, 32, 64, 128])
        hi = _log_int(rng, 40, 500)
        return dict(kind=kind, n=n, L=_log_int(rng, 8, 32), Hkv=rng.choice([1, 5, 8]), len_lo=max(1, hi // 4), len_hi=hi, lens=lens,
                    pages=(n + 3) // 4 * (hi // page + 1) + n + rng.randrange(1, 17), page=page, d=d, dtype=dtype)
    b, hi, page = _log_int(rng, 1, 512), _log_int(rng, 64, 8000), rng.choice([16, 32, 64])
    grow = _log_int(rng, 2, 130)
    return dict(kind=kind, B=b, len_hi=hi, grow=grow, pages=b * ((hi + grow) // page + 2), page=page)


# ------------------------------------------------------------------ trees and lengths: parts of a case, whatever its values
def _trees(case):
    """Parents of every node and the number of live nodes, per sequence: each sequence has a tree of its own."""
    rng, B, T = random.Random(case["lens"] + 17), case["B"], case["T"]
    parents = [[-1] + [i - 1 if case["shape"] == "chain" else rng.randrange(max(0, i - 8), i) for i in range(1, T)] for _ in range(B)]
    live = [rng.randint(max(1, T // 2), T) if case["ragged"] else T for _ in range(B)]
    return parents, live


def _lens(case, n):
    """Key counts of n sequences (of tree cases: with the tree's rows)."""
    rng = random.Random(case["lens"])
    return [rng.randint(max(case["len_lo"], case.get("T", 1)), max(case["len_hi"], case.get("T", 1))) for _ in range(n)]


def _paths(case):
    """An accepted path per sequence: down from the root until a node has no child, or chance ends it."""
    rng = random.Random(case["lens"] + 29)
    out = []
    for parents, live in zip(*_trees(case)):
        path = [0]
        while rng.random() < 0.75:
            kids = [i for i in range(1, live) if parents[i] == path[-1]]
            if not kids:
                break
            path.append(rng.choice(kids))
        out.append(path)
    return out


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _normal(shape, dtype, gen):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen)


def _table(lens, page, seed, width=0):
    """Block table of sequences whose pages were handed out in a random order; -1 past a sequence's end."""
    need = [-(-x // page) for x in lens]
    order = list(range(sum(need)))
    random.Random(seed).shuffle(order)
    rows, at = [], 0
    for n in need:
        rows.append(order[at:at + n] + [-1] * (max(max(need), width) - n))
        at += n
    return _ints(rows), sum(need)


def _sees(parents, T):
    """[B,T,T]: node i sees node j (itself and its ancestors), from the parents on the host."""
    B = len(parents)
    rows = [[0] * T for _ in range(B)]
    for b in range(B):
        for i in range(T):
            rows[b][i] = (1 << i) | (rows[b][parents[b][i]] if i else 0)
    return rows


def _words(rows, T):
    """Bit rows as 32-bit words [B, T, ceil(T / 32)]."""
    W = (T + 31) // 32
    out = [[[((r >> (32 * w)) & 0xffffffff) for w in range(W)] for r in seq] for seq in rows]
    x = torch.tensor(out, dtype=torch.int64)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32).to(DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return {"tree": _prepare_tree, "verify": _prepare_verify, "compact": _prepare_compact, "fork": _prepare_fork,
            "resize": _prepare_resize}[case["kind"]](case, gen, int(seed))


def _prepare_tree(case, gen, seed):
    B, T, hq, hkv, d, dt = case["B"], case["T"], case["Hq"], case["Hkv"], case["d"], DTYPES[case["dtype"]]
    lens, (parents, live) = _lens(case, B), _trees(case)
    st = {"case": case, "scale": 1.0 / math.sqrt(d), "seqlens": _ints(lens), "mask": _words(_sees(parents, T), T),
          "tree_lens": _ints(live) if case["ragged"] else None, "table": None}
    if case["page"]:
        st["table"], pages = _table(lens, case["page"], seed)
        shape, most = (pages, case["page"], hkv, d), st["table"].shape[1] * case["page"]
    else:
        most = max(lens)
        shape = (B, most, hkv, d)
    st["q"], st["k"], st["v"] = _normal((B, T, hq, d), dt, gen), _normal(shape, dt, gen), _normal(shape, dt, gen)
    st["o"], st["lse"] = torch.empty_like(st["q"]), torch.empty(B, hq, T, dtype=torch.float32, device=DEV)
    st["ws"], st["most"] = None, most
    return st


def _prepare_verify(case, gen, seed):
    B, T, V, dt = case["B"], case["T"], case["V"], DTYPES[case["dtype"]]
    parents, live = _trees(case)
    logits = _normal((B, T, V), torch.float32, gen).mul_(3.0)          # a target as peaked as language models are
    target = torch.softmax(logits, -1)
    near = torch.softmax(logits.add_(_normal((B, T, V), torch.float32, gen).mul_(0.7)), -1)   # a draft that mostly agrees
    del logits
    par = _ints(parents)
    rows = torch.gather(near, 1, par.clamp(min=0).long()[:, :, None].expand(B, T, V))   # each node was drawn at its parent
    tokens = torch.multinomial(rows.view(B * T, V), 1, generator=gen).view(B, T).to(torch.int32)
    return {"case": case, "target": target.to(dt), "draft": near.to(dt) if case["draft"] else None, "tokens": tokens, "parents": par,
            "tree_lens": _ints(live) if case["ragged"] else None,
            "u": torch.rand(B, T, device=DEV, generator=gen), "noise": torch.empty(B, V, device=DEV).exponential_(generator=gen).clamp_(min=1e-20),
            "n_accept": torch.empty(B, dtype=torch.int32, device=DEV), "path": torch.empty(B, T, dtype=torch.int32, device=DEV),
            "out": torch.empty(B, T, dtype=torch.int32, device=DEV)}


def _prepare_compact(case, gen, seed):
    B, T, L, hkv, d, dt = case["B"], case["T"], case["L"], case["Hkv"], case["d"], DTYPES[case["dtype"]]
    lens, (_, live), paths = _lens(case, B), _trees(case), _paths(case)
    st = {"case": case, "seqlens": _ints(lens), "tree_lens": _ints(live) if case["ragged"] else None,
          "path": _ints([p + [-1] * (T - len(p)) for p in paths]), "n_accept": _ints([len(p) - 1 for p in paths]),
          "new_lens": torch.empty(B, dtype=torch.int32, device=DEV), "table": None}
    if case["page"]:
        st["table"], pages = _table(lens, case["page"], seed)
        shape = (L, pages, case["page"], hkv, d)
    else:
        shape = (L, B, max(lens), hkv, d)
    st["k"], st["v"] = _normal(shape, dt, gen), _normal(shape, dt, gen)
    return st


def _prepare_fork(case, gen, seed):
    n, L, hkv, d, page, pages, dt = case["n"], case["L"], case["Hkv"], case["d"], case["page"], case["pages"], DTYPES[case["dtype"]]
    S = (n + 3) // 4                                     # prompts; sequence S + i continues prompt i mod S
    lens = _lens(case, S)
    table, used = _table(lens, page, seed)
    if used > pages:
        raise ValueError("the prompts do not fit into the pool")
    table = torch.cat([table, torch.full((n, table.shape[1]), -1, dtype=torch.int32, device=DEV)])
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs[:used] = 1
    shape = (L, pages, page, hkv, d)
    return {"case": case, "k": _normal(shape, dt, gen), "v": _normal(shape, dt, gen), "table": table, "refs": refs,
            "held": _ints([-(-x // page) for x in lens] + [0] * n), "seqlens": _ints(lens + [0] * n),
            "src": _ints([i % S for i in range(n)]), "dst": _ints([S + i for i in range(n)]), "short": _ints([0]),
            "gone": _ints(lens + [0] * n)}


def _prepare_resize(case, gen, seed):
    B, page = case["B"], case["page"]
    rng = random.Random(seed)
    lens = [rng.randint(1, case["len_hi"]) for _ in range(B)]
    table, used = _table(lens, page, seed, width=-(-(case["len_hi"] + case["grow"]) // page) + 1)
    if used > case["pages"]:
        raise ValueError("the sequences do not fit into the pool")
    refs = torch.zeros(case["pages"], dtype=torch.int32, device=DEV)
    refs[:used] = 1
    # a step's first call makes room for the next tree, its second keeps what was accepted; one sequence in 16 has
    # ended, and its place is taken by a new one
    ended = [rng.random() < 1 / 16 for _ in range(B)]
    room = [0 if e else x + case["grow"] for x, e in zip(lens, ended)]
    kept = [x + rng.randint(1, case["grow"]) for x in lens]
    return {"case": case, "table": table, "refs": refs, "held": _ints([-(-x // page) for x in lens]), "room": _ints(room),
            "kept": _ints(kept), "short": _ints([0])}


# ------------------------------------------------------------------ one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _run_own(st, kind)
    return {"tree": _plain_tree, "verify": _plain_verify, "compact": _plain_compact, "fork": _plain_fork,
            "resize": _plain_resize}[kind](st)


def _run_own(st, kind):
    from paper_2410_16663_b200 import binding as fa
    if kind == "tree":
        if st["ws"] is None:          # kept from call to call
            c = st["case"]
            need = fa.fa_decode_tree_workspace_bytes(c["B"], c["T"], c["Hq"], c["Hkv"], st["most"], c["d"])
            st["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
        fa.fa_decode_tree(st["q"], st["k"], st["v"], st["o"], st["lse"], st["seqlens"], st["mask"], st["scale"], st["ws"],
                          tree_lens=st["tree_lens"], block_table=st["table"])
        return {"o": st["o"], "lse": st["lse"]}
    if kind == "verify":
        fa.fa_spec_verify(st["target"], st["draft"], st["tokens"], st["parents"], st["u"], st["noise"], st["n_accept"], st["path"],
                          st["out"], tree_lens=st["tree_lens"])
        return {"n_accept": st["n_accept"], "path": st["path"], "out": st["out"]}
    if kind == "compact":
        fa.fa_cache_compact(st["k"], st["v"], st["seqlens"], st["path"], st["n_accept"], st["new_lens"], tree_lens=st["tree_lens"],
                            block_table=st["table"])
        return {"k": st["k"], "v": st["v"], "new_lens": st["new_lens"]}
    if kind == "fork":                # the samples of the step before end, new ones begin
        fa.fa_pages_resize(st["table"], st["held"], st["refs"], st["gone"], st["short"], st["case"]["page"])
        fa.fa_pages_fork(st["k"], st["v"], st["table"], st["held"], st["seqlens"], st["refs"], st["src"], st["dst"], st["short"])
        return {n: st[n] for n in ("k", "v", "table", "held", "seqlens", "refs", "short")}
    fa.fa_pages_resize(st["table"], st["held"], st["refs"], st["room"], st["short"], st["case"]["page"])
    fa.fa_pages_resize(st["table"], st["held"], st["refs"], st["kept"], st["short"], st["case"]["page"])
    return {n: st[n] for n in ("table", "held", "refs", "short")}


def _bits(words, n):
    """The first n bits of the words in the last dimension, as truth values."""
    j = torch.arange(n, device=words.device)
    return (words[..., j // 32] >> (j % 32)) & 1 != 0


def _plain_tree(st):
    q, k, v, mask, lens = st["q"], st["k"], st["v"], st["mask"], st["seqlens"]
    B, T, hq, d = q.shape
    hkv = k.shape[2]
    if st["table"] is not None:
        at = st["table"].clamp(min=0).long()
        k, v = k[at].reshape(B, -1, hkv, d), v[at].reshape(B, -1, hkv, d)
    S = k.shape[1]
    live = torch.full_like(lens, T) if st["tree_lens"] is None else st["tree_lens"]
    key, row = torch.arange(S, device=DEV), torch.arange(T, device=DEV)
    node = key[None, :] - (lens - live)[:, None]                                       # [B,S]: the key's node, < 0: prefix
    inside = torch.gather(_bits(mask, T), 2, node.clamp(0, T - 1)[:, None, :].expand(B, T, S))
    sees = ((node < 0)[:, None, :] | inside) & (node < live[:, None])[:, None, :] & (row[None, :] < live[:, None])[:, :, None]
    qf = q.float().view(B, T, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, d)
    s = torch.matmul(qf, k.float().permute(0, 2, 3, 1)).mul_(st["scale"])             # [B,hkv,g*T,S]
    s.view(B, hkv, -1, T, S).masked_fill_(~sees[:, None, None], float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m.clamp(min=-1e30)).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.float().permute(0, 2, 1, 3)) / l.clamp(min=1e-30)
    st["o"].copy_(o.view(B, hkv, -1, T, d).permute(0, 3, 1, 2, 4).reshape(B, T, hq, d))
    st["lse"].copy_((m + l.log()).view(B, hq, T))
    return {"o": st["o"], "lse": st["lse"]}


def _plain_verify(st):
    tokens, parents, u = st["tokens"], st["parents"], st["u"]
    p, q = st["target"], st["draft"]
    B, T, V = p.shape
    seq, at = torch.arange(B, device=DEV), torch.arange(T, device=DEV)
    live = torch.full((B,), T, device=DEV) if st["tree_lens"] is None else st["tree_lens"]
    up, x = parents.clamp(min=0).long(), tokens.long()
    px = p[seq[:, None], up, x].float()                                     # of each node's token, after its parent
    qx = q[seq[:, None], up, x].float() if q is not None else torch.ones_like(px)
    cur = torch.zeros(B, dtype=torch.long, device=DEV)
    s, taken = torch.zeros(B, device=DEV), torch.zeros(B, T, dtype=torch.bool, device=DEV)
    taken[:, 0] = True
    gone = torch.zeros(B, T, dtype=torch.bool, device=DEV)                 # rejected nodes
    if st["case"]["shape"] == "chain":
        ok = (u * qx < px) & (at[None, :] < live[:, None])
        ok[:, 0] = True
        taken = ok.long().cumprod(1) > 0
        cur = taken.sum(1) - 1
        missed = (cur + 1 < live)
        s = missed.float()
        gone[seq, (cur + 1).clamp(max=T - 1)] = missed
    else:
        z = torch.ones(B, device=DEV)
        for i in range(1, T):
            tested = (up[:, i] == cur) & (i < live)
            if q is not None:
                r = (px[:, i] - s * qx[:, i]).clamp(min=0)
            else:
                again = (gone & (up == cur[:, None]) & (tokens == tokens[:, i:i + 1])).any(1)
                r = px[:, i].masked_fill(again, 0.0)
            ok = tested & (u[:, i] * z * qx[:, i] < r)
            no = tested & ~ok
            taken[:, i], gone[:, i] = ok, no
            cur = torch.where(ok, i, cur)
            s = torch.where(ok, 0.0, torch.where(no, s + z, s))
            left = (p[seq, cur].float() - s[:, None] * q[seq, cur].float()).clamp(min=0).sum(1) if q is not None else (z - r).clamp(min=0)
            z = torch.where(ok, 1.0, torch.where(no, left, z))
    n = taken.sum(1)
    pc = p[seq, cur].float()
    if q is not None:
        r = (pc - s[:, None] * q[seq, cur].float()).clamp(min=0)
    else:
        out = (gone & (up == cur[:, None])).float()                         # how often a token was rejected at the last node
        r = torch.where(torch.zeros_like(pc).scatter_add_(1, x, out) > 0, 0.0, pc)
    best, first = (r / st["noise"]).max(1)
    spare, other = (pc / st["noise"]).max(1)
    last = torch.where(best > 0, first, torch.where(spare > 0, other, -1))
    order = torch.where(taken, at[None, :], T).sort(1).values               # the accepted nodes come in index order
    st["path"].copy_(torch.where(order < T, order, -1))
    said = torch.gather(tokens, 1, torch.cat([order[:, 1:], order[:, :1]], 1).clamp(max=T - 1))
    st["out"].copy_(torch.where(at[None, :] < n[:, None] - 1, said, torch.where(at[None, :] == n[:, None] - 1, last[:, None].to(said.dtype), -1)))
    st["n_accept"].copy_(n - 1)
    return {"n_accept": st["n_accept"], "path": st["path"], "out": st["out"]}


def _plain_compact(st):
    k, v, path = st["k"], st["v"], st["path"]
    B, T = path.shape
    live = torch.full_like(st["seqlens"], T) if st["tree_lens"] is None else st["tree_lens"]
    prefix, i = st["seqlens"] - live, torch.arange(T, device=DEV)
    moves = (i[None, :] >= 1) & (i[None, :] <= st["n_accept"][:, None])
    to = (prefix[:, None] + i[None, :]).clamp(max=(st["seqlens"] - 1)[:, None]).long()
    src = torch.where(moves, (prefix[:, None] + path).long(), to)
    if st["table"] is None:
        at = torch.arange(B, device=DEV)[:, None] * k.shape[2]
        to, src = to + at, src + at
    else:
        page = k.shape[2]
        to, src = (torch.gather(st["table"], 1, x // page).long() * page + x % page for x in (to, src))
    to, src = to.view(-1), src.view(-1)
    to, src = torch.where(moves.view(-1), to, to[0]), torch.where(moves.view(-1), src, to[0])   # the rest: a root to itself
    for x in (k, v):
        flat = x.view(x.shape[0], -1, x.shape[3], x.shape[4])
        flat[:, to] = flat[:, src]
    st["new_lens"].copy_(prefix + 1 + st["n_accept"])
    return {"k": k, "v": v, "new_lens": st["new_lens"]}


def _resize(table, held, refs, want, short, page):
    e = torch.arange(table.shape[1], device=DEV)[None, :]
    need, had = (want + page - 1) // page, held.clone()
    drop = (e >= need[:, None]) & (e < had[:, None])
    refs.index_add_(0, table.clamp(min=0).view(-1), -drop.view(-1).to(torch.int32))
    rank = torch.cumsum(refs == 0, 0)                                     # of free pages, by index
    grow = (need - had).clamp(min=0)
    upto = torch.cumsum(grow, 0)
    ok = (upto <= rank[-1]) | (grow == 0)
    new = (e >= had[:, None]) & (e < need[:, None]) & ok[:, None]
    fresh = torch.searchsorted(rank, (upto - grow)[:, None] + e - had[:, None] + 1).clamp(max=refs.numel() - 1).to(torch.int32)
    table.copy_(torch.where(new, fresh, torch.where(drop, -1, table)))
    refs.index_add_(0, table.clamp(min=0).view(-1), new.view(-1).to(torch.int32))
    held.copy_(torch.where(ok, need, had))
    short.copy_((~ok).sum())


def _plain_resize(st):
    _resize(st["table"], st["held"], st["refs"], st["room"], st["short"], st["case"]["page"])
    _resize(st["table"], st["held"], st["refs"], st["kept"], st["short"], st["case"]["page"])
    return {n: st[n] for n in ("table", "held", "refs", "short")}


def _plain_fork(st):
    table, refs, held, lens, page = st["table"], st["refs"], st["held"], st["seqlens"], st["case"]["page"]
    _resize(table, held, refs, st["gone"], st["short"], page)
    src, dst = st["src"].long(), st["dst"].long()
    e = torch.arange(table.shape[1], device=DEV)[None, :]
    n, full, part = lens[src], lens[src] // page, lens[src] % page
    rank = torch.cumsum(refs == 0, 0)
    place = torch.cumsum(part > 0, 0)
    ok = (part == 0) | (place <= rank[-1])
    fresh = torch.searchsorted(rank, place).clamp(max=refs.numel() - 1)
    old = table[src]
    mine = ok & (part > 0)
    shared = (e < full[:, None]) & ok[:, None]
    table[dst] = torch.where(shared, old, torch.where((e == full[:, None]) & mine[:, None], fresh[:, None].to(torch.int32), -1))
    refs.index_add_(0, old.clamp(min=0).view(-1), shared.view(-1).to(torch.int32))
    refs.index_add_(0, fresh, mine.to(torch.int32))
    lens[dst] = torch.where(ok, n, 0)
    held[dst] = torch.where(ok, full + (part > 0), 0)
    st["short"].copy_((~ok).sum())
    last = torch.gather(old, 1, full[:, None].clamp(max=old.shape[1] - 1).long())[:, 0].clamp(min=0).long()
    to = torch.where(mine, fresh, last)                                   # (who copies nothing: a page to itself)
    rows = (torch.arange(page, device=DEV)[None, :] < part[:, None])[None, :, :, None, None]
    for x in (st["k"], st["v"]):
        x[:, to] = torch.where(rows, x[:, last], x[:, to])
    return {n: st[n] for n in ("k", "v", "table", "held", "seqlens", "refs", "short")}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind = case["kind"]
    size = 4 if case.get("dtype") == "fp32" else 2
    if kind == "tree":
        parents, live = _trees(case)
        row = case["Hkv"] * case["d"] * size
        nbytes = flops = 0.0
        for x, par, t in zip(_lens(case, case["B"]), parents, live):
            depth = [1] * len(par)
            for i in range(1, len(par)):
                depth[i] = depth[par[i]] + 1
            nbytes += 2 * x * row + 2 * case["T"] * case["Hq"] * case["d"] * size + 4 * case["T"] * case["Hq"]
            flops += 4.0 * case["Hq"] * case["d"] * (t * (x - t) + sum(depth[:t]))
        return {"bytes": nbytes, "flops": flops}
    if kind == "verify":      # the last node's rows and the exponentials; a subtraction, a division and a comparison each
        n = case["B"] * case["V"]
        return {"bytes": float(n * (size * (2 if case["draft"] else 1) + 4)), "flops": 3.0 * n}
    if kind == "compact":
        rows = sum(sum(1 for i, x in enumerate(p) if x != i) for p in _paths(case))
        return {"bytes": 4.0 * rows * case["L"] * case["Hkv"] * case["d"] * size + 8.0 * case["B"], "flops": 0.0}
    if kind == "fork":
        S = (case["n"] + 3) // 4
        lens = _lens(case, S)
        rows = sum(lens[i % S] % case["page"] for i in range(case["n"]))
        return {"bytes": 4.0 * rows * case["L"] * case["Hkv"] * case["d"] * size + 4.0 * case["pages"], "flops": 0.0}
    # two calls: the reference counts, and about half a page table entry per token that comes and goes
    return {"bytes": 2.0 * 4 * case["pages"] + 8.0 * case["B"] * case["grow"] / case["page"], "flops": 0.0}


# ------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"tree": _exact_tree, "verify": _exact_verify, "compact": _exact_compact, "fork": _exact_fork,
            "resize": _exact_resize}[case["kind"]](case, st)


def _exact_tree(case, st):
    B, T, hq, hkv, d = case["B"], case["T"], case["Hq"], case["Hkv"], case["d"]
    g, lens, (parents, live) = hq // hkv, _lens(case, B), _trees(case)
    o = torch.zeros(B, T, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((B, hq, T), float("-inf"), dtype=torch.float64, device=DEV)
    for b in range(B):
        n, t, pre = lens[b], live[b], lens[b] - live[b]
        if case["page"]:
            ids = st["table"][b, :-(-n // case["page"])].long()
            kb, vb = (st[x][ids].reshape(-1, hkv, d)[:n].double() for x in ("k", "v"))
        else:
            kb, vb = (st[x][b, :n].double() for x in ("k", "v"))
        hidden = torch.zeros(t, n, dtype=torch.bool)
        hidden[:, pre:] = True
        for i in range(t):
            j = i
            while j >= 0:
                hidden[i, pre + j] = False
                j = parents[b][j]
        hidden = hidden.to(DEV)
        for h in range(hq):
            x = (st["q"][b, :t, h].double() @ kb[:, h // g].T) / math.sqrt(d)
            x = x.masked_fill(hidden, float("-inf"))
            lse[b, h, :t] = torch.logsumexp(x, 1)
            o[b, :t, h] = torch.softmax(x, 1) @ vb[:, h // g]
    return {"o": o, "lse": lse}


def _exact_verify(case, st):
    B, T = case["B"], case["T"]
    parents, live = _trees(case)
    tokens, u = st["tokens"].tolist(), st["u"].double().tolist()
    n_accept, path, out = [], [], []
    for b in range(B):
        noise = st["noise"][b].double()
        node, walk, said = 0, [0], []
        while True:
            p = st["target"][b, node].double()
            q = st["draft"][b, node].double() if case["draft"] else None
            r, mass = p.clone(), 1.0
            for c in (i for i in range(node + 1, live[b]) if parents[b][i] == node):
                x = tokens[b][c]
                if u[b][c] * mass * (float(q[x]) if q is not None else 1.0) < float(r[x]):
                    break
                if q is not None:
                    r = (r / mass - q).clamp(min=0)            # the residual, normalised at each rejection
                    mass = float(r.sum())
                else:
                    mass = max(mass - float(r[x]), 0.0)
                    r[x] = 0
            else:
                break
            node = c
            walk.append(c)
            said.append(tokens[b][c])
        if float(r.max()) <= 0:
            r = p
        said.append(int(torch.argmax(r / noise)) if float(r.max()) > 0 else -1)
        n_accept.append(len(walk) - 1)
        path.append(walk + [-1] * (T - len(walk)))
        out.append(said + [-1] * (T - len(said)))
    return {"n_accept": _ints(n_accept), "path": _ints(path), "out": _ints(out)}


def _exact_compact(case, st):
    lens, (_, live), paths = _lens(case, case["B"]), _trees(case), _paths(case)
    k, v = st["k"].double(), st["v"].double()
    table = st["table"].tolist() if case["page"] else None
    place = (lambda b, r: (table[b][r // case["page"]], r % case["page"])) if table else (lambda b, r: (b, r))
    for b, p in enumerate(paths):
        pre = lens[b] - live[b]
        for i, x in enumerate(p):
            (s0, r0), (s1, r1) = place(b, pre + i), place(b, pre + x)
            k[:, s0, r0] = k[:, s1, r1]
            v[:, s0, r0] = v[:, s1, r1]
    return {"k": k, "v": v, "new_lens": _ints([n - t + len(p) for n, t, p in zip(lens, live, paths)])}


def _resized(table, held, refs, want, page):
    """One call on host lists; the number of sequences that got nothing."""
    need = [-(-w // page) for w in want]
    for b, n in enumerate(need):
        while held[b] > n:
            held[b] -= 1
            refs[table[b][held[b]]] -= 1
            table[b][held[b]] = -1
    free = [i for i, r in enumerate(refs) if r == 0]
    total = short = 0
    for b, n in enumerate(need):
        grow = n - held[b]
        if grow <= 0:
            continue
        total += grow
        if total > len(free):
            short += 1
            continue
        for i in free[total - grow:total]:
            table[b][held[b]] = i
            refs[i] = 1
            held[b] += 1
    return short


def _exact_resize(case, st):
    table, held, refs = (st[n].tolist() for n in ("table", "held", "refs"))
    _resized(table, held, refs, st["room"].tolist(), case["page"])
    short = _resized(table, held, refs, st["kept"].tolist(), case["page"])
    return {"table": _ints(table), "held": _ints(held), "refs": _ints(refs), "short": _ints([short])}


def _exact_fork(case, st):
    page = case["page"]
    table, held, refs, lens, src, dst = (st[n].tolist() for n in ("table", "held", "refs", "seqlens", "src", "dst"))
    k, v = st["k"].double(), st["v"].double()
    free, short = [i for i, r in enumerate(refs) if r == 0], 0
    for s, t in zip(src, dst):
        full, part = divmod(lens[s], page)
        if part and not free:
            short += 1
            continue
        for j in range(full):
            table[t][j] = table[s][j]
            refs[table[s][j]] += 1
        if part:
            new = table[t][full] = free.pop(0)
            refs[new] = 1
            k[:, new, :part] = k[:, table[s][full], :part]
            v[:, new, :part] = v[:, table[s][full], :part]
        held[t], lens[t] = full + (part > 0), lens[s]
    return {"k": k, "v": v, "table": _ints(table), "held": _ints(held), "seqlens": _ints(lens), "refs": _ints(refs), "short": _ints([short])}
