"""What writes a cache, and attention over latent vectors: what a serving program calls and how its time is watched.

A new token's queries and keys are rotated by their position (kind ``rope``: ``fa_rope``), or rotated on the way to the cache,
where its key and value become a row (``append``: ``fa_cache_append``).  With latent attention that row is one vector for all
heads, 512 elements and 64 rotated ones; new tokens attend to it as it is, with queries that have taken up the key expansion
(``absorbed``: ``fa_decode_latent``), and prompts with keys and values expanded for each head (``expanded``:
``fa_forward_latent``).

``own`` false computes each operator in plain torch operations in 32 bits, ``own`` true calls the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
LATENT, ROPE = 512, 64          # elements of a latent vector, and of the rotated part behind it


def listed():
    return [
        # one user's new token: the queries and keys of 32/8 heads, out of the packed projection
        dict(name="rope_one", kind="rope", n=1, H=40, spare=8, d=128, rot=128, offset=0, pairs=False, stretch=1.0, far=4000, dtype="fp16"),
        # a long prompt far out, neighbouring elements rotated, frequencies stretched for long contexts
        dict(name="rope_prompt", kind="rope", n=16384, H=40, spare=8, d=128, rot=128, offset=0, pairs=True, stretch=8.0, far=500000,
             dtype="bf16"),
        # half of each head is rotated, sizes that are multiples of nothing
        dict(name="rope_part", kind="rope", n=777, H=21, spare=3, d=64, rot=32, offset=32, pairs=False, stretch=1.0, far=30000, dtype="fp16"),
        # one user's new token goes to its cache
        dict(name="append_one", kind="append", B=1, t_lo=1, t_hi=1, Hq=32, Hkv=8, d=128, dv=128, rot=128, offset=0, pairs=False, page=0,
             e4m3=False, before=2000, lens=1, dtype="fp16"),
        # a full server, a few drafted tokens for each sequence, an 8-bit cache on small pages
        dict(name="append_batch", kind="append", B=256, t_lo=1, t_hi=5, Hq=32, Hkv=8, d=128, dv=128, rot=128, offset=0, pairs=False, page=16,
             e4m3=True, before=600, lens=2, dtype="bf16"),
        # the latent vectors of prompts of unequal length, with the rotated queries of 64 heads
        dict(name="append_latent", kind="append", B=12, t_lo=100, t_hi=1500, Hq=64, Hkv=1, d=ROPE, dv=LATENT, rot=ROPE, offset=0, pairs=True,
             page=64, e4m3=False, before=0, lens=3, dtype="bf16"),
        # one user, 16 heads (one GPU's part of a model), a short conversation: the latency of a single step
        dict(name="absorbed_one", kind="absorbed", B=1, T=1, H=16, len_lo=1000, len_hi=1000, lens=1, page=64, dtype="bf16"),
        # a chat batch of such a part, lengths as they come
        dict(name="absorbed_chat", kind="absorbed", B=64, T=1, H=16, len_lo=100, len_hi=12000, lens=2, page=64, dtype="bf16"),
        # all 128 heads on one GPU
        dict(name="absorbed_heads", kind="absorbed", B=32, T=1, H=128, len_lo=1000, len_hi=8000, lens=3, page=0, dtype="fp16"),
        # three tokens at a time, small pages, a head count that is a multiple of nothing
        dict(name="absorbed_few", kind="absorbed", B=7, T=3, H=20, len_lo=500, len_hi=20000, lens=4, page=16, dtype="fp16"),
        # prompts of unequal length, the last of them with keys before their queries
        dict(name="expanded_prompts", kind="expanded", B=9, q_lo=60, q_hi=1500, before=800, H=16, lens=1, causal=True, dtype="bf16"),
        # a long document: the largest
        dict(name="expanded_long", kind="expanded", B=1, q_lo=8192, q_hi=8192, before=0, H=32, lens=2, causal=True, dtype="fp16"),
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
        if w["bytes"] <= m["bytes"] and w["flops"] <= m["flops"]:
            return case


def _draw(rng):
    kind = rng.choice(["rope", "append", "append", "absorbed", "absorbed", "absorbed", "expanded", "expanded"])
    dtype, pairs, lens = rng.choice(["fp16", "bf16"]), rng.random() < 0.5, rng.randrange(1 << 20)
    if kind == "rope":
        d = rng.choice([64, 128, 256])
        rot = rng.choice([d, d, d // 2, d // 4])
        return dict(kind=kind, n=_log_int(rng, 1, 16384), H=_log_int(rng, 1, 72), spare=rng.choice([0, 0, 1, 8]), d=d, rot=rot,
                    offset=rng.choice([0, d - rot]), pairs=pairs, stretch=rng.choice([1.0, 4.0, 32.0]), far=_log_int(rng, 100, 1000000),
                    dtype=dtype)
    if kind == "append":
        t_hi = _log_int(rng, 1, 1500)
        case = dict(kind=kind, B=_log_int(rng, 1, max(1, min(256, 10000 // t_hi))), t_lo=rng.choice([1, t_hi]), t_hi=t_hi, pairs=pairs,
                    page=rng.choice([0, 16, 64, 128]), before=_log_int(rng, 1, 1000), lens=lens, dtype=dtype)
        if rng.random() < 0.4:
            return dict(case, Hq=rng.choice([16, 20, 64, 128]), Hkv=1, d=ROPE, dv=LATENT, rot=ROPE, offset=0, e4m3=False)
        hq, hkv = rng.choice([(32, 32), (32, 8), (64, 8), (8, 8), (5, 5), (8, 1)])
        d = rng.choice([64, 128, 128])
        rot = rng.choice([d, d, d // 2])
        return dict(case, Hq=hq, Hkv=hkv, d=d, dv=d, rot=rot, offset=rng.choice([0, d - rot]), e4m3=rng.random() < 0.4)
    if kind == "absorbed":
        hi = _log_int(rng, 64, 32768)
        return dict(kind=kind, B=_log_int(rng, 1, 128), T=rng.choice([1, 1, 1, 2, 4, 7]), H=rng.choice([8, 16, 20, 32, 64, 128]),
                    len_lo=max(8, hi // rng.choice([1, 4, 64])), len_hi=hi, lens=lens, page=rng.choice([0, 16, 64, 64, 256]), dtype=dtype)
    hi = _log_int(rng, 16, 8192)
    return dict(kind=kind, B=_log_int(rng, 1, 32), q_lo=max(1, hi // rng.choice([1, 4, 32])), q_hi=hi, before=rng.choice([0, 0, 100, 2000]),
                H=rng.choice([4, 16, 20, 32, 128]), lens=lens, causal=rng.random() < 0.8, dtype=dtype)


# ------------------------------------------------------------------ lengths: parts of a case, whatever its values
def _counts(case):
    """New tokens of each sequence (append), its queries (expanded)."""
    rng = random.Random(case["lens"])
    lo, hi = ("t_lo", "t_hi") if case["kind"] == "append" else ("q_lo", "q_hi")
    return [rng.randint(case[lo], case[hi]) for _ in range(case["B"])]


def _before(case):
    """Rows in each sequence's cache ahead of its new tokens (append), keys ahead of its queries (expanded: of every third one)."""
    rng = random.Random(case["lens"] + 17)
    if case["kind"] == "append":
        return [rng.randint(case["before"] // 2, case["before"]) for _ in range(case["B"])]
    return [rng.randint(case["before"] // 2, case["before"]) if b % 3 == 2 else 0 for b in range(case["B"])]


def _lens(case):
    """Keys of each sequence (absorbed), the new tokens' among them."""
    rng = random.Random(case["lens"])
    return [max(case["T"], rng.randint(case["len_lo"], case["len_hi"])) for _ in range(case["B"])]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _cumulated(x):
    out = [0]
    for n in x:
        out.append(out[-1] + n)
    return out


def _normal(shape, dtype, gen):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen)


def _table(lens, page, seed):
    """Block table of sequences whose pages were handed out in a random order; -1 past a sequence's end."""
    need = [-(-x // page) for x in lens]
    order = list(range(sum(need)))
    random.Random(seed).shuffle(order)
    rows, at = [], 0
    for n in need:
        rows.append(order[at:at + n] + [-1] * (max(need) - n))
        at += n
    return _ints(rows), sum(need)


def _frequencies(rot, stretch, trained=8192):
    """Radians per position of each pair, in 64 bits.  Stretched: the pairs that turn less than once over the trained length are slowed
    down, those that turn more than 32 times are left, in between it is a mixture of both."""
    w = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    if stretch == 1.0:
        return w
    keep = ((trained * w / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return w * (keep + (1.0 - keep) / stretch)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return {"rope": _prepare_rope, "append": _prepare_append, "absorbed": _prepare_absorbed, "expanded": _prepare_expanded}[case["kind"]](
        case, gen, int(seed))


def _prepare_rope(case, gen, seed):
    n, H, d, dt = case["n"], case["H"], case["d"], DTYPES[case["dtype"]]
    x = _normal((n, H + case["spare"], d), dt, gen)[:, :H]      # the first heads of a packed projection
    first = random.Random(seed).randint(0, case["far"])
    positions = (first + torch.arange(n, device=DEV)).to(torch.int32)
    # (a stretched context comes with a factor on the rotated elements)
    return {"case": case, "x": x, "out": torch.empty(n, H, d, dtype=dt, device=DEV), "positions": positions,
            "freq": _frequencies(case["rot"], case["stretch"]), "turns": None, "factor": 1.0 + 0.1 * math.log(case["stretch"])}


def _prepare_append(case, gen, seed):
    B, hq, hkv, d, dv, page, dt = (case[x] for x in ("B", "Hq", "Hkv", "d", "dv", "page", "dtype"))
    dt, new, before = DTYPES[dt], _counts(case), _before(case)
    n, lens = sum(new), [x + y for x, y in zip(before, new)]
    st = {"case": case, "n": n, "first": _ints(before), "cu": None if len(set(new)) == 1 else _ints(_cumulated(new)), "table": None,
          "freq": _frequencies(case["rot"], 1.0), "turns": None, "k_scale": 0.02, "v_scale": 0.015,
          "slot": torch.cat([torch.arange(x, y, device=DEV) for x, y in zip(before, lens)]),
          "seq": torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(new, device=DEV), output_size=n)}
    if page:
        st["table"], slabs = _table(lens, page, seed)
        rows = page
    else:
        slabs, rows = B, max(lens)
    st["q"], st["k"], st["v"] = _normal((n, hq, d), dt, gen), _normal((n, hkv, d), dt, gen), _normal((n, hkv, dv), dt, gen)
    st["q_out"] = torch.empty_like(st["q"])
    if dv != d:                                             # a latent vector and its rotated part are one row
        both = _normal((slabs, rows, 1, dv + d), dt, gen)
        st["k_cache"], st["v_cache"] = both[..., dv:], both[..., :dv]
    else:
        st["k_cache"], st["v_cache"] = _normal((slabs, rows, hkv, d), dt, gen), _normal((slabs, rows, hkv, dv), dt, gen)
        if case["e4m3"]:
            st["k_cache"], st["v_cache"] = st["k_cache"].to(torch.float8_e4m3fn), st["v_cache"].to(torch.float8_e4m3fn)
    return st


def _prepare_absorbed(case, gen, seed):
    B, T, H, page, dt = case["B"], case["T"], case["H"], case["page"], DTYPES[case["dtype"]]
    lens = _lens(case)
    st = {"case": case, "lens": lens, "seqlens": _ints(lens), "table": None, "ws": None, "scale": 1.0 / math.sqrt(128 + ROPE)}
    if page:
        st["table"], pages = _table(lens, page, seed)
        shape, st["most"] = (pages, page, LATENT + ROPE), st["table"].shape[1] * page
    else:
        st["most"] = max(lens)
        shape = (B, st["most"], LATENT + ROPE)
    st["cache"] = _normal(shape, dt, gen)
    # (queries that have taken up the key expansion: scores of about the size that the expanded form has)
    st["q"] = _normal((B, T, H, LATENT), dt, gen).mul_(0.5)
    st["q_rope"] = _normal((B, T, H, ROPE), dt, gen)
    st["o"], st["lse"] = torch.empty_like(st["q"]), torch.empty(B, H, T, dtype=torch.float32, device=DEV)
    return st


def _prepare_expanded(case, gen, seed):
    H, dt = case["H"], DTYPES[case["dtype"]]
    nq = _counts(case)
    nk = [x + y for x, y in zip(nq, _before(case))]
    q, kv = _normal((sum(nq), H, 128 + ROPE), dt, gen), _normal((sum(nk), H, 256), dt, gen)
    rows = _normal((sum(nk), LATENT + ROPE), dt, gen)       # the keys' rotated parts are the ends of their latent vectors' rows
    return {"case": case, "q": q[..., :128], "q_rope": q[..., 128:], "k": kv[..., :128], "v": kv[..., 128:], "k_rope": rows[:, LATENT:],
            "o": torch.empty(sum(nq), H, 128, dtype=dt, device=DEV), "lse": torch.empty(H, sum(nq), dtype=torch.float32, device=DEV),
            "cu_q": _ints(_cumulated(nq)), "cu_k": _ints(_cumulated(nk)), "nq": nq, "nk": nk, "scale": 1.0 / math.sqrt(128 + ROPE)}


# ------------------------------------------------------------------ one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _run_own(st, kind)
    return {"rope": _plain_rope, "append": _plain_append, "absorbed": _plain_absorbed, "expanded": _plain_expanded}[kind](st)


def _run_own(st, kind):
    from paper_2410_16663_b200 import binding as fa
    c = st["case"]
    if kind in ("rope", "append") and st["turns"] is None:     # a plan of the model's, made once
        st["turns"] = fa.rope_turns(st["freq"])
    if kind == "rope":
        fa.fa_rope(st["x"], st["out"], st["positions"], st["turns"], offset=c["offset"], interleaved=c["pairs"], factor=st["factor"])
        return {"out": st["out"]}
    if kind == "append":
        fa.fa_cache_append(st["q"], st["q_out"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["first"], turns=st["turns"],
                           cu_seqlens=st["cu"], block_table=st["table"], offset=c["offset"], interleaved=c["pairs"],
                           k_scale=st["k_scale"] if c["e4m3"] else 1.0, v_scale=st["v_scale"] if c["e4m3"] else 1.0)
        return {"q": st["q_out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    if kind == "absorbed":
        if st["ws"] is None:          # kept from call to call
            need = fa.fa_decode_latent_workspace_bytes(c["B"], c["T"], c["H"], st["most"], LATENT)
            st["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
        fa.fa_decode_latent(st["q"], st["q_rope"], st["cache"], st["o"], st["lse"], st["seqlens"], st["scale"], st["ws"],
                            block_table=st["table"])
        return {"o": st["o"], "lse": st["lse"]}
    fa.fa_forward_latent(st["q"], st["q_rope"], st["k"], st["k_rope"], st["v"], st["o"], st["lse"], st["cu_q"], st["cu_k"],
                         max(st["nq"]), max(st["nk"]), c["causal"], st["scale"])
    return {"o": st["o"], "lse": st["lse"]}


def _rotate(x, positions, freq, offset, pairs, factor):
    """x [n,H,d] with the pairs of its columns offset .. rotated, in 32 bits; the angles in 64."""
    angle = positions.double()[:, None] * freq[None, :]
    cos, sin = (angle.cos() * factor).float()[:, None], (angle.sin() * factor).float()[:, None]
    half, out = freq.numel(), x.float().clone()
    part = out[..., offset:offset + 2 * half]
    a, b = (part[..., 0::2], part[..., 1::2]) if pairs else (part[..., :half], part[..., half:])
    a, b = a * cos - b * sin, a * sin + b * cos
    out[..., offset:offset + 2 * half] = torch.stack([a, b], -1).flatten(-2) if pairs else torch.cat([a, b], -1)
    return out


def _plain_rope(st):
    c = st["case"]
    st["out"].copy_(_rotate(st["x"], st["positions"], st["freq"], c["offset"], c["pairs"], st["factor"]))
    return {"out": st["out"]}


def _plain_append(st):
    c, at, seq = st["case"], st["slot"], st["seq"]
    st["q_out"].copy_(_rotate(st["q"], at, st["freq"], c["offset"], c["pairs"], 1.0))
    k, v = _rotate(st["k"], at, st["freq"], c["offset"], c["pairs"], 1.0), st["v"].float()
    if c["e4m3"]:                                           # (the largest value of the type is 448)
        k, v = (k / st["k_scale"]).clamp(-448, 448), (v / st["v_scale"]).clamp(-448, 448)
    if c["page"]:
        slab, row = st["table"][seq, at // c["page"]].long(), at % c["page"]
    else:
        slab, row = seq, at
    for cache, x in ((st["k_cache"], k), (st["v_cache"], v)):
        x = x.to(cache.dtype)
        if c["e4m3"]:
            cache, x = cache.view(torch.uint8), x.view(torch.uint8)
        cache[slab, row] = x
    return {"q": st["q_out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _plain_absorbed(st):
    c, lens, table = st["case"], st["lens"], st["table"]
    T, H, page = c["T"], c["H"], c["page"]
    for b, n in enumerate(lens):
        rows = st["cache"][b, :n] if table is None else st["cache"][table[b, :-(-n // page)].long()].view(-1, LATENT + ROPE)[:n]
        rows = rows.float()
        q = torch.cat([st["q"][b], st["q_rope"][b]], -1).float()                   # [T,H,576]
        s = torch.matmul(q.view(T * H, -1), rows.T).mul_(st["scale"]).view(T, H, n)
        last = torch.arange(n - T, n, device=DEV)
        s.masked_fill_((torch.arange(n, device=DEV)[None, :] > last[:, None])[:, None], float("-inf"))
        m = s.amax(-1, keepdim=True)
        p = s.sub_(m).exp_()
        l = p.sum(-1, keepdim=True)
        st["o"][b] = torch.matmul(p.view(T * H, n), rows[:, :LATENT]).view(T, H, LATENT) / l
        st["lse"][b] = (m + l.log())[..., 0].T
    return {"o": st["o"], "lse": st["lse"]}


def _plain_expanded(st):
    c, q0, k0 = st["case"], 0, 0
    for nq, nk in zip(st["nq"], st["nk"]):
        qs, ks = slice(q0, q0 + nq), slice(k0, k0 + nk)
        part = max(1, (1 << 29) // (nq * nk))                                      # heads at a time
        hidden = torch.arange(nk, device=DEV)[None, :] > torch.arange(nk - nq, nk, device=DEV)[:, None]
        for h in range(0, c["H"], part):
            hs = slice(h, h + part)
            s = torch.matmul(st["q"][qs, hs].float().transpose(0, 1), st["k"][ks, hs].float().permute(1, 2, 0))
            s += torch.matmul(st["q_rope"][qs, hs].float().transpose(0, 1), st["k_rope"][ks].float().T)
            s *= st["scale"]
            if c["causal"]:
                s.masked_fill_(hidden, float("-inf"))
            m = s.amax(-1, keepdim=True)
            p = s.sub_(m).exp_()
            l = p.sum(-1, keepdim=True)
            st["o"][qs, hs] = (torch.matmul(p, st["v"][ks, hs].float().transpose(0, 1)) / l).transpose(0, 1).to(st["o"].dtype)
            st["lse"][hs, qs] = (m + l.log())[..., 0]
        q0, k0 = q0 + nq, k0 + nk
    return {"o": st["o"], "lse": st["lse"]}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "rope":       # a product and a sum of two products for each element of a pair
        n = case["n"] * case["H"]
        return {"bytes": 4.0 * n * case["d"] + 4.0 * case["n"], "flops": 3.0 * n * case["rot"]}
    if kind == "append":
        n, size = sum(_counts(case)), 1 if case["e4m3"] else 2
        kv = case["Hkv"] * (case["d"] + case["dv"])
        return {"bytes": float(n * (4 * case["Hq"] * case["d"] + (2 + size) * kv)), "flops": 3.0 * n * (case["Hq"] + case["Hkv"]) * case["rot"]}
    if kind == "absorbed":
        lens, T, H = _lens(case), case["T"], case["H"]
        nbytes = 2.0 * sum(lens) * (LATENT + ROPE) + case["B"] * T * H * (2.0 * (2 * LATENT + ROPE) + 4)
        pairs = sum(T * x - T * (T - 1) // 2 for x in lens)
        return {"bytes": nbytes, "flops": 2.0 * H * pairs * (2 * LATENT + ROPE)}
    nq = _counts(case)
    nk = [x + y for x, y in zip(nq, _before(case))]
    pairs = sum(x * y - (x * (x - 1) // 2 if case["causal"] else 0) for x, y in zip(nq, nk))
    nbytes = sum(nq) * case["H"] * (2.0 * (128 + ROPE + 128) + 4) + sum(nk) * (2.0 * case["H"] * 256 + 2.0 * ROPE)
    return {"bytes": nbytes, "flops": 2.0 * case["H"] * pairs * (128 + ROPE + 128)}


# ------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"rope": _exact_rope, "append": _exact_append, "absorbed": _exact_absorbed, "expanded": _exact_expanded}[case["kind"]](case, st)


def _turned(x, positions, case, stretch, factor):
    """Each pair as a complex number times that of its angle."""
    x, rot, at = x.double(), case["rot"], case["offset"]
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    w = torch.exp(-2.0 * i / rot * math.log(10000.0))
    if stretch != 1.0:
        over = 8192 * w / (2.0 * math.pi)
        keep = torch.where(over <= 1.0, torch.zeros_like(w), torch.where(over >= 32.0, torch.ones_like(w), (over - 1.0) / 31.0))
        w = keep * w + (1.0 - keep) * w / stretch
    left = at + (2 * torch.arange(rot // 2, device=DEV) if case["pairs"] else torch.arange(rot // 2, device=DEV))
    right = left + (1 if case["pairs"] else rot // 2)
    by = torch.polar(torch.full((), factor, dtype=torch.float64, device=DEV).expand(x.shape[0], 1, rot // 2),
                     (positions.double()[:, None] * w)[:, None, :])
    z = torch.complex(x[:, :, left], x[:, :, right]) * by
    out = x.clone()
    out[:, :, left], out[:, :, right] = z.real, z.imag
    return out


def _exact_rope(case, st):
    return {"out": _turned(st["x"], st["positions"], case, case["stretch"], 1.0 + 0.1 * math.log(case["stretch"]))}


def _exact_append(case, st):
    new, before = _counts(case), _before(case)
    at = torch.tensor([before[b] + t for b in range(case["B"]) for t in range(new[b])], device=DEV)
    q, k, v = _turned(st["q"], at, case, 1.0, 1.0), _turned(st["k"], at, case, 1.0, 1.0), st["v"].double()
    caches = [st["k_cache"].double(), st["v_cache"].double()]
    if case["e4m3"]:         # the cache holds shares of a factor, up to the type's largest
        k, v = (k / st["k_scale"]).clamp(-448.0, 448.0), (v / st["v_scale"]).clamp(-448.0, 448.0)
    n = 0
    for b in range(case["B"]):
        row = torch.arange(before[b], before[b] + new[b], device=DEV)
        for cache, x in zip(caches, (k, v)):
            if case["page"]:
                cache[st["table"][b].long()[row // case["page"]], row % case["page"]] = x[n:n + new[b]]
            else:
                cache[b, before[b]:before[b] + new[b]] = x[n:n + new[b]]
        n += new[b]
    return {"q": q, "k_cache": caches[0], "v_cache": caches[1]}


def _exact_absorbed(case, st):
    B, T, H = case["B"], case["T"], case["H"]
    o = torch.zeros(B, T, H, LATENT, dtype=torch.float64, device=DEV)
    lse = torch.zeros(B, H, T, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lens(case)):
        if case["page"]:
            j = torch.arange(n, device=DEV)
            c = st["cache"][st["table"][b].long()[j // case["page"]], j % case["page"]].double()
        else:
            c = st["cache"][b, :n].double()
        for t in range(T):
            seen = n - T + t + 1
            x = (st["q"][b, t].double() @ c[:seen, :LATENT].T + st["q_rope"][b, t].double() @ c[:seen, LATENT:].T) / math.sqrt(192.0)
            lse[b, :, t] = torch.logsumexp(x, 1)
            o[b, t] = torch.softmax(x, 1) @ c[:seen, :LATENT]
    return {"o": o, "lse": lse}


def _exact_expanded(case, st):
    nq, before, H = _counts(case), _before(case), case["H"]
    o = torch.zeros(sum(nq), H, 128, dtype=torch.float64, device=DEV)
    lse = torch.zeros(H, sum(nq), dtype=torch.float64, device=DEV)
    a = c = 0
    for b in range(case["B"]):
        x, y = nq[b], nq[b] + before[b]
        kr = st["k_rope"][c:c + y].double()
        above = torch.ones(x, y, dtype=torch.bool, device=DEV).triu(before[b] + 1)
        for h in range(H):
            s = st["q"][a:a + x, h].double() @ st["k"][c:c + y, h].double().T + st["q_rope"][a:a + x, h].double() @ kr.T
            s = s / math.sqrt(192.0)
            if case["causal"]:
                s = s.masked_fill(above, float("-inf"))
            lse[h, a:a + x] = torch.logsumexp(s, 1)
            o[a:a + x, h] = torch.softmax(s, 1) @ st["v"][c:c + y, h].double()
        a, c = a + x, c + y
    return {"o": o, "lse": lse}
