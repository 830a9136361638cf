"""Rotation and cache appends against their definitions in float64."""
import random

import pytest
import torch

from oracle import latent as oracle
from paper_2410_16663_b200 import binding as fa

pytestmark = pytest.mark.gpu
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
# What the 32-bit arithmetic adds to a result's own rounding, of |a| + |b| <= 1.5 |(a, b)|: the angle's place in its turn as a float
# (2^-25 of half a turn), sine and cosine (2 ulp), three roundings, all below 2^-23 each.
ARITH = 8 * 2.0 ** -23


def normal(shape, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=DT[dt], device="cuda").normal_(generator=g)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same(got, want, dt, size):
    """Rounded once: half a step of the type, and the arithmetic before it."""
    got = got.double().cpu()
    allow = torch.finfo(DT[dt]).eps / 2 * want.abs() + ARITH * size + 2.0 ** -25
    assert bool(((got - want).abs() <= allow).all()), float(((got - want).abs() - allow).max())


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d, rot, offset", [(128, 128, 0), (64, 16, 48), (64, 32, 8), (256, 64, 64), (16, 16, 0), (576, 64, 512), (1024, 512, 512)])
def test_rope(dt, inter, d, rot, offset):
    n, H = 37, 5
    x = normal((n, H + 3, d), dt, 1)[:, 1:H + 1]
    w = fa.rope_frequencies(rot)
    pos = [0, 1, -5, 2 ** 31 - 1, 500001] + random.Random(2).sample(range(100000), n - 5)
    want = oracle.rotate(x.cpu(), torch.tensor(pos), w.cpu(), offset, inter, 1.25)
    size = 1.5 * 1.25 * x.double().norm(dim=-1, keepdim=True).cpu()
    out = torch.full((n, H, d), float("nan"), dtype=DT[dt], device="cuda")
    fa.fa_rope(x, out, ints(pos), fa.rope_turns(w), offset=offset, interleaved=inter, factor=1.25)
    same(out, want, dt, size)
    keep = torch.ones(d, dtype=torch.bool)
    keep[offset:offset + rot] = False
    assert torch.equal(out[..., keep.cuda()], x[..., keep.cuda()])
    # in place, and back again by the negative turns
    before = x.clone()
    fa.fa_rope(x, x, ints(pos), fa.rope_turns(w), offset=offset, interleaved=inter, factor=1.25)
    assert torch.equal(x, out)
    fa.fa_rope(x, x, ints(pos), -fa.rope_turns(w), offset=offset, interleaved=inter, factor=0.8)
    back = (x.double() - before.double()).norm(dim=-1).max()
    assert float(back) <= 2 * torch.finfo(DT[dt]).eps * float(before.double().norm(dim=-1).max())


@pytest.mark.parametrize("n", [1, 2, 300, 5000])
def test_rope_of_many_tokens(n):
    """The ways the tokens are shared out among the CTAs: one by one, heads apart, several to a CTA."""
    x = normal((n, 40, 128), "bf16", 3)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") + 1000
    w = fa.rope_frequencies(128)
    out = torch.empty_like(x)
    fa.fa_rope(x, out, pos, fa.rope_turns(w))
    at = sorted(set([0, 1 % n, n // 2, n - 1]))
    same(out[at], oracle.rotate(x[at].cpu(), pos[at].cpu(), w.cpu()), "bf16", 1.5 * x[at].double().norm(dim=-1, keepdim=True).cpu())
    for i in at:   # a token's result does not depend on its neighbours
        one = torch.empty_like(x[i:i + 1])
        fa.fa_rope(x[i:i + 1], one, pos[i:i + 1].contiguous(), fa.rope_turns(w))
        assert torch.equal(one[0], out[i])
    assert bool(torch.isfinite(out.float()).all())


def append_case(dt="fp16", B=5, lens=(3, 0, 1, 7, 2), T=0, page=0, Hq=8, Hkv=2, d=128, dv=128, rot=128, offset=0, inter=False, e4m3=False, first=None,
                counts=None, positions=False, latent=False, rows=40, spare=0, with_q=True, with_v=True, seed=1):
    rng = random.Random(seed)
    lens = list(lens) if not T else [T] * B
    cu = None if T else [0] + [sum(lens[:i + 1]) for i in range(B)]
    n = sum(lens) + spare
    first = first or [rng.randrange(0, rows - 12) for _ in range(B)]
    q, k, v = (normal((n, h, w), dt, seed + i) for i, (h, w) in enumerate(((Hq, d), (Hkv, d), (Hkv, dv))))
    table = None
    if page:
        per = -(-rows // page)
        order = list(range(B * per))
        rng.shuffle(order)
        table, slabs, height = [order[b * per:(b + 1) * per] for b in range(B)], B * per + 1, page
    else:
        slabs, height = B, rows
    if latent:
        both = normal((slabs, height, 1, dv + d), dt, seed + 9)
        kc, vc = both[..., dv:], both[..., :dv]
    else:
        kc, vc = normal((slabs, height, Hkv, d), dt, seed + 7), normal((slabs, height, Hkv, dv), dt, seed + 8)
        if e4m3:
            kc, vc = kc.to(torch.float8_e4m3fn), vc.to(torch.float8_e4m3fn)
    pos = [rng.randrange(-10, 100000) for _ in range(n)] if positions else None
    w = fa.rope_frequencies(rot)
    q_out = torch.full_like(q, 7.0)
    before = kc.double().cpu(), vc.double().cpu()
    ks, vs = (0.02, 0.01) if e4m3 else (1.0, 1.0)
    fa.fa_cache_append(q if with_q else None, q_out if with_q else None, k, v if with_v else None, kc, vc if with_v else None, ints(first),
                       turns=fa.rope_turns(w), positions=None if pos is None else ints(pos), counts=None if counts is None else ints(counts),
                       cu_seqlens=None if cu is None else ints(cu), block_table=None if table is None else ints(table), offset=offset,
                       interleaved=inter, k_scale=ks, v_scale=vs)
    places = oracle.append_places(n, B, T, cu, first, counts, rows if not page else -(-rows // page) * page, table, page, slabs)
    owner = oracle.owners(n, B, T, cu)
    at = torch.tensor(pos if pos is not None else [first[b] + t if b >= 0 else 0 for b, t in owner])
    if with_q:
        want = oracle.rotate(q.cpu(), at, w.cpu(), offset, inter)
        mine = [i for i, (b, _) in enumerate(owner) if b >= 0]
        same(q_out[mine], want[mine], dt, 1.5 * q[mine].double().norm(dim=-1, keepdim=True).cpu())
        if len(mine) < n:
            assert bool((q_out[[i for i in range(n) if i not in mine]] == 7.0).all())
    turned = oracle.rotate(k.cpu(), at, w.cpu(), offset, inter)
    for cache, x, old, scale, moved in ((kc, turned, before[0], ks, True), (vc, v.double().cpu(), before[1], vs, False)):
        if cache is vc and not with_v:
            continue
        want, size = old.clone(), torch.zeros_like(old[..., :1])
        touched = torch.zeros(old.shape[:2], dtype=torch.bool)
        for i, place in enumerate(places):
            if place is not None:
                want[place], touched[place] = (x[i] / scale).clamp(-448, 448) if e4m3 else x[i], True
                size[place] = 1.5 * x[i].norm(dim=-1, keepdim=True) / scale
        got = cache.double().cpu()
        assert torch.equal(got[~touched], old[~touched])
        if e4m3:     # half a step of e4m3, of its least normal number below that
            allow = 2.0 ** -4 * want.abs() + 2.0 ** -10 + ARITH * size
            assert bool(((got - want).abs() <= allow)[touched].all())
        elif not moved:
            assert torch.equal(got, want)
        else:
            same(got[touched], want[touched], dt, size[touched])
    return places


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("page", [0, 1, 7, 16, 64])
@pytest.mark.parametrize("e4m3", [False, True])
def test_append(dt, page, e4m3):
    append_case(dt, page=page, e4m3=e4m3, inter=page == 7)


@pytest.mark.parametrize("kw", [
    dict(d=64, dv=64, rot=32, offset=16), dict(d=64, dv=64, rot=32, offset=32, inter=True), dict(Hq=5, Hkv=5, d=256, dv=128),
    dict(B=1, lens=(1,)), dict(T=1), dict(T=3, positions=True), dict(positions=True, page=16), dict(with_q=False), dict(with_v=False),
    dict(counts=[1, 5, 0, 3, -2]), dict(counts=[0, 0, 0, 0, 0], page=16), dict(spare=4), dict(spare=2, page=16, counts=[9] * 5),
    dict(Hq=16, Hkv=1, d=64, dv=512, rot=64, latent=True), dict(Hq=16, Hkv=1, d=64, dv=512, rot=64, latent=True, inter=True, page=16, dt="bf16"),
    dict(first=[37, 39, 40, -1, -9]), dict(first=[47, -3, 10, 2 ** 31 - 4, 46], page=16)], ids=str)
def test_append_forms(kw):
    append_case(**kw)


@pytest.mark.parametrize("B, most", [(1, 700), (70, 9), (300, 3), (1200, 2)])
def test_append_finds_the_sequence(B, most):
    rng = random.Random(B)
    lens = [rng.randint(0, most) for _ in range(B)]
    append_case(B=B, lens=lens, Hq=2, Hkv=1, d=32, dv=16, rot=32, rows=most + 30, first=[rng.randrange(20) for _ in range(B)])


def test_append_passes_over_pages_that_are_not_there():
    k = normal((4, 1, 64), "fp16", 1)
    cache = torch.zeros(3, 16, 1, 64, dtype=torch.float16, device="cuda")
    fa.fa_cache_append(None, None, k, None, cache, None, ints([0, 0, 0, 0]), block_table=ints([[1, 0], [-1, 0], [3, 0], [2 ** 31 - 1, 0]]))
    want = torch.zeros_like(cache)
    want[1, 0] = k[0]
    assert torch.equal(cache, want)


def test_append_past_32_bits():
    """Rows of a cache whose offsets in bytes pass 2^32."""
    B, rows = 3, 1 << 20
    cache = torch.zeros(B, rows, 1, 1024, dtype=torch.uint8, device="cuda")
    k = normal((B, 1, 1024), "bf16", 4)
    first = [rows - 1, 5, rows - 2]
    fa.fa_cache_append(None, None, k, None, cache, None, ints(first), k_scale=0.5)
    for b in range(B):
        got = cache[b, first[b], 0].view(torch.float8_e4m3fn).double().cpu()
        want = k[b, 0].double().cpu() / 0.5
        assert bool(((got - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -10).all())
        cache[b, first[b]] = 0
    assert int(cache.view(torch.int64).abs().max()) == 0


def test_append_takes_nan_and_the_largest():
    k = torch.tensor([float("nan"), float("inf"), 65504.0, -65504.0, 1.0, -0.0, 2.0 ** -24, 448.0], dtype=torch.float16, device="cuda").repeat(1, 1, 8)
    cache = torch.zeros(1, 4, 1, 64, dtype=torch.float8_e4m3fn, device="cuda")
    fa.fa_cache_append(None, None, k, None, cache, None, ints([2]))
    got = cache[0, 2, 0, :8].float().cpu()
    assert bool(torch.isnan(got[0])) and got[1:].tolist() == [448.0, 448.0, -448.0, 1.0, -0.0, 0.0, 448.0]
    plain = torch.zeros(1, 4, 1, 64, dtype=torch.float16, device="cuda")
    fa.fa_cache_append(None, None, k, None, plain, None, ints([2]))
    assert torch.equal(plain[0, 2].view(torch.int16), k[0].view(torch.int16))


def test_append_in_a_graph_and_on_another_stream():
    """A captured step: the lengths of the replay count; what the next step reads follows in the same stream."""
    B = 4
    k, v, q = (normal((B, 1, h, 128), "bf16", i) for i, h in enumerate((2, 2, 8)))
    kc, vc = torch.zeros(B, 64, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, 64, 2, 128, dtype=torch.bfloat16, device="cuda")
    first, turns, out = ints([0, 3, 9, 60]), fa.rope_turns(fa.rope_frequencies(128)), torch.empty_like(q)
    call = lambda: fa.fa_cache_append(q, out, k, v, kc, vc, first, turns=turns)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        first.add_(1)
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert first.tolist() == [1 + step, 4 + step, 10 + step, 61 + step]
        for b in range(B):
            assert torch.equal(vc[b, int(first[b]) - 1], v[b, 0])
    w = fa.rope_frequencies(128).cpu()
    want = oracle.rotate(k[:, 0].cpu(), torch.tensor([2, 5, 11, 62]), w)
    same(torch.stack([kc[b, int(first[b]) - 1] for b in range(B)]), want, "bf16", 1.5 * k[:, 0].double().norm(dim=-1, keepdim=True).cpu())
