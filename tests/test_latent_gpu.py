"""Attention over latent vectors against its definition in float64."""
import random

import pytest
import torch

from oracle import latent as oracle
from paper_2410_16663_b200 import binding as fa

pytestmark = pytest.mark.gpu
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
SCALE = 192 ** -0.5


def normal(shape, dt, seed, by=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=DT[dt], device="cuda").normal_(generator=g).mul_(by)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check(o, lse, want, dt, size=10.0):
    """o, want [n,d].  With u half a step of the type: the output's own rounding (u |O|), that of the probabilities for the second product (u sum P |V|),
    and the 32-bit arithmetic: products of a score add up to at most `size` in magnitude, whose sums over 9 bits of terms are off by 2^-23 * 2^2
    of that at most, the exponentials by 2^-21, the sums over all keys by 2^-15; with size 10 together less than 2^-13 of sum P |V|, and less than
    2^-14 of a log-sum-exp's argument.  fp16 probabilities below 2^-14 of the reference (which is at most the row's largest, so that the row's sum
    is 1 at least) are multiples of 2^-24: rounded by up to 2^-25 whatever their size, which is 2^-25 of sum |V| at most."""
    ref, ref_lse, absv, sumv = want
    u = torch.finfo(DT[dt]).eps / 2
    o, lse = o.double().cpu(), lse.double().cpu()
    extra = max(0.0, size - 10.0) * 2.0 ** -20   # (numerator and denominator)
    allow = u * ref.abs() + (u + 2.0 ** -13 + extra) * absv + 2.0 ** -24 + (2.0 ** -25 * sumv if dt == "fp16" else 0.0)
    assert bool(((o - ref).abs() <= allow).all()), float(((o - ref).abs() / allow.clamp(min=1e-30)).max())
    none = torch.isneginf(ref_lse)
    assert torch.equal(torch.isneginf(lse), none)
    assert bool(((lse - ref_lse).abs() <= 2.0 ** -14 + max(0.0, size - 10.0) * 2.0 ** -21 + 2.0 ** -22 * ref_lse.abs())[~none].all())


def expanded(nq, nk, H, dt, causal, heads=None, rows=None, seed=1, by=1.0):
    cu = lambda x: [0] + [sum(x[:i + 1]) for i in range(len(x))]
    cq, ck = cu(nq), cu(nk)
    q, kv = normal((cq[-1], H, 192), dt, seed, by), normal((ck[-1], H, 256), dt, seed + 1, by)
    both = normal((ck[-1], 576), dt, seed + 2, by)
    o = torch.full((cq[-1], H, 128), float("nan"), dtype=DT[dt], device="cuda")
    lse = torch.full((H, cq[-1]), float("nan"), device="cuda")
    fa.fa_forward_latent(q[..., :128], q[..., 128:], kv[..., :128], both[:, 512:], kv[..., 128:], o, lse, ints(cq), ints(ck), max(nq), max(nk), causal, SCALE)
    for b in range(len(nq)):
        qs, ks = slice(cq[b], cq[b + 1]), slice(ck[b], ck[b + 1])
        for h in heads or range(H):
            k = torch.cat([kv[ks, h, :128], both[ks, 512:]], -1).cpu()
            want = oracle.attention(q[qs, h].cpu(), k, kv[ks, h, 128:].cpu(), SCALE, causal)
            check(o[qs, h], lse[h, qs], want, dt, size=10.0 * by * by)
    assert fa.fa_device_status()[0] == 0
    return q, kv, both, o, lse


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq, nk", [
    ([1], [1]), ([1], [500]), ([128], [128]), ([129], [129]), ([127, 1, 130], [127, 257, 130]), ([64, 0, 300, 5], [64, 40, 701, 5]),
    ([200, 3], [0, 260]), ([50, 40], [10, 39]), ([513], [1000])])
def test_expanded(dt, causal, nq, nk):
    expanded(nq, nk, 3, dt, causal)


@pytest.mark.parametrize("H", [1, 20, 128])
def test_expanded_heads(H):
    expanded([100, 260], [150, 260], H, "bf16", True, heads=[0, H // 2, H - 1])


def test_expanded_many_items():
    """More items than CTAs, several each: the one Q buffer and the ring of K boxes go round."""
    rng = random.Random(5)
    nq = [rng.randint(1, 900) for _ in range(12)]
    expanded(nq, [n + rng.choice([0, 0, 77]) for n in nq], 16, "fp16", True, heads=[0, 7, 15])


def test_expanded_large_scores():
    """Scores of a hundred and more: the reference of the exponentials moves, probabilities are all but one zero."""
    expanded([300], [300], 2, "fp16", True, by=6.0)


def test_expanded_takes_no_rows_of_the_next_sequence():
    """NaN behind a sequence's end, in every tensor the next one owns: it stays in that one's results."""
    q, kv, both = normal((200, 2, 192), "bf16", 1), normal((200, 2, 256), "bf16", 2), normal((200, 576), "bf16", 3)
    clean = torch.empty(100, 2, 128, dtype=torch.bfloat16, device="cuda")
    call = lambda q, kv, both, o, cu: fa.fa_forward_latent(q[..., :128], q[..., 128:], kv[..., :128], both[:, 512:], kv[..., 128:], o, None, ints(cu), ints(cu), 100,
                                                           100, True, SCALE)
    call(q[:100], kv[:100], both[:100], clean, [0, 100])
    q[100:], kv[100:], both[100:] = float("nan"), float("nan"), float("nan")
    o = torch.empty(200, 2, 128, dtype=torch.bfloat16, device="cuda")
    call(q, kv, both, o, [0, 100, 200])
    assert torch.equal(o[:100], clean) and bool(torch.isnan(o[100:]).all())


def test_expanded_rows_behind_the_last_sequence_stay():
    q, kv, both = normal((150, 2, 192), "fp16", 1), normal((150, 2, 256), "fp16", 2), normal((150, 576), "fp16", 3)
    o = torch.full((150, 2, 128), 7.0, dtype=torch.float16, device="cuda")
    fa.fa_forward_latent(q[..., :128], q[..., 128:], kv[..., :128], both[:, 512:], kv[..., 128:], o, None, ints([0, 60, 90]), ints([0, 60, 90]), 60, 60, True, SCALE)
    assert bool((o[90:] == 7.0).all()) and bool(torch.isfinite(o[:90].float()).all())


def test_expanded_without_keys():
    q = normal((5, 2, 192), "fp16", 1)
    none = torch.empty(0, 2, 256, dtype=torch.float16, device="cuda")
    o, lse = torch.full((5, 2, 128), 7.0, dtype=torch.float16, device="cuda"), torch.zeros(2, 5, device="cuda")
    fa.fa_forward_latent(q[..., :128], q[..., 128:], none[..., :128], torch.empty(0, 64, dtype=torch.float16, device="cuda"), none[..., 128:], o, lse, ints([0, 5]),
                         ints([0, 0]), 5, 0, False, SCALE)
    assert bool((o == 0).all()) and bool(torch.isneginf(lse).all())
