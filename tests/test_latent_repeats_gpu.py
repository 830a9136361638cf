"""Attention over latent vectors, called again and again: values of keys that are none are cleared in shared memory while products and loads of other steps are
under way, and none of those may take any harm."""
import random

import pytest
import torch

from paper_2410_16663_b200 import binding as fa
from tests.test_latent_gpu import SCALE, absorbed, expanded, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B, lo, hi, T, H, page", [
    (1, 1000, 1000, 1, 16, 64), (64, 2980, 3000, 1, 16, 0), (64, 100, 3000, 1, 32, 16), (3, 4000, 5000, 1, 32, 32),        # one CTA
    (20, 2000, 2000, 1, 128, 0), (20, 1980, 2000, 1, 64, 64), (32, 500, 4000, 1, 128, 0), (90, 486, 500, 2, 100, 16),      # pairs
    (74, 129, 400, 1, 40, 0), (150, 65, 260, 3, 30, 64), (7, 500, 9000, 3, 20, 64), (150, 1, 260, 3, 30, 32), (7, 500, 9000, 3, 20, 16)])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_the_same_call_gives_the_same_bits(B, lo, hi, T, H, page, dt):
    """All rows behind a sequence's end are NaN; every fourth sequence is held against the definition."""
    rng = random.Random(B)
    lens = [rng.randint(lo, hi) for _ in range(B)]
    q, r, cache, table, ws, o, lse, _ = absorbed(lens, T, H, dt, page=page, samples=range(0, B, 4) if B < 40 else range(0, B, 16))
    now = ints(lens)
    for _ in range(12):
        o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
        ws.fill_(255)
        fa.fa_decode_latent(q, r, cache, o2, lse2, now, SCALE, ws, block_table=table)
        assert torch.equal(o2, o) and torch.equal(lse2, lse)
    assert fa.fa_device_status()[0] == 0


@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("T, H", [(3, 30), (1, 128), (2, 20)])
def test_halves_of_tiles_without_keys(T, H, page):
    """Tiles whose second half has no page, one after the other: the CTA of a pair that has nothing to load there keeps step all the same."""
    rng = random.Random(H)
    lens = [rng.choice([rng.randint(1, 64), 128 + rng.randint(1, 64)]) for _ in range(300)]
    q, r, cache, table, ws, o, lse, _ = absorbed(lens, T, H, "fp16", page=page, samples=range(0, 300, 23))
    now = ints(lens)
    for _ in range(40):
        o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
        fa.fa_decode_latent(q, r, cache, o2, lse2, now, SCALE, ws, block_table=table)
        assert torch.equal(o2, o) and torch.equal(lse2, lse)
    assert fa.fa_device_status()[0] == 0


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("nq, nk, H", [([2000, 1, 700, 129, 64, 1500], [2000, 300, 700, 900, 64, 1777], 16), ([60] * 40, [60 + 7 * i for i in range(40)], 5)])
def test_the_same_prompts_give_the_same_bits(nq, nk, H, dt):
    q, kv, both, o, lse = expanded(nq, nk, H, dt, True, heads=[0])
    cq, ck = ([sum(x[:i]) for i in range(len(x) + 1)] for x in (nq, nk))
    for _ in range(12):
        o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
        fa.fa_forward_latent(q[..., :128], q[..., 128:], kv[..., :128], both[:, 512:], kv[..., 128:], o2, lse2, ints(cq), ints(ck), max(nq), max(nk), True, SCALE)
        assert torch.equal(o2, o) and torch.equal(lse2, lse)
