"""Attention over latent vectors where a sequence's rows make several blocks, the last one shorter, and where what is not finite has to get
through the merge of an item's parts."""
import random

import pytest
import torch

from oracle import latent as oracle
from paper_2410_16663_b200 import binding as fa
from tests.test_latent_gpu import SCALE, absorbed, check, ints, normal

pytestmark = pytest.mark.gpu


def every_head(result, lens, T, H, dt, samples=None, by=0.5):
    """All heads and tokens of a call of `absorbed`, whose own look is at four heads."""
    q, r, cache, table, _, o, lse, _ = result
    size = SCALE * (512 * 0.64 * by + 64 * 0.64)
    for b in samples or range(len(lens)):
        n = lens[b]
        if table is None:
            rows = cache[b, :n]
        else:
            at = torch.arange(n, device="cuda")
            rows = cache.view(-1, 576)[table[b, at // cache.shape[1]].long() * cache.shape[1] + at % cache.shape[1]]
        rows, live = rows.cpu(), min(T, n)
        x = torch.cat([q[b], r[b]], -1)[T - live:].cpu()
        for h in range(H):
            check(o[b, T - live:, h], lse[b, h, T - live:], oracle.attention(x[:, h], rows, rows[:, :512], SCALE, True), dt, size=size)


def strided(result, lens):
    """The same with queries whose heads lie before their tokens: bit for bit the same result."""
    q, r, cache, table, ws, o, lse, _ = result
    B, T, H, _ = q.shape
    far = torch.full((B, H, T, 640), float("nan"), dtype=q.dtype, device="cuda")
    q2, r2 = far[..., :512].transpose(1, 2), far[..., 576:].transpose(1, 2)
    q2.copy_(q), r2.copy_(r)
    o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
    fa.fa_decode_latent(q2, r2, cache, o2, lse2, ints(lens), SCALE, ws, block_table=table)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("T, H", [(3, 43), (7, 37), (2, 67), (1, 33), (43, 3)])
def test_blocks_that_are_not_alike(T, H, page):
    """129 rows are blocks of 65 and 64, 259 of 87, 87 and 85, 134 of 67 and 67; each of them has an odd half."""
    lens = [700, 40, 0, 129]
    result = absorbed(lens, T, H, "bf16", page=page)
    every_head(result, lens, T, H, "bf16")
    strided(result, lens)


@pytest.mark.parametrize("dt, page", [("fp16", 0), ("bf16", 32)])
def test_blocks_of_more_items_than_workers(dt, page):
    """Sequences of several tiles and three blocks each, some without keys: workers' runs end inside items of every block."""
    rng = random.Random(7)
    lens = [rng.choice([0, rng.randint(100, 900), rng.randint(100, 900), rng.randint(100, 900)]) for _ in range(60)]
    some = list(range(0, 60, 7))
    result = absorbed(lens, 7, 37, dt, page=page, samples=some)
    every_head(result, lens, 7, 37, dt, samples=some)
    strided(result, lens)


@pytest.mark.parametrize("B, n, T, H, page", [
    (2, 400, 1, 40, 0), (2, 400, 1, 128, 64), (2, 400, 2, 100, 16),      # pairs, many parts of an item
    (20, 900, 1, 128, 0), (20, 900, 1, 40, 16),                          # pairs, a few parts
    (90, 300, 1, 64, 0),                                                 # pairs, more items than workers
    (30, 900, 1, 16, 0), (30, 900, 1, 32, 16), (200, 200, 1, 20, 0)])    # one CTA, a few parts, more items than workers
@pytest.mark.parametrize("column", [3, 511, 560])
def test_nan_in_one_number_of_a_seen_row(B, n, T, H, page, column):
    """It makes the tokens that see it NaN, through every merge, and stays in its sequence."""
    result = absorbed([n - 7 * (b % 3) for b in range(B)], T, H, "fp16", page=page, samples=[0])
    q, r, cache, table, ws, o, lse, _ = result
    lens = [n - 7 * (b % 3) for b in range(B)]
    bad = {0: 17, 1: lens[1] - T, B - 1: lens[B - 1] // 2}
    for b, key in bad.items():
        if table is None:
            cache[b, key, column] = float("nan")
        else:
            cache[int(table[b, key // page]), key % page, column] = float("nan")
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    fa.fa_decode_latent(q, r, cache, o2, lse2, ints(lens), SCALE, ws, block_table=table)
    for b in range(B):
        if b in bad:
            assert bool(torch.isnan(o2[b]).all()) and bool(torch.isnan(lse2[b]).all()), b
        else:
            assert torch.equal(o2[b], o[b]) and torch.equal(lse2[b], lse[b]), b
