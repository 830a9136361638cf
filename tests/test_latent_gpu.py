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


# ------------------------------------------------------------------ the absorbed form
def pool_of(rows, page, rng):
    """rows: per sequence [n,576].  A pool whose pages are NaN wherever no row is, and the table; pages in a random order."""
    need = [max(1, -(-len(r) // page)) for r in rows]
    order = list(range(sum(need) + 2))
    rng.shuffle(order)
    pool = torch.full((len(order), page, 576), float("nan"), dtype=rows[0].dtype, device="cuda")
    table, at = [], 0
    for r, n in zip(rows, need):
        ids = order[at:at + n]
        at += n
        for i, page_at in enumerate(ids):
            part = r[i * page:(i + 1) * page]
            pool[page_at, :len(part)] = part
        table.append(ids + [-1] * (max(need) - n))
    return pool, ints(table)


def absorbed(lens, T, H, dt, page=0, seed=1, by=0.5, parts=True, room=0, samples=None):
    rng, B = random.Random(seed), len(lens)
    rows = [normal((n, 576), dt, seed + b) for b, n in enumerate(lens)]
    table = None
    if page:
        cache, table = pool_of(rows, page, rng)
        most = table.shape[1] * page
    else:
        most = max(max(lens), T) + room
        cache = torch.full((B, most, 576), float("nan"), dtype=DT[dt], device="cuda")
        for b, r in enumerate(rows):
            cache[b, :len(r)] = r
    if parts:     # two parts of one tensor
        both = normal((B, T, H, 576), dt, seed + 100)
        q, q_rope = both[..., :512], both[..., 512:]
        q.mul_(by)
    else:
        q, q_rope = normal((B, T, H, 512), dt, seed + 100, by), normal((B, T, H, 64), dt, seed + 101)
    o, lse = torch.full((B, T, H, 512), float("nan"), dtype=DT[dt], device="cuda"), torch.full((B, H, T), float("nan"), device="cuda")
    ws = torch.full((fa.fa_decode_latent_workspace_bytes(B, T, H, most),), 0xff, dtype=torch.uint8, device="cuda")
    if page and -(-T // page) > table.shape[1]:
        pytest.skip("the tokens do not fit into the table")
    fa.fa_decode_latent(q, q_rope, cache, o, lse, ints(lens), SCALE, ws, block_table=table)
    # products of a score: 512 of 0.8 by and 64 of 0.8 squared on average
    size = SCALE * (512 * 0.64 * by + 64 * 0.64)
    for b in samples or range(B):
        n = lens[b]
        live = min(T, n)        # tokens that see a key
        x = torch.cat([q[b], q_rope[b]], -1)[T - live:].cpu()
        for h in sorted(set([0, 1 % H, H // 2, H - 1])):
            want = oracle.attention(x[:, h], rows[b].cpu(), rows[b][:, :512].cpu(), SCALE, True)
            check(o[b, T - live:, h], lse[b, h, T - live:], want, dt, size=size)
        assert bool((o[b, :T - live] == 0).all()) and bool(torch.isneginf(lse[b, :, :T - live]).all())
    assert bool(torch.isfinite(o.float()).all()) and fa.fa_device_status()[0] == 0
    return q, q_rope, cache, table, ws, o, lse, most


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("page", [0, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("T, H", [(1, 16), (1, 20), (3, 5), (2, 16)])
def test_absorbed(dt, page, T, H):
    absorbed([700, 1, 128, 0, 129, 2, 383], T, H, dt, page=page)


@pytest.mark.parametrize("T, H", [(1, 1), (1, 33), (1, 64), (1, 100), (1, 128), (2, 128), (7, 20), (64, 3), (5, 128)])
def test_absorbed_row_blocks(T, H):
    absorbed([300, 65, 1000], T, H, "bf16", page=64, parts=False)
    absorbed([64, 300, 513], T, H, "fp16")


@pytest.mark.parametrize("H", [16, 128])
def test_absorbed_one_long_sequence(H):
    absorbed([30011], 1, H, "fp16", page=64)


@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("T, H", [(1, 16), (1, 32), (2, 20), (3, 40)])
def test_absorbed_long_runs_of_small_pages(T, H, page):
    """Several tiles of a sequence for every worker, so that the buffers of small pages go round more than once."""
    absorbed([30011, 20000, 17], T, H, "fp16", page=page)


def test_absorbed_many_short_sequences():
    """More sequences than CTAs, several of them without keys; runs of many items."""
    rng = random.Random(3)
    lens = [rng.choice([0, 1, 2, 127, 128, 129, 200]) for _ in range(400)]
    absorbed(lens, 1, 16, "bf16", page=16, samples=range(0, 400, 9))
    absorbed(lens[:170], 2, 40, "fp16", samples=range(0, 170, 9))


def test_absorbed_large_scores():
    absorbed([900, 130], 2, 16, "fp16", by=20.0)
    absorbed([900, 130], 2, 64, "fp16", by=20.0)


def test_absorbed_without_keys_at_all():
    o, lse = absorbed([0, 0, 0], 1, 16, "fp16", room=40)[5:7]
    assert bool((o == 0).all()) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("H", [16, 32, 128])
def test_absorbed_lengths_are_clamped(H):
    """Lengths past the cache or below zero are those of the cache and none."""
    q, r, cache, _, ws, o, lse, most = absorbed([300, 300], 1, H, "bf16")
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    fa.fa_decode_latent(q, r, cache, o2, lse2, ints([10 ** 9, -5]), SCALE, ws)
    assert torch.equal(o2[0], o[0]) and torch.equal(lse2[0], lse[0]) and bool((o2[1] == 0).all()) and bool(torch.isneginf(lse2[1]).all())


@pytest.mark.parametrize("H", [16, 128])
def test_absorbed_pages_that_are_not_there_read_as_zeros(H):
    """A page number outside the pool: rows of zeros, no fault."""
    cache, q, r = normal((4, 64, 576), "fp16", 1), normal((1, 1, H, 512), "fp16", 2, 0.5), normal((1, 1, H, 64), "fp16", 3)
    o, ws = torch.empty_like(q), torch.empty(fa.fa_decode_latent_workspace_bytes(1, 1, H, 256), dtype=torch.uint8, device="cuda")
    for bad in (-1, 4, 2 ** 31 - 1):
        fa.fa_decode_latent(q, r, cache, o, None, ints([256]), SCALE, ws, block_table=ints([[2, bad, 0, 1]]))
        rows = torch.cat([cache[2], torch.zeros_like(cache[0]), cache[0], cache[1]])
        want = oracle.attention(torch.cat([q, r], -1)[0, 0, :1].cpu(), rows.cpu(), rows[:, :512].cpu(), SCALE, False)
        got = o[0, 0, :1].double().cpu()
        assert bool(((got - want[0]).abs() <= 2.0 ** -11 * want[0].abs() + (2.0 ** -11 + 2.0 ** -13) * want[2] + 2.0 ** -25 * want[3] + 2.0 ** -24).all())


def test_absorbed_nan_in_a_row_that_is_seen_stays_in_its_sequence():
    q, r, cache, _, ws, o, lse, _ = absorbed([300, 400], 1, 16, "fp16")
    cache[0, 17] = float("nan")
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    fa.fa_decode_latent(q, r, cache, o2, lse2, ints([300, 400]), SCALE, ws)
    assert bool(torch.isnan(o2[0]).all()) and bool(torch.isnan(lse2[0]).all()) and torch.equal(o2[1], o[1]) and torch.equal(lse2[1], lse[1])


@pytest.mark.parametrize("H", [16, 32, 128])
def test_absorbed_in_a_graph(H):
    """Lengths and rows of the replay count, and a workspace that two graphs share in turn."""
    lens = [200, 900, 40]
    q, r, cache, _, ws, o, lse, _ = absorbed(lens, 1, H, "bf16", room=600)
    now, cache2 = ints(lens), normal(cache.shape, "bf16", 77)
    out = [torch.empty_like(o), torch.empty_like(o)]
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g, to, c in zip(graphs, out, (cache, cache2)):
        with torch.cuda.graph(g):
            fa.fa_decode_latent(q, r, c, to, None, now, SCALE, ws)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], o)
    want = torch.empty_like(o)
    now.copy_(ints([1500, 0, 777]))
    cache.nan_to_num_(0.25)
    for g in graphs:
        g.replay()
    for to, c in zip(out, (cache, cache2)):
        fa.fa_decode_latent(q, r, c, want, None, now, SCALE, ws)
        assert torch.equal(to, want)


def test_absorbed_offsets_past_32_bits():
    """A cache of more than 4 GiB: the last sequence's rows."""
    B, n = 3, 1300000
    cache = torch.zeros(B, n, 576, dtype=torch.float16, device="cuda")
    cache[2, n - 300:] = normal((300, 576), "fp16", 1)
    q, r = normal((B, 1, 16, 512), "fp16", 2, 0.5), normal((B, 1, 16, 64), "fp16", 3)
    o, ws = torch.empty_like(q), torch.empty(fa.fa_decode_latent_workspace_bytes(B, 1, 16, n), dtype=torch.uint8, device="cuda")
    fa.fa_decode_latent(q, r, cache, o, None, ints([0, 0, n]), SCALE, ws)
    x = torch.cat([q, r], -1)[2, 0, :2].cpu()
    want = oracle.attention(x, cache[2, n - 300:].cpu(), cache[2, n - 300:, :512].cpu(), SCALE, False)
    # with the zeros before them: their scores are 0, their values nothing
    rest = torch.log1p((n - 300) * torch.exp(-want[1]))[:, None]
    got = o[2, 0, :2].double().cpu()
    ref = want[0] * torch.exp(-rest)
    assert bool(((got - ref).abs() <= 2.0 ** -10 * want[2] * torch.exp(-rest) + 2.0 ** -11 * ref.abs() + 2.0 ** -24).all())


@pytest.mark.parametrize("T, H", [(3, 5), (4, 20), (2, 128)])
def test_absorbed_queries_of_any_strides(T, H):
    """Heads before tokens, a tensor with room between the rows: the result is that of the same queries put together."""
    q, r, cache, table, ws, o, lse, most = absorbed([300, 41, 0, 700], T, H, "bf16", page=32)
    far = normal((4, H, T, 1024), "bf16", 5)
    q2, r2 = far[..., :512].transpose(1, 2), far[..., 640:704].transpose(1, 2)
    q2.copy_(q), r2.copy_(r)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    fa.fa_decode_latent(q2, r2, cache, o2, lse2, ints([300, 41, 0, 700]), SCALE, ws, block_table=table)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)


@pytest.mark.parametrize("H", [16, 40, 128])
def test_calls_at_once(H):
    """Two calls on two streams, with workspaces of their own, while a third takes its turns on one: each gives what it gives alone."""
    cases = [absorbed([400, 3000, 77], 1, H, dt, page=page) for dt, page in (("fp16", 64), ("bf16", 0), ("fp16", 16))]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    lens = ints([400, 3000, 77])
    torch.cuda.synchronize()
    outs = []
    for turn in range(6):
        for i, (q, r, cache, table, ws, o, lse, _) in enumerate(cases):
            with torch.cuda.stream(streams[i % 2]):
                o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
                fa.fa_decode_latent(q, r, cache, o2, lse2, lens, SCALE, ws, block_table=table)
                outs.append((o2, o, lse2, lse))
    torch.cuda.synchronize()
    for o2, o, lse2, lse in outs:
        assert torch.equal(o2, o) and torch.equal(lse2, lse)


@pytest.mark.parametrize("H, T", [(16, 1), (40, 2), (128, 1)])
def test_a_prompt_and_the_tokens_after_it(H, T):
    """A layer's calls as they follow one another: the prompt's latent vectors and rotated keys go to a paged cache, its queries are rotated on the
    way and attend in the expanded form; then new tokens are appended and attend in the absorbed form, to what the appends have written."""
    dt, page, lens = "fp16", 16, [70, 131, 1]
    B, n = len(lens), sum(lens)
    g = torch.Generator(device="cuda").manual_seed(3)
    w_k = torch.empty(H, 128, 512, device="cuda").normal_(generator=g).mul_(512 ** -0.5)       # key and value expansion of each head
    w_v = torch.empty(H, 128, 512, device="cuda").normal_(generator=g).mul_(512 ** -0.5)
    turns = fa.rope_turns(fa.rope_frequencies(64))
    need = [-(-(x + T) // page) for x in lens]
    pages, at, table = list(range(sum(need))), 0, []
    random.Random(1).shuffle(pages)
    for x in need:
        table.append(pages[at:at + x] + [-1] * (max(need) - x))
        at += x
    table = ints(table)
    cache = torch.full((sum(need), page, 576), float("nan"), dtype=torch.float16, device="cuda")
    cu = ints([0, 70, 201, 202])
    # the prompt
    q, c, kr = normal((n, H, 192), dt, 11), normal((n, 1, 512), dt, 12), normal((n, 1, 64), dt, 13)
    raw = q.clone()
    fa.fa_cache_append(q[..., 128:], q[..., 128:], kr, c, cache[..., 512:], cache[..., :512], ints([0] * B), turns=turns, cu_seqlens=cu, block_table=table)
    slots = torch.cat([table[b, torch.arange(x, device="cuda") // page].long() * page + torch.arange(x, device="cuda") % page for b, x in enumerate(lens)])
    rows = cache.view(-1, 576)[slots]
    assert torch.equal(rows[:, :512], c[:, 0]) and torch.equal(q[..., :128], raw[..., :128])
    k = torch.einsum("nc,hdc->nhd", rows[:, :512].float(), w_k).half()
    v = torch.einsum("nc,hdc->nhd", rows[:, :512].float(), w_v).half()
    o, lse = torch.empty(n, H, 128, dtype=torch.float16, device="cuda"), torch.empty(H, n, device="cuda")
    fa.fa_forward_latent(q[..., :128], q[..., 128:], k, rows[:, 512:], v, o, lse, cu, cu, max(lens), max(lens), True, SCALE)
    at = 0
    for x in lens:
        for h in (0, H - 1):
            want = oracle.attention(q[at:at + x, h].cpu(), torch.cat([k[at:at + x, h], rows[at:at + x, 512:]], -1).cpu(), v[at:at + x, h].cpu(), SCALE, True)
            check(o[at:at + x, h], lse[h, at:at + x], want, dt)
        at += x
    # T tokens more; the second sequence's do not get room
    q2, c2, kr2 = normal((B, T, H, 192), dt, 21), normal((B, T, 1, 512), dt, 22), normal((B, T, 1, 64), dt, 23)
    before = cache.clone()
    fa.fa_cache_append(q2[..., 128:], q2[..., 128:], kr2, c2, cache[..., 512:], cache[..., :512], ints(lens), turns=turns, counts=ints([T, 0, T]), block_table=table)
    changed = (cache.view(torch.int16) != before.view(torch.int16)).any(-1).sum()
    assert int(changed) == 2 * T
    now = [lens[0] + T, lens[1], lens[2] + T]
    absorbed_q = torch.einsum("bthd,hdc->bthc", q2[..., :128].float(), w_k).half()
    ol, lse2 = torch.empty(B, T, H, 512, dtype=torch.float16, device="cuda"), torch.empty(B, H, T, device="cuda")
    ws = torch.empty(fa.fa_decode_latent_workspace_bytes(B, T, H, table.shape[1] * page), dtype=torch.uint8, device="cuda")
    fa.fa_decode_latent(absorbed_q, q2[..., 128:], cache, ol, lse2, ints(now), SCALE, ws, block_table=table)
    for b, x in enumerate(now):
        slots = table[b, torch.arange(x, device="cuda") // page].long() * page + torch.arange(x, device="cuda") % page
        rows = cache.view(-1, 576)[slots]
        live = min(T, x)
        for h in (0, H - 1):
            want = oracle.attention(torch.cat([absorbed_q[b, T - live:, h], q2[b, T - live:, h, 128:]], -1).cpu(), rows.cpu(), rows[:, :512].cpu(), SCALE, True)
            check(ol[b, T - live:, h], lse2[b, h, T - live:], want, dt, size=40.0)
            # And the two forms agree: of the absorbed output expanded, and of expanded keys and values.  Queries, keys, values and outputs are rounded to half a
            # step (2^-11) each on the way: scores move by 2^-11 of some tens of products' root sum square, below 0.01, and the output by less than 0.02 of its size.
            kk, vv = rows[:, :512].double() @ w_k[h].double().T, rows[:, :512].double() @ w_v[h].double().T
            full = oracle.attention(q2[b, T - live:, h].cpu(), torch.cat([kk, rows[:, 512:].double()], -1).cpu(), vv.cpu(), SCALE, True)[0]
            got = (ol[b, T - live:, h].double() @ w_v[h].double().T).cpu()
            assert float((got - full).norm() / full.norm()) < 0.02


@pytest.mark.parametrize("H", [5, 32, 128])
@pytest.mark.parametrize("most", [1, 10, 64, 65, 128, 129])
def test_absorbed_small_caches(H, most):
    """Caches that are less than a tile, one tile (of which nothing is to merge) and a little more."""
    absorbed([most, 0, max(1, most // 2)], 1, H, "fp16")


@pytest.mark.parametrize("H", [16, 128])
def test_absorbed_scale_of_zero(H):
    """All keys weigh the same."""
    cache, q, r = normal((2, 200, 576), "fp16", 1), normal((2, 1, H, 512), "fp16", 2), normal((2, 1, H, 64), "fp16", 3)
    o, lse, ws = torch.empty_like(q), torch.empty(2, H, 1, device="cuda"), torch.empty(fa.fa_decode_latent_workspace_bytes(2, 1, H, 200), dtype=torch.uint8, device="cuda")
    fa.fa_decode_latent(q, r, cache, o, lse, ints([200, 7]), 0.0, ws)
    for b, n in enumerate((200, 7)):
        want = cache[b, :n, :512].double().mean(0)
        allow = 2.0 ** -11 * want.abs() + 2.0 ** -13 * cache[b, :n, :512].double().abs().mean(0)
        assert bool(((o[b, 0].double() - want).abs() <= allow).all()) and bool((lse[b].double() - torch.log(torch.tensor(float(n)))).abs().max() < 1e-4)
