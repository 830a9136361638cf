"""The operators of a speculative decoding step on the GPU, against plain restatements in 64 bits on the host."""
import random

import pytest
import torch

from oracle import speculative as ref
from tests.util import assert_close_to_oracle, guard_alloc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def fa():
    from paper_2410_16663_b200 import binding
    return binding


def ints(x, dev=DEV):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def random_tree(T, rng, back=6):
    return [-1] + [rng.randrange(max(0, i - back), i) for i in range(1, T)]


def paged_copy(cache, lens, page, gen, extra=3, wide=0):
    """A contiguous host cache [B,S,H,d] as a pool whose pages are in a random order, and its table (unused entries -1)."""
    B, S, H, d = cache.shape
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + extra, generator=gen).tolist()
    pool = torch.full((len(order), page, H, d), float("nan"), dtype=cache.dtype)
    table = torch.full((B, max(need + [1]) + wide), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        for j in range(n):
            table[b, j] = order.pop()
            rows = cache[b, j * page:min((j + 1) * page, S)]
            pool[table[b, j], :rows.shape[0]] = rows
    return pool, table


def check_tree(fa, B, T, Hq, Hkv, d, dtype, lens, page=0, tree_lens=None, see=None, seed=0, shared=False, with_lse=True, smax=0,
               poison_hidden_keys=False, scale=None, wide=0):
    gen, rng = torch.Generator().manual_seed(seed), random.Random(seed)
    S = max(max(lens), T, smax, 1)
    q, k, v = (torch.randn(*s, generator=gen).to(dtype) for s in ((B, T, Hq, d), (B, S, Hkv, d), (B, S, Hkv, d)))
    if see is None:
        see = torch.stack([ref.ancestors(random_tree(T, rng)) for _ in range(1 if shared else B)])
    see_b = see.expand(B, T, T) if shared else see
    scale = d ** -0.5 if scale is None else scale
    live = [max(0, min(T if tree_lens is None else tree_lens[b], T, lens[b])) for b in range(B)]
    if poison_hidden_keys:      # nodes that nobody sees: their keys may be anything
        for b in range(B):
            for j in range(live[b]):
                if not see_b[b, :live[b], j].any():
                    k[b, lens[b] - live[b] + j] = float("nan")
    o_ref, l_ref = ref.tree_attention(q, k, v, lens, see_b, scale, tree_lens)
    absv = ref.tree_attention(q, k, v, lens, see_b, scale, tree_lens, abs_v=True)[0] if dtype == torch.bfloat16 else None
    for b in range(B):
        k[b, lens[b]:], v[b, lens[b]:] = float("nan"), float("nan")
        q[b, live[b]:] = float("nan")                 # queries of no node
    table = None
    if page:
        k, table = paged_copy(k, lens, page, torch.Generator().manual_seed(seed + 1), wide=wide)
        v, _ = paged_copy(v, lens, page, torch.Generator().manual_seed(seed + 1), wide=wide)
    words = ref.bits_to_words(see[0] if shared else see)
    dev = lambda x: None if x is None else x.to(DEV)
    o, check_o = guard_alloc((B, T, Hq, d), dtype, DEV)
    lse, check_l = guard_alloc((B, Hq, T), torch.float32, DEV) if with_lse else (None, lambda: None)
    tab = dev(table)
    skv = S if table is None else table.shape[1] * page
    for variant in (0, 1, 2):     # by the sizes, and each of the two kernels
        need = fa.fa_decode_tree_workspace_bytes(B, T, Hq, Hkv, skv, d, variant)
        ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device=DEV)
        o.fill_(float("nan"))
        fa.fa_decode_tree(dev(q), dev(k), dev(v), o, lse, ints(lens), dev(words), scale, ws[:need],
                          tree_lens=None if tree_lens is None else ints(tree_lens), block_table=tab, variant=variant)
        torch.cuda.synchronize()
        assert fa.fa_device_status()[0] == 0
        check_o(), check_l()
        assert (ws[need:] == 0xff).all(), "workspace overrun"
        assert_close_to_oracle(o, lse if with_lse else l_ref, o_ref, l_ref, stored_bf16=dtype == torch.bfloat16, p_absv=absv, what=f"variant {variant}")
        for b in range(B):
            assert not o[b, live[b]:].float().any()


HEADS = [(4, 4), (8, 2), (8, 1), (10, 2), (7, 1), (16, 2)]


@pytest.mark.parametrize("T", [1, 2, 3, 7, 16, 17, 31, 32, 33, 61, 64, 65])
@pytest.mark.parametrize("d,dtype", [(128, torch.float16), (64, torch.bfloat16)])
def test_tree_nodes_and_heads(fa, T, d, dtype):
    hq, hkv = HEADS[T % len(HEADS)]
    lens = [max(T, 300), T, T + 129]
    check_tree(fa, 3, T, hq, hkv, d, dtype, lens, seed=T)


@pytest.mark.parametrize("page", [0, 16, 32, 64, 128, 384])
@pytest.mark.parametrize("hq,hkv,T,d", [(4, 4, 12, 128), (12, 2, 20, 128), (8, 1, 40, 64), (8, 2, 5, 64)])
def test_tree_over_pages_and_tile_ends(fa, page, hq, hkv, T, d):
    # the tree's rows end before, at and behind the ends of tiles and pages, and lie across them
    lens = [T, T + 1, 127, 128, 129, 128 + T // 2, 255 + T, 256, 511, 640 + T]
    check_tree(fa, len(lens), T, hq, hkv, d, torch.float16, lens, page=page, seed=page + T, wide=2)


@pytest.mark.parametrize("g,T", [(1, 128), (1, 129), (2, 64), (4, 32), (3, 43), (4, 64), (5, 52), (8, 32), (8, 33), (16, 16), (16, 17),
                                 (1, 256), (1, 255), (3, 200), (130, 2), (300, 1)])
def test_tree_rows_per_kv_head(fa, g, T):
    # rows that share a kv head: below, at and above one and two tiles of 128
    lens = [T + 70, 500 + T]
    check_tree(fa, 2, T, 2 * g, 2, 128, torch.bfloat16 if g % 2 else torch.float16, lens, seed=g * 1000 + T)


def test_tree_lengths_that_do_not_fit(fa):
    # no keys, fewer keys than nodes, trees of no node, lengths past the cache
    check_tree(fa, 5, 9, 8, 2, 128, torch.float16, [0, 4, 200, 9, 1], tree_lens=[9, 9, 0, 12, 1], seed=3)
    check_tree(fa, 4, 40, 8, 2, 64, torch.bfloat16, [0, 17, 300, 40], tree_lens=[40, 40, -3, 40], seed=4)
    lens, mask = ints([100000, -5]), ref.bits_to_words(torch.ones(2, 4, 4, dtype=torch.bool)).to(DEV)
    q, k = torch.randn(2, 4, 4, 64, device=DEV).half(), torch.randn(2, 50, 4, 64, device=DEV).half()
    o, lse = torch.empty_like(q), torch.empty(2, 4, 4, device=DEV)
    o_ref, l_ref = ref.tree_attention(q.cpu(), k.cpu(), k.cpu(), [50, 0], torch.ones(2, 4, 4, dtype=torch.bool), 0.125)
    for variant in (1, 2):
        ws = torch.empty(fa.fa_decode_tree_workspace_bytes(2, 4, 4, 4, 50, 64, variant), dtype=torch.uint8, device=DEV)
        fa.fa_decode_tree(q, k, k, o, lse, lens, mask, 0.125, ws, variant=variant)
        assert_close_to_oracle(o, lse, o_ref, l_ref)


@pytest.mark.parametrize("T,hq,hkv", [(9, 4, 2), (50, 8, 2), (90, 8, 2)])
def test_tree_masks_that_are_none(fa, T, hq, hkv):
    gen = torch.Generator().manual_seed(5)
    see = torch.rand(4, T, T, generator=gen) < 0.3      # any bits, a node without its own among them
    see[0] = False                                      # nobody sees a node
    see[1, :, 1] = False                                # nobody sees node 1
    see[2, 3] = False                                   # row 3 sees the prefix alone
    check_tree(fa, 4, T, hq, hkv, 128, torch.float16, [T, 130 + T, T, 400], see=see, tree_lens=[T, T, T - 2, T - 1],
               poison_hidden_keys=True, seed=6)


@pytest.mark.parametrize("T", [6, 48])
def test_tree_shared_mask_no_lse_and_room_behind(fa, T):
    check_tree(fa, 3, T, 8, 2, 128, torch.bfloat16, [200, T, 333], shared=True, with_lse=False, smax=900, seed=8)


@pytest.mark.parametrize("T,B,smax,d", [(4, 1, 5000, 128), (30, 1, 5000, 128), (30, 6, 9000, 64), (64, 2, 9000, 128), (3, 40, 2500, 128), (33, 40, 1500, 128)])
def test_tree_over_long_caches(fa, T, B, smax, d):
    rng = random.Random(B)
    lens = [rng.randint(T, smax) for _ in range(B - 1)] + [smax]
    check_tree(fa, B, T, 8, 2, d, torch.float16, lens, seed=T + B)


def test_tree_scores_far_apart(fa):
    # scores of several hundred: the reference of the exponentials moves within a row, and most keys weigh nothing
    for T, seed in ((5, 1), (40, 2)):
        gen = torch.Generator().manual_seed(seed)
        q = (torch.randn(1, T, 4, 128, generator=gen) * 6).half()
        k, v = (torch.randn(1, 1200, 2, 128, generator=gen) * 4).half(), torch.randn(1, 1200, 2, 128, generator=gen).half()
        see = ref.ancestors(random_tree(T, random.Random(seed)))[None]
        o_ref, l_ref = ref.tree_attention(q, k, v, [1200], see, 0.3)
        for variant in (1, 2):
            o, lse = torch.empty_like(q, device=DEV), torch.empty(1, 4, T, device=DEV)
            ws = torch.empty(fa.fa_decode_tree_workspace_bytes(1, T, 4, 2, 1200, 128, variant), dtype=torch.uint8, device=DEV)
            fa.fa_decode_tree(q.to(DEV), k.to(DEV), v.to(DEV), o, lse, ints([1200]), ref.bits_to_words(see).to(DEV), 0.3, ws, variant=variant)
            assert_close_to_oracle(o, lse, o_ref, l_ref, stored_fp16_ulp=True)


def test_tree_of_a_chain_is_the_append(fa):
    # the same rows by fa_decode_ex: both against each other, within two roundings of the output and of the probabilities
    B, T, S = 3, 8, 700
    gen = torch.Generator(device=DEV).manual_seed(9)
    q, k, v = (torch.empty(*s, dtype=torch.float16, device=DEV).normal_(generator=gen) for s in ((B, T, 8, 128), (B, S, 2, 128), (B, S, 2, 128)))
    lens = ints([700, 8, 300])
    mask = ref.bits_to_words(torch.tril(torch.ones(T, T, dtype=torch.bool))).to(DEV)
    a, b = torch.empty_like(q), torch.empty_like(q)
    ws2 = torch.empty(fa.fa_decode_append_workspace_bytes(B, T, 8, 2, S, 128), dtype=torch.uint8, device=DEV)
    fa.fa_decode_ex(q, k, v, b, None, lens, 128 ** -0.5, ws2)
    for variant in (1, 2):
        ws = torch.empty(fa.fa_decode_tree_workspace_bytes(B, T, 8, 2, S, 128, variant), dtype=torch.uint8, device=DEV)
        fa.fa_decode_tree(q, k, v, a, None, lens, mask, 128 ** -0.5, ws, variant=variant)
        assert float((a.double() - b.double()).abs().max()) <= 4e-3


@pytest.mark.parametrize("T", [3, 40])
def test_tree_pages_past_32_bits(fa, T):
    # a pool of more than 2^31 elements, whose pages in use are its last ones
    if torch.cuda.mem_get_info()[0] < 24e9:
        pytest.skip("needs 24 GB")
    pages, page, H, d = 140000, 16, 8, 128
    pool_k = torch.empty(pages, page, H, d, dtype=torch.float16, device=DEV)
    pool_v = torch.empty(pages, page, H, d, dtype=torch.float16, device=DEV)
    gen = torch.Generator().manual_seed(11)
    n = 100
    ids = list(range(pages - 7, pages))
    k, v = torch.randn(7, page, H, d, generator=gen).half(), torch.randn(7, page, H, d, generator=gen).half()
    pool_k[pages - 7:], pool_v[pages - 7:] = k.to(DEV), v.to(DEV)
    q = torch.randn(1, T, 16, d, generator=gen).half()
    see = ref.ancestors(random_tree(T, random.Random(1)))[None]
    o_ref, l_ref = ref.tree_attention(q, k.reshape(1, -1, H, d), v.reshape(1, -1, H, d), [n], see, 0.1)
    for variant in (1, 2):
        o, lse = torch.empty_like(q, device=DEV), torch.empty(1, 16, T, device=DEV)
        ws = torch.empty(fa.fa_decode_tree_workspace_bytes(1, T, 16, H, 7 * page, d, variant), dtype=torch.uint8, device=DEV)
        fa.fa_decode_tree(q.to(DEV), pool_k, pool_v, o, lse, ints([n]), ref.bits_to_words(see).to(DEV), 0.1, ws, block_table=ints([ids]), variant=variant)
        assert_close_to_oracle(o, lse, o_ref, l_ref)


@pytest.mark.parametrize("T", [4, 40])
@pytest.mark.parametrize("page", [16, 128])
def test_tree_pages_that_are_none(fa, T, page):
    # table entries outside the pool read as zeros, whatever they are
    gen = torch.Generator().manual_seed(12)
    H, d, n = 2, 64, 4 * page
    k, v = torch.randn(4, page, H, d, generator=gen).half(), torch.randn(4, page, H, d, generator=gen).half()
    q = torch.randn(1, T, 8, d, generator=gen).half()
    see = ref.ancestors(random_tree(T, random.Random(2)))[None]
    for bad in (-1, 4, 1 << 30, -(1 << 31), (1 << 31) - 1, (1 << 28) + 1):
        kz, vz = k.clone(), v.clone()
        kz[1], vz[1] = 0, 0
        o_ref, l_ref = ref.tree_attention(q, kz.view(1, n, H, d), vz.view(1, n, H, d), [n], see, 0.125)
        for variant in (1, 2):
            o, lse = torch.empty_like(q, device=DEV), torch.empty(1, 8, T, device=DEV)
            ws = torch.empty(fa.fa_decode_tree_workspace_bytes(1, T, 8, H, n, d, variant), dtype=torch.uint8, device=DEV)
            fa.fa_decode_tree(q.to(DEV), k.to(DEV), v.to(DEV), o, lse, ints([n]), ref.bits_to_words(see).to(DEV), 0.125, ws,
                              block_table=ints([[0, bad, 2, 3]]), variant=variant)
            assert_close_to_oracle(o, lse, o_ref, l_ref)


@pytest.mark.parametrize("smax", [40, 127, 128, 129, 200, 1001])
def test_tree_at_the_end_of_the_caches(fa, smax):
    # the last sequence ends with the caches' last row; other rows of the allocation hold NaN
    for T, hq, hkv, d in ((20, 8, 1, 128), (33, 4, 4, 64), (40, 8, 1, 64)):
        B, gen = 2, torch.Generator().manual_seed(smax)
        lens = [max(T, smax // 2), smax]
        q = torch.randn(B, T, hq, d, generator=gen).half()
        k, check_k = guard_alloc((B, smax, hkv, d), torch.float16, DEV, pad=64 * hkv * d)
        v, check_v = guard_alloc((B, smax, hkv, d), torch.float16, DEV, pad=64 * hkv * d)
        k.copy_(torch.randn(k.shape, generator=gen)), v.copy_(torch.randn(v.shape, generator=gen))
        see = torch.stack([ref.ancestors(random_tree(T, random.Random(b))) for b in range(B)])
        o_ref, l_ref = ref.tree_attention(q, k.cpu(), v.cpu(), lens, see, 0.1)
        for variant in (1, 2):
            o, lse = torch.empty_like(q, device=DEV), torch.empty(B, hq, T, device=DEV)
            ws = torch.empty(fa.fa_decode_tree_workspace_bytes(B, T, hq, hkv, smax, d, variant), dtype=torch.uint8, device=DEV)
            fa.fa_decode_tree(q.to(DEV), k, v, o, lse, ints(lens), ref.bits_to_words(see).to(DEV), 0.1, ws, variant=variant)
            assert_close_to_oracle(o, lse, o_ref, l_ref)
        check_k(), check_v()


# ------------------------------------------------------------------ verification
def check_verify(fa, B, T, V, dtype, draft, seed, trees=None, live=None, p=None, q=None, tokens=None, u=None, noise=None):
    gen, rng = torch.Generator().manual_seed(seed), random.Random(seed)
    trees = trees or [random_tree(T, rng, back=4) for _ in range(B)]
    if p is None:
        logits = 2 * torch.randn(B, T, V, generator=gen)
        p = torch.softmax(logits, -1).to(dtype)
        q = torch.softmax(logits + 0.7 * torch.randn(B, T, V, generator=gen), -1).to(dtype)
    if tokens is None:
        up = torch.tensor(trees).clamp(min=0)
        rows = torch.gather(q.float(), 1, up[:, :, None].expand(B, T, V)).view(B * T, V)
        tokens = torch.multinomial(rows, 1, generator=gen).view(B, T)
    u = torch.rand(B, T, generator=gen) if u is None else u
    noise = torch.empty(B, V).exponential_(generator=gen).clamp_(min=1e-20) if noise is None else noise
    n, path, out = torch.full((B,), -9, dtype=torch.int32, device=DEV), *(torch.full((B, T), -9, dtype=torch.int32, device=DEV) for _ in range(2))
    fa.fa_spec_verify(p.to(DEV), q.to(DEV) if draft else None, tokens.to(torch.int32).to(DEV), ints(trees), u.to(DEV), noise.to(DEV), n, path, out,
                      tree_lens=None if live is None else ints(live))
    n, path, out = n.tolist(), path.tolist(), out.tolist()
    for b in range(B):
        t = T if live is None else max(1, min(live[b], T))
        want, said = ref.verify(p[b], q[b] if draft else None, tokens[b], trees[b], u[b], noise[b], t)
        assert n[b] == len(want) - 1, b
        assert path[b] == want + [-1] * (T - len(want)), b
        assert out[b] == said + [-1] * (T - len(said)), b
    return n, out


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (1, 5, 33), (7, 9, 1000), (3, 64, 1001), (2, 256, 130), (40, 6, 4100), (2, 17, 20002)])
def test_verify_trees(fa, B, T, V, dtype, draft):
    rng = random.Random(B + T)
    check_verify(fa, B, T, V, dtype, draft, seed=B * T + V)
    check_verify(fa, B, T, V, dtype, draft, seed=B * T + V + 1, live=[rng.randint(-1, T + 2) for _ in range(B)])
    check_verify(fa, B, T, V, dtype, draft, seed=B * T + V + 2, trees=[[-1] + list(range(T - 1))] * B)        # a chain


@pytest.mark.parametrize("draft", [True, False])
def test_verify_many_children(fa, draft):
    # every node a child of the root, tokens that come again: a residual for each rejection
    V, T, B = 37, 40, 20
    gen = torch.Generator().manual_seed(1)
    p = torch.softmax(torch.randn(B, T, V, generator=gen), -1)
    q = torch.softmax(torch.randn(B, T, V, generator=gen), -1)
    tokens = torch.multinomial(q[:, 0], T, replacement=True, generator=gen)
    check_verify(fa, B, T, V, torch.float32, draft, seed=2, trees=[[-1] + [0] * (T - 1)] * B, p=p, q=q, tokens=tokens,
                 u=torch.rand(B, T, generator=gen) * 0.3 + 0.7)


def test_verify_ends_of_the_range(fa):
    V, T = 8, 3
    one = torch.zeros(1, T, V)
    one[0, :, 5] = 1.0
    chain, even = [[-1, 0, 1]], torch.full((1, T, V), 1 / V)
    tok = torch.tensor([[0, 5, 5]])
    u = torch.tensor([[0.5, 0.999999, 0.999999]])
    # the draft is certain and right: all stand, the last token is the target's only one
    assert check_verify(fa, 1, T, V, torch.float32, True, 0, trees=chain, p=one, q=one, tokens=tok, u=u)[1] == [[5, 5, 5]]
    # the target has nothing where the draft was: never accepted, not even at u = 0
    assert check_verify(fa, 1, T, V, torch.float32, True, 0, trees=chain, p=one, q=even, tokens=torch.tensor([[0, 2, 2]]), u=u * 0)[0] == [0]
    # equal scores: the lowest token
    assert check_verify(fa, 1, T, V, torch.float32, False, 0, trees=chain, p=even, q=even, tokens=torch.tensor([[0, 9, 9]]), u=u,
                        noise=torch.ones(1, V))[1] == [[0, -1, -1]]
    # a residual without mass: the target's row takes its place; a row without mass: -1
    half = torch.zeros(1, T, V)
    half[0, :, 2:4] = 0.5
    assert check_verify(fa, 1, T, V, torch.float32, True, 0, trees=chain, p=half, q=2 * half, tokens=torch.tensor([[0, 6, 6]]), u=u,
                        noise=torch.ones(1, V))[1] == [[2, -1, -1]]
    assert check_verify(fa, 1, T, V, torch.float32, True, 0, trees=chain, p=0 * even, q=even, tokens=torch.tensor([[0, 6, 6]]), u=u)[1] == [[-1] * 3]
    # tokens and parents that are none; NaN in rows that are not read
    bad = torch.tensor([[0, -7, 1 << 30]])
    assert check_verify(fa, 1, T, V, torch.float32, True, 0, trees=chain, p=even, q=even, tokens=bad, u=u * 0)[0] == [0]
    nan = even.clone()
    nan[0, 1:] = float("nan")
    assert check_verify(fa, 1, T, V, torch.float32, True, 0, trees=chain, p=nan, q=even, tokens=torch.tensor([[0, 3, 3]]),
                        u=torch.tensor([[0.0, 1.0, 0.0]]), noise=torch.ones(1, V))[0] == [0]
    n, out, path = ints([7]), ints([[7] * T]), ints([[7] * T])
    fa.fa_spec_verify(even.to(DEV), even.to(DEV), ints([[0, 1, 1]]), ints([[-1, 5, -3]]), torch.zeros(1, T, device=DEV), torch.ones(1, V, device=DEV), n, path, out)
    assert n.tolist() == [0] and path.tolist() == [[0, -1, -1]] and out.tolist() == [[0, -1, -1]]


def test_verify_rows_that_are_not_aligned(fa):
    # the same numbers at a start that four entries at a time cannot be read from
    B, T, V = 2, 5, 4096
    gen = torch.Generator().manual_seed(7)
    p = torch.softmax(2 * torch.randn(B, T, V, generator=gen), -1)
    args = dict(tokens=torch.randint(0, V, (B, T), generator=gen).to(torch.int32).to(DEV), parents=ints([[-1, 0, 0, 1, 1]] * B),
                uniforms=torch.rand(B, T, generator=gen).to(DEV))
    noise = torch.empty(B, V).exponential_(generator=gen)
    got = []
    for off in (0, 1, 3):
        at = lambda x: torch.cat([torch.zeros(off, device=DEV), x.to(DEV).flatten()])[off:].view(x.shape)
        n, path, out = ints([0] * B), ints([[0] * T] * B), ints([[0] * T] * B)
        fa.fa_spec_verify(at(p), at(p.roll(1, 2)), noise=at(noise), n_accept=n, path=path, out_tokens=out, **args)
        got.append((n.tolist(), path.tolist(), out.tolist()))
    assert got[0] == got[1] == got[2]


# ------------------------------------------------------------------ the cache
@pytest.mark.parametrize("page", [0, 16, 64, 7])
@pytest.mark.parametrize("dtype,row", [(torch.float16, (2, 64)), (torch.uint8, (1, 48)), (torch.bfloat16, (8, 128)), (torch.float32, (1, 4))])
def test_compact(fa, page, dtype, row):
    gen, rng = torch.Generator().manual_seed(page), random.Random(page)
    B, T, L = 7, 40, 3
    lens = [0, 1, 40, 41, 99, 130, 75]
    tree = [T, T, T, T, 17, 30, 0]
    path = [[0] + sorted(rng.sample(range(1, T), T // 2)) + [-1] * (T - 1 - T // 2) for _ in range(B)]
    path[3] = list(range(T))                          # everything stands: nothing moves
    path[5][3] = 1000                                 # no node
    acc = [3, 0, T // 2, T - 1, 60, 9, 5]
    S = 140 if not page else -(-140 // page) * page
    k, v = (torch.randint(0, 250, (L, B, S, *row), generator=gen).to(dtype) for _ in range(2))
    table = None
    if page:
        n = S // page
        table = torch.randperm(B * n, generator=gen).view(B, n).to(torch.int32)
        k, v = (x.view(L, B * n, page, *row) for x in (k, v))
    kd, vd, new = k.to(DEV), v.to(DEV), torch.full((B,), -9, dtype=torch.int32, device=DEV)
    fa.fa_cache_compact(kd, vd, ints(lens), ints(path), ints(acc), new, tree_lens=ints(tree), block_table=None if table is None else table.to(DEV))
    want = ref.compact(k, v, lens, path, acc, tree, table, T)
    assert new.tolist() == want
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)


def test_compact_long_paths_and_strided_layers(fa):
    # a path of 200 nodes, 12 more than it needs to step over 8 at a time; layers that are not next to each other
    gen = torch.Generator().manual_seed(2)
    T, S = 256, 300
    pool = torch.randn(6, 2, 1, S, 2, 64, generator=gen).half()
    k, v = pool[:, 0].clone(), pool[:, 1].clone()
    path = [[0] + list(range(50, 250)) + [-1] * 55]
    both = pool.to(DEV)
    new = ints([0])
    fa.fa_cache_compact(both[:, 0], both[:, 1], ints([S]), ints(path), ints([200]), new)
    assert ref.compact(k, v, [S], path, [200], None, None, T) == new.tolist()
    assert torch.equal(both[:, 0].cpu(), k) and torch.equal(both[:, 1].cpu(), v)


def check_resize(fa, table, held, refs, want, page):
    t, h, r, s = ints(table), ints(held), ints(refs), ints([-9])
    fa.fa_pages_resize(t, h, r, ints(want), s, page)
    short = ref.pages_resize(table, held, refs, want, page)
    assert s.tolist() == [short]
    assert h.tolist() == held
    assert r.tolist() == refs
    assert t.tolist() == table
    return short


@pytest.mark.parametrize("num_pages", [1, 5, 37, 1024, 16384, 16385, 40000, 131072, 140001, 300000])
def test_resize_random_steps(fa, num_pages):
    rng = random.Random(num_pages)
    page, B = 16, min(64, num_pages)
    most = min(num_pages, 2 + 3 * num_pages // B)
    most = min(most, 4000)
    table, held, refs = [[-1] * most for _ in range(B)], [0] * B, [0] * num_pages
    for i in rng.sample(range(num_pages), num_pages // 7):
        refs[i] = rng.randint(1, 3)                   # pages that belong to others
    shorts = 0
    for step in range(6):
        want = [rng.choice([0, h * page, rng.randint(0, most * page), max(0, h * page - rng.randint(0, 99)), h * page + rng.randint(0, 40)])
                for h in held]
        shorts += check_resize(fa, table, held, refs, want, page)
    assert all(r >= 0 for r in refs)
    check_resize(fa, table, held, refs, [-1] * B, page)
    assert held == [0] * B


def test_resize_shortage_and_limits(fa):
    # what an earlier sequence asks for and does not get is not given to a later one; a table too narrow; pages given back in the same call
    table, held, refs = [[0, 1, -1, -1], [-1] * 4, [-1] * 4, [2, -1, -1, -1]], [2, 0, 0, 1], [1, 1, 1, 0, 0]
    assert check_resize(fa, table, held, refs, [0, 80, 16, 48], 16) == 1            # row 1 asks for five entries of four
    table, held, refs = [[0, -1, -1, -1], [-1] * 4, [-1] * 4], [1, 0, 0], [1, 0, 0, 0]
    assert check_resize(fa, table, held, refs, [16, 64, 16], 16) == 2
    table, held, refs = [[3, 1, 0, 2]], [4], [1, 2, 1, 1]
    assert check_resize(fa, table, held, refs, [0], 16) == 0 and refs == [0, 1, 0, 0]


def test_resize_many_sequences(fa):
    B = 4096
    rng = random.Random(0)
    table, held, refs = [[-1] * 4 for _ in range(B)], [0] * B, [0] * 9000
    check_resize(fa, table, held, refs, [rng.randint(0, 64) for _ in range(B)], 16)
    check_resize(fa, table, held, refs, [rng.randint(0, 64) for _ in range(B)], 16)


def test_resize_wants_past_32_bits(fa):
    # 4096 sequences that together want 2^31 - 2 to some more than 2^31 pages, of a pool of 3000: the first two have what they want,
    # nobody else gets or is said to hold a page
    if torch.cuda.mem_get_info()[0] < 24e9:
        pytest.skip("needs 24 GB")
    B, most, num_pages = 4096, (1 << 19) + 1024, 3000
    table = torch.full((B, most), -1, dtype=torch.int32, device=DEV)
    held, refs, short = ints([0] * B), ints([0] * num_pages), ints([-9])
    for total in ((1 << 31) - 2, (1 << 31) - 1, 1 << 31, (B - 2) * most + 1200):
        left, want = total - 1200, [1000, 200]
        for i in range(2, B):
            want.append(min(most, left - (B - 1 - i)))           # (everybody wants a page)
            left -= want[-1]
        assert sum(want) == total and min(want) > 0
        fa.fa_pages_resize(table, held, refs, ints(want), short, 1)
        assert short.tolist() == [B - 2]
        assert held.tolist() == [1000, 200] + [0] * (B - 2)
        assert table[0, :1000].tolist() == list(range(1000)) and table[1, :200].tolist() == list(range(1000, 1200))
        assert int((table >= 0).sum()) == 1200 and refs.tolist() == [1] * 1200 + [0] * 1800
        fa.fa_pages_resize(table, held, refs, ints([0] * B), short, 1)
        assert short.tolist() == [0] and not refs.any()


@pytest.mark.parametrize("page,num_pages,n", [(16, 60, 9), (1, 400, 5), (64, 17000, 3), (7, 13, 12), (128, 30, 1), (16, 150000, 40)])
def test_fork(fa, page, num_pages, n):
    gen, rng = torch.Generator().manual_seed(page), random.Random(page)
    L, row = (2, (2, 64)) if num_pages < 1000 else (1, (1, 8))
    S = max(1, n // 3)
    most = max(2, min(num_pages // (S + 1), 6))
    lens = [rng.randint(0, most * page) for _ in range(S)] + [0] * n
    lens[0] = most * page - (page > 1)
    order = rng.sample(range(num_pages), num_pages)
    table, held, refs = [[-1] * most for _ in lens], [0] * len(lens), [0] * num_pages
    for b in range(S):
        held[b] = -(-lens[b] // page)
        for e in range(held[b]):
            table[b][e] = order.pop()
            refs[table[b][e]] = 1
    src, dst = [rng.randrange(S) for _ in range(n)], [S + i for i in range(n)]
    src[0] = 0
    k, v = (torch.randn(L, num_pages, page, *row, generator=gen).half() for _ in range(2))
    kd, vd, t, h, ln, r, s = k.to(DEV), v.to(DEV), ints(table), ints(held), ints(lens), ints(refs), ints([-9])
    fa.fa_pages_fork(kd, vd, t, h, ln, r, ints(src), ints(dst), s)
    short = ref.pages_fork(k, v, table, held, lens, refs, src, dst, page)
    assert s.tolist() == [short]
    assert (t.tolist(), h.tolist(), ln.tolist(), r.tolist()) == (table, held, lens, refs)
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)
    # the new sequences end again: the pages of the first are as before
    fa.fa_pages_resize(t, h, r, ints([x if i < S else 0 for i, x in enumerate(lens)]), s, page)
    ref.pages_resize(table, held, refs, [x if i < S else 0 for i, x in enumerate(lens)], page)
    assert (t.tolist(), h.tolist(), r.tolist()) == (table, held, refs)


def test_fork_without_pages_and_bad_pairs(fa):
    page, L = 16, 1
    k, v = torch.randn(L, 3, page, 1, 64).half(), torch.randn(L, 3, page, 1, 64).half()
    table, held, lens, refs = [[0, 1], [-1, -1], [-1, -1], [-1, -1]], [2, 0, 0, 0], [20, 0, 0, 0], [1, 1, 0]
    kd, vd, t, h, ln, r, s = k.to(DEV), v.to(DEV), ints(table), ints(held), ints(lens), ints(refs), ints([-9])
    src, dst = [0, 9, 0, 0, -1], [1, 2, 4, 3, 2]
    fa.fa_pages_fork(kd, vd, t, h, ln, r, ints(src), ints(dst), s)
    assert ref.pages_fork(k, v, table, held, lens, refs, src, dst, page) == 1 and s.tolist() == [1]
    assert (t.tolist(), h.tolist(), ln.tolist(), r.tolist()) == (table, held, lens, refs)
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)


# ------------------------------------------------------------------ streams and graphs
def test_a_step_in_a_graph_and_on_a_side_stream(fa):
    """Reserve, attend, verify, compact, give back: captured once, replayed with other lengths, trees and numbers; each replay
    against the same calls on a side stream behind a long kernel, which in turn are what the tests above compare."""
    B, T, Hq, Hkv, d, page, V, L = 3, 6, 8, 2, 64, 16, 500, 2
    num_pages, most = 80, 16
    gen = torch.Generator(device=DEV).manual_seed(3)
    new = lambda *s, dt=torch.float16: torch.empty(*s, dtype=dt, device=DEV).normal_(generator=gen)
    st = dict(k=new(L, num_pages, page, Hkv, d), v=new(L, num_pages, page, Hkv, d), q=new(B, T, Hq, d), p=torch.softmax(2 * new(B, T, V, dt=torch.float32), -1),
              table=ints([[-1] * most] * B), held=ints([0] * B), refs=ints([0] * num_pages), want=ints([40, 70, 20]), lens=ints([40, 70, 20]),
              mask=ints([[[1 << i | 1] for i in range(T)]] * B), tokens=ints([[0, 3, 4, 5, 6, 7]] * B), parents=ints([[-1, 0, 0, 0, 0, 0]] * B),
              u=torch.rand(B, T, device=DEV, generator=gen), noise=torch.empty(B, V, device=DEV).exponential_(generator=gen))
    names = ("o", "lse", "n", "path", "out", "new_lens", "short")

    def step(x, y):
        fa.fa_pages_resize(x["table"], x["held"], x["refs"], x["want"], y["short"], page)
        fa.fa_decode_tree(x["q"], x["k"][1], x["v"][1], y["o"], y["lse"], x["lens"], x["mask"], 0.125, y["ws"], block_table=x["table"])
        fa.fa_spec_verify(x["p"], None, x["tokens"], x["parents"], x["u"], x["noise"], y["n"], y["path"], y["out"])
        fa.fa_cache_compact(x["k"], x["v"], x["lens"], y["path"], y["n"], y["new_lens"], block_table=x["table"])
        fa.fa_pages_resize(x["table"], x["held"], x["refs"], y["new_lens"], y["short"], page)

    def outputs():
        return dict(o=torch.zeros(B, T, Hq, d, dtype=torch.float16, device=DEV), lse=torch.zeros(B, Hq, T, device=DEV), n=ints([0] * B),
                    path=ints([[0] * T] * B), out=ints([[0] * T] * B), new_lens=ints([0] * B), short=ints([0]),
                    ws=torch.zeros(fa.fa_decode_tree_workspace_bytes(B, T, Hq, Hkv, most * page, d), dtype=torch.uint8, device=DEV))

    copy = lambda x: {n: t.clone() for n, t in x.items()}
    first, y = copy(st), outputs()
    step(copy(st), outputs())                        # (one call outside of the capture: kernels are set up once)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(first, y)
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=DEV)
    for lens in ([40, 70, 20], [100, 6, 33], [7, 200, 64]):
        st["lens"].copy_(ints(lens)), st["want"].copy_(ints(lens))
        st["u"].uniform_(generator=gen), st["q"].normal_(generator=gen)
        for n, t in first.items():
            t.copy_(st[n])
        graph.replay()
        z, second = outputs(), None
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(3):
                big = torch.tanh(big @ big)
            second = copy(st)                        # (made on the side stream, behind the products)
            step(second, z)
        side.synchronize()
        assert all(torch.equal(y[n], z[n]) for n in names)
        assert all(torch.equal(first[n], second[n]) for n in ("table", "held", "refs", "k", "v"))
        assert z["new_lens"].tolist() == [a - T + 1 + b for a, b in zip(lens, z["n"].tolist())] and z["short"].tolist() == [0]
    assert fa.fa_device_status()[0] == 0


def test_steps_of_a_serving_loop(fa):
    """The example's loop: forked sequences decode some steps; the pages' counts, tables and lengths agree with one another at the end,
    and the cache holds the rows of exactly the tokens that stand, with the attention's own inputs written again."""
    from paper_2410_16663_b200 import speculate
    samples, prompt, nodes, steps, page = 5, 333, 13, 4, 16
    said, cache = speculate.run(samples, prompt, nodes, steps, layers=2, vocab=512, page=page)
    torch.cuda.synchronize()
    assert fa.fa_device_status()[0] == 0 and int(cache.short) == 0
    lens, held, table, refs = (t.tolist() for t in (cache.lens, cache.held, cache.table, cache.refs))
    gained = [sum(1 + int(n[b]) for _, n in said) for b in range(samples)]
    assert lens == [prompt + g for g in gained]
    assert held == [-(-x // page) for x in lens]
    count = [0] * len(refs)
    for b in range(samples):
        assert all(e >= 0 for e in table[b][:held[b]]) and all(e == -1 for e in table[b][held[b]:])
        for e in table[b][:held[b]]:
            count[e] += 1
    assert count == refs and max(refs) == samples and sum(r == samples for r in refs) == prompt // page
    for out, n in said:
        for b in range(samples):
            k = int(n[b])
            assert (out[b, :k + 1] >= 0).all() and (out[b, k + 1:] == -1).all()
    # layer 0's keys depend on the tokens alone: the last token's row of every step stands first in its tree, the accepted ones follow
    gen = torch.Generator(device=DEV)
    gen.manual_seed(0)
    model = speculate.Model(2, 8, 2, 128, 512, torch.bfloat16, DEV, gen)
    for b in range(samples):
        tokens = []
        for i, (out, n) in enumerate(said):
            k = int(n[b])
            first = int(said[i - 1][0][b, int(said[i - 1][1][b])]) if i else None
            tokens += [first] + out[b, :k].tolist()
        rows = torch.arange(prompt, lens[b], device=DEV)
        got = cache.k[0, cache.table[b, rows // page].long(), rows % page]
        known = [i for i, t in enumerate(tokens) if t is not None]
        x = model.embed[torch.tensor([tokens[i] for i in known], device=DEV)][None]
        want = model.project(x, 0)[1][0]
        assert torch.allclose(got[known].float(), want.float(), rtol=2e-2, atol=2e-2)


def test_steps_of_a_serving_loop_that_rejects_and_moves(fa, monkeypatch):
    """The example's loop once more, with what its calls decided: drafts are rejected and stand, accepted rows move, every sequence says
    several tokens, and layer 0's keys and values are those of the tokens that stand."""
    from paper_2410_16663_b200 import speculate
    log, compact = [], fa.fa_cache_compact

    def logged(k, v, lens, path, n, new, **kw):
        log.append((path.clone(), n.clone()))
        return compact(k, v, lens, path, n, new, **kw)

    monkeypatch.setattr(fa, "fa_cache_compact", logged)
    samples, prompt, nodes, steps, page = 5, 333, 13, 6, 16
    said, cache = speculate.run(samples, prompt, nodes, steps, layers=2, vocab=512, page=page, seed=1)
    assert fa.fa_device_status()[0] == 0 and int(cache.short) == 0
    accepted = torch.stack([n for _, n in log])
    assert (accepted == 0).any() and (accepted >= 2).any()
    assert sum(int(path[b, i]) > i for path, n in log for b in range(samples) for i in range(1, int(n[b]) + 1)) >= 10
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    model = speculate.Model(2, 8, 2, 128, 512, torch.bfloat16, DEV, gen)
    for b in range(samples):
        tokens = []
        for i, (out, n) in enumerate(said):
            tokens += [int(said[i - 1][0][b, int(said[i - 1][1][b])]) if i else -1] + out[b, :int(n[b])].tolist()
        assert len(set(tokens)) >= 5
        rows = torch.arange(prompt + 1, int(cache.lens[b]), device=DEV)
        x = model.embed[torch.tensor(tokens[1:], device=DEV)][None]
        for pool, part in ((cache.k, 1), (cache.v, 2)):
            got = pool[0, cache.table[b, rows // page].long(), rows % page]
            assert torch.allclose(got.float(), model.project(x, 0)[part][0].float(), rtol=2e-2, atol=2e-2)
