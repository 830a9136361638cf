"""The many-rows kernel of the tree attention, whose CTAs share items and pass on a table of what to merge: every relation of items to
CTAs, calls one after the other without the host in between, and replays of a captured call with other lengths."""
import random

import pytest
import torch

from oracle import speculative as ref
from tests.test_speculative_gpu import ints, paged_copy, random_tree
from tests.util import assert_close_to_oracle, guard_alloc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def fa():
    from paper_2410_16663_b200 import binding
    return binding


def ctas(d):
    """Of a launch: two to an SM with d = 64."""
    return torch.cuda.get_device_properties(0).multi_processor_count * (2 if d == 64 else 1)


class Case:
    """Inputs of a call, on the device with NaN wherever nothing may be read, and what it has to give."""

    def __init__(self, B, T, Hq, Hkv, d, dtype, lens, page=0, tree_lens=None, seed=0):
        gen, rng = torch.Generator().manual_seed(seed), random.Random(seed)
        S = max(max(lens), T, 1)
        q, k, v = (torch.randn(*s, generator=gen).to(dtype) for s in ((B, T, Hq, d), (B, S, Hkv, d), (B, S, Hkv, d)))
        see = torch.stack([ref.ancestors(random_tree(T, rng)) for _ in range(B)])
        self.sizes, self.scale, self.dtype = (B, T, Hq, Hkv, d), d ** -0.5, dtype
        self.live = [max(0, min(T if tree_lens is None else tree_lens[b], T, lens[b])) for b in range(B)]
        self.o_ref, self.l_ref = ref.tree_attention(q, k, v, lens, see, self.scale, tree_lens)
        self.absv = ref.tree_attention(q, k, v, lens, see, self.scale, tree_lens, abs_v=True)[0] if dtype == torch.bfloat16 else None
        for b in range(B):
            k[b, lens[b]:], v[b, lens[b]:], q[b, self.live[b]:] = float("nan"), float("nan"), float("nan")
        table = None
        if page:
            k, table = paged_copy(k, lens, page, torch.Generator().manual_seed(seed + 1))
            v, _ = paged_copy(v, lens, page, torch.Generator().manual_seed(seed + 1))
        dev = lambda x: None if x is None else x.to(DEV)
        self.q, self.k, self.v, self.table, self.mask = dev(q), dev(k), dev(v), dev(table), dev(ref.bits_to_words(see))
        self.lens, self.trees = ints(lens), None if tree_lens is None else ints(tree_lens)
        self.keys = S if table is None else table.shape[1] * page

    def workspace(self, fa, variant):
        B, T, Hq, Hkv, d = self.sizes
        return torch.full((fa.fa_decode_tree_workspace_bytes(B, T, Hq, Hkv, self.keys, d, variant),), 0xff, dtype=torch.uint8, device=DEV)

    def call(self, fa, o, lse, ws, variant, q=None):
        fa.fa_decode_tree(self.q if q is None else q, self.k, self.v, o, lse, self.lens, self.mask, self.scale, ws, tree_lens=self.trees,
                          block_table=self.table, variant=variant)

    def check(self, fa, variants=(0, 1, 2)):
        B, T, Hq, Hkv, d = self.sizes
        for variant in variants:
            o, check_o = guard_alloc((B, T, Hq, d), self.dtype, DEV)     # (NaN: what is not written is seen, in both)
            lse, check_l = guard_alloc((B, Hq, T), torch.float32, DEV)
            ws, again = self.workspace(fa, variant), (torch.empty_like(o), torch.empty_like(lse))
            self.call(fa, o, lse, ws, variant)
            self.call(fa, *again, ws, variant)                           # the same workspace, as the first call left it
            torch.cuda.synchronize()
            assert fa.fa_device_status()[0] == 0
            check_o(), check_l()
            assert_close_to_oracle(o, lse, self.o_ref, self.l_ref, stored_bf16=self.dtype == torch.bfloat16, p_absv=self.absv, what=f"variant {variant}")
            assert torch.equal(o, again[0]) and torch.equal(lse, again[1]), f"variant {variant}: another result"
            for b in range(B):
                assert not o[b, self.live[b]:].float().any() and torch.isneginf(lse[b, :, self.live[b]:]).all()


def some_lengths(n, T, most, seed):
    """Lengths of n sequences: empty ones, the tree alone, ends of tiles, and anything up to ``most``."""
    rng = random.Random(seed)
    lens = [rng.choice([0, 1, T, T + 1, 127, 128, 129, most, rng.randint(T, most), rng.randint(T, most), rng.randint(T, most)]) for _ in range(n)]
    return [max(0, min(x, most)) for x in lens[:-1]] + [most]


@pytest.mark.parametrize("d,dtype,B,hq,hkv,T,most,page", [
    (128, torch.float16, 24, 16, 8, 40, 700, 0),      # one row tile
    (128, torch.bfloat16, 40, 32, 8, 40, 500, 16),    # two row tiles
    (128, torch.float16, 20, 32, 8, 80, 400, 128),    # two blocks of them
    (64, torch.bfloat16, 40, 8, 8, 20, 700, 0),
    (64, torch.float16, 33, 16, 8, 80, 500, 64),      # two blocks of one row tile
    (128, torch.float16, 64, 16, 16, 8, 128, 0),      # more items per CTA than there are segments between its warps
    (128, torch.bfloat16, 70, 32, 16, 70, 128, 16),
    (64, torch.float16, 100, 16, 16, 8, 128, 32),
])
def test_more_items_than_ctas(fa, d, dtype, B, hq, hkv, T, most, page):
    rows = hq // hkv * T
    assert B * hkv * -(-rows // (128 if d == 64 else 256)) >= ctas(d)
    lens = some_lengths(B, T, most, seed=B + T)
    trees = None if T % 3 else [random.Random(b).randint(-1, T + 2) for b in range(B)]
    Case(B, T, hq, hkv, d, dtype, lens, page, trees, seed=B * T).check(fa, (0, 2))


@pytest.mark.parametrize("more", [-1, 0, 1])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("T", [20, 130])
def test_as_many_items_as_ctas(fa, d, more, T):
    """One item less than CTAs, which are merged by item, as many, and one more, merged by CTA: of equal lengths, where items and runs
    of tiles end together, and of different ones."""
    B = ctas(d) + more
    if T > 128 and d == 64:
        B = (ctas(d) + 1) // 2 + more                # (two blocks of rows)
    for lens in ([200] * B, some_lengths(B, T, 400, seed=B), [max(T, 300)] + [0] * (B - 1), [0] * (B - 1) + [max(T, 700)]):
        Case(B, T, 1, 1, d, torch.float16, lens, seed=T + B).check(fa, (2,))


@pytest.mark.parametrize("d,g,hkv,T", [(128, 64, 2, 1), (128, 64, 2, 4), (128, 64, 1, 5), (128, 64, 2, 9), (128, 128, 1, 1), (128, 128, 2, 2), (128, 128, 1, 3),
                                       (128, 128, 1, 5), (128, 32, 2, 8), (128, 32, 1, 9), (64, 64, 2, 2), (64, 64, 1, 3), (64, 64, 2, 5), (64, 128, 1, 1),
                                       (64, 128, 1, 4), (64, 32, 2, 4), (64, 32, 1, 9)])
def test_a_tile_of_few_whole_nodes(fa, d, g, hkv, T):
    """32 and more query heads per kv head: a tile of 128 rows is four nodes and fewer, and blocks of rows are whole nodes."""
    lens = [T, T + 127, 300, 0, 1000]
    Case(len(lens), T, g * hkv, hkv, d, torch.float16 if T % 2 else torch.bfloat16, lens, seed=g + T).check(fa)


@pytest.mark.parametrize("d,dtype,B,hq,hkv,T,lens,page", [
    (128, torch.float16, 3, 8, 2, 7, [300, 7, 136], 0), (64, torch.bfloat16, 3, 4, 4, 33, [300, 33, 162], 0), (128, torch.bfloat16, 2, 8, 1, 64, [2500, 70], 16),
    (64, torch.float16, 2, 8, 1, 64, [2500, 70], 64), (128, torch.float16, 2, 3, 1, 200, [900, 270], 0), (128, torch.float16, 1, 4, 2, 30, [5000], 0)])
def test_every_kernel_writes_its_own_log_sums(fa, d, dtype, B, hq, hkv, T, lens, page):
    Case(B, T, hq, hkv, d, dtype, lens, page, seed=T).check(fa)


GRAPHS = [(128, 6, 8, 2, 40, 1500, 16), (128, 40, 8, 4, 40, 300, 0), (128, 3, 32, 8, 64, 900, 128), (64, 5, 16, 2, 33, 1200, 64), (64, 40, 8, 8, 20, 260, 16)]


@pytest.mark.parametrize("d,B,hq,hkv,T,most,page", GRAPHS)
def test_calls_that_feed_one_another(fa, d, B, hq, hkv, T, most, page):
    """Three calls of the many-rows kernel on one workspace, each with the outputs of the one before as its queries, and one of another size
    between them that leaves its own parts and table there: captured and replayed with other lengths and queries, on a side stream behind a
    backlog, and one by one with the host waiting and a new workspace each time.  All the same to the last bit."""
    case = Case(B, T, hq, hkv, d, torch.float16, some_lengths(B, T, most, seed=1), page, seed=d + B)
    other = Case(2, 24, 4 * hkv, hkv, d, torch.float16, [500, 333], 0, seed=9)
    case.q.nan_to_num_()                             # (rows of no node: their outputs are zeros and are the next call's queries)
    if not page:
        case.k.nan_to_num_(), case.v.nan_to_num_()   # (lengths change)
    names = ("q", "lens", "mask")
    first = {n: getattr(case, n).clone() for n in names}

    def chain(outs, lses, ws):
        q = case.q
        for i, (o, lse) in enumerate(zip(outs, lses)):
            case.call(fa, o, lse, ws if ws is not None else case.workspace(fa, 2), 2, q)
            if ws is None:
                torch.cuda.synchronize()
            if i == 1:
                other.call(fa, outs[-1].new_empty(other.q.shape) if ws is None else spare[0], None, other.workspace(fa, 2) if ws is None else ws, 2)
                if ws is None:
                    torch.cuda.synchronize()
            q = o

    def outputs():
        nan = lambda *s, dt: torch.full(s, float("nan"), dtype=dt, device=DEV)
        return [nan(*case.q.shape, dt=torch.float16) for _ in range(3)], [nan(B, hq, T, dt=torch.float32) for _ in range(3)]

    spare = [torch.empty_like(other.q)]
    need = max(case.workspace(fa, 2).numel(), other.workspace(fa, 2).numel())
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
    captured = outputs()
    chain(*outputs(), ws)                            # (one call outside of the capture: kernels are set up once)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(*captured, ws)
    side, gen = torch.cuda.Stream(), torch.Generator(device=DEV).manual_seed(3)
    big = torch.randn(4096, 4096, device=DEV) / 64
    held = first["lens"].tolist()
    for turn in range(4):
        if turn:                                     # other lengths (of a table: no more than has pages), queries and masks
            rng = random.Random(turn)
            lens = [rng.choice([0, 1, x // 2, x, rng.randint(0, x)]) if turn < 3 else x for x in held]
            case.lens.copy_(ints(lens))
            case.q.normal_(generator=gen)
            case.mask.copy_(first["mask"].roll(turn, 0))
        for x in captured[0] + captured[1]:
            x.fill_(float("nan"))
        for _ in range(5):
            big = torch.tanh(big @ big)
        graph.replay()
        behind, alone = outputs(), outputs()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(5):
                big = torch.tanh(big @ big)
            chain(*behind, ws)
        side.synchronize()
        chain(*alone, None)
        for a, b, c in zip(*(x[0] + x[1] for x in (captured, behind, alone))):
            assert torch.equal(a, c) and torch.equal(b, c) and not torch.isnan(c).any()
        if turn == 0:
            dead = [b for b in range(B) if case.live[b] < T]
            ok = [b for b in range(B) if b not in dead]
            assert_close_to_oracle(alone[0][0][ok], alone[1][0][ok], case.o_ref[ok], case.l_ref[ok])
    assert fa.fa_device_status()[0] == 0
