"""The serving loop of speculate.py on the host: its calls of the library are answered by the restatements in 64 bits."""
import random

import pytest
import torch

from oracle import speculative as ref


class Library:
    """The calls that the loop makes, on host tensors; ``log`` keeps (path, n_accept) of every step."""

    def __init__(self):
        self.log = []

    def fa_pages_resize(self, table, held, refs, want, short, page):
        t, h, r = table.tolist(), held.tolist(), refs.tolist()
        short.fill_(ref.pages_resize(t, h, r, want.tolist(), page))
        for x, y in ((table, t), (held, h), (refs, r)):
            x.copy_(torch.tensor(y, dtype=torch.int32))

    def fa_pages_fork(self, k, v, table, held, lens, refs, src, dst, short):
        t, h, n, r = table.tolist(), held.tolist(), lens.tolist(), refs.tolist()
        short.fill_(ref.pages_fork(k, v, t, h, n, r, src.tolist(), dst.tolist(), k.shape[2]))
        for x, y in ((table, t), (held, h), (lens, n), (refs, r)):
            x.copy_(torch.tensor(y, dtype=torch.int32))

    def tree_mask(self, parents):
        return torch.stack([ref.bits_to_words(ref.ancestors(p)) for p in parents.tolist()])

    def fa_decode_tree_workspace_bytes(self, *sizes):
        return 16

    def fa_decode_tree(self, q, k, v, o, lse, lens, mask, scale, ws, tree_lens=None, block_table=None):
        T = q.shape[1]
        see = torch.stack([(mask[..., j // 32] >> (j % 32) & 1).bool() for j in range(T)], -1)
        o.copy_(ref.tree_attention(q, k, v, lens.tolist(), see, scale, None if tree_lens is None else tree_lens.tolist(), block_table)[0])

    def fa_spec_verify(self, p, q, tokens, parents, u, noise, n, path, out, tree_lens=None):
        B, T = tokens.shape
        for b in range(B):
            live = T if tree_lens is None else max(1, min(int(tree_lens[b]), T))
            nodes, said = ref.verify(p[b], q[b], tokens[b], parents[b], u[b], noise[b], live)
            n[b] = len(nodes) - 1
            path[b], out[b] = -1, -1
            path[b, :len(nodes)], out[b, :len(said)] = torch.tensor(nodes), torch.tensor(said)
        self.log.append((path.clone(), n.clone()))

    def fa_cache_compact(self, k, v, lens, path, n, new, tree_lens=None, block_table=None):
        new.copy_(torch.tensor(ref.compact(k, v, lens.tolist(), path, n.tolist(), None if tree_lens is None else tree_lens.tolist(), block_table,
                                           path.shape[1])))


@pytest.fixture
def loop(monkeypatch):
    from paper_2410_16663_b200 import build
    build.build()
    from paper_2410_16663_b200 import speculate
    monkeypatch.setattr(speculate, "fa", Library())
    return speculate


def state(cache):
    return [t.clone() for t in (cache.k, cache.v, cache.table, cache.held, cache.lens, cache.refs)]


@pytest.mark.parametrize("pages,served", [(6, []), (7, [0]), (8, [0, 1]), (9, [0, 1, 2])])
def test_a_sequence_without_room_sits_the_step_out(loop, pages, served):
    """Three sequences of 20 rows on two 16-row pages each, and too few pages for a tree of 13 in each.  Nothing of another sequence's
    is written, who was not served keeps rows and pages and says nothing, and the shortage is counted."""
    B, T, page, V = 3, 13, 16, 40
    gen = torch.Generator().manual_seed(1)
    cache = loop.PagedCache(2, pages, page, 2, 8, B, 64, torch.float32, "cpu")
    model = loop.Model(2, 4, 2, 8, V, torch.float32, "cpu", gen)
    cache.resize(torch.tensor([20] * B, dtype=torch.int32))
    cache.lens = torch.tensor([20] * B, dtype=torch.int32)
    cache.k.normal_(generator=gen), cache.v.normal_(generator=gen)
    before = state(cache)
    rng = random.Random(0)
    parents = torch.tensor([[-1] + [rng.randrange(max(0, i - 3), i) for i in range(1, T)] for _ in range(B)], dtype=torch.int32)
    tokens = torch.randint(0, V, (B, T), generator=gen).to(torch.int32)
    draft = torch.full((B, T, V), 1.0 / V)
    out, n, _ = loop.step(model, cache, tokens, parents, draft, gen, None)
    assert int(cache.short) == B - len(served)
    for b in range(B):
        if b in served:
            assert int(cache.lens[b]) == 20 + 1 + int(n[b]) and (out[b, :int(n[b]) + 1] >= 0).all() and (out[b, int(n[b]) + 1:] == -1).all()
            # the token that stood, and the accepted ones: their rows, behind the twenty
            said = tokens[b, :1].tolist() + out[b, :int(n[b])].tolist()
            want = model.project(model.embed[torch.tensor(said)][None], 0)[1][0]
            got = ref.gather_rows(cache.k[0], cache.table, b, int(cache.lens[b]))[20:]
            assert torch.allclose(got, want, rtol=1e-4, atol=1e-4)
        else:
            assert int(cache.lens[b]) == 20 and int(n[b]) == 0 and (out[b] == -1).all()
            assert torch.equal(cache.table[b], before[2][b]) and int(cache.held[b]) == 2
        for layer in range(2):      # nobody's twenty rows changed
            for x, y in ((cache.k, before[0]), (cache.v, before[1])):
                assert torch.equal(ref.gather_rows(x[layer], cache.table, b, 20), ref.gather_rows(y[layer], before[2], b, 20))
    assert cache.held.tolist() == [-(-int(x) // page) for x in cache.lens] and int(cache.refs.sum()) == int(cache.held.sum())
    # the next step's shortage is counted on top, and what the call that gives back reports does not take it away
    cache.reserve(1000)
    assert int(cache.short) == B - len(served) + B


def test_a_loop_of_a_pool_that_is_too_small(loop):
    """Steps go on where some sequences are not served: the lengths are those of the tokens that were said."""
    gen = torch.Generator().manual_seed(2)
    B, T, page, V = 4, 6, 4, 30
    cache = loop.PagedCache(1, 13, page, 1, 8, B, 60, torch.float32, "cpu")
    model = loop.Model(1, 2, 1, 8, V, torch.float32, "cpu", gen)
    cache.resize(torch.tensor([5] * B, dtype=torch.int32))
    cache.lens = torch.tensor([5] * B, dtype=torch.int32)
    said = [0] * B
    for _ in range(5):
        tokens = torch.randint(0, V, (B, T), generator=gen).to(torch.int32)
        out, n, _ = loop.step(model, cache, tokens, loop.random_trees(B, T, gen, "cpu"), torch.full((B, T, V), 1.0 / V), gen, None)
        said = [s + int((o >= 0).sum()) for s, o in zip(said, out)]
    assert cache.lens.tolist() == [5 + s for s in said] and max(said) >= 5 and int(cache.short) > 0
    assert int(cache.refs.max()) == 1 and int(cache.refs.sum()) == int(cache.held.sum())


# ------------------------------------------------------------------ what the example's check of its cache can see
SAMPLES, PROMPT, NODES, STEPS, PAGE = 5, 41, 13, 5, 16


def run_and_check(loop, check):
    said, cache = loop.run(SAMPLES, PROMPT, NODES, STEPS, layers=2, Hq=4, Hkv=2, d=16, vocab=64, page=PAGE, dtype=torch.float32, device="cpu")
    model = loop.Model(2, 4, 2, 16, 64, torch.float32, "cpu", torch.Generator().manual_seed(0))
    return said, cache, check(said, cache, model, PROMPT)


def rows_that_differ(said, cache, model, prompt):
    """Rows of layer 0's keys, which depend on the tokens alone, that are not those of the tokens that stand."""
    bad = 0
    for b in range(len(said[0][1])):
        tokens = []
        for i, (out, n) in enumerate(said):
            tokens += [int(said[i - 1][0][b, int(said[i - 1][1][b])]) if i else None] + out[b, :int(n[b])].tolist()
        known = [i for i, t in enumerate(tokens) if t is not None]
        got = ref.gather_rows(cache.k[0], cache.table, b, int(cache.lens[b]))[prompt:]
        assert len(got) == len(tokens)
        want = model.project(model.embed[torch.tensor([tokens[i] for i in known])][None], 0)[1][0]
        bad += int(((got[known] - want).abs().amax((1, 2)) > 1e-3).sum())
    return bad


def test_the_loop_accepts_rejects_and_moves(loop):
    """A loop whose every token is the same, or whose drafts all stand, would show nothing of verification and compaction."""
    said, cache, bad = run_and_check(loop, rows_that_differ)
    assert bad == 0 and int(cache.short) == 0
    lib = loop.fa
    accepted = torch.stack([n for _, n in lib.log])
    assert (accepted == 0).any() and (accepted >= 2).any() and 0.3 < float(accepted.float().mean()) < NODES / 2
    moved = sum(int(path[b, i]) > i for path, n in lib.log for b in range(SAMPLES) for i in range(1, int(n[b]) + 1))
    assert moved >= 10
    for b in range(SAMPLES):
        assert len({t for out, n in said for t in out[b, :int(n[b]) + 1].tolist()}) >= 5


@pytest.mark.parametrize("mistake", ["nothing moves", "the next row", "a path backwards"])
def test_the_check_of_the_cache_sees_a_compaction_that_is_wrong(loop, monkeypatch, mistake):
    right = ref.compact

    def wrong(k, v, lens, path, n, tree_lens=None, table=None, T=None):
        if mistake == "nothing moves":
            return right(k.clone(), v.clone(), lens, path, n, tree_lens, table, T)
        if mistake == "the next row":
            return right(k, v, lens, [[min(int(x) + (i > 0), T - 1) for i, x in enumerate(row)] for row in path], n, tree_lens, table, T)
        return right(k, v, lens, [[int(row[0])] + [int(x) for x in row[1:1 + int(m)]][::-1] + [-1] * (T - 1 - int(m)) for row, m in zip(path, n)], n, tree_lens, table, T)

    monkeypatch.setattr(ref, "compact", wrong)
    assert run_and_check(loop, rows_that_differ)[2] > 0


def test_the_example_model_is_not_certain(loop):
    """At the sizes of the GPU test: what follows a token is spread over several, and another for another token."""
    gen = torch.Generator().manual_seed(0)
    model = loop.Model(2, 8, 2, 128, 512, torch.bfloat16, "cpu", gen)
    p = model.probabilities(model.embed[torch.arange(64)])
    assert float(p.amax(-1).mean()) < 0.6 and float((p * p).sum(-1).reciprocal().mean()) > 3
    assert int((p.argmax(-1) == torch.arange(64)).sum()) <= 4 and p.argmax(-1).unique().numel() > 30
