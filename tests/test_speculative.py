"""The operators of a speculative decoding step on the host: the argument checks of the C entry points (which come before any
CUDA call), the binding's own, and the pins of the oracle that the GPU tests compare with."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from oracle import speculative as ref


@pytest.fixture(scope="module")
def fa():
    from paper_2410_16663_b200 import build
    build.build()
    from paper_2410_16663_b200 import binding
    return binding


def tree_params(fa, **kw):
    buf = torch.zeros(1 << 16, dtype=torch.float16)
    at = (buf.data_ptr() + 15) & ~15
    p = fa.fa_tree_params()
    p.q = p.k = p.v = p.o = p.seqlens_k = p.mask = p.workspace = at
    p.B, p.T, p.Hq, p.Hkv, p.Skv_max, p.d, p.dtype, p.scale = 2, 4, 4, 2, 256, 128, fa.FA_DTYPE_FP16, 0.1
    p.mask_stride, p.workspace_bytes = 4, 1 << 30
    for name, value in kw.items():
        setattr(p, name, at + value[1] if isinstance(value, tuple) else value)
    p._keep = buf
    return p


def test_tree_attention_refuses_bad_arguments(fa):
    call = lambda **kw: fa.lib.fa_decode_tree(ctypes.byref(tree_params(fa, **kw)), None)
    assert fa.lib.fa_decode_tree(None, None) == fa.FA_ERR_NULL
    assert call(B=0) == fa.FA_OK
    for kw in (dict(B=-1), dict(T=0), dict(T=-3), dict(Hq=5), dict(Hkv=0), dict(Skv_max=-1), dict(mask_stride=-4), dict(d=0)):
        assert call(**kw) == fa.FA_ERR_SHAPE, kw
    for kw in (dict(T=257), dict(T=200, Skv_max=199), dict(d=256), dict(d=96), dict(dtype=fa.FA_DTYPE_FP32), dict(scale=-0.1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(B=65536), dict(Hq=70000, Hkv=1), dict(variant=3), dict(variant=-1)):
        assert call(**kw) == fa.FA_ERR_UNSUPPORTED, kw
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(mask=None), dict(seqlens_k=None)):
        assert call(**kw) == fa.FA_ERR_NULL, kw
    for kw in (dict(q=("at", 2)), dict(k=("at", 8)), dict(v=("at", 8)), dict(o=("at", 4)), dict(workspace=("at", 4)), dict(mask=("at", 2)),
               dict(tree_lens=("at", 1)), dict(lse=("at", 2)), dict(seqlens_k=("at", 2))):
        assert call(**kw) == fa.FA_ERR_ALIGN, kw
    need = fa.fa_decode_tree_workspace_bytes(2, 4, 4, 2, 256, 128)
    assert need > 0 and fa.fa_decode_tree_workspace_bytes(2, 4, 4, 2, 256, 96) == 0 and fa.fa_decode_tree_workspace_bytes(2, 0, 4, 2, 256, 128) == 0
    assert call(workspace_bytes=need - 1) == fa.FA_ERR_WORKSPACE and call(workspace=None) == fa.FA_ERR_WORKSPACE
    for d in (128, 64):
        more = fa.fa_decode_tree_workspace_bytes(2, 40, 4, 2, 256, d, 2)
        assert more > 0 and call(T=40, d=d, variant=2, workspace_bytes=more - 1) == fa.FA_ERR_WORKSPACE
        assert fa.fa_decode_tree_workspace_bytes(64, 64, 32, 8, 8192, d) == fa.fa_decode_tree_workspace_bytes(64, 64, 32, 8, 8192, d, 2)
    paged = dict(block_table=("at", 0), num_pages=8, page_size=64, max_pages=4, table_stride=4)
    for kw in (dict(page_size=48), dict(page_size=0), dict(table_stride=3), dict(num_pages=-1), dict(num_pages=0),
               dict(max_pages=1 << 26, table_stride=1 << 26)):
        assert call(**{**paged, **kw}) == fa.FA_ERR_SHAPE, kw
    assert call(**{**paged, "block_table": ("at", 2)}) == fa.FA_ERR_ALIGN
    assert call(**{**paged, "max_pages": 0}) == fa.FA_ERR_UNSUPPORTED        # no room for the tree's own rows


def test_verification_refuses_bad_arguments(fa):
    buf = torch.zeros(4096, dtype=torch.float32)
    at = (buf.data_ptr() + 15) & ~15
    names = ["p", "q", "tokens", "parents", "tree_lens", "u", "noise", "n_accept", "path", "out"]

    def call(**kw):
        a = dict(dict.fromkeys(names, at), B=1, T=2, V=8, dtype=fa.FA_DTYPE_FP32)
        a.update(kw)
        return fa.lib.fa_spec_verify(*[a[n] for n in names], a["B"], a["T"], a["V"], a["dtype"], None)

    assert call(B=0) == fa.FA_OK
    for kw in (dict(B=-1), dict(T=0), dict(V=0)):
        assert call(**kw) == fa.FA_ERR_SHAPE, kw
    for kw in (dict(T=257), dict(V=(1 << 30) + 1), dict(B=65536), dict(dtype=3), dict(dtype=-1)):
        assert call(**kw) == fa.FA_ERR_UNSUPPORTED, kw
    for n in names:
        if n not in ("q", "tree_lens"):
            assert call(**{n: None}) == fa.FA_ERR_NULL, n
        assert call(**{n: at + 2}) == fa.FA_ERR_ALIGN, n
    assert call(p=at + 1, dtype=fa.FA_DTYPE_BF16) == fa.FA_ERR_ALIGN


def test_cache_operators_refuse_bad_arguments(fa):
    buf = torch.zeros(4096, dtype=torch.float32)
    at = (buf.data_ptr() + 15) & ~15

    def compact(**kw):
        a = dict(k=at, v=at, table=None, lens=at, tree_lens=None, path=at, n=at, new=at, L=1, ls=0, B=1, T=2, S=8, np=0, ps=0, mp=0, ts=0, row=256)
        a.update(kw)
        return fa.lib.fa_cache_compact(*a.values(), None)

    assert compact(B=0) == fa.FA_OK
    paged = dict(table=at, np=4, ps=16, mp=2, ts=2)
    for kw in (dict(B=-1), dict(T=0), dict(L=-1), dict(row=0), dict(ls=-16), dict(S=-1), {**paged, "ps": 0}, {**paged, "ts": 1},
               {**paged, "np": -1}, {**paged, "mp": 1 << 28, "ts": 1 << 28}):
        assert compact(**kw) == fa.FA_ERR_SHAPE, kw
    assert compact(B=65536) == fa.FA_ERR_UNSUPPORTED
    for n in ("k", "v", "lens", "path", "n", "new"):
        assert compact(**{n: None}) == fa.FA_ERR_NULL, n
    for kw in (dict(row=24), dict(ls=8), dict(k=at + 8), dict(v=at + 4), dict(path=at + 2), dict(new=at + 1), dict(tree_lens=at + 2),
               {**paged, "table": at + 2}):
        assert compact(**kw) == fa.FA_ERR_ALIGN, kw

    def resize(**kw):
        a = dict(table=at, held=at, refs=at, want=at, short=at, B=1, np=8, ps=16, mp=2, ts=2)
        a.update(kw)
        return fa.lib.fa_pages_resize(*a.values(), None)

    assert resize(B=0) == fa.FA_OK
    for kw in (dict(B=-1), dict(np=-1), dict(ps=0), dict(mp=-1), dict(ts=1)):
        assert resize(**kw) == fa.FA_ERR_SHAPE, kw
    assert resize(B=4097) == fa.FA_ERR_UNSUPPORTED
    for n in ("table", "held", "refs", "want", "short"):
        assert resize(**{n: None}) == fa.FA_ERR_NULL and resize(**{n: at + 2}) == fa.FA_ERR_ALIGN, n

    def fork(**kw):
        a = dict(k=at, v=at, table=at, held=at, lens=at, refs=at, src=at, dst=at, short=at, n=1, L=1, ls=0, B=2, np=8, ps=16, mp=2, ts=2, row=256)
        a.update(kw)
        return fa.lib.fa_pages_fork(*a.values(), None)

    assert fork(n=0) == fa.FA_OK
    for kw in (dict(n=-1), dict(B=-1), dict(L=-1), dict(ls=-16), dict(np=-1), dict(ps=0), dict(mp=-1), dict(ts=1), dict(row=0),
               dict(mp=1 << 28, ts=1 << 28)):
        assert fork(**kw) == fa.FA_ERR_SHAPE, kw
    for kw in (dict(n=4097), dict(L=32768)):
        assert fork(**kw) == fa.FA_ERR_UNSUPPORTED, kw
    for n in ("k", "v", "table", "held", "lens", "refs", "src", "dst", "short"):
        assert fork(**{n: None}) == fa.FA_ERR_NULL, n
    for kw in (dict(row=40), dict(ls=8), dict(k=at + 8), dict(v=at + 8), dict(src=at + 2), dict(lens=at + 1), dict(table=at + 2)):
        assert fork(**kw) == fa.FA_ERR_ALIGN, kw


def test_binding_refuses_what_the_library_cannot_see(fa):
    q = torch.zeros(1, 2, 4, 128, dtype=torch.float16)
    k = torch.zeros(1, 64, 2, 128, dtype=torch.float16)
    lens, mask = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, 1, dtype=torch.int32)
    ok = dict(q=q, k=k, v=k, o=q, lse=None, seqlens_k=lens, mask=mask, scale=0.1, workspace=None)
    for kw in (dict(mask=mask.long()), dict(mask=torch.zeros(1, 2, 2, dtype=torch.int32)), dict(mask=torch.zeros(3, 1, dtype=torch.int32)),
               dict(k=k.float()), dict(o=q.float()), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(seqlens_k=lens.long())):
        with pytest.raises(ValueError):
            fa.fa_decode_tree(**{**ok, **kw})
    p = torch.zeros(1, 2, 8)
    ints, f = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, 2)
    base = [p, p, ints, ints, f, torch.zeros(1, 8), torch.zeros(1, dtype=torch.int32), ints, ints]
    for i, bad in ((0, p.double()), (1, p.half()), (2, ints.long()), (4, f.double()), (5, torch.zeros(8, 2).T[:1]), (7, ints.long())):
        args = list(base)
        args[i] = bad
        with pytest.raises(ValueError):
            fa.fa_spec_verify(*args)
    kk = torch.zeros(2, 4, 16, 2, 64)
    i1 = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        fa.fa_cache_compact(kk, kk.half(), i1, ints, i1, i1)
    with pytest.raises(ValueError):
        fa.fa_pages_fork(kk, kk, ints, i1, i1, torch.zeros(5, dtype=torch.int32), i1, i1, i1)
    with pytest.raises(ValueError):
        fa.fa_pages_resize(ints, i1, torch.zeros(8, dtype=torch.int32)[::2], i1, i1, 16)


def test_oracle_verification_draws_from_the_target():
    """Whatever the draft proposes, the first emitted token is distributed as the target's first row: 6000 trees with two children
    each over a vocabulary of 5; a frequency of probability p is within 5 sqrt(p (1 - p) / n) of it."""
    gen = torch.Generator().manual_seed(3)
    n, V = 6000, 5
    p = torch.softmax(torch.randn(3, V, generator=gen), -1)
    for with_q in (True, False):
        q = torch.softmax(torch.randn(3, V, generator=gen), -1)
        count = torch.zeros(V, dtype=torch.float64)
        for _ in range(n):
            tokens = [0] + (torch.multinomial(q[0], 2, replacement=True, generator=gen).tolist() if with_q else [1, 3])
            u = torch.rand(3, generator=gen)
            noise = torch.empty(V).exponential_(generator=gen)
            _, out = ref.verify(p, q if with_q else None, tokens, [-1, 0, 0], u, noise, 3)
            count[out[0]] += 1
        pd = p[0].double()
        assert ((count / n - pd).abs() <= 5 * (pd * (1 - pd) / n).sqrt()).all(), (with_q, count / n, pd)


def test_oracle_tree_attention_of_a_chain_is_causal():
    import oracle
    gen = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(1, s, h, 64, generator=gen, dtype=torch.float64).half() for s, h in ((6, 4), (19, 2), (19, 2)))
    see = ref.ancestors([-1, 0, 1, 2, 3, 4])[None]
    o, lse = ref.tree_attention(q, k, v, [19], see, 0.125)
    o2, l2 = oracle.attention_full(q, k, v, True, 0.125)
    assert float((o - o2).abs().max()) < 1e-12 and float((lse - l2).abs().max()) < 1e-12


def test_words_of_a_mask():
    see = torch.zeros(1, 40, dtype=torch.bool)
    see[0, [0, 31, 32, 39]] = True
    assert ref.bits_to_words(see).tolist() == [[1 - (1 << 31), 1 + (1 << 7)]]


def test_compaction_refuses_new_lengths_among_its_inputs(fa):
    """new_lens[b] is written while other CTAs may still have to read b's length, tree, path and table entries: in place, rows would
    move at a wrong prefix.  Next to them it may lie (what is behind the check, the device, then answers)."""
    B, T, pages = 3, 4, 2
    buf = torch.zeros(4096, dtype=torch.int32)
    at = (buf.data_ptr() + 15) & ~15
    words = lambda i: at + 4 * i
    a = dict(k=at, v=at, table=None, lens=words(100), tree_lens=words(200), path=words(300), n=words(400), new=words(500), L=1, ls=0, B=B, T=T, S=8,
             np=4, ps=16, mp=pages, ts=pages + 3, row=256)
    call = lambda **kw: fa.lib.fa_cache_compact(*{**a, **kw}.values(), None)
    if torch.cuda.is_available():
        pytest.skip("a device would take host pointers")
    free = call()
    assert free in (fa.FA_ERR_DEVICE, fa.FA_ERR_CUDA)
    for name, n in (("lens", B), ("tree_lens", B), ("n", B), ("path", B * T)):
        for new in (a[name], a[name] + 4 * (n - 1), a[name] - 4 * (B - 1)):
            assert call(new=new) == fa.FA_ERR_UNSUPPORTED, name
        for new in (a[name] + 4 * n, a[name] - 4 * B):
            assert call(new=new) == free, name
    table = words(600)
    end = table + 4 * ((B - 1) * (pages + 3) + pages)
    assert call(table=table, new=end - 4) == fa.FA_ERR_UNSUPPORTED and call(table=table, new=end) == free
    assert call(tree_lens=None) == free


def test_pages_refuse_a_pool_past_their_sums(fa):
    buf = torch.zeros(64, dtype=torch.int32)
    at = (buf.data_ptr() + 15) & ~15
    assert fa.lib.fa_pages_resize(at, at, at, at, at, 1, (1 << 31) - 1, 16, 2, 2, None) == fa.FA_ERR_UNSUPPORTED
    assert fa.lib.fa_pages_fork(at, at, at, at, at, at, at, at, at, 1, 1, 0, 2, (1 << 31) - 1, 16, 2, 2, 256, None) == fa.FA_ERR_UNSUPPORTED


def test_tree_workspace_of_heads_that_do_not_divide(fa):
    """Sizes that the call refuses need no workspace, and asking for it ends in an answer (in a process of its own: fewer query heads
    than kv heads would be a division by zero)."""
    ask = "from paper_2410_16663_b200 import binding as fa\nprint([fa.fa_decode_tree_workspace_bytes(1, 4, hq, hkv, 256, 128, v) " \
          "for hq, hkv in ((2, 4), (5, 2), (1 << 30, 1)) for v in (0, 1, 2)])"
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", ask], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, (out.returncode, out.stderr[-500:])
    assert out.stdout.split() == str([0] * 9).split()


def test_mask_of_parents_that_are_none(fa):
    """Entries past a tree's length may hold anything: no index outside the tree is followed, nor a node that comes later."""
    for T in (1, 5, 33, 70):
        parents = [-1] + [(i - 1) // 2 for i in range(1, T)]
        assert torch.equal(fa.tree_mask(torch.tensor(parents, dtype=torch.int32)), ref.bits_to_words(ref.ancestors(parents)))
        for none in (T, T - 1, T + 7, (1 << 31) - 1, -(1 << 31), -2):
            odd = parents[:T // 2] + [none] * (T - T // 2)
            clean = parents[:T // 2] + [none if 0 <= none < i else -1 for i in range(T // 2, T)]
            want = ref.bits_to_words(ref.ancestors(clean))
            assert torch.equal(fa.tree_mask(torch.tensor(odd, dtype=torch.int32)), want)
            assert torch.equal(fa.tree_mask(torch.tensor([parents, odd], dtype=torch.int32))[1], want)


class Recorder:
    """Takes the place of the library: what the binding passes on."""

    def __getattr__(self, name):
        def call(*args):
            self.last = (name, args)
            return 0
        return call


@pytest.fixture
def calls(fa, monkeypatch):
    recorder = Recorder()
    monkeypatch.setattr(fa, "lib", recorder)
    monkeypatch.setattr(fa, "_stream", lambda: 0)
    return recorder


def refused(call, right, **wrong):
    """``right`` goes through; every replacement of one argument is refused before anything is passed on."""
    call(**right)
    for name, values in wrong.items():
        for value in values:
            with pytest.raises(ValueError):
                call(**{**right, name: value})


def test_binding_refuses_sizes_that_do_not_go_together(fa, calls):
    """A tensor that is smaller than the call takes it for would be read or written past its end."""
    half, i32, f32 = (lambda *s, t=t: torch.zeros(*s, dtype=t) for t in (torch.float16, torch.int32, torch.float32))
    B, T, Hq, Hkv, d, S = 3, 5, 4, 2, 64, 20
    tree = dict(q=half(B, T, Hq, d), k=half(B, S, Hkv, d), v=half(B, S, Hkv, d), o=half(B, T, Hq, d), lse=f32(B, Hq, T), seqlens_k=i32(B),
                mask=i32(B, T, 1), scale=0.1, workspace=None, tree_lens=i32(B))
    refused(fa.fa_decode_tree, tree, k=[half(B, S, Hkv, 128), half(B, S + 1, Hkv, d)], v=[half(B, S, Hkv, 128), half(B, S, 1, d), half(B - 1, S, Hkv, d)],
            o=[half(B, T, Hq, 128), half(B, T - 1, Hq, d)], lse=[f32(B, Hq, T - 1)], seqlens_k=[i32(B - 1)], tree_lens=[i32(1)])
    few = {**tree, "k": half(B - 1, S, Hkv, d), "v": half(B - 1, S, Hkv, d)}        # fewer caches than sequences
    with pytest.raises(ValueError):
        fa.fa_decode_tree(**few)
    paged = {**few, "block_table": i32(B, 2)}
    refused(fa.fa_decode_tree, paged, block_table=[i32(B - 1, 2)])
    fa.fa_decode_tree(**{**tree, "seqlens_k": i32(B + 4), "tree_lens": None, "lse": None})          # vectors may be longer
    p = f32(B, T, 9)
    verify = dict(target_probs=p, draft_probs=p, tokens=i32(B, T), parents=i32(B, T), uniforms=f32(B, T), noise=f32(B, 9), n_accept=i32(B), path=i32(B, T),
                  out_tokens=i32(B, T), tree_lens=i32(B))
    less = [i32(B, T - 1), i32(B - 1, T), i32(B, T + 1)]
    refused(fa.fa_spec_verify, verify, draft_probs=[f32(B, T, 8), f32(B, T - 1, 9), f32(1, T, 9)], tokens=less, parents=less, path=less, out_tokens=less,
            uniforms=[f32(B, T - 1)], noise=[f32(B, 8), f32(1, 9)], n_accept=[i32(B - 1)], tree_lens=[i32(B - 1)])
    kv = half(2, B, S, Hkv, d)
    compact = dict(k=kv, v=kv, seqlens_k=i32(B), path=i32(B, T), n_accept=i32(B), new_lens=i32(B), tree_lens=i32(B))
    refused(fa.fa_cache_compact, compact, path=[i32(B + 1, T)], seqlens_k=[i32(B - 1)], n_accept=[i32(B - 1)], new_lens=[i32(B - 1)], tree_lens=[i32(B - 1)],
            block_table=[i32(B - 1, 2)])
    refused(fa.fa_pages_resize, dict(block_table=i32(B, 4), held=i32(B), refs=i32(7), want=i32(B), n_short=i32(1), page_size=16), held=[i32(B - 1)],
            want=[i32(B - 1)], n_short=[i32(0)])
    refused(fa.fa_pages_fork, dict(k=kv, v=kv, block_table=i32(4, 4), held=i32(4), seqlens_k=i32(4), refs=i32(B), src=i32(2), dst=i32(2), n_short=i32(1)),
            held=[i32(3)], seqlens_k=[i32(3)], src=[i32(1)], dst=[i32(1)], n_short=[i32(0)], refs=[i32(B + 1)])


def test_binding_reads_no_stride_of_an_extent_of_one(fa, calls):
    """torch calls a tensor contiguous whatever the strides of its extents of 1 are: a page of one row, one layer."""
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    B, T = 2, 3
    for k, layer, row in ((torch.zeros(3, 2, 7, 2, 64).half(), 7 * 2 * 2 * 64 * 2, 256), (torch.zeros(1, 3, 7, 2, 64).half().movedim(0, 2), 7 * 2 * 64 * 2, 256),
                          (torch.zeros(2, 5, 2, 64).half().as_strided((1, 2, 5, 2, 64), (3, 640, 128, 64, 1)), 0, 256)):
        fa.fa_cache_compact(k, k, i32(B), i32(B, T), i32(B), i32(B), block_table=i32(B, 4))
        name, args = calls.last
        assert name == "fa_cache_compact" and (args[8], args[9], args[17]) == (k.shape[0], layer, row)
        fa.fa_pages_fork(k, k, i32(B, 4), i32(B), i32(B), i32(k.shape[1]), i32(1), i32(1), i32(1))
        name, args = calls.last
        assert name == "fa_pages_fork" and (args[10], args[11], args[17]) == (k.shape[0], layer, row)


def test_nobody_is_short_where_there_is_nothing_to_do(fa, monkeypatch):
    """An empty batch and an empty list of pairs: the count of an earlier call does not stand (the library itself leaves it, and says so)."""
    monkeypatch.setattr(fa, "_stream", lambda: 0)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    short, kv = i32(1) + 7, torch.zeros(1, 3, 16, 1, 64).half()
    assert fa.lib.fa_pages_resize(None, None, None, None, short.data_ptr(), 0, 3, 16, 2, 2, None) == fa.FA_OK and short.tolist() == [7]
    assert fa.fa_pages_resize(i32(0, 2), i32(0), i32(3), i32(0), short, 16) == fa.FA_OK and short.tolist() == [0]
    short += 7
    assert fa.fa_pages_fork(kv, kv, i32(2, 2), i32(2), i32(2), i32(3), i32(0), i32(0), short) == fa.FA_OK and short.tolist() == [0]


@pytest.mark.parametrize("d,B,T,hq,hkv,keys,kernel", [
    # one cluster per row block
    (128, 1, 8, 32, 8, 512, 1), (128, 1, 32, 32, 8, 2048, 1), (128, 2, 6, 32, 8, 5133, 1), (128, 1, 26, 32, 8, 3235, 2), (128, 1, 16, 32, 8, 8192, 2),
    # whole sequences per CTA, two row blocks and more
    (128, 16, 8, 32, 8, 512, 1), (128, 16, 8, 32, 8, 812, 1), (128, 16, 6, 32, 8, 1543, 2), (128, 64, 8, 32, 8, 512, 2), (128, 6, 20, 32, 8, 250, 1),
    (128, 8, 20, 32, 8, 153, 2), (128, 8, 32, 32, 8, 236, 2),
    # cut into chunks that are merged
    (128, 1, 40, 32, 8, 349, 1), (128, 4, 16, 32, 8, 512, 2), (128, 4, 32, 32, 8, 512, 2), (128, 2, 40, 64, 8, 289, 2), (128, 8, 8, 32, 2, 989, 2),
    # 16 rows per kv head: one row block
    (128, 64, 4, 32, 8, 2048, 1), (64, 64, 4, 32, 8, 2048, 1),
    (64, 2, 6, 32, 8, 34601, 1), (64, 4, 5, 32, 8, 31842, 2), (64, 64, 5, 32, 8, 1161, 1), (64, 12, 6, 32, 8, 1601, 1), (64, 12, 6, 32, 8, 4560, 2),
    (64, 3, 10, 32, 8, 8707, 1), (64, 6, 10, 32, 8, 9403, 2), (64, 32, 10, 32, 8, 1151, 1), (64, 16, 10, 32, 8, 3711, 2),
    (64, 4, 16, 32, 8, 2048, 1), (64, 1, 32, 32, 8, 6183, 1), (64, 3, 20, 32, 8, 4995, 2), (64, 8, 40, 32, 8, 208, 1), (64, 16, 48, 32, 8, 247, 2),
    (64, 2, 40, 32, 8, 279, 1), (64, 4, 32, 32, 8, 512, 2), (64, 3, 61, 40, 5, 7951, 2), (64, 3, 80, 32, 8, 837, 2)])
def test_the_tree_kernel_is_the_faster_one_where_both_were_timed(fa, d, B, T, hq, hkv, keys, kernel):
    """The default's choice, seen by the workspace that it asks for, at sizes on both sides of each line that the rule's comment gives times for."""
    sizes = [fa.fa_decode_tree_workspace_bytes(B, T, hq, hkv, keys, d, variant) for variant in (0, 1, 2)]
    assert sizes[1] != sizes[2] and sizes[0] == sizes[kernel]
