"""Rotation and cache appends: what the calls refuse, on the CPU, and the plan of the angles."""
import ctypes
import math
from fractions import Fraction

import pytest
import torch

from paper_2410_16663_b200 import binding as fa

PI = Fraction(3141592653589793238462643383279502884197, 10 ** 39)
A = 1 << 12   # an aligned address that nothing is read from


def rope_args(**kw):
    a = dict(x=A, out=A, positions=A, turns=A, n=4, H=2, d=128, rot=128, offset=0, inter=0, factor=1.0, xt=256, xh=128, ot=256, oh=128,
             dtype=fa.FA_DTYPE_FP16)
    a.update(kw)
    return [a[k] for k in ("x", "out", "positions", "turns", "n", "H", "d", "rot", "offset", "inter", "factor", "xt", "xh", "ot", "oh", "dtype")]


@pytest.mark.parametrize("change, code", [
    (dict(n=-1), fa.FA_ERR_SHAPE), (dict(H=0), fa.FA_ERR_SHAPE), (dict(d=0), fa.FA_ERR_SHAPE), (dict(rot=-16), fa.FA_ERR_SHAPE),
    (dict(offset=8), fa.FA_ERR_SHAPE), (dict(rot=64, offset=-8), fa.FA_ERR_SHAPE), (dict(xt=-8), fa.FA_ERR_SHAPE), (dict(xt=4), fa.FA_ERR_SHAPE),
    (dict(oh=1), fa.FA_ERR_SHAPE), (dict(d=120, rot=64), fa.FA_ERR_UNSUPPORTED), (dict(d=2048), fa.FA_ERR_UNSUPPORTED),
    (dict(d=1024, rot=528), fa.FA_ERR_UNSUPPORTED), (dict(rot=24), fa.FA_ERR_UNSUPPORTED), (dict(rot=64, offset=4), fa.FA_ERR_UNSUPPORTED),
    (dict(dtype=2), fa.FA_ERR_UNSUPPORTED), (dict(factor=math.inf), fa.FA_ERR_UNSUPPORTED), (dict(factor=math.nan), fa.FA_ERR_UNSUPPORTED),
    (dict(H=1 << 20), fa.FA_ERR_UNSUPPORTED), (dict(x=0), fa.FA_ERR_NULL), (dict(out=0), fa.FA_ERR_NULL), (dict(positions=0), fa.FA_ERR_NULL),
    (dict(turns=0), fa.FA_ERR_NULL), (dict(x=A + 8), fa.FA_ERR_ALIGN), (dict(turns=A + 4), fa.FA_ERR_ALIGN), (dict(positions=A + 2), fa.FA_ERR_ALIGN),
    (dict(n=0, x=0), fa.FA_OK)])
def test_rope_refusals(change, code):
    assert fa.lib.fa_rope(*rope_args(**change), None) == code


def append_params(**kw):
    p = fa.fa_append_params()
    base = dict(q=A, q_out=A, k=A, v=A, k_cache=A, v_cache=A, turns=A, positions=0, first_rows=A, counts=0, cu_seqlens=0, block_table=0, n=4, B=2,
                T=2, Hq=4, Hkv=2, d=128, dv=128, rot_dim=128, rot_offset=0, interleaved=0, dtype=0, cache_dtype=0, Skv_max=64, num_pages=0,
                page_size=0, max_pages=0, table_stride=0, factor=1.0, k_scale=1.0, v_scale=1.0, q_stride=(512, 128), q_out_stride=(512, 128),
                k_stride=(256, 128), v_stride=(256, 128), k_cache_stride=(64 * 256, 256), v_cache_stride=(64 * 256, 256))
    base.update(kw)
    for name, x in base.items():
        if isinstance(x, tuple):
            for i in range(2):
                getattr(p, name)[i] = x[i]
        else:
            setattr(p, name, x)
    return p


@pytest.mark.parametrize("change, code", [
    (dict(n=-1), fa.FA_ERR_SHAPE), (dict(n=5), fa.FA_ERR_SHAPE), (dict(B=-1), fa.FA_ERR_SHAPE), (dict(Hkv=0), fa.FA_ERR_SHAPE), (dict(Hq=0), fa.FA_ERR_SHAPE),
    (dict(dv=0), fa.FA_ERR_SHAPE), (dict(rot_offset=16), fa.FA_ERR_SHAPE), (dict(Skv_max=-1), fa.FA_ERR_SHAPE),
    (dict(k_stride=(12, 128)), fa.FA_ERR_SHAPE), (dict(k_cache_stride=(64 * 256, 252)), fa.FA_ERR_SHAPE), (dict(v_cache_stride=(-8, 256)), fa.FA_ERR_SHAPE),
    (dict(cache_dtype=3, k_cache_stride=(64 * 256, 264)), fa.FA_ERR_SHAPE),
    (dict(block_table=A, num_pages=4, page_size=0, max_pages=2, table_stride=2), fa.FA_ERR_SHAPE),
    (dict(block_table=A, num_pages=4, page_size=16, max_pages=3, table_stride=2), fa.FA_ERR_SHAPE),
    (dict(block_table=A, num_pages=4, page_size=1 << 20, max_pages=1 << 12, table_stride=1 << 12), fa.FA_ERR_SHAPE),
    (dict(dv=72), fa.FA_ERR_UNSUPPORTED), (dict(dtype=2), fa.FA_ERR_UNSUPPORTED), (dict(cache_dtype=1), fa.FA_ERR_UNSUPPORTED),
    (dict(cache_dtype=3, k_scale=0.0), fa.FA_ERR_UNSUPPORTED), (dict(cache_dtype=3, v_scale=math.inf), fa.FA_ERR_UNSUPPORTED),
    (dict(cache_dtype=3, k_scale=math.nan), fa.FA_ERR_UNSUPPORTED), (dict(factor=math.nan), fa.FA_ERR_UNSUPPORTED),
    (dict(k=0), fa.FA_ERR_NULL), (dict(k_cache=0), fa.FA_ERR_NULL), (dict(first_rows=0), fa.FA_ERR_NULL), (dict(q_out=0), fa.FA_ERR_NULL),
    (dict(v_cache=0), fa.FA_ERR_NULL), (dict(k=A + 8), fa.FA_ERR_ALIGN), (dict(v_cache=A + 4), fa.FA_ERR_ALIGN), (dict(counts=A + 2), fa.FA_ERR_ALIGN),
    (dict(n=0, T=0, k=0), fa.FA_OK)])
def test_append_refusals(change, code):
    assert fa.lib.fa_cache_append(ctypes.byref(append_params(**change)), None) == code


def test_append_null_block():
    assert fa.lib.fa_cache_append(None, None) == fa.FA_ERR_NULL


def test_the_binding_refuses_what_the_library_cannot_see():
    f, i = torch.zeros, torch.int32
    k, first, turns = f(4, 2, 64, dtype=torch.half), f(2, dtype=i), f(32, dtype=torch.int64)
    cache = f(2, 8, 2, 64, dtype=torch.half)
    ok = dict(q=None, q_out=None, k=k, v=None, k_cache=cache, v_cache=None, first_rows=first, turns=turns)
    for change in (dict(k=k.float()), dict(k_cache=cache.float()), dict(first_rows=first.long()), dict(k=k[..., ::2]), dict(k_cache=cache[:, :, :1]),
                   dict(k_cache=cache.transpose(1, 2)), dict(turns=turns.int()), dict(q=k, q_out=k[:3]), dict(v=k[:, :1], v_cache=cache),
                   dict(counts=f(1, dtype=i)), dict(positions=f(3, dtype=i)), dict(cu_seqlens=f(5, dtype=i)), dict(k=f(5, 2, 64, dtype=torch.half)),
                   dict(v=k, v_cache=cache.view(torch.uint8)[..., :64].contiguous())):
        with pytest.raises(ValueError):
            fa.fa_cache_append(**{**ok, **change})
    x = f(4, 2, 64, dtype=torch.half)
    for change in (dict(x=x.float()), dict(out=x[:3]), dict(positions=f(3, dtype=i)), dict(positions=f(4, dtype=torch.int64)), dict(x=x[..., ::2], out=x[..., ::2])):
        with pytest.raises(ValueError):
            fa.fa_rope(**{**dict(x=x, out=x, positions=f(4, dtype=i), turns=turns), **change})
    with pytest.raises(ValueError):
        fa.rope_turns(f(32))


def test_turns_hold_every_angle():
    """The integer product's low 64 bits are the angle's place in its turn, as exact arithmetic gives it: two pi in 64 bits and the division by
    it are off by less than 2^-52 of the angle each, the whole turns taken off by nothing, the share by less than two of its units."""
    w = torch.cat([fa.rope_frequencies(64, device="cpu"), torch.tensor([math.pi, 4.0, -0.3], dtype=torch.float64)])
    turns = fa.rope_turns(w)
    for pos in (0, 1, 7, 4095, 500000, 2 ** 31 - 1, -3):
        for share, f in zip(turns.tolist(), w.tolist()):
            want = pos * Fraction(f) / (2 * PI)
            off = Fraction(pos * share % 2 ** 64, 2 ** 64) - want
            off = abs(off - round(off))
            assert off <= abs(want) / 2 ** 51 + Fraction(abs(pos), 2 ** 63)


def test_scaled_frequencies():
    w = fa.rope_frequencies(128, device="cpu")
    assert torch.equal(fa.rope_frequencies(128, stretch=4.0, device="cpu"), w / 4)
    by_parts = fa.rope_frequencies(128, stretch=8.0, trained=4096, device="cpu")
    over = 4096 * w / (2 * math.pi)
    assert torch.equal(by_parts[over >= 32], w[over >= 32]) and torch.allclose(by_parts[over <= 1], w[over <= 1] / 8, rtol=1e-15)
    mid = (over > 1) & (over < 32)
    assert bool(mid.any()) and bool(((by_parts < w) & (by_parts > w / 8))[mid].all())


@pytest.mark.parametrize("change, code", [
    (dict(q_out_stride=(0, 128)), fa.FA_ERR_SHAPE), (dict(q_out_stride=(512, 0)), fa.FA_ERR_SHAPE), (dict(q_out_stride=(512, 120)), fa.FA_ERR_SHAPE),
    (dict(k_cache_stride=(64 * 256, 0)), fa.FA_ERR_SHAPE), (dict(k_cache_stride=(0, 256)), fa.FA_ERR_SHAPE), (dict(v_cache_stride=(64 * 256, 128)), fa.FA_ERR_SHAPE),
    (dict(Skv_max=1, k_cache_stride=(256, 0), n=0, T=0), fa.FA_OK), (dict(q_out_stride=(128, 1024), n=0, T=0), fa.FA_OK)])
def test_outputs_that_lie_over_themselves_are_refused(change, code):
    """Rows or heads one over the other (an expanded tensor) would hold whatever came last; dimensions of one, and heads before tokens, stay open."""
    assert fa.lib.fa_cache_append(ctypes.byref(append_params(**change)), None) == code


def test_rope_outputs_that_lie_over_themselves_are_refused():
    for change in (dict(ot=0), dict(oh=0), dict(oh=8)):
        assert fa.lib.fa_rope(*rope_args(**change), None) == fa.FA_ERR_SHAPE


@pytest.mark.parametrize("change, code", [
    (dict(q_out_stride=(128, 128)), fa.FA_ERR_SHAPE), (dict(q_out_stride=(504, 128)), fa.FA_ERR_SHAPE), (dict(q_out_stride=(128, 504)), fa.FA_ERR_SHAPE),
    (dict(k_cache_stride=(256, 256)), fa.FA_ERR_SHAPE), (dict(v_cache_stride=(256, 256)), fa.FA_ERR_SHAPE), (dict(k_cache_stride=(64 * 256 - 8, 256)), fa.FA_ERR_SHAPE),
    (dict(v_cache_stride=(256, 504)), fa.FA_ERR_SHAPE), (dict(k_cache_stride=(1 << 41, 1 << 41)), fa.FA_ERR_SHAPE),
    (dict(block_table=A, num_pages=1 << 30, page_size=1 << 20, max_pages=4, table_stride=4, k_cache_stride=(1 << 41, 1 << 40)), fa.FA_ERR_SHAPE),
    (dict(k=0, q_out_stride=(512, 128)), fa.FA_ERR_NULL), (dict(k=0, q_out_stride=(128, 512)), fa.FA_ERR_NULL), (dict(k=0, q_out_stride=(576, 144)), fa.FA_ERR_NULL),
    (dict(k=0, k_cache_stride=(256, 512), v_cache_stride=(256, 1024)), fa.FA_ERR_NULL), (dict(k=0, v_cache_stride=(63 * 1152 + 256, 1152)), fa.FA_ERR_NULL),
    (dict(k=0, n=1, B=1, T=1, q_out_stride=(0, 128), k_cache_stride=(0, 256)), fa.FA_ERR_NULL)])
def test_outputs_that_lie_over_themselves_by_both_strides_are_refused(change, code):
    """Each stride is wide enough, but steps of the one end where steps of the other do.  (What is open gets as far as the missing k.)"""
    assert fa.lib.fa_cache_append(ctypes.byref(append_params(**change)), None) == code


def test_rope_outputs_that_lie_over_themselves_by_both_strides_are_refused():
    for change in (dict(ot=128, oh=128), dict(ot=248, oh=128), dict(ot=128, oh=504)):
        assert fa.lib.fa_rope(*rope_args(**change), None) == fa.FA_ERR_SHAPE
    for change in (dict(ot=128, oh=512), dict(ot=256, oh=128), dict(n=1, ot=0), dict(H=1, oh=0, ot=128), dict(xt=128, xh=128), dict(xt=0, xh=0)):
        assert fa.lib.fa_rope(*rope_args(**{**change, "x": 0}), None) == fa.FA_ERR_NULL
