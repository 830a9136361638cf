"""Attention over latent vectors: what the calls refuse, on the CPU."""
import ctypes
import math

import pytest
import torch

from paper_2410_16663_b200 import binding as fa

A = 1 << 12   # an aligned address that nothing is read from


def set_fields(p, **kw):
    for name, x in kw.items():
        if isinstance(x, tuple):
            for i in range(2):
                getattr(p, name)[i] = x[i]
        else:
            setattr(p, name, x)
    return p


def forward_params(**kw):
    base = dict(q=A, q_rope=A, k=A, k_rope=A, v=A, o=A, lse=0, cu_seqlens_q=A, cu_seqlens_k=A, q_stride=(768, 192), q_rope_stride=(768, 192),
                k_stride=(1024, 256), v_stride=(1024, 256), k_rope_stride=576, B=2, H=4, total_q=10, total_k=20, max_seqlen_q=8, max_seqlen_k=16, d=128,
                d_rope=64, causal=1, dtype=0, scale=0.1)
    return set_fields(fa.fa_latent_params(), **{**base, **kw})


@pytest.mark.parametrize("change, code", [
    (dict(B=-1), fa.FA_ERR_SHAPE), (dict(H=0), fa.FA_ERR_SHAPE), (dict(total_q=-1), fa.FA_ERR_SHAPE), (dict(max_seqlen_q=11), fa.FA_ERR_SHAPE),
    (dict(max_seqlen_k=21), fa.FA_ERR_SHAPE), (dict(q_stride=(768, 100)), fa.FA_ERR_SHAPE), (dict(q_rope_stride=(32, 192)), fa.FA_ERR_SHAPE),
    (dict(k_stride=(1024, 0)), fa.FA_ERR_SHAPE), (dict(v_stride=(-8, 256)), fa.FA_ERR_SHAPE), (dict(k_rope_stride=0), fa.FA_ERR_SHAPE),
    (dict(k_rope_stride=580), fa.FA_ERR_SHAPE), (dict(d=64), fa.FA_ERR_UNSUPPORTED), (dict(d_rope=128), fa.FA_ERR_UNSUPPORTED),
    (dict(dtype=2), fa.FA_ERR_UNSUPPORTED), (dict(scale=-1.0), fa.FA_ERR_UNSUPPORTED), (dict(scale=math.inf), fa.FA_ERR_UNSUPPORTED),
    (dict(scale=math.nan), fa.FA_ERR_UNSUPPORTED), (dict(B=65536), fa.FA_ERR_UNSUPPORTED), (dict(H=65536), fa.FA_ERR_UNSUPPORTED),
    (dict(q=0), fa.FA_ERR_NULL), (dict(q_rope=0), fa.FA_ERR_NULL), (dict(k=0), fa.FA_ERR_NULL), (dict(k_rope=0), fa.FA_ERR_NULL), (dict(v=0), fa.FA_ERR_NULL),
    (dict(o=0), fa.FA_ERR_NULL), (dict(cu_seqlens_q=0), fa.FA_ERR_NULL), (dict(q_rope=A + 8), fa.FA_ERR_ALIGN), (dict(k_rope=A + 2), fa.FA_ERR_ALIGN),
    (dict(lse=A + 2), fa.FA_ERR_ALIGN), (dict(cu_seqlens_k=A + 1), fa.FA_ERR_ALIGN), (dict(total_q=0, max_seqlen_q=0, q=0), fa.FA_OK), (dict(B=0, q=0), fa.FA_OK)])
def test_forward_refusals(change, code):
    assert fa.lib.fa_forward_latent(ctypes.byref(forward_params(**change)), None) == code


def test_the_binding_refuses_what_the_library_cannot_see():
    z = lambda *s: torch.zeros(*s, dtype=torch.half)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    ok = dict(q=z(4, 2, 128), q_rope=z(4, 2, 64), k=z(6, 2, 128), k_rope=z(6, 64), v=z(6, 2, 128), o=z(4, 2, 128), lse=None, cu_seqlens_q=cu, cu_seqlens_k=cu,
              max_seqlen_q=4, max_seqlen_k=6, causal=True, scale=0.1)
    for change in (dict(k=z(6, 2, 128).float()), dict(k_rope=z(5, 64)), dict(v=z(6, 1, 128)), dict(o=z(4, 2, 256)[..., :128]), dict(lse=z(2, 4)),
                   dict(lse=torch.zeros(7)), dict(cu_seqlens_q=cu.long()), dict(q_rope=z(3, 2, 64)), dict(k_rope=z(64, 6).T), dict(q=z(4, 2, 256)[..., ::2])):
        with pytest.raises(ValueError):
            fa.fa_forward_latent(**{**ok, **change})


def decode_params(**kw):
    base = dict(q=A, q_rope=A, cache=A, o=A, lse=0, seqlens_k=A, block_table=0, q_stride=(4096, 2048, 512), q_rope_stride=(512, 256, 64), B=2, T=2, H=4,
                Skv_max=100, d=512, d_rope=64, dtype=0, num_pages=0, page_size=0, max_pages=0, table_stride=0, scale=0.1, workspace=A, workspace_bytes=1 << 40)
    p = fa.fa_latent_decode_params()
    for name, x in {**base, **kw}.items():
        if isinstance(x, tuple):
            for i in range(3):
                getattr(p, name)[i] = x[i]
        else:
            setattr(p, name, x)
    return p


PAGED = dict(block_table=A, num_pages=8, page_size=16, max_pages=4, table_stride=4)


@pytest.mark.parametrize("change, code", [
    (dict(B=-1), fa.FA_ERR_SHAPE), (dict(T=0), fa.FA_ERR_SHAPE), (dict(H=0), fa.FA_ERR_SHAPE), (dict(Skv_max=-1), fa.FA_ERR_SHAPE), (dict(d=0), fa.FA_ERR_SHAPE),
    (dict(q_stride=(4096, 2048, 508)), fa.FA_ERR_SHAPE), (dict(q_rope_stride=(512, 256, 32)), fa.FA_ERR_SHAPE), (dict(q_stride=(4096, 0, 512)), fa.FA_ERR_SHAPE),
    (dict(PAGED, page_size=24), fa.FA_ERR_SHAPE), (dict(PAGED, table_stride=3), fa.FA_ERR_SHAPE), (dict(PAGED, num_pages=0), fa.FA_ERR_SHAPE),
    (dict(PAGED, max_pages=1 << 28, table_stride=1 << 28), fa.FA_ERR_SHAPE), (dict(T=65), fa.FA_ERR_UNSUPPORTED), (dict(T=64, Skv_max=63), fa.FA_ERR_UNSUPPORTED),
    (dict(d=256), fa.FA_ERR_UNSUPPORTED), (dict(d_rope=128), fa.FA_ERR_UNSUPPORTED), (dict(dtype=2), fa.FA_ERR_UNSUPPORTED), (dict(scale=-0.1), fa.FA_ERR_UNSUPPORTED),
    (dict(scale=math.nan), fa.FA_ERR_UNSUPPORTED), (dict(B=65536), fa.FA_ERR_UNSUPPORTED), (dict(H=65536), fa.FA_ERR_UNSUPPORTED),
    (dict(B=65535, T=64, H=8192, Skv_max=1 << 28), fa.FA_ERR_UNSUPPORTED), (dict(q=0), fa.FA_ERR_NULL), (dict(q_rope=0), fa.FA_ERR_NULL),
    (dict(cache=0), fa.FA_ERR_NULL), (dict(o=0), fa.FA_ERR_NULL), (dict(seqlens_k=0), fa.FA_ERR_NULL), (dict(cache=A + 8), fa.FA_ERR_ALIGN), (dict(o=A + 2), fa.FA_ERR_ALIGN),
    (dict(workspace=A + 4), fa.FA_ERR_ALIGN), (dict(seqlens_k=A + 2), fa.FA_ERR_ALIGN), (dict(lse=A + 1), fa.FA_ERR_ALIGN), (dict(PAGED, block_table=A + 2), fa.FA_ERR_ALIGN),
    (dict(workspace=0), fa.FA_ERR_WORKSPACE), (dict(workspace_bytes=1000), fa.FA_ERR_WORKSPACE), (dict(B=0, q=0), fa.FA_OK)], ids=str)
def test_decode_refusals(change, code):
    assert fa.lib.fa_decode_latent(ctypes.byref(decode_params(**change)), None) == code


def test_decode_workspace():
    size = fa.fa_decode_latent_workspace_bytes
    assert size(2, 2, 4, 100) > 0 and size(2, 65, 4, 100) == size(0, 1, 4, 100) == size(1, 0, 4, 100) == size(1, 1, 0, 100) == size(1, 1, 4, 0) == size(1, 1, 4, 100, 256) == 0
    assert fa.lib.fa_decode_latent(ctypes.byref(decode_params(workspace_bytes=size(2, 2, 4, 100) - 1)), None) == fa.FA_ERR_WORKSPACE


def test_the_decode_binding_refuses_what_the_library_cannot_see():
    z, i = lambda *s: torch.zeros(*s, dtype=torch.half), torch.int32
    ok = dict(q=z(2, 1, 4, 512), q_rope=z(2, 1, 4, 64), cache=z(2, 20, 576), o=z(2, 1, 4, 512), lse=None, seqlens_k=torch.zeros(2, dtype=i), scale=0.1, workspace=None)
    for change in (dict(cache=z(2, 20, 576).float()), dict(cache=z(2, 20, 512)), dict(cache=z(1, 20, 576)), dict(o=z(2, 1, 4, 576)[..., :512]), dict(o=z(2, 1, 3, 512)),
                   dict(q_rope=z(2, 1, 3, 64)), dict(lse=z(2, 4, 1)), dict(lse=torch.zeros(7)), dict(seqlens_k=torch.zeros(1, dtype=i)),
                   dict(seqlens_k=torch.zeros(2)), dict(q=z(2, 1, 4, 1024)[..., ::2]), dict(block_table=torch.zeros(1, 4, dtype=i)),
                   dict(block_table=torch.zeros(2, 4))):
        with pytest.raises(ValueError):
            fa.fa_decode_latent(**{**ok, **change})


@pytest.mark.parametrize("change, code", [
    (dict(PAGED, max_pages=(1 << 27) - 1, table_stride=1 << 27), fa.FA_ERR_UNSUPPORTED), (dict(Skv_max=0x7fffffff), fa.FA_ERR_UNSUPPORTED),
    (dict(H=128, Skv_max=0x7fffffff - 255), fa.FA_ERR_UNSUPPORTED), (dict(Skv_max=0x7fffffff - 256, q=0), fa.FA_ERR_NULL),
    (dict(PAGED, max_pages=(1 << 27) - 17, table_stride=1 << 27, q=0), fa.FA_ERR_NULL)], ids=str)
def test_a_capacity_whose_end_passes_32_bits_is_refused(change, code):
    """The position behind the last tile's last key, and half a tile beyond it, are formed in 32 bits.  (What is open gets as far as the missing q.)"""
    assert fa.lib.fa_decode_latent(ctypes.byref(decode_params(**change)), None) == code


def test_decode_workspace_holds_what_a_call_can_use():
    """Two partial results for each worker at most -- a CTA (up to 32 rows) or a pair of them (of up to 128 rows), of 160 SMs -- of 512 + 1 floats a row; a cache of
    one tile has none.  And a workspace for the most tokens, heads and keys does for fewer."""
    size = fa.fa_decode_latent_workspace_bytes
    rest = 32 + 160 * 16
    for B, T, H, slots, rows in ((1, 1, 128, 160, 128), (64, 1, 128, 160, 128), (2, 64, 128, 160, 128), (4, 1, 100, 160, 100), (4, 1, 16, 320, 16), (4, 2, 16, 320, 32)):
        assert size(B, T, H, 10000) <= slots * rows * 513 * 4 + rest, (B, T, H)
        assert size(B, T, H, 64) <= rest
    for H in (1, 5, 16, 20, 33, 43, 64, 128):
        for most in (64, 65, 100, 128, 129, 10000):
            sizes = [size(3, T, H, most) for T in range(1, 65)]
            assert sizes == sorted(sizes), (H, most)
            assert size(3, 2, H, most) <= size(3, 2, H + 1, most) and size(3, 2, H, most) <= size(3, 2, H, most + 1)
