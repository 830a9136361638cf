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
