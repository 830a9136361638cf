"""A layer of grouped heads as its calls follow one another: a prompt's and the new tokens' rows go to the caches by `fa_cache_append`, queries
rotated on the way, and the decode calls read what the appends have written."""
import random

import pytest
import torch

from oracle import latent as oracle
from paper_2410_16663_b200 import binding as fa
from tests.test_latent_gpu import DT, check, ints, normal
from tests.test_rope_append_gpu import ARITH, same

pytestmark = pytest.mark.gpu


def decode(q, kc, vc, o, lse, lens, table, e4m3, ks, vs, rows):
    B, T, Hq, d = q.shape
    scale = d ** -0.5
    ws = torch.empty(max(fa.fa_decode_append_workspace_bytes(B, T, Hq, kc.shape[2], rows, d), fa.fa_decode_workspace_bytes(B, Hq, kc.shape[2], rows, d), 16),
                     dtype=torch.uint8, device="cuda")
    if not e4m3:
        fa.fa_decode_ex(q, kc, vc, o, lse, lens, scale, ws, block_table=table)
    elif table is None:
        (fa.fa_decode_fp8 if q.dtype is torch.float16 else fa.fa_decode_fp8_bf16)(q, kc, vc, o, lse, lens, scale, ks, vs, ws)
    else:
        (fa.fa_decode_fp8_paged if q.dtype is torch.float16 else fa.fa_decode_fp8_paged_bf16)(q, kc, vc, table, o, lse, lens, scale, ks, vs, ws)


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("e4m3, T", [(False, 1), (False, 3), (True, 1)])
@pytest.mark.parametrize("page", [0, 16, 128])
def test_appended_rows_are_what_decode_reads(dt, e4m3, T, page):
    Hq, Hkv, d, before = 8, 2, 128, [70, 131, 0, 128]
    B, n, rows = len(before), sum(before), 160
    ks, vs = (0.02, 0.013) if e4m3 else (1.0, 1.0)
    table, rng = None, random.Random(4)
    if page:
        per = -(-rows // page)
        order = list(range(B * per))
        rng.shuffle(order)
        table, slabs, height = ints([order[b * per:(b + 1) * per] for b in range(B)]), B * per, page
    else:
        slabs, height = B, rows
    kc, vc = (torch.full((slabs, height, Hkv, d), float("nan"), dtype=DT[dt], device="cuda") for _ in range(2))
    if e4m3:
        kc, vc = kc.to(torch.float8_e4m3fn), vc.to(torch.float8_e4m3fn)
    freq = fa.rope_frequencies(d)
    turns = fa.rope_turns(freq)
    cu = ints([sum(before[:b]) for b in range(B + 1)])
    # queries, keys and values are the heads of one projection's output; queries are rotated in place
    prompt, new = normal((n, Hq + 2 * Hkv, d), dt, 1), normal((B, T, Hq + 2 * Hkv, d), dt, 2)
    raw, raw_new = prompt.clone(), new.clone()
    for x, first, cu_seqlens in ((prompt, [0] * B, cu), (new, before, None)):
        q, k, v = x[..., :Hq, :], x[..., Hq:Hq + Hkv, :], x[..., Hq + Hkv:, :]
        fa.fa_cache_append(q, q, k, v, kc, vc, ints(first), turns=turns, cu_seqlens=cu_seqlens, block_table=table, k_scale=ks, v_scale=vs)
    assert torch.equal(prompt[:, Hq:], raw[:, Hq:]) and torch.equal(new[:, :, Hq:], raw_new[:, :, Hq:])
    lens = [x + T for x in before]
    o, lse = torch.full((B, T, Hq, d), float("nan"), dtype=DT[dt], device="cuda"), torch.full((B, Hq, T), float("nan"), device="cuda")
    q = new[:, :, :Hq].contiguous()
    decode(q, kc, vc, o, lse, ints(lens), table, e4m3, ks, vs, rows if not page else table.shape[1] * page)
    for b, m in enumerate(lens):
        at = torch.arange(m, device="cuda")
        where = b * height + at if table is None else table[b, at // page].long() * page + at % page
        got_k, got_v = (c.view(-1, Hkv, d)[where].double().cpu() for c in (kc, vc))
        all_k, all_v = (torch.cat([raw[cu[b]:cu[b + 1], x], raw_new[b, :, x]]).cpu() for x in (slice(Hq, Hq + Hkv), slice(Hq + Hkv, None)))
        turned = oracle.rotate(all_k, at.cpu(), freq.cpu())
        size = 1.5 * all_k.double().norm(dim=-1, keepdim=True)
        if e4m3:   # half a step of e4m3, of its least normal number below that
            for got, want, by in ((got_k, turned, ks), (got_v, all_v.double(), vs)):
                want = (want / by).clamp(-448, 448)
                assert bool(((got - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -10 + ARITH * size / by).all())
            got_k, got_v = got_k * ks, got_v * vs
        else:
            same(got_k, turned, dt, size)
            assert torch.equal(got_v, all_v.double())
        same(q[b], oracle.rotate(raw_new[b, :, :Hq].cpu(), torch.arange(m - T, m), freq.cpu()), dt, 1.5 * raw_new[b, :, :Hq].double().norm(dim=-1, keepdim=True).cpu())
        for h in range(Hq):
            hk = h // (Hq // Hkv)
            # products of a score add up to |q| |k| / sqrt(d) at most
            most = float(q[b, :, h].double().norm(dim=-1).max() * got_k[:, hk].norm(dim=-1).max()) * d ** -0.5
            check(o[b, :, h], lse[b, h], oracle.attention(q[b, :, h].cpu(), got_k[:, hk], got_v[:, hk], d ** -0.5, True), dt, size=max(10.0, most))
    assert fa.fa_device_status()[0] == 0
