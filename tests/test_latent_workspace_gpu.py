"""The workspace of attention over latent vectors: what a call writes lies inside the bytes that it asks for."""
import pytest
import torch

from paper_2410_16663_b200 import binding as fa
from tests.test_latent_gpu import SCALE, absorbed, ints

pytestmark = pytest.mark.gpu
AROUND = 1 << 20


def guarded(size):
    """size bytes between two stretches that hold 0x5a, and a look at whether they still do."""
    flat = torch.full((size + 2 * AROUND,), 0x5a, dtype=torch.uint8, device="cuda")
    return flat[AROUND:AROUND + size], lambda: bool((flat[:AROUND] == 0x5a).all()) and bool((flat[AROUND + size:] == 0x5a).all())


@pytest.mark.parametrize("T, H", [(1, 5), (1, 32), (1, 40), (3, 30), (1, 128), (2, 128), (3, 43)])
@pytest.mark.parametrize("most", [3, 63, 64, 65, 128, 129, 1000])
def test_a_call_stays_inside_its_workspace(T, H, most):
    lens = [most, 0, max(1, most // 2), most - 1] * 30
    q, r, cache, _, _, o, lse, _ = absorbed(lens, T, H, "fp16", samples=[0])
    ws, untouched = guarded(fa.fa_decode_latent_workspace_bytes(len(lens), T, H, cache.shape[1]))
    o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
    fa.fa_decode_latent(q, r, cache, o2, lse2, ints(lens), SCALE, ws)
    assert torch.equal(o2, o) and torch.equal(lse2, lse) and untouched()


@pytest.mark.parametrize("T", [1, 2, 3, 4])
def test_a_workspace_for_the_most_tokens_does_for_fewer(T):
    """12 heads: up to two tokens are one CTA's rows, three and four a pair's."""
    lens = [900, 41, 300]
    q, r, cache, _, _, o, lse, most = absorbed(lens, T, 12, "bf16")
    ws, untouched = guarded(fa.fa_decode_latent_workspace_bytes(3, 4, 12, most))
    o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
    fa.fa_decode_latent(q, r, cache, o2, lse2, ints(lens), SCALE, ws)
    assert torch.equal(o2, o) and torch.equal(lse2, lse) and untouched()
