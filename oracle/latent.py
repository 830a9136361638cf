"""Rotation, cache appends and attention over latent vectors from their definitions, in float64 on the CPU.  Test infrastructure."""
import math

import torch


def rotate(x, positions, frequencies, offset=0, interleaved=False, factor=1.0):
    """x [n,H,d] with the pairs of its columns offset .. offset + 2 len(frequencies) turned by positions [n] times frequencies."""
    out = x.double().clone()
    angle = positions.double()[:, None] * frequencies.double()[None, :]
    turn = torch.polar(torch.full_like(angle, factor), angle)[:, None, :]
    half = frequencies.numel()
    i = torch.arange(half)
    a, b = (offset + 2 * i, offset + 2 * i + 1) if interleaved else (offset + i, offset + half + i)
    z = torch.complex(out[:, :, a], out[:, :, b]) * turn
    out[:, :, a], out[:, :, b] = z.real, z.imag
    return out


def owners(n, B, T, cu):
    """(sequence, place in it) of every token; sequence -1: nobody's."""
    if cu is None:
        return [(i // T, i % T) for i in range(n)]
    out = [(-1, -1)] * n
    for b in range(B):
        for t in range(cu[b], min(cu[b + 1], n)):
            out[t] = (b, t - cu[b])
    return out


def append_places(n, B, T, cu, first, counts, rows, table=None, page=0, pages=0):
    """The (slab, row) of every token's cache row, None where it has none."""
    out = []
    for b, t in owners(n, B, T, cu):
        row = None if b < 0 else first[b] + t
        if row is None or (counts is not None and t >= counts[b]) or not 0 <= row < rows:
            out.append(None)
        elif table is None:
            out.append((b, row))
        else:
            at = table[b][row // page]
            out.append((at, row % page) if 0 <= at < pages else None)
    return out


def attention(q, k, v, scale, causal):
    """q [n,dk], k [m,dk], v [m,dv]: (o [n,dv], lse [n], sum P |V| [n,dv], sum |V| [dv]); causal: the n queries are the last of the m
    positions.  A row that sees nothing gives zeros and -inf."""
    n, m = q.shape[0], k.shape[0]
    s = q.double() @ k.double().T * scale
    if causal:
        s = s.masked_fill(torch.arange(m)[None, :] > torch.arange(m - n, m)[:, None], -math.inf)
    lse = torch.logsumexp(s, 1) if m else torch.full((n,), -math.inf, dtype=torch.float64)
    p = torch.where(torch.isneginf(lse)[:, None], torch.zeros_like(s), torch.exp(s - lse.clamp(min=-1e300)[:, None]))
    return p @ v.double(), lse, p @ v.double().abs(), v.double().abs().sum(0)
