"""Plain restatements, in 64 bits and on host lists, of the operators of a speculative decoding step: attention for a tree of
drafted tokens, verification, compaction of the accepted rows, and the pages of a pool.  Test infrastructure only."""
from __future__ import annotations

import torch


def bits_to_words(see):
    """Truth values [..., T] as 32-bit words [..., ceil(T/32)] (int32)."""
    T = see.shape[-1]
    W = (T + 31) // 32
    pad = torch.zeros(*see.shape[:-1], W * 32, dtype=torch.int64)
    pad[..., :T] = see.to(torch.int64)
    w = (pad.view(*see.shape[:-1], W, 32) << torch.arange(32)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def ancestors(parents):
    """[T,T] truth values of one tree: node i sees itself and the nodes above it."""
    T = len(parents)
    see = torch.zeros(T, T, dtype=torch.bool)
    for i in range(T):
        j = i
        while j >= 0:
            see[i, j] = True
            j = parents[j]
    return see


def gather_rows(cache, table, b, n):
    """The first n rows of sequence b, [n,Hkv,d], of a contiguous cache (table None) or of a pool."""
    if table is None:
        return cache[b, :n]
    page = cache.shape[1]
    rows = [cache[int(table[b, j // page]), j % page] for j in range(n)]
    return torch.stack(rows) if rows else cache.new_zeros(0, *cache.shape[2:])


def tree_attention(q, k, v, lens, see, scale, tree_lens=None, table=None, abs_v=False):
    """q [B,T,Hq,d]; see [B,T,T]; returns O [B,T,Hq,d] and LSE [B,Hq,T] in fp64, on the host."""
    B, T, Hq, d = q.shape
    Hkv = k.shape[2]
    g = Hq // Hkv
    o = torch.zeros(B, T, Hq, d, dtype=torch.float64)
    lse = torch.full((B, Hq, T), float("-inf"), dtype=torch.float64)
    for b in range(B):
        n = max(0, int(lens[b]))
        live = max(0, min(T if tree_lens is None else int(tree_lens[b]), T, n))
        pre = n - live
        kb, vb = (gather_rows(x, table, b, n).double() for x in (k, v))
        if abs_v:
            vb = vb.abs()
        hidden = torch.zeros(live, n, dtype=torch.bool)
        hidden[:, pre:] = ~see[b, :live, :live]
        for h in range(Hq):
            x = (scale * (q[b, :live, h].double() @ kb[:, h // g].T)).masked_fill(hidden, float("-inf"))
            m = x.amax(1, keepdim=True).clamp(min=-1e300) if n else torch.zeros(live, 1, dtype=torch.float64)
            w = (x - m).exp()
            l = w.sum(1, keepdim=True)
            lse[b, h, :live] = (m + l.log())[:, 0]
            o[b, :live, h] = (w @ vb[:, h // g]) / l.clamp(min=1e-300)
    return o, lse


def verify(p, q, tokens, parents, u, noise, live):
    """One sequence, host tensors; returns (accepted nodes with the root, emitted tokens)."""
    p = p.double()
    q = None if q is None else q.double()
    V = p.shape[1]
    node, path, out = 0, [0], []
    while True:
        left, mass, step = p[node].clone(), 1.0, None
        for c in range(1, live):
            if int(parents[c]) != node:
                continue
            x = int(tokens[c])
            have = float(left[x]) if 0 <= x < V else 0.0
            odds = 1.0 if q is None else float(q[node, x]) if 0 <= x < V else 0.0
            if float(u[c]) * mass * odds < have:
                step = c
                break
            if q is not None:
                left = (left / mass - q[node]).clamp(min=0)
                mass = float(left.sum())
            else:
                mass = max(mass - have, 0.0)
                if 0 <= x < V:
                    left[x] = 0
        if step is None:
            break
        node = step
        path.append(step)
        out.append(int(tokens[step]))
    if not float(left.max()) > 0:
        left = p[node]
    out.append(int(torch.argmax(left / noise.double())) if float(left.max()) > 0 else -1)
    return path, out


def compact(k, v, lens, path, n_accept, tree_lens=None, table=None, T=None):
    """Moves the rows of k, v [L,slabs,rows,...] (host tensors, in place); returns the new lengths."""
    new = []
    most = k.shape[2] if table is None else table.shape[1] * k.shape[2]
    for b in range(len(lens)):
        n = max(0, min(int(lens[b]), most))
        live = max(0, min(T if tree_lens is None else int(tree_lens[b]), T, n))
        acc = max(0, min(int(n_accept[b]), live - 1))
        pre = n - live
        for i in range(1, acc + 1):
            x = int(path[b][i])
            if not i < x < live:
                continue
            (s0, r0), (s1, r1) = (((b, r) if table is None else (int(table[b][r // k.shape[2]]), r % k.shape[2])) for r in (pre + i, pre + x))
            for c in (k, v):
                c[:, s0, r0] = c[:, s1, r1]
        new.append(pre + 1 + acc if live else n)
    return new


def pages_resize(table, held, refs, want, page):
    """On host lists, in place; returns the number of sequences that could not be served."""
    most = len(table[0])
    need = [-(-max(w, 0) // page) for w in want]
    for b, n in enumerate(need):
        for e in range(n, held[b]):
            refs[table[b][e]] -= 1
            table[b][e] = -1
        if n < held[b]:
            held[b] = n
    free = [i for i, r in enumerate(refs) if r == 0]
    total = short = 0
    for b, n in enumerate(need):
        if n <= held[b]:
            continue
        if n > most:
            short += 1
            continue
        total += n - held[b]
        if total > len(free):
            short += 1
            continue
        for i in free[total - (n - held[b]):total]:
            table[b][held[b]], refs[i] = i, 1
            held[b] += 1
    return short


def pages_fork(k, v, table, held, lens, refs, src, dst, page):
    """On host lists and host pools, in place; returns the number of pairs without a page."""
    free, short = [i for i, r in enumerate(refs) if r == 0], 0
    for s, t in zip(src, dst):
        if not (0 <= s < len(lens) and 0 <= t < len(lens)):
            continue
        full, part = divmod(lens[s], page)
        table[t] = [-1] * len(table[t])
        if part and not free:
            short += 1
            held[t] = lens[t] = 0
            continue
        for e in range(full):
            table[t][e] = table[s][e]
            refs[table[s][e]] += 1
        if part:
            new = table[t][full] = free.pop(0)
            refs[new] = 1
            k[:, new, :part] = k[:, table[s][full], :part]
            v[:, new, :part] = v[:, table[s][full], :part]
        held[t], lens[t] = full + (part > 0), lens[s]
    return short
