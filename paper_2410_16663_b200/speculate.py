"""Speculative decoding over a paged cache, step by step: how the library's calls go together.

A prompt's rows are in a page pool of every layer; ``fa_pages_fork`` makes more sequences of it, which share its full pages.
Then each step drafts a tree of tokens for every sequence and
  1. ``fa_pages_resize``    makes room for the tree's rows (who gets none sits the step out),
  2. the model writes their keys and values and, layer by layer, ``fa_decode_tree`` attends over cache and tree,
  3. ``fa_spec_verify``     decides which tokens stand, and draws the one after them,
  4. ``fa_cache_compact``   moves the accepted rows together, in all layers,
  5. ``fa_pages_resize``    gives back the pages past the new length.
The model here is a stand-in of random weights (embeddings, one matrix per layer for each of Q, K and V, and one for the vocabulary),
and so is the draft, which is the same model without the attention and with noise.  Nothing in a step waits for the GPU.

  python -m paper_2410_16663_b200.speculate --samples 8 --prompt 1000 --nodes 24 --steps 5
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as fa


class PagedCache:
    """Page pools of all layers and the state that ``fa_pages_resize`` and ``fa_pages_fork`` keep.  ``short`` counts the
    sequences that were not served, over all calls.  Behind the pools' pages lies one that is nobody's."""

    def __init__(self, layers, pages, page, Hkv, d, sequences, rows, dtype, device):
        self.page, self.pages = page, pages
        self.all_k = torch.zeros(layers, pages + 1, page, Hkv, d, dtype=dtype, device=device)
        self.all_v = torch.zeros_like(self.all_k)
        self.k, self.v = self.all_k[:, :pages], self.all_v[:, :pages]
        ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)
        self.table = torch.full((sequences, -(-rows // page)), -1, dtype=torch.int32, device=device)
        self.held, self.lens, self.refs, self.short, self.missed = ints(sequences), ints(sequences), ints(pages), ints(1), ints(1)

    def resize(self, rows):
        fa.fa_pages_resize(self.table, self.held, self.refs, rows, self.missed, self.page)
        self.short += self.missed

    def reserve(self, n):
        """Room for n more rows of every sequence; returns who has it, [B] truth values."""
        rows = self.lens + n
        self.resize(rows)
        return self.held * self.page >= rows

    def fork(self, src, dst):
        fa.fa_pages_fork(self.k, self.v, self.table, self.held, self.lens, self.refs, src, dst, self.missed)
        self.short += self.missed

    def write(self, layer, first, k, v, served):
        """Rows k, v [B,n,Hkv,d] of the sequences that ``served`` [B] says, from row first [B] on.  (The others' go to the page that is
        nobody's: an index of -1 would be the pool's last page, and leaving rows out would wait for the GPU to count them.)"""
        rows = first[:, None] + torch.arange(k.shape[1], device=k.device)[None, :]
        entries = (rows // self.page).clamp(max=self.table.shape[1] - 1)
        pages = torch.where(served[:, None], torch.gather(self.table, 1, entries), self.pages).long()
        self.all_k[layer, pages, rows % self.page] = k
        self.all_v[layer, pages, rows % self.page] = v

    def compact(self, path, n_accept, tree_lens):
        """The accepted rows of each sequence's tree, which end its cache, move together; the lengths follow."""
        new = torch.empty_like(self.lens)
        fa.fa_cache_compact(self.k, self.v, self.lens, path, n_accept, new, tree_lens=tree_lens, block_table=self.table)
        self.lens = new


class Model:
    """A stand-in: embeddings, a matrix for each of Q, K and V per layer, and one for the vocabulary at the end.  (Not the embeddings
    again: a token of a random model would then be followed by itself, with certainty.)"""

    def __init__(self, layers, Hq, Hkv, d, vocab, dtype, device, gen):
        new = lambda *s: torch.empty(*s, dtype=dtype, device=device).normal_(0.0, 1.0, generator=gen)
        self.Hq, self.Hkv, self.d, width = Hq, Hkv, d, Hq * d
        self.embed = new(vocab, width)
        self.w = [[new(width, h * d) / math.sqrt(width) for h in (Hq, Hkv, Hkv)] for _ in range(layers)]
        self.head = new(vocab, width)

    def project(self, x, layer):
        return [(x @ w).view(*x.shape[:2], -1, self.d) for w in self.w[layer]]

    def probabilities(self, x):
        x = x / x.float().square().mean(-1, keepdim=True).sqrt().to(x.dtype)
        return torch.softmax((x @ self.head.T).float() / math.sqrt(x.shape[-1]) * 3.0, -1)


def step(model, cache, tokens, parents, draft, gen, ws):
    """One step: tokens, parents int32 [B,T], draft [B,T,V] the draft's distributions after each node.  Returns (out_tokens, n_accept,
    the target's distributions).  A sequence for whose tree the pool has no pages keeps its rows and says nothing: its out_tokens
    are -1 and its n_accept is 0."""
    B, T = tokens.shape
    served = cache.reserve(T)                                      # room for the tree
    first = cache.lens
    live = torch.where(served, T, 0).to(torch.int32)
    cache.lens = cache.lens + live
    mask = fa.tree_mask(parents)
    x = model.embed[tokens.long()]
    for layer in range(len(model.w)):
        q, k, v = model.project(x, layer)
        cache.write(layer, first, k, v, served)
        o = torch.empty_like(q)
        fa.fa_decode_tree(q, cache.k[layer], cache.v[layer], o, None, cache.lens, mask, 1.0 / math.sqrt(model.d), ws, tree_lens=live,
                          block_table=cache.table)
        x = x + o.view(B, T, -1)
    target = model.probabilities(x)
    dev = tokens.device
    n_accept = torch.empty(B, dtype=torch.int32, device=dev)
    path, out = torch.empty(B, T, dtype=torch.int32, device=dev), torch.empty(B, T, dtype=torch.int32, device=dev)
    uniforms = torch.rand(B, T, device=dev, generator=gen)
    noise = torch.empty(B, target.shape[-1], device=dev).exponential_(generator=gen).clamp_(min=1e-20)
    fa.fa_spec_verify(target, draft, tokens, parents, uniforms, noise, n_accept, path, out, tree_lens=live)
    cache.compact(path, n_accept, live)                            # the accepted rows, in all layers
    cache.resize(cache.lens)                                       # and the pages behind them
    return torch.where(served[:, None], out, -1), torch.where(served, n_accept, 0), target


def random_trees(B, T, gen, device):
    """Parents [B,T]: a node hangs off one of the four before it."""
    node = torch.arange(T, device=device)
    low = (node - 4).clamp(min=0)
    up = low + (torch.rand(B, T, device=device, generator=gen) * (node - low)).long()
    return torch.where(node == 0, -1, torch.minimum(up, (node - 1).clamp(min=0))).to(torch.int32)


def draft_trees(model, last, parents, gen):
    """A tree of drafted tokens for every sequence: node 0 is the token ``last`` [B,1], every other node is drawn from the draft's
    distribution after its parent.  Returns tokens int32 [B,T] and the distributions [B,T,V]."""
    B, T = parents.shape
    tokens, row = last.repeat(1, T), torch.arange(B, device=last.device)

    def after(x):
        x = model.embed[x]
        return model.probabilities(x + torch.empty_like(x).normal_(0.0, 0.3, generator=gen))

    draft = [after(last[:, 0])]
    for i in range(1, T):
        up = torch.stack(draft, 1)[row, parents[:, i].long()]
        tokens[:, i] = torch.multinomial(up, 1, generator=gen)[:, 0]
        draft.append(after(tokens[:, i]))
    return tokens.to(torch.int32), torch.stack(draft, 1)


def run(samples=4, prompt=1000, nodes=24, steps=4, layers=4, Hq=8, Hkv=2, d=128, vocab=4096, page=16, dtype=torch.bfloat16, seed=0,
        device="cuda"):
    """Forks ``samples`` sequences off one prompt and decodes ``steps`` steps of each.  Returns (emitted tokens per step and
    sequence, lengths, cache)."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    most = prompt + steps * nodes + nodes
    pages = -(-prompt // page) + samples * (-(-(steps + 1) * nodes // page) + 2)
    cache = PagedCache(layers, pages, page, Hkv, d, samples + 1, most, dtype, device)
    model = Model(layers, Hq, Hkv, d, vocab, dtype, device, gen)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=device)
    # the prompt is sequence 0 (its rows would come from a prefill), the samples are sequences 1 .. samples
    cache.resize(ints([prompt] + [0] * samples))
    cache.lens = ints([prompt] + [0] * samples)
    for layer in range(layers):
        for pool in (cache.k, cache.v):
            rows = torch.empty(prompt, Hkv, d, dtype=dtype, device=device).normal_(generator=gen)
            at = torch.arange(prompt, device=device)
            pool[layer, cache.table[0, at // page].long(), at % page] = rows
    cache.fork(ints([0] * samples), ints(list(range(1, samples + 1))))
    cache.resize(torch.cat([ints([0]), cache.lens[1:]]))           # the prompt's own sequence ends: its pages live on with the samples
    cache.table, cache.held, cache.lens = cache.table[1:].contiguous(), cache.held[1:].contiguous(), cache.lens[1:].contiguous()
    need = fa.fa_decode_tree_workspace_bytes(samples, nodes, Hq, Hkv, cache.table.shape[1] * page, d)
    ws = torch.empty(max(16, need), dtype=torch.uint8, device=device)
    last = torch.randint(0, vocab, (samples, 1), device=device, generator=gen)
    said = []
    for _ in range(steps):
        parents = random_trees(samples, nodes, gen, device)
        tokens, draft = draft_trees(model, last, parents, gen)
        out, n_accept, _ = step(model, cache, tokens, parents, draft, gen, ws)
        new = torch.gather(out, 1, n_accept[:, None].long())        # the token after the last that stands
        last = torch.where(new >= 0, new, last)
        said.append((out, n_accept))
    return said, cache


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--samples", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--nodes", type=int, default=24)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args()
    run(a.samples, a.prompt, a.nodes, 1, a.layers)                  # (kernels are loaded, pools are warm)
    torch.cuda.synchronize()
    said, cache = run(a.samples, a.prompt, a.nodes, a.steps, a.layers)
    for i, (out, n) in enumerate(said):
        print(f"step {i}: accepted {n.tolist()}, first tokens {out[:, 0].tolist()}")
    print(f"lengths {cache.lens.tolist()}, {int((cache.refs > 0).sum())} of {cache.refs.numel()} pages in use, "
          f"{int((cache.refs > 1).sum())} shared; not served: {int(cache.short)}; status {fa.fa_device_status()[0]}")


if __name__ == "__main__":
    main()
