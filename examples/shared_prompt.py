"""One prompt, several continuations: the shared paged cache end to end.

Prompts are read once (append, prompt attention), forked into continuations that share their pages, each
continuation decodes blocks of draft tokens (append, then the decode kernel over the block's rows), keeps
a different number of them (rollback), some are dropped (their pages come back), and the pool is
compacted. Queries, keys and values come from small tables indexed by token, so that equal tokens give
equal cache rows; the attention of every layer runs as in a decoder of the given head layout.

    python examples/shared_prompt.py [--heads 32 --kv-heads 8 --head-dim 128 --layers 2]
"""
from __future__ import annotations

import argparse
import os
import sys
from typing import List

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2511_09844_gb300 import sd2  # noqa: E402

PAGE = 16


class Cache:
    """The pool with the tables of the live sequences; all of it on the GPU."""

    def __init__(self, layers: int, pages: int, kv_heads: int, head_dim: int, stride: int):
        self.pool = torch.zeros(layers, pages, 2, kv_heads, PAGE, head_dim, dtype=torch.bfloat16, device="cuda")
        self.table = torch.zeros(1, stride, dtype=torch.int32, device="cuda")
        self.length = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.pages = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ref = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def fork(self, parent: List[int], keep: List[int] = None, grow: List[int] = None):
        f = sd2.pages_fork(self.pool, self.table, self.length, _i(parent), None if keep is None else _i(keep),
                           None if grow is None else _i(grow), err=self.err)
        self.table, self.length, self.pages, self.ref = f.table, f.length, f.pages, f.ref

    def compact(self):
        c = sd2.pages_compact(self.pool, self.table, self.pages, self.ref, err=self.err)
        self.table, self.ref = c.table, c.ref
        return int(c.n_live)

    def check(self):
        if int(self.err):
            raise RuntimeError(f"device error bits {int(self.err)}")


def _i(v) -> torch.Tensor:
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Model:
    """Queries, keys and values of every layer, looked up by token."""

    def __init__(self, layers: int, heads: int, kv_heads: int, head_dim: int, vocab: int = 512, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim, self.layers = heads, kv_heads, head_dim, layers
        self.qkv = torch.randn(layers, vocab, heads + 2 * kv_heads, head_dim, generator=g, device="cuda").bfloat16()

    def read(self, cache: Cache, rows: List[List[int]]):
        """Append each sequence's new tokens and attend from them: outputs [layer][sequence][row, heads * hd]."""
        tokens = torch.tensor([t for r in rows for t in r], device="cuda")
        cu = [0]
        for r in rows:
            cu.append(cu[-1] + len(r))
        cache.length = cache.length + _i([len(r) for r in rows])
        out = []
        for layer in range(self.layers):
            x = self.qkv[layer][tokens]
            q, k, v = x.split((self.heads, self.kv_heads, self.kv_heads), dim=1)
            sd2.pages_append(k, v, cache.pool, cache.table, layer, _i(cu), cache.length, err=cache.err)
            o = sd2.attention_prompt(q, cache.pool, cache.table, layer, _i(cu), cache.length, err=cache.err)
            out.append(list(o.split([len(r) for r in rows])))
        return out

    def decode(self, cache: Cache, rows: List[List[int]], max_len: int):
        """The same for short blocks, through the decode kernel."""
        tokens = torch.tensor([t for r in rows for t in r], device="cuda")
        n, cu = [len(r) for r in rows], [0]
        for r in rows:
            cu.append(cu[-1] + len(r))
        cache.length = cache.length + _i(n)
        lens = cache.length.tolist()
        pos = _i([lens[s] - n[s] + i for s in range(len(rows)) for i in range(n[s])])
        out = []
        for layer in range(self.layers):
            x = self.qkv[layer][tokens]
            q, k, v = x.split((self.heads, self.kv_heads, self.kv_heads), dim=1)
            sd2.pages_append(k, v, cache.pool, cache.table, layer, _i(cu), cache.length, err=cache.err)
            o = sd2.attention(q.float().contiguous(), cache.pool, cache.table, layer, pos, _i(cu[:-1]), _i(n),
                              _i(list(range(len(rows)))), max(n), 1, 64 * ((max_len + 63) // 64), err=cache.err)
            out.append(list(o.split(n)))
        return out


def run(heads: int = 32, kv_heads: int = 8, head_dim: int = 128, layers: int = 2, prompts=(70, 200, 33), copies: int = 3,
        block: int = 5, seed: int = 0):
    """The whole story; returns (model, steps), a step being (outputs, the tokens of every sequence up to and with its
    new rows, the number of new rows)."""
    r = torch.Generator().manual_seed(seed)
    draw = lambda n: torch.randint(0, 512, (n,), generator=r).tolist()  # noqa: E731
    model = Model(layers, heads, kv_heads, head_dim, seed=seed)
    longest = max(prompts) + 4 * block
    cache = Cache(layers, pages=2 + copies * sum(-(-(p + 4 * block) // PAGE) for p in prompts), kv_heads=kv_heads,
                  head_dim=head_dim, stride=-(-longest // PAGE) + 1)
    steps = []
    # the prompts: empty sequences with room, read in one packed pass
    seqs = [draw(p) for p in prompts]
    cache.fork([-1] * len(prompts), grow=list(prompts))
    steps.append((model.read(cache, seqs), [list(s) for s in seqs], [len(s) for s in seqs]))
    # every prompt into `copies` continuations with room for a block
    parent = [i for i in range(len(prompts)) for _ in range(copies)]
    cache.fork(parent, grow=[block] * len(parent))
    shared = int((cache.ref > 1).sum())
    seqs = [list(seqs[p]) for p in parent]
    for step in range(2):
        new = [draw(block) for _ in seqs]
        before = [len(s) for s in seqs]
        seqs = [s + n for s, n in zip(seqs, new)]
        steps.append((model.decode(cache, new, longest), [list(s) for s in seqs], [block] * len(seqs)))
        # keep some of each block; the last sequence is dropped after the first round
        kept = [b + 1 + (i + step) % block for i, b in enumerate(before)]
        live = list(range(len(seqs) - (1 if step == 0 else 0)))
        cache.fork(live, keep=[kept[i] for i in live], grow=[block] * len(live))
        seqs = [seqs[i][:kept[i]] for i in live]
    held = int((cache.ref > 0).sum())
    n_live = cache.compact()
    new = [draw(block) for _ in seqs]
    seqs = [s + n for s, n in zip(seqs, new)]
    steps.append((model.read(cache, new), [list(s) for s in seqs], [block] * len(seqs)))
    cache.check()
    print(f"{len(prompts)} prompts, {len(parent)} continuations sharing {shared} pages; {held} pages held at the end, now ids 0..{n_live - 1}")
    return model, steps


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--layers", type=int, default=2)
    a = ap.parse_args()
    run(a.heads, a.kv_heads, a.head_dim, a.layers)


if __name__ == "__main__":
    main()
