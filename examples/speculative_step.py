"""Speculative decoding with the operators of a decoding step.

One layer of a model with random weights in 4 bits -- attention over a paged
cache, then a feed-forward network -- serves a few requests: a prompt each,
then, step after step, a tree of drafted tokens, of which a path is accepted.
Every step is

    q, k, v = x.Wqkv               decode.q4_linear
    maps    = tables.step(...)     where each new token goes
    cache.store(k, v, maps.slots)
    a       = decode.tree_attention(q, cache, tables.table, lens, maps.offsets, ...)
    x       = x + a.Wo;  x + relu(x.Wup + bias).Wdown

and nothing is read back from the GPU between them.  For its check the program
then decodes the accepted tokens once more, one at a time, into a cache of its
own: a drafted token sees the tokens that it descends from, and so its row of
the tree's step has to be the row of the step that decodes it alone.

    python examples/speculative_step.py
"""
import argparse
import os
import random
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2006_12645_amd import decode  # noqa: E402


class Layer:
    def __init__(self, width, heads, key_heads, hidden, dtype, group=64):
        self.width, self.heads, self.key_heads, self.dim = width, heads, key_heads, width // heads
        self.qkv = self._weight(width, (heads + 2 * key_heads) * self.dim, dtype, group)
        self.out = self._weight(width, width, dtype, group)
        self.up = self._weight(width, hidden, dtype, group)
        self.down = self._weight(hidden, width, dtype, group)
        self.up_bias = (torch.randn(hidden, device="cuda") * 0.1).to(dtype)

    @staticmethod
    def _weight(K, N, dtype, group):
        """Round a random matrix to 4 bits: a scale and a zero point for every
        `group` values of a column."""
        w = torch.randn(K, N, device="cuda") * K ** -0.5
        parts = w.view(K // group, group, N)
        low, high = parts.amin(1), parts.amax(1)
        scale = ((high - low) / 15).to(dtype)
        zero = (-low / scale.float()).round().to(dtype)
        codes = (parts / scale.float().unsqueeze(1) + zero.float().unsqueeze(1)).round().clamp(0, 15).to(torch.uint8).view(K, N)
        return decode.Q4Weight(decode.q4_pack(codes), decode.q4_groups(scale), decode.q4_groups(zero), K=K, N=N, group=group)

    def __call__(self, x, cache, tables, maps, lens, max_new):
        H, G, D = self.heads, self.key_heads, self.dim
        qkv = decode.q4_linear(x, self.qkv).view(-1, H + 2 * G, D)
        cache.store(qkv[:, H:H + G], qkv[:, H + G:], maps.slots)
        a = decode.tree_attention(qkv[:, :H], cache, tables.table, lens, maps.offsets, max_new=max_new, mask=maps.mask)
        x = x + decode.q4_linear(a.view(-1, self.width), self.out)
        return x + decode.q4_linear(decode.q4_linear(x, self.up, self.up_bias, act="relu"), self.down)


class Server:
    """A cache and its tables for some requests, and a layer over it."""

    def __init__(self, layer, requests, longest, block, tokens, dtype, tree):
        blocks = requests * (-(-longest // block)) + requests
        shape = (blocks, block, layer.key_heads, layer.dim)
        self.layer, self.block = layer, block
        self.cache = decode.PagedCache(torch.empty(shape, dtype=dtype, device="cuda"), torch.empty(shape, dtype=dtype, device="cuda"))
        self.tables = decode.BlockTables.empty(requests, -(-longest // block), blocks, block, tokens=tokens, tree=tree)

    def step(self, x, lens, new, max_new, parents=None):
        """Rows x of the new tokens, one after the other (padded to the tables'
        size); lens, new: int32 tensors."""
        maps = self.tables.step(lens, new, parents)
        return self.layer(x, self.cache, self.tables, maps, lens, max_new), maps


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def padded(rows, tokens):
    out = rows.new_zeros((tokens, rows.shape[1]))
    out[: len(rows)] = rows
    return out


def run(requests=4, steps=3, drafts=16, prompt=40, width=1024, heads=8, key_heads=2, hidden=4096, block=16, dtype=torch.float16, seed=0):
    """Serves, checks, and returns the largest difference between a drafted
    token's row and that of the same token decoded alone, over the rows' root
    mean square."""
    torch.manual_seed(seed)
    rng = random.Random(seed)
    layer = Layer(width, heads, key_heads, hidden, dtype)
    longest = prompt + steps * (drafts + 1)
    tree = Server(layer, requests, longest, block, requests * max(prompt, drafts), dtype, tree=True)
    alone = Server(layer, requests, longest, block, requests * prompt, dtype, tree=False)
    # prompts: chains, here as trees whose every token hangs from the one before it (at most 64 tokens)
    lens = [rng.randint(prompt // 2, prompt) for _ in range(requests)]
    rows = torch.randn(sum(lens), width, device="cuda").to(dtype)
    chain = ints([i - 1 for n in lens for i in range(n)] + [-1] * (tree.tables.tokens - sum(lens)))
    none = ints([0] * requests)
    got, _ = tree.step(padded(rows, tree.tables.tokens), none, ints(lens), prompt, chain)
    want, _ = alone.step(padded(rows, alone.tables.tokens), none, ints(lens), prompt)
    worst = float((got[: len(rows)] - want[: len(rows)]).abs().max() / want[: len(rows)].float().square().mean().sqrt())
    for _ in range(steps):
        count = [rng.randint(drafts // 2, drafts) for _ in lens]
        parents = [[rng.randint(max(-1, t - 4), t - 1) for t in range(c)] for c in count]
        rows = torch.randn(sum(count), width, device="cuda").to(dtype)
        flat = sum(parents, [])
        got, maps = tree.step(padded(rows, tree.tables.tokens), ints(lens), ints(count), drafts,
                              ints(flat + [-1] * (tree.tables.tokens - len(flat))))
        assert not maps.status.any(), "no room"
        # accept a path from a root to a random token
        first, paths = 0, []
        for c, up in zip(count, parents):
            path, t = [], rng.randrange(c)
            while t >= 0:
                path.append(first + t)
                t = up[t]
            paths.append(path[::-1])
            first += c
        # the same tokens, one a request and step
        for i in range(max(map(len, paths))):
            now = [1 if i < len(p) else 0 for p in paths]
            at = [p[i] for p in paths if i < len(p)]
            want, maps = alone.step(padded(rows[at], alone.tables.tokens), ints([n + min(i, len(p)) for n, p in zip(lens, paths)]), ints(now), 1)
            assert not maps.status.any(), "no room"
            difference = (got[at].float() - want[: len(at)].float()).abs().max()
            worst = max(worst, float(difference / want[: len(at)].float().square().mean().sqrt()))
        # The accepted tokens' keys stand where the tree had them, not in their
        # order: they are stored again, by their slots in a chain.
        kept = [p for path in paths for p in path]
        chain = ints([i - 1 for p in paths for i in range(len(p))] + [-1] * (tree.tables.tokens - len(kept)))
        tree.step(padded(rows[kept], tree.tables.tokens), ints(lens), ints([len(p) for p in paths]), drafts, chain)
        lens = [n + len(p) for n, p in zip(lens, paths)]
    return worst


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--steps", type=int, default=3)
    ap.add_argument("--drafts", type=int, default=16)
    a = ap.parse_args()
    worst = run(requests=a.requests, steps=a.steps, drafts=a.drafts)
    print(f"{a.steps} steps of {a.requests} requests with trees of up to {a.drafts} drafts: rows of accepted tokens "
          f"differ from those decoded alone by at most {worst:.2g} of their root mean square")


if __name__ == "__main__":
    main()
