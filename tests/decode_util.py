"""Plain 64-bit implementations of the decoding operators and the inputs of
their tests."""
import math

import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # unit roundoff


# ------------------------------------------------------------------ linear

def dequantized(codes, scales, zeros, group):
    """(K, N) codes and (G, N) scales and zeros as a 64-bit matrix."""
    g = torch.arange(codes.shape[0], device=codes.device) // group
    z = 8.0 if zeros is None else zeros.double()[g]
    return (codes.double() - z) * scales.double()[g]


def activated(x, act):
    return {"none": lambda v: v, "relu": lambda v: v.clamp_min(0), "sigmoid": torch.sigmoid, "tanh": torch.tanh}[act](x)


# ------------------------------------------------------------------ tables

class TableModel:
    """The block tables in plain Python lists, one request after the other."""

    def __init__(self, requests, width, num_blocks, block):
        self.table = [[-1] * width for _ in range(requests)]
        self.held = [0] * requests
        self.free = list(range(num_blocks - 1, -1, -1))
        self.width, self.block = width, block

    def step(self, lens, new, parents, tokens):
        lens, new = [max(0, n) for n in lens], [max(0, c) for c in new]
        need = [-(-(n + c) // self.block) for n, c in zip(lens, new)]
        ends, total = [], 0
        for c in new:
            total += c
            ends.append(total)
        status = [2 if need[r] > self.width else 3 if ends[r] > tokens or (parents is not None and new[r] > 64) else 0
                  for r in range(len(lens))]
        for r, row in enumerate(self.table):
            for col in range(need[r], self.held[r]):
                self.free.append(row[col])
                row[col] = -1
            self.held[r] = min(self.held[r], need[r])
        short = False
        for r, row in enumerate(self.table):
            want = need[r] - self.held[r]
            if status[r] or want <= 0:
                continue
            short = short or want > len(self.free)
            if short:
                status[r] = 1
                continue
            for col in range(self.held[r], need[r]):
                row[col] = self.free.pop()
            self.held[r] = need[r]
        offsets = [min(v, tokens) for v in [0] + ends]
        slots, positions, mask = [-1] * tokens, [-1] * tokens, [0] * tokens
        for r in range(len(lens)):
            first, here = offsets[r], offsets[r + 1] - offsets[r]
            if parents is not None and here > 64:
                continue
            for i in range(here):
                pos = lens[r] + i
                if status[r] == 0:
                    slots[first + i] = self.table[r][pos // self.block] * self.block + pos % self.block
                depth = i
                if parents is not None:
                    p = parents[first + i]
                    mask[first + i] = 1 << i | (mask[first + p] if 0 <= p < i else 0)
                    depth = bin(mask[first + i]).count("1") - 1
                positions[first + i] = lens[r] + depth
        mask = [m - (1 << 64) if m >> 63 else m for m in mask]
        return offsets, slots, positions, status, mask if parents is not None else None


# --------------------------------------------------------------- attention

def attention(q, k_cache, v_cache, table, lens, counts, mask, scale):
    """(out, sum of weights times |v|) in 64 bits, on the CPU; rows past the
    last request's tokens are left at zero.  `mask`: a list of words or None."""
    H, D = k_cache.shape[2], k_cache.shape[3]
    block = k_cache.shape[1]
    share = q.shape[1] // H
    q, k_cache, v_cache, table = q.double().cpu(), k_cache.cpu(), v_cache.cpu(), table.cpu()
    out, spread = torch.zeros_like(q), torch.zeros_like(q)
    at = 0
    for r, (n, c) in enumerate(zip(lens, counts)):
        pos = torch.arange(min(n + c, table.shape[1] * block))
        page = table[r, pos // block].long()
        there = (page >= 0) & (page < k_cache.shape[0])
        pos, page = pos[there], page[there]
        k, v = k_cache[page, pos % block].double(), v_cache[page, pos % block].double()
        for i in range(c):
            draft = pos - n
            sees = draft <= i if mask is None else \
                (draft < 0) | torch.tensor([0 <= d < 64 and bool(mask[at + i] >> d & 1) for d in draft.tolist()], dtype=torch.bool)
            if not sees.any():
                continue
            for h in range(q.shape[1]):
                kk, vv = k[sees, h // share], v[sees, h // share]
                p = torch.softmax(scale * (kk @ q[at + i, h]), 0)
                out[at + i, h] = p @ vv
                spread[at + i, h] = p @ vv.abs()
        at += c
    return out, spread


def check_attention(got, ref, spread, dtype, what=""):
    """Each weight is rounded to the cache's type (u relative, and their sum
    with them: 2 u of the sum of weights times |v|), a score's fp32 sum moves
    its weight by less than 2^-14, and the result is rounded once."""
    u = U[dtype]
    err = (got.double().cpu() - ref).abs()
    bound = u * ref.abs() + (2 * u + 2.0 ** -14) * spread
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((err / bound.clamp_min(1e-30)).max()), bad.nonzero()[:3].tolist())


class Batch:
    """A paged cache with these requests in it: blocks in random order, NaN
    wherever no request's token is."""

    def __init__(self, seed, lens, counts, *, heads, share, dim, block, dtype, head_major=False, pad=0, q_scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.counts, self.scale, self.dtype = lens, counts, 1.0 / math.sqrt(dim), dtype
        need = [-(-(n + c) // block) for n, c in zip(lens, counts)]
        blocks, width = sum(need) + 2, max(need + [1]) + 1
        order = torch.randperm(blocks, generator=g)
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32)
        shape = (blocks, heads, block, dim) if head_major else (blocks, block, heads, dim)
        k, v = torch.full(shape, math.nan), torch.full(shape, math.nan)
        if head_major:
            k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
        at = 0
        for r, (n, c) in enumerate(zip(lens, counts)):
            mine = order[at:at + need[r]]
            at += need[r]
            self.table[r, : need[r]] = mine
            pos = torch.arange(n + c)
            k[mine[pos // block], pos % block] = torch.randn((n + c, heads, dim), generator=g)
            v[mine[pos // block], pos % block] = torch.randn((n + c, heads, dim), generator=g)
        tokens = sum(counts)
        # q as a slice of a fused projection, and rows of padding after it
        wide = torch.randn((tokens + pad, (share + 2) * heads, dim), generator=g) * q_scale
        self.offsets = torch.tensor([sum(counts[:r]) for r in range(len(counts) + 1)], dtype=torch.int32)
        self.k, self.v = k.to(dtype), v.to(dtype)
        self.q = wide.to(dtype)[:, : share * heads]

    def reference(self, mask=None):
        tokens = sum(self.counts)
        return attention(self.q[:tokens], self.k, self.v, self.table, self.lens, self.counts, mask, self.scale)


def signed(words):
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64).view(-1, 1)
