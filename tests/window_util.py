"""A plain 64-bit implementation of attention with a window and sinks."""
import torch


def seen(n, c, window, sinks, words=None, ends=None):
    """(c, positions) truth values: which positions each of the c new tokens
    after n cached ones sees.  words: their masks; ends: positions there are."""
    total = n + c if ends is None else min(n + c, ends)
    pos = torch.arange(total)
    out = torch.zeros((c, total), dtype=torch.bool)
    for i in range(c):
        fresh = range(i + 1) if words is None else [j for j in range(c) if j < 64 and words[i] >> j & 1]
        text = n + len(fresh)  # its length
        out[i, :n] = ((pos < sinks) | (pos >= text - window))[: min(n, total)]
        for place, j in enumerate(fresh):
            if n + j < total:
                out[i, n + j] = n + place < sinks or n + place >= text - window
    return out


def attention(q, k, v, table, lens, counts, mask, scale, window, sinks):
    """(out, sum of weights times |v|) in 64 bits, on the CPU; k and v are a
    paged cache's, (num_blocks, block_size, heads, dim)."""
    H, block = k.shape[2], k.shape[1]
    share = q.shape[1] // H
    q, k, v, table = q.double().cpu(), k.double().cpu(), v.double().cpu(), table.cpu()
    out, spread = torch.zeros_like(q), torch.zeros_like(q)
    at = 0
    for r, (n, c) in enumerate(zip(lens, counts)):
        sees = seen(n, c, window, sinks, None if mask is None else mask[at:at + c], table.shape[1] * block)
        pos = torch.arange(sees.shape[1])
        page = table[r, pos // block].long()
        sees &= (page >= 0) & (page < k.shape[0])
        used = sees.any(0)
        pos, page, sees = pos[used], page[used], sees[:, used]
        rows = sees.any(1)
        for h in range(q.shape[1]):
            kk, vv = k[page, pos % block, h // share], v[page, pos % block, h // share]
            s = (scale * (q[at:at + c, h] @ kk.t())).masked_fill(~sees, -float("inf"))
            p = torch.where(sees & rows.view(-1, 1), torch.softmax(s, 1), 0.0)
            there = vv.isfinite().all()
            for i in range(c) if not there else ():  # (0 times an infinity is not a term)
                out[at + i, h] = p[i, sees[i]] @ vv[sees[i]]
            if there:
                out[at:at + c, h] = p @ vv
            spread[at:at + c, h] = p @ vv.abs().nan_to_num(0.0, 0.0)
        at += c
    return out, spread
