"""The cache in 4 bits in plain 64-bit arithmetic: its stored form, how it is
rounded to, and attention over it."""
import math

import torch

from paper_2006_12645_amd import decode

import decode_util as D
import window_util as W


def width_of(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def element_places(dim, keys):
    """(byte, shift) of each element of a stored row."""
    width, places = width_of(dim), []
    for d in range(dim):
        word = d // 8
        if keys:
            word = (width // 32) * (word % 4) + word // 4
        places.append((4 * word + d % 8 // 2, 4 * (d % 2)))
    return places


def codes_of(stored, dim, keys):
    """(..., dim) codes of (..., width / 2) bytes."""
    byte, shift = (torch.tensor(v) for v in zip(*element_places(dim, keys)))
    return stored.cpu().long()[..., byte] >> shift & 15


def values(stored, scales, dim, group, keys):
    """What rows stand for, in 64 bits; and their scales, element by element."""
    of = torch.arange(dim) // group
    pair = scales.double().cpu()[..., of, :]
    return pair[..., 0] * (codes_of(stored, dim, keys) - 8) + pair[..., 1], pair[..., 0]


def rounded(x, group):
    """(codes, scales, offsets) of rows x (..., dim): the definition, each fp32
    step in 64 bits and rounded."""
    single, dtype, x = lambda v: v.float().double(), x.dtype, x.double().cpu()  # noqa: E731
    fifteenth = single(torch.tensor(2 / 15, dtype=torch.float64))
    codes, scales, offsets = torch.empty(x.shape, dtype=torch.long), [], []
    for d in range(0, x.shape[-1], group):
        v = x[..., d:d + group]
        low, high = v.amin(-1, keepdim=True), v.amax(-1, keepdim=True)  # (NaN if one is)
        finite = v.isfinite().all(-1, keepdim=True)
        scale = single(single(high / 2 - low / 2) * fifteenth).to(dtype).double()
        scale = torch.where(finite & (scale >= 2.0 ** -100), scale, 0.0)
        offset = torch.where(finite, single(low + 8 * scale), math.nan).to(dtype).double()
        steps = single(single(v - offset) * single(1 / scale))
        codes[..., d:d + group] = torch.where(scale > 0, (steps.round() + 8).clamp(0, 15), 8).long()
        scales.append(scale)
        offsets.append(offset)
    return codes, torch.cat(scales, -1), torch.cat(offsets, -1)


def empty(blocks, block, heads, dim, dtype, group):
    """A cache of any codes with scales and offsets that are NaN."""
    cache = decode.Q4Cache.empty(blocks, block, heads, dim, dtype, group=group)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=torch.Generator().manual_seed(7), dtype=torch.uint8))
    cache.k_scales.fill_(math.nan)
    cache.v_scales.fill_(math.nan)
    return cache


class Batch(D.Batch):
    """The requests of a decode_util.Batch in a cache of 4 bits."""

    def __init__(self, seed, lens, counts, *, heads, share, dim, block, dtype, group, **kw):
        super().__init__(seed, lens, counts, heads=heads, share=share, dim=dim, block=block, dtype=dtype, **kw)
        self.group, self.dim = group, dim
        self.cache = empty(self.k.shape[0], block, heads, dim, dtype, group)
        at = [(int(self.table[r, p // block]) * block + p % block) for r, (n, c) in enumerate(zip(lens, counts)) for p in range(n + c)]
        slots = torch.tensor(at, dtype=torch.int32)
        rows = lambda t: t.reshape(-1, heads, dim)[slots.long()].cuda()  # noqa: E731
        self.cache.store(rows(self.k), rows(self.v), slots.cuda())

    def read(self):
        """k, v and the scales of v as a paged cache's, (num_blocks, block_size, heads, dim), in 64 bits."""
        c = self.cache
        k, _ = values(c.k, c.k_scales, self.dim, self.group, True)
        v, scale = values(c.v, c.v_scales, self.dim, self.group, False)
        return [t.permute(0, 2, 1, 3) for t in (k, v, scale)]

    def arguments(self):
        return (self.q.cuda(), self.cache, self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), self.offsets.cuda())

    def attend(self, masks=None, **kw):
        return decode.tree_attention(*self.arguments(), max_new=max(self.counts), mask=None if masks is None else D.signed(masks).cuda(), **kw)

    def check(self, got, masks=None, window=None, sinks=0, what="", lens=None):
        """A score's fp32 sums move its weight by less than 2^-14; the second
        product's fp32 sums are of 16 + code and 24, so that each key's error is at
        most 2^-13 of its weight times |value| + 8 scales.  There the weight times
        the scale is rounded: to 16 bits and more in fp16, within that, and to bf16
        once in bf16, where it multiplies code - 8 (what is taken from 16 + code is
        24 times the sum of the rounded ones) and so adds at most 2^-8 of the weight
        times scale |code - 8|.  The result is rounded once."""
        tokens = sum(self.counts)
        k, v, scale = self.read()
        lens = self.lens if lens is None else lens
        args = (self.table, lens, self.counts, masks, self.scale, 1 << 40 if window is None else window, sinks)
        ref, _ = W.attention(self.q[:tokens], k, v, *args)
        size, _ = W.attention(self.q[:tokens], k, v.abs() + 8 * scale.abs(), *args)
        got = got[:tokens].double().cpu()
        if self.dtype is torch.bfloat16:
            c = self.cache
            steps = scale.abs() * (codes_of(c.v, self.dim, False) - 8).abs().permute(0, 2, 1, 3)
            size = size + 2.0 ** 5 * W.attention(self.q[:tokens], k, steps, *args)[0]  # (2^-8 over 2^-13)
        finite = ref.isfinite()
        assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isfinite(), finite), (what, "NaN")
        err, bound = (got - ref).abs()[finite], (D.U[self.dtype] * ref.abs() + 2.0 ** -13 * size)[finite]
        bad = ~(err <= bound)
        assert not bad.any(), (what, int(bad.sum()), float((err / bound.clamp_min(1e-30)).max()))
