"""A decoding step: few-row products with 4-bit weights, the block tables and
slot maps of a paged key/value cache, the cache itself, and the attention of
each request's new tokens over it (one token, a chain or a tree of drafts).

Argument marshalling over libgba.so, like :mod:`paper_2006_12645_amd.gba`:
every step of the computation is a HIP kernel, launched on `stream` or torch's
current one.  The stored forms are those of include/gba.h.  The three handles
(Q4Weight, BlockTables, PagedCache) check the tensors a program keeps once and
hold them; a call checks what it is given, in the extension _gba_decode, since
these calls are bound by the host.  Calls read nothing back from the GPU and may
be captured in a HIP graph.
"""
import ctypes
import math
import os
from typing import NamedTuple, Optional

import torch

from . import gba

DTYPES = {torch.float16: gba.GBA_F16, torch.bfloat16: gba.GBA_BF16}


def _gpu(name, t, dtype, device=None):
    if t.dtype is not dtype or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor of {dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on another device than what it is used with")


def _ints(name, t, shape, device=None):
    """A contiguous int32 CUDA tensor of this shape."""
    _gpu(name, t, torch.int32, device)
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of shape {tuple(shape)}, got {tuple(t.shape)}")


_raw_stream = torch._C._cuda_getCurrentRawStream

_binding = None


def _calls():
    """The extension with the calls (loaded once, after libgba.so).  Raises if
    it has not been built."""
    global _binding
    if _binding is None:
        gba.lib()
        path = os.path.join(gba.PKG, "_gba_decode.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
        from . import _gba_decode
        _gba_decode.set_error(gba.GbaError)
        _binding = _gba_decode
    return _binding


class Q4Weight:
    """A K x N matrix in 4 bits: W[k, j] = scale * (code - zero), one scale
    and zero (8 without `zeros`) for every `group` (32, 64 or 128) k of a
    column.

    codes: int32 (ceil(N/16), ceil(K/128), 64, 4), as q4_pack makes it; scales
    and zeros: fp16 or bf16 (ceil(N/16), ceil(K/group), 16), as q4_groups
    makes them from (ceil(K/group), N).
    """

    def __init__(self, codes, scales, zeros=None, *, K, N, group=128):
        if group not in (32, 64, 128):
            raise ValueError("group must be 32, 64 or 128")
        if scales.dtype not in DTYPES or not scales.is_cuda:
            raise TypeError("scales must be a float16 or bfloat16 CUDA tensor")
        _gpu("codes", codes, torch.int32, scales.device)
        columns, chunks, groups = -(-N // 16), -(-K // 128), -(-K // group)
        if codes.shape != (columns, chunks, 64, 4) or not codes.is_contiguous():
            raise ValueError(f"codes must be a contiguous {(columns, chunks, 64, 4)} tensor, got {tuple(codes.shape)}")
        for name, t in (("scales", scales), ("zeros", zeros)):
            if t is None:
                continue
            _gpu(name, t, scales.dtype, scales.device)
            if t.shape != (columns, groups, 16) or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {(columns, groups, 16)} tensor, got {tuple(t.shape)}")
        self.codes, self.scales, self.zeros = codes, scales, zeros
        self.K, self.N, self.group, self.dtype, self.device = K, N, group, scales.dtype, scales.device
        self._desc = gba.Q4WeightDesc(DTYPES[scales.dtype], group, K, N, codes.data_ptr(), scales.data_ptr(),
                                      None if zeros is None else zeros.data_ptr())
        self._at, self._index, self._linear = ctypes.addressof(self._desc), scales.device.index, _calls().linear


def q4_pack(codes, stream=None):
    """The stored form of a (K, N) uint8 matrix of codes (their low four bits)."""
    _gpu("codes", codes, torch.uint8)
    K, N = codes.shape
    ld = gba._row_major_ld(codes, "codes")
    with torch.cuda.stream(stream):  # (None: as it is)
        packed = torch.empty((-(-N // 16), -(-K // 128), 64, 4), dtype=torch.int32, device=codes.device)
        gba._check(gba.lib().gba_q4_pack(K, N, codes.data_ptr(), ld, packed.data_ptr(), gba._stream_handle(stream, codes.device)),
                   "gba_q4_pack")
    return packed


def q4_groups(per_group):
    """The stored form of (groups, N) scales or zeros: (ceil(N/16), groups, 16)."""
    G, N = per_group.shape
    out = torch.zeros((G, -(-N // 16) * 16), dtype=per_group.dtype, device=per_group.device)
    out[:, :N] = per_group
    return out.view(G, -1, 16).permute(1, 0, 2).contiguous()


def q4_linear(x, w, bias=None, act="none", out=None, stream=None):
    """out = act(x @ W + bias) for a few rows x (M, K) and a Q4Weight.

    x, bias (N,) and out (M, N; allocated when None) are of the weight's
    dtype, x and out row-major with any row stride.
    """
    if stream is not None:
        with torch.cuda.stream(stream):  # its memory for what is allocated
            return w._linear(w._at, w._index, x, bias, out, gba.ACTS[act], stream.cuda_stream)
    return w._linear(w._at, w._index, x, bias, out, gba.ACTS[act], _raw_stream(w._index))


class StepMaps(NamedTuple):
    """What a step needs to know of its new tokens (int32; mask int64)."""
    offsets: torch.Tensor             # (requests + 1,): where each request's tokens begin
    slots: torch.Tensor               # (tokens,): slot in the cache, or -1
    positions: torch.Tensor           # (tokens,): position in the text (a tree's: by depth), or -1
    status: torch.Tensor              # (requests,): 0, 1 no blocks left, 2 too long for the table, 3 too many tokens
    mask: Optional[torch.Tensor] = None  # (tokens,) words, (tokens, 1): which of its request's new tokens one descends from


class BlockTables:
    """The block tables of a batch and the stack of free blocks, on the GPU.

    table (requests, width), held (requests,), free_blocks (num_blocks,) and
    free_count (1,): int32, contiguous, changed in place by step().  tokens:
    room for a step's new tokens (padded entries are -1).  tree: steps take
    parents and give masks.
    """

    def __init__(self, table, held, free_blocks, free_count, block_size, *, tokens, tree=False):
        requests, width = table.shape
        _ints("table", table, (requests, width))
        _ints("held", held, (requests,), table.device)
        _ints("free_blocks", free_blocks, free_blocks.shape[:1], table.device)
        _ints("free_count", free_count, (1,), table.device)
        if block_size < 1 or tokens < 0:
            raise ValueError("block_size must be positive and tokens not negative")
        self.table, self.held, self.free_blocks, self.free_count = table, held, free_blocks, free_count
        self.block_size, self.tokens, self.tree = block_size, tokens, bool(tree)
        self.requests, self.device = requests, table.device
        self._plan = torch.empty(4 * (requests + 1), dtype=torch.int32, device=table.device)  # the step's own scratch
        self._desc = gba.BlockTablesDesc(requests, width, free_blocks.shape[0], block_size, table.data_ptr(), held.data_ptr(),
                                         free_blocks.data_ptr(), free_count.data_ptr(), self._plan.data_ptr())
        self._at, self._index, self._step = ctypes.addressof(self._desc), table.device.index, _calls().step

    @classmethod
    def empty(cls, requests, width, num_blocks, block_size, *, tokens, tree=False, device="cuda"):
        """Tables of requests that hold nothing; every block is free (block 0 is taken first)."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.full((requests, width), -1, **i32), torch.zeros(requests, **i32),
                   torch.arange(num_blocks - 1, -1, -1, **i32), torch.full((1,), num_blocks, **i32), block_size,
                   tokens=tokens, tree=tree)

    def maps(self):
        """Uninitialised StepMaps for step(out=...)."""
        i32 = dict(dtype=torch.int32, device=self.device)
        R, T = self.requests, self.tokens
        mask = torch.empty((T, 1), dtype=torch.int64, device=self.device) if self.tree else None
        return StepMaps(torch.empty(R + 1, **i32), torch.empty(T, **i32), torch.empty(T, **i32), torch.empty(R, **i32), mask)

    def step(self, lens, new, parents=None, out=None, stream=None):
        """Room for each request's new[r] tokens after the lens[r] that it
        keeps: gives back blocks it no longer needs, takes free ones, and
        returns the StepMaps of the new tokens (see gba_tables_step).

        lens, new: int32 (requests,).  parents, with tree=True: int32
        (tokens,), each new token's parent among its request's new ones, -1
        for a root.  out: StepMaps to write (a captured graph's).
        """
        if stream is not None:
            with torch.cuda.stream(stream):
                return StepMaps(*self._step(self._at, self._index, lens, new, parents, self.tokens, self.tree, out, stream.cuda_stream))
        return StepMaps(*self._step(self._at, self._index, lens, new, parents, self.tokens, self.tree, out, _raw_stream(self._index)))


class PagedCache:
    """Keys and values of num_blocks blocks of block_size tokens: k and v,
    (num_blocks, block_size, heads, dim), fp16 or bf16, dim contiguous."""

    def __init__(self, k, v):
        if k.dtype not in DTYPES or not k.is_cuda:
            raise TypeError("k must be a float16 or bfloat16 CUDA tensor")
        _gpu("v", v, k.dtype, k.device)
        if k.dim() != 4 or v.shape != k.shape:
            raise ValueError("k and v must be (num_blocks, block_size, heads, dim)")
        if k.shape[3] > 1 and (k.stride(3) != 1 or v.stride(3) != 1):
            raise ValueError("dim must be contiguous")
        self.k, self.v, self.dtype, self.device = k, v, k.dtype, k.device
        self.num_blocks, self.block_size, self.heads, self.dim = k.shape
        self._scale = 1.0 / math.sqrt(max(self.dim, 1))
        self._desc = gba.PagedCacheDesc(DTYPES[k.dtype], *k.shape, k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3])
        self._at, self._index = ctypes.addressof(self._desc), k.device.index
        self._store, self._attend = _calls().store, _calls().attend

    def store(self, k, v, slots, stream=None):
        """Write the rows k[t], v[t] (tokens, heads, dim) at slots[t] (int32;
        tokens whose slot is outside the cache are left out, the others' slots
        differ)."""
        self._store(self._at, self._index, k, v, slots, _raw_stream(self._index) if stream is None else stream.cuda_stream)


# Scratch of calls with workspace="auto", one per (device, stream): calls in a
# stream's order share one.  A smaller one that was replaced is kept, since a
# graph captured earlier may hold its address; as sizes at least double, those
# kept are together smaller than the one in use.
_scratch = {}
_retired = []


def _more_scratch(nbytes, device, key):
    """A larger scratch buffer of the current stream, of at least nbytes, zeros."""
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError(f"workspace='auto' would allocate {nbytes} bytes while the stream is being captured into a graph; "
                           "pass a zero-filled uint8 CUDA tensor of at least that size as `workspace`, or make one call "
                           "before the capture")
    size = max(nbytes, 1 << 20)
    if key in _scratch:
        _retired.append(_scratch[key])
        size = max(size, 2 * _scratch[key].numel())
    _scratch[key] = torch.zeros(size, dtype=torch.uint8, device=device)
    return _scratch[key]


def tree_attention(q, cache, table, lens, offsets, *, max_new, mask=None, scale=None, out=None, workspace="auto", stream=None):
    """Attention of each request's new tokens over the cache.

    q: (tokens, q_heads, dim) of the cache's dtype, q_heads a multiple of the
    cache's heads; the keys and values of the tokens are in the cache already.
    table (requests, width), lens (requests,) (cached tokens before the new
    ones), offsets (requests + 1,): int32.  max_new: no request has more new
    tokens.  mask: int64 (tokens, 1) or (tokens,), which of its request's new
    tokens each one sees (a StepMaps'); None: those up to itself.  scale:
    1 / sqrt(dim) by default.  workspace: "auto" (a scratch buffer of this
    stream, which a graph captured on it goes on using: its replays must not
    overlap the stream's other calls), None (long requests are not split) or a
    uint8 CUDA tensor, zeros before its first use.
    Rows of padded tokens are not written.
    """
    if stream is not None:
        with torch.cuda.stream(stream):
            return tree_attention(q, cache, table, lens, offsets, max_new=max_new, mask=mask, scale=scale, out=out, workspace=workspace)
    index = cache._index
    raw = _raw_stream(index)
    auto = isinstance(workspace, str)
    ws = _scratch.get((index, raw)) if auto else workspace
    if scale is None:
        scale = cache._scale
    got = cache._attend(cache._at, index, q, table, lens, offsets, max_new, mask, scale, out, ws, auto, raw)
    if type(got) is int:  # the bytes that it needs
        ws = _more_scratch(got, cache.device, (index, raw))
        got = cache._attend(cache._at, index, q, table, lens, offsets, max_new, mask, scale, out, ws, False, raw)
    return got
