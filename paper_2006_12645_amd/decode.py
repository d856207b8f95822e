"""A decoding step: few-row products with 4-bit weights, the block tables and
slot maps of a paged key/value cache, the cache itself, and the attention of
each request's new tokens over it (one token, a chain or a tree of drafts).

Argument marshalling over libgba.so, like :mod:`paper_2006_12645_amd.gba`:
every step of the computation is a HIP kernel, launched on `stream` or torch's
current one.  The stored forms are those of include/gba.h.  The three handles
(Q4Weight, BlockTables, PagedCache) check the tensors a program keeps once and
hold them; a call checks what it is given.  Calls read nothing back from the
GPU and may be captured in a HIP graph.
"""
import ctypes
import math
from typing import NamedTuple, Optional

import torch

from . import gba

DTYPES = {torch.float16: gba.GBA_F16, torch.bfloat16: gba.GBA_BF16}


def _gpu(name, t, dtype):
    if t.dtype is not dtype or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor of {dtype}")


def _ints(name, t, shape, dtype=torch.int32):
    """A contiguous int32 CUDA tensor of this shape."""
    if t.dtype is not dtype or not t.is_cuda:
        raise TypeError(f"{name} must be an int32 CUDA tensor")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of shape {tuple(shape)}, got {tuple(t.shape)}")


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(stream, index):
    """The HIP stream to launch on: `stream`, else torch's current one of device `index`."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(index)
    return gba._stream_handle(stream, torch.device("cuda", index))


def _empty(shape, dtype, device, stream):
    """torch.empty, of the memory of the stream that the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


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
        if codes.dtype is not torch.int32 or not codes.is_cuda:
            raise TypeError("codes must be an int32 CUDA tensor")
        columns, chunks, groups = -(-N // 16), -(-K // 128), -(-K // group)
        if codes.shape != (columns, chunks, 64, 4) or not codes.is_contiguous():
            raise ValueError(f"codes must be a contiguous {(columns, chunks, 64, 4)} tensor, got {tuple(codes.shape)}")
        for name, t in (("scales", scales), ("zeros", zeros)):
            if t is None:
                continue
            _gpu(name, t, scales.dtype)
            if t.shape != (columns, groups, 16) or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {(columns, groups, 16)} tensor, got {tuple(t.shape)}")
        self.codes, self.scales, self.zeros = codes, scales, zeros
        self.K, self.N, self.group, self.dtype, self.device = K, N, group, scales.dtype, scales.device
        self._desc = gba.Q4WeightDesc(DTYPES[scales.dtype], group, K, N, codes.data_ptr(), scales.data_ptr(),
                                      None if zeros is None else zeros.data_ptr())
        self._ref = ctypes.byref(self._desc)
        self._index, self._call = scales.device.index, gba.lib().gba_q4_linear


def q4_pack(codes, stream=None):
    """The stored form of a (K, N) uint8 matrix of codes (their low four bits)."""
    _gpu("codes", codes, torch.uint8)
    K, N = codes.shape
    ld = gba._row_major_ld(codes, "codes")
    packed = _empty((-(-N // 16), -(-K // 128), 64, 4), torch.int32, codes.device, stream)
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
    # A call of a few rows is bound by this function and the launch: plain
    # comparisons, and the weight's handle holds what does not change.
    M, K = x.shape
    dtype, N = w.dtype, w.N
    if K != w.K:
        raise ValueError(f"x has {K} columns, the weight {w.K} rows")
    if x.dtype is not dtype or not x.is_cuda:
        raise TypeError(f"x must be a CUDA tensor of the weight's dtype, {dtype}")
    lda, unit = x.stride()
    if M <= 1:
        lda = K if K > 0 else 1
    if unit != 1 and K > 1 or lda < K:
        raise ValueError("x must be a row-major (M, K) matrix")
    b = None
    if bias is not None:
        if bias.dtype is not dtype or not bias.is_cuda:
            raise TypeError(f"bias must be a CUDA tensor of the weight's dtype, {dtype}")
        if bias.dim() != 1 or bias.shape[0] != N or (N > 1 and bias.stride(0) != 1):
            raise ValueError("bias must be a contiguous (N,) vector")
        b = bias.data_ptr()
    if out is None:
        out = x.new_empty((M, N)) if stream is None else _empty((M, N), dtype, x.device, stream)
        ldc = N if N > 0 else 1
    else:
        if out.dtype is not dtype or not out.is_cuda:
            raise TypeError(f"out must be a CUDA tensor of the weight's dtype, {dtype}")
        if out.shape != (M, N) or (N > 1 and out.stride(1) != 1):
            raise ValueError("out must be a row-major (M, N) matrix")
        ldc = gba._row_major_ld(out, "out")
    status = w._call(w._ref, M, x.data_ptr(), lda, b, gba.ACTS[act], out.data_ptr(), ldc, _stream_of(stream, w._index))
    if status:
        raise gba.GbaError(status, "gba_q4_linear")
    return out


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
        _ints("held", held, (requests,))
        _ints("free_blocks", free_blocks, free_blocks.shape[:1])
        _ints("free_count", free_count, (1,))
        if block_size < 1 or tokens < 0:
            raise ValueError("block_size must be positive and tokens not negative")
        self.table, self.held, self.free_blocks, self.free_count = table, held, free_blocks, free_count
        self.block_size, self.tokens, self.tree = block_size, tokens, tree
        self.requests, self.device = requests, table.device
        self._plan = torch.empty(4 * (requests + 1), dtype=torch.int32, device=table.device)  # the step's own scratch
        self._sizes = [requests + 1, tokens, tokens, requests]
        self._desc = gba.BlockTablesDesc(requests, width, free_blocks.shape[0], block_size, table.data_ptr(), held.data_ptr(),
                                         free_blocks.data_ptr(), free_count.data_ptr(), self._plan.data_ptr())
        self._ref = ctypes.byref(self._desc)
        self._index, self._call, self._shape = table.device.index, gba.lib().gba_tables_step, (requests,)
        # where the maps stand in one allocation: each at a multiple of 16 bytes
        self._at = [0]
        for n in self._sizes:
            self._at.append(self._at[-1] + -(-n // 4) * 4)

    @classmethod
    def empty(cls, requests, width, num_blocks, block_size, *, tokens, tree=False, device="cuda"):
        """Tables of requests that hold nothing; every block is free (block 0 is taken first)."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.full((requests, width), -1, **i32), torch.zeros(requests, **i32),
                   torch.arange(num_blocks - 1, -1, -1, **i32), torch.full((1,), num_blocks, **i32), block_size,
                   tokens=tokens, tree=tree)

    def maps(self, stream=None):
        """Uninitialised StepMaps for step(out=...)."""
        flat = _empty(self._at[4], torch.int32, self.device, stream)
        mask = _empty((self.tokens, 1), torch.int64, self.device, stream) if self.tree else None
        return StepMaps(*(flat.narrow(0, at, n) for at, n in zip(self._at, self._sizes)), mask)

    def step(self, lens, new, parents=None, out=None, stream=None):
        """Room for each request's new[r] tokens after the lens[r] that it
        keeps: gives back blocks it no longer needs, takes free ones, and
        returns the StepMaps of the new tokens (see gba_tables_step).

        lens, new: int32 (requests,).  parents, with tree=True: int32
        (tokens,), each new token's parent among its request's new ones, -1
        for a root.  out: StepMaps to write (a captured graph's).
        """
        T = self.tokens
        _ints("lens", lens, self._shape)
        _ints("new", new, self._shape)
        if (parents is not None) != self.tree:
            raise ValueError("parents come with tree=True" if parents is not None else "a tree's steps need parents")
        if parents is not None:
            _ints("parents", parents, (T,))
        if out is None:
            out = self.maps(stream)
        else:
            for name, t, n in zip(out._fields, out, self._sizes):
                _ints(name, t, (n,))
            if self.tree:
                m = out.mask
                if m is None or m.dtype is not torch.int64 or not m.is_cuda or m.shape != (T, 1) or not m.is_contiguous():
                    raise ValueError("out.mask must be a contiguous int64 (tokens, 1) CUDA tensor")
        status = self._call(self._ref, lens.data_ptr(), new.data_ptr(), None if parents is None else parents.data_ptr(), T,
                            out.offsets.data_ptr(), out.slots.data_ptr(), out.positions.data_ptr(), out.status.data_ptr(),
                            out.mask.data_ptr() if self.tree else None, _stream_of(stream, self._index))
        if status:
            raise gba.GbaError(status, "gba_tables_step")
        return out


class PagedCache:
    """Keys and values of num_blocks blocks of block_size tokens: k and v,
    (num_blocks, block_size, heads, dim), fp16 or bf16, dim contiguous."""

    def __init__(self, k, v):
        if k.dtype not in DTYPES or not k.is_cuda:
            raise TypeError("k must be a float16 or bfloat16 CUDA tensor")
        _gpu("v", v, k.dtype)
        if k.dim() != 4 or v.shape != k.shape:
            raise ValueError("k and v must be (num_blocks, block_size, heads, dim)")
        if k.shape[3] > 1 and (k.stride(3) != 1 or v.stride(3) != 1):
            raise ValueError("dim must be contiguous")
        self.k, self.v, self.dtype, self.device = k, v, k.dtype, k.device
        self.num_blocks, self.block_size, self.heads, self.dim = k.shape
        self._desc = gba.PagedCacheDesc(DTYPES[k.dtype], *k.shape, k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3])
        self._ref = ctypes.byref(self._desc)
        L = gba.lib()
        self._index, self._store, self._attend = k.device.index, L.gba_cache_store, L.gba_tree_attention

    def store(self, k, v, slots, stream=None):
        """Write the rows k[t], v[t] (tokens, heads, dim) at slots[t] (int32;
        tokens whose slot is outside the cache are left out)."""
        dtype, tokens = self.dtype, slots.shape[0]
        want = (tokens, self.heads, self.dim)
        if k.dtype is not dtype or v.dtype is not dtype or not k.is_cuda or not v.is_cuda:
            raise TypeError(f"k and v must be CUDA tensors of the cache's dtype, {dtype}")
        if k.shape != want or v.shape != want:
            raise ValueError(f"k and v must be {want}, got {tuple(k.shape)} and {tuple(v.shape)}")
        kt, kh, k1 = k.stride()
        vt, vh, v1 = v.stride()
        if (k1 != 1 or v1 != 1) and self.dim > 1:
            raise ValueError("dim must be contiguous in k and v")
        _ints("slots", slots, (tokens,))
        status = self._store(self._ref, tokens, k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, slots.data_ptr(),
                             _stream_of(stream, self._index))
        if status:
            raise gba.GbaError(status, "gba_cache_store")


# Scratch of calls with workspace="auto", one per (device, stream): calls in a
# stream's order share one.  A smaller one that was replaced is kept, since a
# graph captured earlier may hold its address.
_scratch = {}
_retired = []


def _scratch_for(nbytes, device, stream):
    key = (device.index, gba._stream_handle(stream, device))
    ws = _scratch.get(key)
    if ws is None or ws.numel() < nbytes:
        if gba.stream_capturing(torch.cuda.current_stream(device) if stream is None else stream):
            raise RuntimeError(f"workspace='auto' would allocate {nbytes} bytes while the stream is being captured into a "
                               "graph; pass a uint8 CUDA tensor of at least that size as `workspace`, or make one call "
                               "before the capture")
        if ws is not None:
            _retired.append(ws)
        ws = _empty(max(nbytes, 1 << 20), torch.uint8, device, stream)
        _scratch[key] = ws
    return ws


def attention_workspace_size(desc):
    """Bytes of workspace a filled AttentionDesc would use to split long requests."""
    n = ctypes.c_size_t(0)
    gba._check(gba.lib().gba_tree_attention_workspace_size(ctypes.byref(desc), ctypes.byref(n)), "gba_tree_attention_workspace_size")
    return n.value


def tree_attention(q, cache, table, lens, offsets, *, max_new, mask=None, scale=None, out=None, workspace="auto", stream=None):
    """Attention of each request's new tokens over the cache.

    q: (tokens, q_heads, dim) of the cache's dtype, q_heads a multiple of the
    cache's heads; the keys and values of the tokens are in the cache already.
    table (requests, width), lens (requests,) (cached tokens before the new
    ones), offsets (requests + 1,): int32.  max_new: no request has more new
    tokens.  mask: int64 (tokens, 1) or (tokens,), which of its request's new
    tokens each one sees (a StepMaps'); None: those up to itself.  scale:
    1 / sqrt(dim) by default.  workspace: "auto" (a scratch buffer of this
    stream), None (long requests are not split) or a uint8 CUDA tensor.
    Rows of padded tokens are not written.
    """
    dtype = cache.dtype
    tokens, heads, dim = q.shape
    requests, width = table.shape
    for name, t in (("q", q), ("out", out)):
        if t is not None and (t.dtype is not dtype or not t.is_cuda):
            raise TypeError(f"{name} must be a CUDA tensor of the cache's dtype, {dtype}")
    if dim != cache.dim or heads % max(cache.heads, 1) != 0:
        raise ValueError(f"q must be (tokens, a multiple of {cache.heads}, {cache.dim}), got {tuple(q.shape)}")
    _ints("table", table, (requests, width))
    _ints("lens", lens, (requests,))
    _ints("offsets", offsets, (requests + 1,))
    if mask is not None:
        if mask.dtype is not torch.int64 or not mask.is_cuda:
            raise TypeError("mask must be an int64 CUDA tensor")
        if mask.numel() != tokens or not mask.is_contiguous():
            raise ValueError("mask must be one contiguous word for each token")
    if out is None:
        out = _empty((tokens, heads, dim), dtype, q.device, stream)
    elif out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    if dim > 1 and (q.stride(2) != 1 or out.stride(2) != 1):
        raise ValueError("dim must be contiguous in q and out")
    qs, os = q.stride(), out.stride()
    d = gba.AttentionDesc(cache._desc, requests, width, tokens, max_new, heads, 1.0 / math.sqrt(dim) if scale is None else scale,
                          q.data_ptr(), qs[0], qs[1], out.data_ptr(), os[0], os[1], table.data_ptr(), lens.data_ptr(),
                          offsets.data_ptr(), None if mask is None else mask.data_ptr(), None, 0)
    if workspace is not None:
        need = attention_workspace_size(d)
        if need > 0:
            ws = _scratch_for(need, q.device, stream) if isinstance(workspace, str) else workspace
            if ws.dtype is not torch.uint8 or not ws.is_cuda:
                raise TypeError("workspace must be a uint8 CUDA tensor")
            d.workspace, d.workspace_bytes = ws.data_ptr(), ws.numel()
    gba._check(gba.lib().gba_tree_attention(ctypes.byref(d), gba._stream_handle(stream, q.device)), "gba_tree_attention")
    return out
