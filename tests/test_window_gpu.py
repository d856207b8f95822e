"""Attention with a window and sinks against a plain 64-bit implementation."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode, gba  # noqa: E402

import decode_util as D  # noqa: E402
import window_util as W  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gba.lib()
    yield


def tree_masks(rng, counts):
    masks = []
    for c in counts:
        mine = []
        for i in range(c):
            p = rng.randint(max(-1, i - 4), i - 1)
            mine.append(1 << i | (mine[p] if p >= 0 else 0))
        masks += mine
    return masks


def arguments(b):
    return (b.q.cuda(), decode.PagedCache(b.k.cuda(), b.v.cuda()), b.table.cuda(), torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda())


def attend(b, masks=None, **kw):
    return decode.tree_attention(*arguments(b), max_new=max(b.counts), mask=None if masks is None else D.signed(masks).cuda(), **kw)


def check(b, masks, window, sinks, dtype, **kw):
    print("CASE window", window, sinks, b.lens[:6], b.counts[:6], dtype, kw, flush=True)
    tokens = sum(b.counts)
    ref, spread = W.attention(b.q[:tokens], b.k, b.v, b.table, b.lens, b.counts, masks, b.scale, window, sinks)
    D.check_attention(attend(b, masks, window=window, sinks=sinks, **kw)[:tokens], ref, spread, dtype, (window, sinks))


# heads, query heads a key head, dim, block
LAYOUTS = [(1, 1, 64, 16), (2, 4, 128, 16), (1, 8, 80, 7), (2, 1, 8, 1), (1, 3, 256, 32), (1, 16, 96, 100), (2, 2, 120, 64)]
BOUNDS = [(1, 0), (2, 1), (31, 0), (32, 4), (33, 33), (100, 5), (64, 200), (2 ** 31 + 5, 0), (300, 2 ** 40)]


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_single_tokens(layout, dtype):
    heads, share, dim, block = LAYOUTS[layout]
    lens = [0, 1, 15, 16, 17, 31, 32, 63, 64, 65, 127, 129, 200, 333]
    b = D.Batch(layout, lens, [1] * len(lens), heads=heads, share=share, dim=dim, block=block, dtype=dtype, head_major=layout % 2 == 1)
    for window, sinks in BOUNDS:
        check(b, None, window, sinks, dtype)


@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_several_tokens(layout, tree):
    heads, share, dim, block = LAYOUTS[layout]
    rng = random.Random(layout)
    dtype = [HALF, BF16][layout % 2]
    lens, counts = [0, 0, 1, 5, 64, 100, 300, 7], [1, 64, 0, 33, 17, 2, 5, 0]
    b = D.Batch(20 + layout, lens, counts, heads=heads, share=share, dim=dim, block=block, dtype=dtype, head_major=layout % 2 == 0)
    masks = tree_masks(rng, counts) if tree else None
    for window, sinks in BOUNDS:
        check(b, masks, window, sinks, dtype)


def test_any_mask():
    """Bits of later tokens, of none, and past the request's tokens."""
    rng = random.Random(9)
    lens, counts = [0, 0, 3, 40, 500], [5, 64, 8, 20, 64]
    b = D.Batch(31, lens, counts, heads=2, share=2, dim=64, block=16, dtype=BF16)
    masks = [0 if rng.random() < 0.3 else rng.getrandbits(64) for _ in range(sum(counts))]
    for window, sinks in [(1, 0), (7, 0), (20, 2), (20, 45), (64, 5), (200, 0)]:
        check(b, masks, window, sinks, BF16)


@pytest.mark.parametrize("share,dim", [(1, 64), (4, 128), (3, 64), (2, 256), (1, 80)])
def test_prompts(share, dim):
    """Chains that are longer than the window, with cached tokens before them."""
    lens, counts = [0, 37, 700, 64], [700, 401, 300, 1]
    b = D.Batch(41, lens, counts, heads=1, share=share, dim=dim, block=16, dtype=HALF)
    for window, sinks in [(1, 0), (33, 3), (128, 0), (257, 70), (2000, 1)]:
        for workspace in ("auto", None):
            check(b, None, window, sinks, HALF, workspace=workspace)


@pytest.mark.parametrize("share,dim,counts", [(1, 64, [1, 1]), (4, 128, [1, 3]), (4, 128, [40, 64]), (8, 64, [64, 5]), (8, 128, [64, 64])])
def test_long_requests(share, dim, counts):
    """Windows that are split across workgroups, with and without the room for it."""
    rng = random.Random(share)
    b = D.Batch(51 + dim, [9000, 3000], counts, heads=1, share=share, dim=dim, block=16, dtype=BF16)
    masks = tree_masks(rng, counts)
    for window, sinks in [(2500, 0), (4001, 100), (8999, 1)]:
        for workspace in ("auto", None):
            check(b, masks, window, sinks, BF16, workspace=workspace)


def test_many_requests():
    rng = random.Random(77)
    lens = [rng.choice([0, 1, rng.randint(0, 900)]) for _ in range(150)]
    counts = [rng.choice([0, 1, 1, 3]) for _ in lens]
    b = D.Batch(61, lens, counts, heads=2, share=2, dim=64, block=16, dtype=HALF)
    for window, sinks in [(5, 1), (300, 4), (600, 0)]:
        check(b, None, window, sinks, HALF)


@pytest.mark.parametrize("shape", [(2, 4, 128, 16, [6, 1, 3]), (1, 2, 128, 7, [9, 14]), (1, 1, 80, 16, [40, 64]), (2, 2, 64, 32, [50, 64]),
                                   (1, 4, 128, 16, [64, 33]), (1, 3, 256, 16, [7, 20]), (1, 1, 64, 16, [300, 90])],
                         ids=lambda s: "-".join(str(x) for x in s[:4]))
def test_what_a_row_does_not_see_has_no_effect(shape):
    """NaN before the window of all rows, infinities before that of the last one
    and in the tile of the sinks."""
    heads, share, dim, block, counts = shape
    window, sinks = 70, 3
    lens = [1000, 333, 90][: len(counts)]
    b = D.Batch(17, lens, counts, heads=heads, share=share, dim=dim, block=block, dtype=BF16)
    for r, (n, c) in enumerate(zip(lens, counts)):
        sees = W.seen(n, c, window, sinks)
        some, last = sees.any(0), sees[c - 1]
        for pos in range(n + c):
            page = int(b.table[r, pos // block])
            if not some[pos]:
                b.k[page, pos % block] = b.v[page, pos % block] = math.nan
            elif not last[pos] and pos % 5 == 0:
                b.v[page, pos % block, :, 1::3] = math.inf
    ref, spread = W.attention(b.q, b.k, b.v, b.table, lens, counts, None, b.scale, window, sinks)
    print("CASE window unseen", shape, flush=True)
    got = attend(b, window=window, sinks=sinks).double().cpu()
    finite = ref.isfinite()
    assert torch.equal(got.isfinite(), finite) and torch.equal(ref.isposinf(), got.isposinf()) and not finite.all()
    zero = torch.zeros_like(ref)
    D.check_attention(torch.where(finite, got, zero), torch.where(finite, ref, zero), torch.where(finite, spread, zero), BF16)


def test_a_window_over_everything_is_none():
    rng = random.Random(3)
    counts = [3, 17, 1, 64]
    b = D.Batch(5, [50, 700, 1, 0], counts, heads=2, share=4, dim=128, block=16, dtype=HALF)
    for masks in (None, tree_masks(rng, counts)):
        want = attend(b, masks)
        for window, sinks in [(10 ** 6, 0), (5, 10 ** 6)]:
            print("CASE window over all", window, sinks, flush=True)
            assert torch.equal(attend(b, masks, window=window, sinks=sinks), want)


def test_a_chain_as_a_tree_and_as_a_chain():
    counts = [40, 7]
    b = D.Batch(6, [100, 20], counts, heads=1, share=2, dim=64, block=16, dtype=HALF)
    chain = [(1 << i + 1) - 1 for c in counts for i in range(c)]
    for window, sinks in [(1, 0), (5, 0), (30, 25), (64, 4)]:
        a, t = attend(b, None, window=window, sinks=sinks), attend(b, chain, window=window, sinks=sinks)
        ref, spread = W.attention(b.q, b.k, b.v, b.table, b.lens, counts, chain, b.scale, window, sinks)
        D.check_attention(a, ref, spread, HALF)
        D.check_attention(t, ref, spread, HALF)


def test_padding_and_missing_blocks():
    b = D.Batch(81, [50, 20], [2, 3], heads=2, share=2, dim=64, block=16, dtype=HALF, pad=3)
    out = torch.full(b.q.shape, 5.0, dtype=HALF, device="cuda")
    b.table[0, 2], b.table[1, 0] = -1, 10 ** 6
    print("CASE window padding", flush=True)
    got = attend(b, window=30, sinks=2, out=out)
    assert got.data_ptr() == out.data_ptr() and (got[5:] == 5).all()
    check(b, None, 30, 2, HALF)


def test_on_another_stream_and_in_a_graph():
    """A graph follows new lengths: its windows move."""
    b = D.Batch(91, [9000, 500, 9], [4, 4, 4], heads=2, share=4, dim=128, block=16, dtype=BF16)
    q, cache, table, lens, offsets = arguments(b)
    q = q.contiguous()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, ws = torch.empty_like(q), torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode.tree_attention(q, cache, table, lens, offsets, max_new=4, window=3000, sinks=4, out=out, workspace=ws)
    for less in (0, 5, 400, 0):
        now = torch.tensor([max(0, n - less) for n in b.lens], dtype=torch.int32)
        lens.copy_(now)
        out.zero_()
        print("CASE window graph", less, flush=True)
        graph.replay()
        torch.cuda.synchronize()
        there = decode.tree_attention(q, cache, table, lens, offsets, max_new=4, window=3000, sinks=4, stream=side)
        side.synchronize()
        assert torch.equal(out, there)
        ref, spread = W.attention(b.q, b.k, b.v, b.table, now.tolist(), b.counts, None, b.scale, 3000, 4)
        D.check_attention(out, ref, spread, BF16)
    assert not ws[: 1 << 18].any()


def test_refusals():
    b = D.Batch(1, [5], [1], heads=1, share=1, dim=64, block=16, dtype=HALF)
    for kw in (dict(window=0), dict(window=-3), dict(window=4, sinks=-1)):
        with pytest.raises(gba.GbaError):
            attend(b, **kw)
    with pytest.raises(ValueError):
        attend(b, sinks=4)
