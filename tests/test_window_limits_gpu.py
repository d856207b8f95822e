"""Windows and caches in 4 bits next to the largest positions."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402

import decode_util as D  # noqa: E402
import q4_cache_util as Q  # noqa: E402
import window_util as W  # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
I32 = dict(dtype=torch.int32, device="cuda")


def end_of_a_long_text(count, share, dim, window, sinks):
    """The last blocks, and the first, of a text that ends just below 2^31; the
    others are not in the cache.  (q, k, v, table, length, and the same positions
    one after the other with the window and sinks that leave the same ones)"""
    block = 16
    width = (2 ** 31 - 1) // block
    n = width * block - count - 3
    table = torch.full((1, width), -1, **I32)
    pages = sorted({0, 1} | set(range((n - window) // block - 1, width)))
    for i, page in enumerate(pages):
        table[0, page] = i
    g = torch.Generator().manual_seed(count)
    k, v = (torch.randn((len(pages), block, 1, dim), generator=g).to(BF16) for _ in range(2))
    q = torch.randn((count, share, dim), generator=g).to(BF16)
    kept = len(pages) * block - 3 - count
    return q, k, v, table, n, torch.arange(len(pages), dtype=torch.int32).view(1, -1), kept


@pytest.mark.parametrize("count,share,dim", [(1, 1, 64), (3, 8, 64), (16, 8, 64), (90, 1, 128)])
def test_a_window_at_the_end_of_nearly_2_31_tokens(count, share, dim):
    window, sinks = 100, 5
    print("CASE long window", count, share, dim, flush=True)
    q, k, v, table, n, flat, kept = end_of_a_long_text(count, share, dim, window, sinks)
    scale = 1 / math.sqrt(dim)
    ref, spread = W.attention(q, k, v, flat, [kept], [count], None, scale, window, sinks)
    args = (table, torch.tensor([n], **I32), torch.tensor([0, count], **I32))
    for workspace in ("auto", None):
        got = decode.tree_attention(q.cuda(), decode.PagedCache(k.cuda(), v.cuda()), *args, max_new=count, window=window, sinks=sinks, workspace=workspace)
        D.check_attention(got, ref, spread, BF16, workspace)
    b = Q.Batch.__new__(Q.Batch)
    b.cache = Q.empty(k.shape[0], 16, 1, dim, BF16, 32)
    b.cache.store(k.view(-1, 1, dim).cuda(), v.view(-1, 1, dim).cuda(), torch.arange(k.shape[0] * 16, **I32))
    b.dim, b.group, b.dtype, b.scale, b.q, b.table, b.lens, b.counts = dim, 32, BF16, scale, q, flat, [kept], [count]
    for workspace in ("auto", None):
        got = decode.tree_attention(q.cuda(), b.cache, *args, max_new=count, window=window, sinks=sinks, workspace=workspace)
        b.check(got, None, window, sinks, workspace)


def test_four_bits_over_nearly_2_31_tokens():
    """Without a window: all but a few blocks are not in the cache."""
    print("CASE long codes", flush=True)
    q, k, v, table, n, flat, kept = end_of_a_long_text(2, 4, 64, 50, 0)
    b = Q.Batch.__new__(Q.Batch)
    b.cache = Q.empty(k.shape[0], 16, 1, 64, BF16, 64)
    b.cache.store(k.view(-1, 1, 64).cuda(), v.view(-1, 1, 64).cuda(), torch.arange(k.shape[0] * 16, **I32))
    b.dim, b.group, b.dtype, b.scale, b.q, b.table, b.lens, b.counts = 64, 64, BF16, 0.125, q, flat, [kept], [2]
    b.check(decode.tree_attention(q.cuda(), b.cache, table, torch.tensor([n], **I32), torch.tensor([0, 2], **I32), max_new=2))


@pytest.mark.parametrize("more", [100, 2 ** 31 - 1 - 64])
def test_lengths_past_the_table(more):
    """A text that is longer than the table: what the table has of it is seen, by
    all without a window, and with one as far as the window and sinks reach."""
    block, dim = 16, 64
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((4, block, 1, dim), generator=g).to(BF16) for _ in range(2))
    q = torch.randn((2, 1, dim), generator=g).to(BF16)
    table = torch.arange(4, dtype=torch.int32).view(1, 4)
    n = 64 + more
    b = Q.Batch.__new__(Q.Batch)
    b.cache = Q.empty(4, block, 1, dim, BF16, 64)
    b.cache.store(k.view(-1, 1, dim).cuda(), v.view(-1, 1, dim).cuda(), torch.arange(64, **I32))
    b.dim, b.group, b.dtype, b.scale, b.q, b.table, b.lens, b.counts = dim, 64, BF16, 0.125, q, table, [64], [2]
    args = (table.cuda(), torch.tensor([n], **I32), torch.tensor([0, 2], **I32))
    for window, sinks in [(None, 0), (50, 7), (more + 30, 0), (2 ** 31 + 70, 3)]:
        print("CASE past the table", more, window, sinks, flush=True)
        # the 64 positions as those before two new tokens that are not there: the window reaches as far into them
        reach = 1 << 40 if window is None else window - more
        sees = torch.zeros((2, 64), dtype=torch.bool)
        for i in range(2):
            pos = torch.arange(64)
            sees[i] = (pos < sinks) | (pos >= 64 + i + 1 - reach)
        kk, vv, scale = b.read()
        flat = lambda t: t.reshape(64, dim)  # noqa: E731
        got4 = decode.tree_attention(q.cuda(), b.cache, *args, max_new=2, window=window, sinks=sinks).double().cpu()[:, 0]
        got16 = None if window is None else decode.tree_attention(q.cuda(), decode.PagedCache(k.cuda(), v.cuda()), *args, max_new=2, window=window, sinks=sinks).double().cpu()[:, 0]
        for got, keys, values, size in ((got4, flat(kk), flat(vv), flat(scale) * 8), (got16, flat(k.double()), flat(v.double()), 0)):
            if got is None:
                continue
            for i in range(2):
                if not sees[i].any():
                    assert not got[i].any()
                    continue
                p = torch.softmax(0.125 * (keys[sees[i]] @ q[i, 0].double()), 0)
                ref, spread = p @ values[sees[i]], p @ (values.abs() + size)[sees[i]]
                # one rounding of the result, two of the weights' kind, and of the scores' fp32 sums
                assert ((got[i] - ref).abs() <= 2.0 ** -8 * ref.abs() + (2 * 2.0 ** -8 + 2.0 ** -13) * spread).all()


def test_a_query_that_is_not_finite_is_nan():
    for bad in (math.inf, -math.inf, math.nan):
        for count in (1, 20):
            b = Q.Batch(3, [100], [count], heads=2, share=2, dim=64, block=16, dtype=BF16, group=32)
            b.q[count - 1, 1, 40] = bad
            got = b.attend()
            rows = torch.zeros((count, 4), dtype=torch.bool)
            rows[count - 1, 1] = True
            assert torch.equal(got.isnan().all(2).cpu(), rows) and torch.equal(got.isfinite().all(2).cpu(), ~rows)


@pytest.mark.parametrize("workspace", ["auto", None], ids=["runs", "one"])
@pytest.mark.parametrize("count", [1, 20, 64])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_query_or_a_key_that_is_not_finite_in_one_of_many_runs(bad, count, workspace):
    b = Q.Batch(13, [9000, 12000], [count, count], heads=4, share=2, dim=128, block=16, dtype=BF16, group=64)
    b.q[2 * count - 1, 3, 40] = bad
    page = int(b.table[0, 400])
    b.cache.k_scales[page, 2, 5, 1, 0] = bad
    print("CASE q4 not finite in a run", bad, count, workspace, flush=True)
    for window, sinks in [(None, 0), (8000, 5)]:
        got = b.attend(workspace=workspace, window=window, sinks=sinks)
        rows = torch.zeros(got.shape[:2], dtype=torch.bool)
        rows[2 * count - 1, 3] = True
        rows[:count, 4:6] = True
        assert torch.equal(got.isnan().all(2).cpu(), rows) and torch.equal(got.isfinite().all(2).cpu(), ~rows)
