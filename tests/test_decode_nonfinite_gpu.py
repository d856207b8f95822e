"""Infinities and NaN that a row does see: they reach the result, however a
request is split."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16

# kept tokens, new tokens, key heads, query heads a key head, dim, block: one
# run; runs that the last workgroup joins; runs that a second kernel joins, few
# rows and, from 4096 rows on, many
SHAPES = {"whole": ([100, 3], [2, 1], 2, 2, 64, 16), "in_place": ([1500, 1000], [1, 2], 2, 2, 64, 16), "rows_apart": ([9000, 700], [3, 1], 2, 4, 128, 16),
          "odd_blocks": ([3000], [5], 1, 2, 80, 7), "shared_tiles": ([2000, 900], [20, 64], 1, 4, 128, 16),
          "many_rows": ([3000, 400], [64, 64], 4, 8, 64, 16)}
CALLS = [(name, ws) for name in SHAPES for ws in ("auto", None)]


def batch(name, dtype, seed):
    lens, counts, heads, share, dim, block = SHAPES[name]
    return D.Batch(seed, lens, counts, heads=heads, share=share, dim=dim, block=block, dtype=dtype)


def attend(b, ws):
    return decode.tree_attention(b.q.cuda().contiguous(), decode.PagedCache(b.k.cuda(), b.v.cuda()), b.table.cuda(),
                                 torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda(), max_new=max(b.counts), workspace=ws)


def put(b, r, pos, k=None, v=None):
    block = b.k.shape[1]
    page = int(b.table[r, pos // block])
    if k is not None:
        b.k[page, pos % block] = k
    if v is not None:
        b.v[page, pos % block, :, 1::3] = v


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("name,ws", CALLS)
def test_a_query_that_is_nan(name, ws, dtype):
    """All scores of the row are NaN, so it is, and no other row."""
    print("CASE nan query", name, ws, dtype, flush=True)
    b = batch(name, dtype, 5)
    b.q = b.q.clone()
    b.q[0, 1, 3] = math.nan
    b.q[-1, 0] = math.nan
    got = attend(b, ws)
    odd = torch.zeros(got.shape[:2], dtype=torch.bool)
    odd[0, 1] = odd[-1, 0] = True
    assert torch.equal(got.isnan().all(2).cpu(), odd)
    assert torch.equal(got.isnan().any(2).cpu(), odd)


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("name,ws", CALLS)
def test_a_key_that_is_nan(name, ws, dtype):
    """A cached key that every row of its request sees."""
    print("CASE nan key", name, ws, dtype, flush=True)
    b = batch(name, dtype, 6)
    put(b, 0, b.lens[0] // 2, k=math.nan)
    got = attend(b, ws).isnan().cpu()
    assert got[: b.counts[0]].all() and not got[b.counts[0]:].any()


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("place", [0.0, 0.4, 0.95])
@pytest.mark.parametrize("name,ws", CALLS)
def test_a_value_that_is_infinite(name, ws, place, dtype):
    """A cached value that every row of its request sees: its elements are what
    the formula says, the others as without it."""
    print("CASE infinite value", name, ws, place, dtype, flush=True)
    b = batch(name, dtype, 7)
    put(b, 0, int(place * b.lens[0]), v=-math.inf)
    ref, spread = b.reference()
    got = attend(b, ws)
    finite = ref.isfinite()
    assert torch.equal(ref.isneginf(), got.isneginf().cpu()) and not got.isnan().any() and not got.isposinf().any()
    zero = torch.zeros_like(ref)
    D.check_attention(torch.where(finite, got.double().cpu(), zero), torch.where(finite, ref, zero), torch.where(finite, spread, zero), dtype)
