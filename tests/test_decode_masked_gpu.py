"""Attention with infinities and NaN where a row does not look: in the keys and
values of new tokens that other rows see."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16

# heads, query heads a key head, dim, block size, new tokens: 16 rows and more
# of each request, as they are shared by 1, 2, 4 and 8 waves; blocks that are no
# multiple of 16 tokens
SHAPES = [(2, 1, 64, 16, [6, 1, 3]), (2, 4, 128, 16, [5, 8, 1]), (1, 2, 128, 7, [9, 14]), (1, 1, 80, 16, [40, 64]),
          (2, 2, 64, 32, [50, 64]), (1, 4, 128, 16, [64, 33]), (1, 3, 256, 16, [7, 20]), (1, 2, 256, 5, [12]), (2, 8, 64, 16, [64, 2])]


def branches(rng, counts):
    """Trees in which the last token has no descendant, so that no other row sees it."""
    masks = []
    for c in counts:
        mine = []
        for i in range(c):
            parent = rng.randint(-1, i - 1)
            mine.append(1 << i | (mine[parent] if parent >= 0 else 0))
        masks += mine
    return masks


def plant(b, r, draft, k=None, v=None):
    pos = b.lens[r] + draft
    block = b.k.shape[1]
    page = int(b.table[r, pos // block])
    if k is not None:
        b.k[page, pos % block] = k
    if v is not None:
        b.v[page, pos % block, :, 1::3] = v


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("tree", [True, False], ids=["tree", "chain"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:4]))
def test_what_a_row_does_not_see_has_no_effect(shape, tree, dtype):
    heads, share, dim, block, counts = shape
    print("masked", shape, tree, dtype, flush=True)
    rng = random.Random(5)
    lens = [rng.choice([0, 17, 300, 1000]) for _ in counts]
    b = D.Batch(17, lens, counts, heads=heads, share=share, dim=dim, block=block, dtype=dtype)
    masks = branches(rng, counts) if tree else None
    odd = []  # (first row of the request, rows, draft with a NaN key)
    at = 0
    for r, c in enumerate(counts):
        if c > 2:
            plant(b, r, c // 2, v=[math.inf, -math.inf, math.nan][r % 3])
            plant(b, r, c - 2, v=-math.inf)
            plant(b, r, c - 1, k=math.nan, v=math.nan)
            odd.append((at, c, c - 1))
        at += c
    ref, spread = b.reference(masks)
    cache = decode.PagedCache(b.k.cuda(), b.v.cuda())
    got = decode.tree_attention(b.q.cuda().contiguous(), cache, b.table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), b.offsets.cuda(),
                                max_new=max(counts), mask=D.signed(masks).cuda() if tree else None).double().cpu()
    here = torch.ones(at, dtype=torch.bool)
    for first, c, draft in odd:  # a row that sees a NaN key: its result is not specified
        for i in range(c):
            here[first + i] = not (masks[first + i] >> draft & 1 if tree else i >= draft)
    ref, spread, got = ref[here], spread[here], got[here]
    assert torch.equal(ref.isnan(), got.isnan())
    assert torch.equal(ref.isposinf(), got.isposinf()) and torch.equal(ref.isneginf(), got.isneginf())
    assert ref.isfinite().any() and (not odd or not ref.isfinite().all())
    finite = ref.isfinite()
    zero = torch.zeros_like(ref)
    D.check_attention(torch.where(finite, got, zero), torch.where(finite, ref, zero), torch.where(finite, spread, zero), dtype)


def test_a_row_that_sees_nothing_is_zero_beside_nan():
    print("masked empty row", flush=True)
    b = D.Batch(3, [0, 0], [3, 20], heads=2, share=2, dim=128, block=16, dtype=HALF)
    b.k[:], b.v[:] = math.nan, math.nan
    got = decode.tree_attention(b.q.cuda().contiguous(), decode.PagedCache(b.k.cuda(), b.v.cuda()), b.table.cuda(),
                                torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda(), max_new=20,
                                mask=torch.zeros(23, dtype=torch.int64, device="cuda"))
    assert not got.any()
