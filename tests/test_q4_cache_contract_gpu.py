"""What include/gba.h says of attention over a cache in 4 bits: queries that are
not finite in rows that see nothing, and how much of a weight the second product
has of each type."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402

import q4_cache_util as Q  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("window", [None, 3])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
def test_a_query_that_is_not_finite_and_sees_nothing(dtype, bad, window):
    b = Q.Batch(5, [0, 40, 0], [3, 2, 1], heads=1, share=2, dim=64, block=16, dtype=dtype, group=32)
    b.q[:, 1, 7] = bad
    masks = [0, 2, 0, 1, 3, 0]  # of 0 cached tokens, 40 and 0
    print("CASE q4 nothing seen", dtype, bad, window, flush=True)
    got = b.attend(masks, window=window)
    for row, sees in enumerate((False, True, False, True, True, False)):
        assert got[row, 1].isnan().all() if sees else not got[row].any(), row
        assert got[row, 0].isfinite().all(), row


@pytest.mark.parametrize("dtype,u", [(HALF, 2.0 ** -16), (BF16, 2.0 ** -8)], ids=["f16", "bf16"])
def test_weights_of_the_second_product(dtype, u):
    """One key of code 15 and scale 1 among some of code 8 and scale 0, offsets 0: the
    result is 7 times the key's weight w over the sum of all, with w rounded once
    to bf16 (u = 2^-8), or to two bf16 numbers, each next to what it stands for
    (2^-8 of what the first left, which is 2^-8 of w), and the result once.  (The sums
    of 31 w and of 24 w: 55 w 2^-24 each, below 2^-16 w.)"""
    n = 9
    cache = Q.empty(1, 16, 1, 64, dtype, 64)
    cache.k.fill_(0x88)
    cache.v.fill_(0x88)
    cache.k_scales[..., 0], cache.k_scales[..., 1] = 0.0, 0.0
    cache.v_scales[..., 0], cache.v_scales[..., 1] = 0.0, 0.0
    cache.k_scales[0, 0, 0, 0, 1] = 1.0   # key 0: all of its elements are 1
    cache.v[0, 0, 0] = 0xFF
    cache.v_scales[0, 0, 0, 0, 0] = 1.0
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.zeros((40, 1, 64), dtype=dtype, device="cuda")
    q[:, 0, 0] = torch.linspace(-3, 3, 40).to(dtype)
    print("CASE q4 weights", dtype, flush=True)
    got = decode.tree_attention(q, cache, i(*([0] * 40)).view(40, 1), i(*([n - 1] * 40)), i(*range(41)), max_new=1, scale=1.0).double().cpu()[:, 0]
    s = q.double().cpu()[:, 0, 0]
    w = 7 * s.exp() / (s.exp() + n - 1)
    r = 2.0 ** -11 if dtype is HALF else 2.0 ** -8
    assert ((got - w.view(-1, 1)).abs() <= (r + u + 2.0 ** -16) * w.view(-1, 1)).all()
