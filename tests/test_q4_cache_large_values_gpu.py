"""Attention over a cache in 4 bits whose values, keys or queries are next to
bf16's largest, where a sum of (16 + code) scales, or of 24 scales, is no fp32
number although the result is one.

Scales and offsets are multiplied by powers of two, so the references and bounds
are those of ordinary values, multiplied likewise."""
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402

import decode_util as D  # noqa: E402
import q4_cache_util as Q  # noqa: E402
from test_window_gpu import tree_masks  # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

# heads, query heads a key head, dim, block, group, cached tokens, new tokens:
# whole requests, runs, trees, every layout of groups
SHAPES = {"whole": (2, 4, 128, 16, 64, [100, 3, 0], [1, 2, 5]), "runs": (1, 8, 64, 16, 32, [9000, 700], [2, 1]), "trees": (2, 4, 128, 32, 32, [300, 1000], [64, 17]),
          "wide": (1, 2, 256, 16, 128, [500, 40], [1, 20]), "one group": (2, 3, 64, 48, 64, [3000], [4]), "padded": (1, 5, 136, 16, 32, [200], [3])}
CALLS = [(name, ws, window) for name in SHAPES for ws in ("auto", None) for window in (None, 90)]


def batch(name, seed):
    heads, share, dim, block, group, lens, counts = SHAPES[name]
    b = Q.Batch(seed, lens, counts, heads=heads, share=share, dim=dim, block=block, dtype=BF16, group=group)
    return b, tree_masks(random.Random(seed), counts) if max(counts) > 5 else None


def multiply(scales, power):
    """By 2^power, in steps that are numbers of the type."""
    for step in [60] * (power // 60) + [power % 60] if power > 0 else [-60] * (-power // 60) + [-(-power % 60)]:
        scales.mul_(2.0 ** step)


def largest(pairs):
    assert not pairs.isinf().any()
    return float(pairs.float().nan_to_num(0.0).abs().max())


@pytest.mark.parametrize("name,ws,window", CALLS)
def test_values(name, ws, window):
    b, masks = batch(name, 3)
    multiply(b.cache.v_scales, 124)
    assert largest(b.cache.v_scales) > 2.0 ** 124
    print("CASE q4 large values", name, ws, window, flush=True)
    b.check(b.attend(masks, window=window, sinks=3 if window else 0, workspace=ws), masks, window, 3 if window else 0)


@pytest.mark.parametrize("power", [70, 79, 80, 100, 122])
@pytest.mark.parametrize("name,ws,window", CALLS)
def test_values_of_one_token(name, ws, window, power):
    """One token's values are large, all others as ever: rows that see it have its
    sums, in one of many runs and groups."""
    b, masks = batch(name, 4)
    for r, n in enumerate(b.lens):
        pos = max(n - 20, 0)
        page, at = int(b.table[r, pos // b.cache.block_size]), pos % b.cache.block_size
        multiply(b.cache.v_scales[page, 0, at, 0], power)
    print("CASE q4 large token", name, ws, window, power, flush=True)
    b.check(b.attend(masks, window=window, sinks=3 if window else 0, workspace=ws), masks, window, 3 if window else 0)


@pytest.mark.parametrize("name,ws,window", CALLS)
def test_values_that_no_row_sees(name, ws, window):
    """Large values, and some that are not finite, at places that no row sees change nothing."""
    b, masks = batch(name, 5)
    args = dict(window=50, sinks=2, workspace=ws)
    want = b.attend(masks, **args)
    for r, n in enumerate(b.lens):
        for pos in range(2, n - 50):
            page, at = int(b.table[r, pos // b.cache.block_size]), pos % b.cache.block_size
            b.cache.v_scales[page, :, at] = 3e38 if pos % 3 else float("nan")
    print("CASE q4 large unseen", name, ws, flush=True)
    assert torch.equal(b.attend(masks, **args), want)


@pytest.mark.parametrize("name,ws,window", CALLS)
def test_keys(name, ws, window):
    """Keys whose group spans more than fp32 holds of 24 scales, and small queries."""
    b, masks = batch(name, 6)
    multiply(b.cache.k_scales, 126)
    b.q, scale = b.q * 2.0 ** -100, b.scale * 2.0 ** -26
    assert 24 * largest(b.cache.k_scales[..., 0]) > 2.0 ** 128
    print("CASE q4 large keys", name, ws, window, flush=True)
    got = b.attend(masks, window=window, sinks=3 if window else 0, workspace=ws, scale=scale)
    b.scale = scale
    b.check(got, masks, window, 3 if window else 0)


@pytest.mark.parametrize("name,ws,window", CALLS)
def test_queries(name, ws, window):
    """Queries next to the largest and small keys; of two rows of a tile, one has
    ordinary queries and scores near 0."""
    b, masks = batch(name, 7)
    multiply(b.cache.k_scales, -90)
    b.q, scale = b.q * 2.0 ** 120, b.scale * 2.0 ** -30
    b.q[0, 0] *= 2.0 ** -120
    assert largest(b.q) > 2.0 ** 121
    print("CASE q4 large queries", name, ws, window, flush=True)
    got = b.attend(masks, window=window, sinks=3 if window else 0, workspace=ws, scale=scale)
    b.scale = scale
    b.check(got, masks, window, 3 if window else 0)


@pytest.mark.parametrize("half", [60, 63])
@pytest.mark.parametrize("sign", [1, -1])
def test_a_large_softmax_scale(sign, half):
    """Scores of ordinary size by a scale near the largest and small keys and queries."""
    b, masks = batch("whole", 8)
    multiply(b.cache.k_scales, -half)
    b.q, scale = b.q * 2.0 ** -half, sign * b.scale * 2.0 ** (2 * half)
    print("CASE q4 large scale", sign, half, flush=True)
    got = b.attend(masks, scale=scale)
    b.scale = scale
    b.check(got, masks)
