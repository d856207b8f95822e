"""Windows, and the cache in 4 bits, of more requests than are split, and of so many
that their runs have no counters."""
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402

import decode_util as D  # noqa: E402
import q4_cache_util as Q  # noqa: E402
import window_util as W  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


def wide(table, width):
    """The table of requests that could have `width` blocks."""
    return torch.cat([table, torch.full((table.shape[0], width - table.shape[1]), -1, dtype=torch.int32)], 1)


def attend(b, width, **kw):
    return decode.tree_attention(b.q.cuda().contiguous(), decode.PagedCache(b.k.cuda(), b.v.cuda()), wide(b.table, width).cuda(),
                                 torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda(), max_new=max(b.counts), **kw)


@pytest.mark.parametrize("requests,heads,share,dim,window,sinks,width", [(1100, 2, 2, 64, 20, 3, 40), (1500, 1, 1, 128, 300, 0, 100), (513, 64, 1, 64, 10 ** 6, 4, 8192)])
def test_windows(requests, heads, share, dim, window, sinks, width):
    rng = random.Random(requests)
    lens = [rng.choice([0, 1, rng.randint(0, 40), 330 if r % 97 == 0 else 5]) for r in range(requests)]
    counts = [rng.choice([0, 1, 1, 2]) for _ in lens]
    b = D.Batch(requests, lens, counts, heads=heads, share=share, dim=dim, block=16, dtype=HALF)
    ref, spread = W.attention(b.q, b.k, b.v, b.table, lens, counts, None, b.scale, window, sinks)
    for workspace in ("auto", None):
        print("CASE many windows", requests, heads, workspace, flush=True)
        D.check_attention(attend(b, width, window=window, sinks=sinks, workspace=workspace), ref, spread, HALF, workspace)


@pytest.mark.parametrize("requests,heads,share,dim,group", [(1100, 2, 2, 64, 64), (2000, 1, 4, 128, 32)])
def test_four_bits(requests, heads, share, dim, group):
    rng = random.Random(requests)
    lens = [rng.choice([0, 1, rng.randint(0, 40), 330 if r % 97 == 0 else 5]) for r in range(requests)]
    counts = [rng.choice([0, 1, 1, 2]) for _ in lens]
    b = Q.Batch(requests, lens, counts, heads=heads, share=share, dim=dim, block=16, dtype=BF16, group=group)
    for window, sinks in [(None, 0), (20, 3), (300, 0)]:
        print("CASE many codes", requests, heads, window, flush=True)
        b.check(b.attend(window=window, sinks=sinks), None, window, sinks)
