"""The join of many rows (from 4096 of them on), and batches of more requests than are split."""
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


def attend(b, max_new, mask=None):
    return decode.tree_attention(b.q.cuda().contiguous(), decode.PagedCache(b.k.cuda(), b.v.cuda()), b.table.cuda(),
                                 torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda(), max_new=max_new, mask=mask)


# kept and new tokens, key heads, query heads a key head, dim: each of tokens * query heads >= 4096
@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("lens,counts,heads,share,dim", [([2000, 300, 0, 900], [64, 40, 20, 33], 4, 8, 64), ([1500, 700], [70, 200], 2, 8, 128),
                                                         ([600, 2100], [61, 4], 8, 8, 80), ([1000], [130], 16, 2, 64)])
def test_many_rows(lens, counts, heads, share, dim, dtype):
    print("CASE join rows", lens, counts, heads, share, dim, dtype, flush=True)
    b = D.Batch(sum(counts), lens, counts, heads=heads, share=share, dim=dim, block=16, dtype=dtype)
    assert b.q.shape[0] * b.q.shape[1] >= 4096
    ref, spread = b.reference()
    D.check_attention(attend(b, max(counts)), ref, spread, dtype)


@pytest.mark.parametrize("requests", [1024, 1025])
def test_as_many_requests_as_are_split_and_one_more(requests):
    print("CASE many requests", requests, flush=True)
    rng = random.Random(requests)
    lens = [rng.choice([0, 1, 7, rng.randint(0, 40)]) for _ in range(requests)]
    lens[500] = 900
    counts = [rng.choice([0, 1, 1, 2]) for _ in lens]
    counts[500] = 2
    b = D.Batch(5, lens, counts, heads=1, share=2, dim=64, block=16, dtype=HALF)
    ref, spread = b.reference()
    D.check_attention(attend(b, 2), ref, spread, HALF)
