"""Attention with offsets that no step makes: falling ones and numbers of any
size."""
import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu
HALF = torch.float16


def attend(b, offsets, max_new, tokens):
    out = torch.full((tokens, *b.q.shape[1:]), 5.0, dtype=b.dtype, device="cuda")
    q = torch.zeros_like(out)
    q[: len(b.q)] = b.q.cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    return decode.tree_attention(q, decode.PagedCache(b.k.cuda(), b.v.cuda()), b.table.cuda(), torch.tensor(b.lens, **i32),
                                 torch.tensor(offsets, **i32), max_new=max_new, out=out)


def test_rows_that_several_requests_claim():
    """Requests 0 and 3 are split, so that their rows are written by the join,
    which finds none of them; request 2 is not, and writes its own."""
    print("CASE falling offsets", flush=True)
    b = D.Batch(2, [5000, 10, 100, 3000], [1, 1, 5, 1], heads=1, share=2, dim=64, block=16, dtype=HALF)
    b.q = b.q[2:7]  # request 2's
    ref, spread = D.attention(b.q, b.k, b.v, b.table[2:3], [100], [5], None, b.scale)
    got = attend(b, [0, 100, 0, 5, 20], 100, 100)
    D.check_attention(got[:5], ref, spread, HALF)
    assert (got[5:] == 5).all()


@pytest.mark.parametrize("tail", [[2 ** 31 - 1, -2 ** 31, -1], [2 ** 31 - 1, -2 ** 31 + 3, 2 ** 31 - 1], [2 ** 31 - 4, -2 ** 31, 8]])
def test_offsets_of_any_size(tail):
    print("CASE wild offsets", tail, flush=True)
    b = D.Batch(3, [30, 40, 50, 60], [3, 5, 1, 1], heads=2, share=2, dim=64, block=16, dtype=HALF)
    b.q = b.q[:8]
    ref, spread = D.attention(b.q, b.k, b.v, b.table[:2], [30, 40], [3, 5], None, b.scale)
    D.check_attention(attend(b, [0, 3] + tail, 8, 8), ref, spread, HALF)


@pytest.mark.parametrize("max_new", [64, 10 ** 6, 2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 60])
def test_a_bound_on_new_tokens_beyond_any_request(max_new):
    print("CASE large max_new", max_new, flush=True)
    b = D.Batch(4, [30, 900, 50], [3, 5, 1], heads=2, share=2, dim=64, block=16, dtype=HALF)
    ref, spread = b.reference()
    D.check_attention(attend(b, b.offsets.tolist(), max_new, 9), ref, spread, HALF)
