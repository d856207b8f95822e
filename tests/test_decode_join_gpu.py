"""Both ways of joining a request's runs: by the workgroup that ends last, for
few runs, and by a second kernel.  Each twice and in turn on one workspace, so
that what a call leaves there meets the next one."""
import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode, gba  # noqa: E402

import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu

# requests of so many keys, new tokens, key heads, query heads a key head, head size
SHAPES = [([1000], [1], 4, 4, 128), ([3000, 2000, 900, 10], [1, 2, 1, 3], 4, 2, 64), ([600, 400], [5, 6], 1, 8, 64), ([1500], [3], 2, 2, 256),
          ([2000, 700], [20, 16], 2, 3, 128), ([5000], [9], 1, 6, 128)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_calls_of_different_shapes_share_a_workspace(dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ws = torch.zeros(128 << 20, dtype=torch.uint8, device="cuda")
    cases = []
    for i, (lens, counts, heads, share, dim) in enumerate(SHAPES):
        b = D.Batch(300 + i, lens, counts, heads=heads, share=share, dim=dim, block=16, dtype=dtype)
        cases.append((b, b.reference()))
    for _ in range(2):
        for b, (ref, spread) in cases:
            print("CASE join", b.lens, b.counts, dtype, flush=True)
            got = decode.tree_attention(b.q.contiguous().cuda(), decode.PagedCache(b.k.cuda(), b.v.cuda()), b.table.cuda(),
                                        torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda(), max_new=max(b.counts), workspace=ws)
            D.check_attention(got, ref, spread, dtype, (b.lens, b.counts))
    assert not ws[: 1 << 18].any()


def test_the_last_workgroup_joins_in_order():
    """A request's runs are added in their order whichever ends last: the same
    bits every time."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    b = D.Batch(400, [1700, 1300], [2, 2], heads=2, share=4, dim=128, block=16, dtype=torch.bfloat16)
    args = (b.q.contiguous().cuda(), decode.PagedCache(b.k.cuda(), b.v.cuda()), b.table.cuda(), torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda())
    print("CASE join order", flush=True)
    first = decode.tree_attention(*args, max_new=2)
    for _ in range(20):
        assert torch.equal(decode.tree_attention(*args, max_new=2), first)
