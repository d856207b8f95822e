"""Attention where one key has nearly all of the weight and a value of zero: the
result is made of the other keys' small weights alone."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("gap", [10, 13, 16, 18, 20])
@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("share,count,workspace", [(1, 1, "auto"), (1, 1, None), (4, 8, "auto"), (4, 8, None), (4, 15, None), (4, 25, "auto"),
                                                   (4, 64, "auto"), (4, 64, None)])
def test_small_weights_add_up(share, count, workspace, dtype, gap):
    """Key 0 of 3000 scores `gap` above the others, which are within half of
    each other; values of one sign.  A weight is rounded to the type, in fp16
    to no less than 2^-25 of the unit in which the largest one is at least
    2^11.  Of 3000 such errors of either sign, each up to 2^-36 |v|, a sum of 2^-36
    |v| sqrt(3000 / 3) is left; beside check_attention's bound there is room for
    twelve times that, 2^-39 of the sum of all |v|."""
    print("CASE dominant", share, count, workspace, dtype, gap, flush=True)
    n, dim = 3000, 64
    b = D.Batch(int(gap) + share, [n], [count], heads=2, share=share, dim=dim, block=16, dtype=dtype)
    g = torch.Generator().manual_seed(7)
    pos = torch.arange(n + count)
    page, at = b.table[0, pos // 16].long(), pos % 16
    # the first element of q is 8, of which 1 / sqrt(64) makes 1, and the others are zeros: a score is its key's first element
    b.q = torch.zeros_like(b.q)
    b.q[:, :, 0] = 8
    k = torch.randn((n + count, 2, dim), generator=g)
    k[:, :, 0] = torch.rand((n + count, 2), generator=g) - 0.5
    k[0, :, 0] = gap
    v = (torch.rand((n + count, 2, dim), generator=g) + 0.5) * (100 if gap > 12 else 1)
    v[0] = 0
    b.k[page, at], b.v[page, at] = k.to(dtype), v.to(dtype)
    ref, spread = b.reference()
    # (as if it were a part of the spread, of which check_attention allows 2 u + 2^-14)
    spread = spread + 2.0 ** -39 * float(v.abs().sum(0).max()) / (2 * D.U[dtype] + 2.0 ** -14)
    got = decode.tree_attention(b.q.cuda().contiguous(), decode.PagedCache(b.k.cuda(), b.v.cuda()), b.table.cuda(),
                                torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda(), max_new=count, workspace=workspace)
    D.check_attention(got, ref, spread, dtype)
    assert math.isfinite(float(got.float().abs().max())) and float(ref.min()) > 2.0 ** -13
