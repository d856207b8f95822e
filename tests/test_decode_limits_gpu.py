"""Sizes next to 2^31."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("count,share,dim,block,before,workspace", [
    (1, 1, 8, 16, 20, "auto"), (1, 1, 8, 16, 0, "auto"), (1, 1, 8, 16, 0, None), (3, 8, 64, 16, 5, "auto"), (16, 4, 64, 16, 1, "auto"),
    (64, 4, 64, 16, 0, "auto"), (2, 2, 128, 24, 0, "auto")])
def test_attention_of_a_request_of_nearly_2_31_tokens(count, share, dim, block, before, workspace):
    """A table of as many blocks as fit, whose last `before` tokens are not used; all entries but five are
    not in the cache, so that their tokens are not seen."""
    print("CASE long positions", count, share, dim, block, before, workspace, flush=True)
    width = (2 ** 31 - 1) // block
    end = width * block - before
    n = end - count
    g = torch.Generator().manual_seed(count)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    last = (end - 1) // block
    pages = sorted({0, width // 3, width // 2, last - 1 - count // block, last - 1} | set(range(n // block, last + 1)))
    for i, page in enumerate(pages):
        table[0, page] = i
    k, v = (torch.randn((len(pages), block, 1, dim), generator=g).to(BF16) for _ in range(2))
    q = torch.randn((count, share, dim), generator=g).to(BF16)
    # the same positions one after the other: those that are not in the cache have no effect
    pos = [page * block + i for page in pages for i in range(block) if page * block + i < end]
    flat_k = torch.cat(list(k))[: len(pos)].unsqueeze(0)
    flat_v = torch.cat(list(v))[: len(pos)].unsqueeze(0)
    kept = len(pos) - count
    assert pos[kept] == n
    ref, spread = D.attention(q, flat_k, flat_v, torch.zeros((1, 1), dtype=torch.int32), [kept], [count], None, 1 / math.sqrt(dim))
    i32 = dict(dtype=torch.int32, device="cuda")
    got = decode.tree_attention(q.cuda(), decode.PagedCache(k.cuda(), v.cuda()), table, torch.tensor([n], **i32),
                                torch.tensor([0, count], **i32), max_new=count, workspace=workspace)
    D.check_attention(got, ref, spread, BF16)
