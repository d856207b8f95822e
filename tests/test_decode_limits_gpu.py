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


@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
def test_product_with_nearly_2_31_rows_of_weights(zeros):
    """The last whole eight k before 2^31 are beyond K; NaN stands there."""
    print("CASE long product", zeros, flush=True)
    K, N = 2 ** 31 - 100, 3
    chunks = -(-K // 128)
    f16 = dict(dtype=HALF, device="cuda")
    row = torch.zeros(2 ** 31 + 64, **f16)
    at = [0, 12345, K // 2, K - 1000, K - 29, K - 2, K - 1]
    for i, k in enumerate(at):
        row[k] = i + 1
    row[K:] = math.nan
    codes = torch.zeros((1, chunks, 64, 4), dtype=torch.int32, device="cuda")  # every code is 0
    scales = torch.full((1, chunks, 16), 0.125, **f16)
    z = torch.full((1, chunks, 16), 4.0, **f16) if zeros else None
    w = decode.Q4Weight(codes, scales, z, K=K, N=N, group=128)
    got = decode.q4_linear(row[:K].view(1, K), w)
    assert got.tolist() == [[-0.125 * (4 if zeros else 8) * 28] * N]
