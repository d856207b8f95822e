"""Two requests of nearly 2^31 tokens each and so many heads that one run is aimed
at: their mean length passes 2^31, and each is one run."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu


def test_two_requests_of_nearly_2_31_tokens():
    print("CASE long batch", flush=True)
    heads, share, dim, block, count = 128, 4, 8, 16, 64
    width = (2 ** 31 - 1) // block
    n = width * block - count
    g = torch.Generator().manual_seed(1)
    # six blocks a request: the first, one in the middle, and those of the last 64 tokens
    table = torch.full((2, width), -1, dtype=torch.int32, device="cuda")
    pages = [0, width // 2] + list(range(width - 4, width))
    for r in range(2):
        for i, page in enumerate(pages):
            table[r, page] = 6 * r + i
    k, v = (torch.randn((12, block, heads, dim), generator=g).half() for _ in range(2))
    q = torch.randn((2 * count, heads * share, dim), generator=g).half()
    i32 = dict(dtype=torch.int32, device="cuda")
    got = decode.tree_attention(q.cuda(), decode.PagedCache(k.cuda(), v.cuda()), table, torch.tensor([n, n], **i32),
                                torch.tensor([0, count, 2 * count], **i32), max_new=count).cpu()
    for r in range(2):
        for h in (0, heads - 1):
            mine = slice(r * count, (r + 1) * count), slice(h * share, (h + 1) * share)
            flat_k, flat_v = (torch.cat(list(t[6 * r:6 * r + 6, :, h:h + 1])).unsqueeze(0) for t in (k, v))
            ref, spread = D.attention(q[mine], flat_k, flat_v, torch.zeros((1, 1), dtype=torch.int32), [32], [count], None, 1 / math.sqrt(dim))
            D.check_attention(got[mine], ref, spread, torch.float16)
