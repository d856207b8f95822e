"""What the automatic workspaces of attention keep."""
import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402

pytestmark = pytest.mark.gpu


def test_a_batch_that_grows_by_ones_keeps_little():
    """All buffers that were replaced are together no larger than the one in
    use, and that one is less than twice what the largest call needs."""
    cache = decode.PagedCache(*(torch.zeros((40, 16, 8, 128), dtype=torch.float16, device="cuda") for _ in range(2)))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        key = (0, stream.cuda_stream)
        decode._scratch.pop(key, None)
        before = len(decode._retired)
        needs = []
        for requests in range(1, 65):
            print("CASE scratch", requests, flush=True)
            i32 = dict(dtype=torch.int32, device="cuda")
            q = torch.zeros((requests, 32, 128), dtype=torch.float16, device="cuda")
            decode.tree_attention(q, cache, torch.zeros((requests, 40), **i32), torch.full((requests,), 600, **i32),
                                  torch.arange(requests + 1, **i32), max_new=64)
            needs.append(decode._scratch[key].numel())
        retired = [t.numel() for t in decode._retired[before:]]
        assert sum(retired) <= needs[-1]
        assert len(set(needs)) < 10
    stream.synchronize()
