"""The handles refuse tensors of different GPUs (stand-ins for tensors: no GPU is needed)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402


class Tensor:
    """What the handles look at of a contiguous CUDA tensor."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.int32, gpu=0):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", gpu)

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        strides = torch.empty(self.shape, device="meta").stride()
        return strides if i is None else strides[i]

    def data_ptr(self):
        raise AssertionError("used before it was refused")


H = torch.float16


@pytest.mark.parametrize("codes,scales,zeros", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (0, 1, None)])
def test_weight(codes, scales, zeros):
    with pytest.raises(ValueError, match="another device"):
        decode.Q4Weight(Tensor(2, 1, 64, 4, gpu=codes), Tensor(2, 1, 16, dtype=H, gpu=scales),
                        None if zeros is None else Tensor(2, 1, 16, dtype=H, gpu=zeros), K=128, N=32)


@pytest.mark.parametrize("odd", range(1, 4))
def test_tables(odd):
    t = [Tensor(4, 8), Tensor(4), Tensor(32), Tensor(1)]
    t[odd].device = torch.device("cuda", 1)
    with pytest.raises(ValueError, match="another device"):
        decode.BlockTables(*t, 16, tokens=4)


def test_cache():
    with pytest.raises(ValueError, match="another device"):
        decode.PagedCache(Tensor(4, 16, 2, 64, dtype=H), Tensor(4, 16, 2, 64, dtype=H, gpu=1))
