"""Products with 4-bit weights of inputs that are infinite, NaN or so large
that a sum of a(16 + q) is not finite while the sum of a(q - z) is."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16

# rows, K, N: up to 16, 32 and 64 rows, aligned and not, one and several column
# blocks a workgroup
SHAPES = [(1, 300, 40), (7, 1003, 8210), (3, 2100, 16400), (20, 520, 100), (32, 519, 33), (50, 520, 8200), (70, 333, 20)]


def weight(g, K, N, group, dtype, zeros):
    G = -(-K // group)
    codes = torch.randint(0, 16, (K, N), generator=g, dtype=torch.uint8)
    scales = (2.0 ** torch.randint(-4, -1, (G, N), generator=g)).to(dtype)
    z = torch.randint(0, 16, (G, N), generator=g).to(dtype) if zeros else None
    w = decode.Q4Weight(decode.q4_pack(codes.cuda()), decode.q4_groups(scales.cuda()),
                        None if z is None else decode.q4_groups(z.cuda()), K=K, N=N, group=group)
    return w, D.dequantized(codes, scales, z, group)


@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_what_is_not_finite(shape, group, zeros, dtype, act):
    """Whole numbers and scales that are powers of two, so that finite results
    are exact; an infinite input times a code equal to the zero point is NaN."""
    M, K, N = shape
    print("CASE linear not finite", shape, group, zeros, dtype, act, flush=True)
    g = torch.Generator().manual_seed(M + group)
    w, ref = weight(g, K, N, group, dtype, zeros)
    x = torch.randint(-4, 5, (M, K), generator=g).to(dtype)
    x[0, K // 3] = math.inf
    if M > 2:
        x[1, K - 1] = -math.inf
        x[M - 1, 5] = math.nan
    if M > 5:
        x[4, 0], x[4, K // 2] = math.inf, -math.inf
    want = x.double() @ ref
    # (torch's own product may take 0 for inf * 0)
    odd = ~x.isfinite()
    for i in odd.any(1).nonzero().view(-1).tolist():
        want[i] = (x[i].double().view(-1, 1) * ref).sum(0)
    want = torch.where(want.isnan(), want, D.activated(want, act)).to(dtype)
    got = decode.q4_linear(x.cuda(), w, act=act).cpu()
    assert torch.equal(want.isnan(), got.isnan())
    assert torch.equal(want[~want.isnan()], got[~want.isnan()])


@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_large_finite_inputs(shape, zeros):
    """Rows of 2^117 (and of 1): sums of 128 terms of at least 16 and at most 31 of
    them pass 2^128, the largest number; those of q - z are below 2^10 of them,
    whole, and the sums of scaled groups too."""
    M, K, N = shape
    print("CASE linear large", shape, zeros, flush=True)
    g = torch.Generator().manual_seed(M)
    w, _ = weight(g, K, N, 128, BF16, zeros)
    x = torch.ones((M, K), dtype=BF16)
    x[::2] = 2.0 ** 117
    small = decode.q4_linear(torch.ones_like(x).cuda(), w).float().cpu()
    want = small.double() * x[:, :1].double()
    want = torch.where(want.abs() < 2.0 ** 128, want, torch.sign(want) * math.inf).to(BF16)
    assert torch.equal(decode.q4_linear(x.cuda(), w).cpu(), want)
