"""Attention of few tokens among very many rows, which are padding."""
import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode, gba  # noqa: E402
import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,share,width,workspace", [(2 ** 20 + 5, 65, 64, "auto"), (2 ** 20 + 5, 65, 64, None), (2 ** 23 + 1, 1, 16, "auto"),
                                                          (2 ** 23 + 1, 1, 64, None), (2 ** 23 + 1, 1, 64, "auto")])
def test_many_rows_of_padding(tokens, share, width, workspace):
    """Six tokens of two requests in up to 2^26 rows of q and more.  Only where a second kernel
    would have 2^32 threads is the call refused."""
    print("CASE padded rows", tokens, share, width, workspace, flush=True)
    b = D.Batch(width, [8 * width, 30], [4, 2], heads=1, share=share, dim=8, block=16, dtype=torch.float16)
    table = torch.full((2, width), -1, dtype=torch.int32)
    table[:, : b.table.shape[1]] = b.table[:, :width]
    ref, spread = b.reference()
    q = torch.zeros((tokens, share, 8), dtype=torch.float16, device="cuda")
    q[:6] = b.q.cuda()
    out = torch.full_like(q, 5.0)

    def call():
        return decode.tree_attention(q, decode.PagedCache(b.k.cuda(), b.v.cuda()), table.cuda(), torch.tensor(b.lens, dtype=torch.int32).cuda(),
                                     b.offsets.cuda(), max_new=4, out=out, workspace=workspace)

    if tokens > 2 ** 23 and width * 16 > 256 and workspace == "auto":
        # (a few runs, which the workgroup that ends last joins, need no second kernel)
        with pytest.raises(gba.GbaError):
            b2 = torch.zeros((2, 4096), dtype=torch.int32, device="cuda")
            decode.tree_attention(q, decode.PagedCache(b.k.cuda(), b.v.cuda()), b2, torch.tensor(b.lens, dtype=torch.int32).cuda(),
                                  b.offsets.cuda(), max_new=4, out=out)
        assert (out == 5).all()
    D.check_attention(call()[:6], ref, spread, torch.float16)
    assert (out[6:] == 5).all()
