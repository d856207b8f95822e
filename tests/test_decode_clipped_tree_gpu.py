"""Trees of more than 64 tokens of which the step's buffers take 64 or fewer."""
import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests,tokens,new", [(1, 30, 100), (2, 64, 65), (3, 100, 70), (40, 500, 90), (40, 41 * 64, 66)])
def test_entries_of_a_clipped_tree(requests, tokens, new):
    """The last request has too many tokens, the others 4 each: its entries are
    -1, -1 and 0, however many of them there are."""
    print("CASE clipped tree", requests, tokens, new, flush=True)
    i32 = dict(dtype=torch.int32, device="cuda")
    tables = decode.BlockTables.empty(requests, 32, 32 * requests, 16, tokens=tokens, tree=True)
    count = [4] * (requests - 1) + [new]
    maps = tables.step(torch.full((requests,), 5, **i32), torch.tensor(count, **i32), torch.full((tokens,), -1, **i32))
    first = 4 * (requests - 1)
    assert maps.offsets.tolist() == [4 * r for r in range(requests)] + [min(first + new, tokens)]
    assert maps.status.tolist() == [0] * (requests - 1) + [3]
    assert maps.positions.tolist() == [5] * first + [-1] * (tokens - first)
    assert maps.mask.view(-1).tolist() == [1, 2, 4, 8] * (requests - 1) + [0] * (tokens - first)
    assert (maps.slots[:first] >= 0).all() and (maps.slots[first:] == -1).all()
    assert tables.held.tolist() == [1] * (requests - 1) + [0]
