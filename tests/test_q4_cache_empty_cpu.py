"""Q4Cache.empty refuses what the cache itself refuses, before it allocates."""
import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode  # noqa: E402


@pytest.mark.parametrize("bad", [dict(group=0), dict(group=-64), dict(group=48), dict(dim=0), dict(dim=60), dict(dim=264), dict(dim=-8)])
def test_sizes(bad, monkeypatch):
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: pytest.fail("allocated"))
    kw = dict(dim=64, group=64)
    kw.update(bad)
    with pytest.raises(ValueError, match="group" if "group" in bad else "dim"):
        decode.Q4Cache.empty(4, 16, 2, kw["dim"], torch.float16, group=kw["group"], device="cpu")
