"""Row counts of an attention that do not fit 32 bits are refused, before
anything is launched."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import gba  # noqa: E402

FAKE = 0x10000  # a 256-byte aligned non-null address; never dereferenced here


@pytest.mark.parametrize("call", ["gba_tree_attention", "gba_tree_attention_workspace_size"])
@pytest.mark.parametrize("max_new,tokens,q_heads", [(2 ** 31 - 1, 2 ** 31 - 1, 4), (2 ** 40, 2 ** 31 - 1, 4), (2 ** 62, 2 ** 31 - 1, 6), (2 ** 30, 2 ** 30, 8),
                                                    (2 ** 17, 2 ** 17, 65534)])
def test_rows_beyond_32_bits(max_new, tokens, q_heads, call):
    cache = gba.PagedCacheDesc(gba.GBA_F16, 8, 16, 2, 64, FAKE, FAKE, 2048, 128, 64, 2048, 128, 64)
    d = gba.AttentionDesc(cache, 2, 4, tokens, max_new, q_heads, 0.125, FAKE, 64 * q_heads, 64, FAKE, 64 * q_heads, 64, FAKE, FAKE, FAKE, None, None, 0)
    arg = None if call == "gba_tree_attention" else ctypes.byref(ctypes.c_size_t())
    assert getattr(gba.lib(), call)(ctypes.byref(d), arg) == gba.GBA_EUNSUPPORTED


def test_more_new_tokens_than_rows_need_no_more_room():
    """No request has more new tokens than there are rows, whatever max_new says."""
    cache = gba.PagedCacheDesc(gba.GBA_F16, 8, 16, 2, 64, FAKE, FAKE, 2048, 128, 64, 2048, 128, 64)
    sizes = []
    for max_new in (6, 7, 1000, 2 ** 31, 2 ** 32 + 1, 2 ** 60):
        d = gba.AttentionDesc(cache, 2, 400, 6, max_new, 4, 0.125, FAKE, 256, 64, FAKE, 256, 64, FAKE, FAKE, FAKE, None, None, 0)
        n = ctypes.c_size_t()
        assert gba.lib().gba_tree_attention_workspace_size(ctypes.byref(d), ctypes.byref(n)) == gba.GBA_OK
        sizes.append(n.value)
    assert len(set(sizes)) == 1 and sizes[0] > 0
