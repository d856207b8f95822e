"""Workspaces of windows: a call whose requests and heads fill the chip many times
over is not split for a small gain, and none has more than half a gigabyte of
sums."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import gba  # noqa: E402

import test_bounded_cpu as S  # noqa: E402
import test_decode_cpu as C  # noqa: E402

FAKE = C.FAKE
MOST = (1 << 29) + (1 << 18) + 8 * gba.GBA_MAX_REQUESTS + 256  # sums, counters, the requests' runs


def bytes_of(q4, requests, heads, dim, window, width, *, new=1, share=1, block=16):
    out, q = ctypes.c_size_t(), heads * share
    common = (requests, width, requests * new, new, q)
    rows = (0.125, FAKE, q * dim, dim, FAKE, q * dim, dim, FAKE, FAKE, FAKE, None, None, 0)
    if q4:
        cache = S.cache_desc(num_blocks=65536, heads=heads, dim=dim, block_size=block)
        st = gba.lib().gba_q4_attend_workspace_size(ctypes.byref(gba.Q4AttentionDesc(cache, *common, window, 4, *rows)), ctypes.byref(out))
    else:
        cache = C.cache_desc(num_blocks=65536, heads=heads, dim=dim, block_size=block, k_block=block * heads * dim, k_token=heads * dim, k_head=dim,
                             v_block=block * heads * dim, v_token=heads * dim, v_head=dim)
        st = gba.lib().gba_window_attention_workspace_size(ctypes.byref(gba.AttentionDesc(cache, *common, *rows)), window, 4, ctypes.byref(out))
    assert st == S.OK
    return out.value


@pytest.mark.parametrize("q4", [False, True], ids=["16", "4"])
@pytest.mark.parametrize("requests,heads,dim,window,width", [(1020, 32, 256, 131072, 8192), (1013, 64, 64, 2 ** 20, 65536), (513, 64, 64, 10 ** 6, 8192)])
def test_many_requests_are_left_whole(requests, heads, dim, window, width, q4):
    assert bytes_of(q4, requests, heads, dim, window, width) == 0


@pytest.mark.parametrize("q4", [False, True], ids=["16", "4"])
def test_sums_have_a_bound(q4):
    seen = set()
    for requests in (1, 2, 7, 33, 100, 255, 257, 500, 1000, 1024):
        for heads in (1, 2, 8, 31, 64):
            for dim in (64, 128, 256):
                for new, share in ((1, 1), (1, 8), (1, 33), (16, 4), (64, 4), (64, 16)):
                    for window in (1024, 8192, 131072, 2 ** 20, 2 ** 40):
                        for width in (512, 8192, 65536):
                            need = bytes_of(q4, requests, heads, dim, window, width, new=new, share=share)
                            assert need <= MOST, (requests, heads, dim, new, share, window, width, need)
                            seen.add(need)
    assert len(seen) > 50


@pytest.mark.parametrize("q4", [False, True], ids=["16", "4"])
def test_few_requests_are_split_as_before(q4):
    """One request of one head and one of eight: runs enough for the chip."""
    for heads, dim in ((1, 64), (8, 128)):
        assert bytes_of(q4, 1, heads, dim, 131072, 8192) - (1 << 18) > 8 * 16 * (dim + 2) * 4 * heads
