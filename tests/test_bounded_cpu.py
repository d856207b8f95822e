"""The entry points of windows and of the cache in 4 bits on the CPU: struct
mirrors, what they refuse before anything is launched, tensors of different
GPUs, and the registers of their kernels."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode, gba  # noqa: E402

import test_decode_cpu as C  # noqa: E402
import test_decode_devices_cpu as V  # noqa: E402
import test_decode_resources_cpu as R  # noqa: E402

FAKE, BIG, OK, EINVAL, EUNSUPPORTED = C.FAKE, C.BIG, C.OK, C.EINVAL, C.EUNSUPPORTED


@pytest.mark.parametrize("struct,mirror", [("gba_q4_cache", gba.Q4CacheDesc), ("gba_q4_attention", gba.Q4AttentionDesc)])
def test_structs_match_the_header(struct, mirror, tmp_path):
    C.test_structs_match_the_header(struct, mirror, tmp_path)


def window(cache=(), call="gba_window_attention", window=100, sinks=4, **kw):
    d = gba.AttentionDesc(C.cache_desc(**dict(cache)), 2, 4, 6, 3, 4, 0.125, FAKE, 256, 64, FAKE, 256, 64, FAKE, FAKE, FAKE, None, None, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    if call == "gba_window_attention":
        return gba.lib().gba_window_attention(ctypes.byref(d), window, sinks, None)
    return gba.lib().gba_window_attention_workspace_size(ctypes.byref(d), window, sinks, ctypes.byref(ctypes.c_size_t()))


@pytest.mark.parametrize("call", ["gba_window_attention", "gba_window_attention_workspace_size"])
@pytest.mark.parametrize("kw,status", [
    (dict(window=0), EINVAL), (dict(window=-1), EINVAL), (dict(sinks=-1), EINVAL), (dict(window=0, tokens=0), EINVAL),
    (dict(cache=dict(dtype=3)), EINVAL), (dict(requests=-1), EINVAL), (dict(q_heads=3), EINVAL), (dict(q=None), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(workspace=FAKE + 16), EINVAL), (dict(cache=dict(dim=60)), EUNSUPPORTED),
    (dict(q=FAKE + 8), EUNSUPPORTED), (dict(mask=FAKE, max_new=65), EUNSUPPORTED), (dict(tokens=BIG), EUNSUPPORTED),
    (dict(requests=gba.GBA_MAX_REQUESTS + 1), EUNSUPPORTED)])
def test_window_refusals(kw, status, call):
    assert window(call=call, **kw) == status


def test_window_of_nothing():
    for kw in (dict(tokens=0), dict(requests=0), dict(max_new=0), dict(q_heads=0)):
        assert window(q=None, out=None, lens=None, offsets=None, table=None, **kw) == OK
    assert gba.lib().gba_window_attention(None, 1, 0, None) == EINVAL
    assert gba.lib().gba_window_attention_workspace_size(None, 1, 0, ctypes.byref(ctypes.c_size_t())) == EINVAL


def cache_desc(**kw):
    c = gba.Q4CacheDesc(gba.GBA_F16, 64, 8, 16, 2, 64, FAKE, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [
    (dict(dtype=2), EINVAL), (dict(group=16), EINVAL), (dict(group=0), EINVAL), (dict(group=256), EINVAL), (dict(num_blocks=-1), EINVAL),
    (dict(block_size=0), EINVAL), (dict(heads=-1), EINVAL), (dict(dim=-8), EINVAL), (dict(k_codes=None), EINVAL), (dict(v_codes=None), EINVAL),
    (dict(k_scales=None), EINVAL), (dict(v_scales=None), EINVAL), (dict(block_size=24), EUNSUPPORTED), (dict(dim=60), EUNSUPPORTED),
    (dict(dim=264), EUNSUPPORTED), (dict(heads=65536), EUNSUPPORTED), (dict(num_blocks=2 ** 27), EUNSUPPORTED), (dict(k_codes=FAKE + 8), EUNSUPPORTED),
    (dict(v_codes=FAKE + 4), EUNSUPPORTED), (dict(k_scales=FAKE + 4), EUNSUPPORTED), (dict(v_scales=FAKE + 8), EUNSUPPORTED)]


def rows(load=False, cache=(), **kw):
    a = dict(tokens=4, k=FAKE, kt=128, kh=64, v=FAKE, vt=128, vh=64, slots=FAKE)
    a.update(kw)
    c = ctypes.byref(cache_desc(**dict(cache)))
    if load:
        return gba.lib().gba_q4_cache_load(c, a["tokens"], a["slots"], a["k"], a["kt"], a["kh"], a["v"], a["vt"], a["vh"], None)
    return gba.lib().gba_q4_cache_store(c, a["tokens"], a["k"], a["kt"], a["kh"], a["v"], a["vt"], a["vh"], a["slots"], None)


@pytest.mark.parametrize("load", [False, True], ids=["store", "load"])
@pytest.mark.parametrize("kw,status", [(dict(cache=c), s) for c, s in BAD_CACHES] + [
    (dict(tokens=-1), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(slots=None), EINVAL), (dict(k=FAKE + 1), EUNSUPPORTED),
    (dict(v=FAKE + 1), EUNSUPPORTED), (dict(slots=FAKE + 2), EUNSUPPORTED), (dict(tokens=BIG), EUNSUPPORTED),
    (dict(tokens=0, k=None, v=None, slots=None), OK), (dict(cache=dict(heads=0), k=None), OK)])
def test_store_and_load_refusals(kw, status, load):
    assert rows(load, **kw) == status


def test_store_and_load_refuse_no_cache():
    assert gba.lib().gba_q4_cache_store(None, 1, FAKE, 1, 1, FAKE, 1, 1, FAKE, None) == EINVAL
    assert gba.lib().gba_q4_cache_load(None, 1, FAKE, FAKE, 1, 1, FAKE, 1, 1, None) == EINVAL
    assert rows(cache=dict(num_blocks=0, k_codes=None, v_codes=None, k_scales=None, v_scales=None)) == OK


def attend(cache=(), size=False, **kw):
    d = gba.Q4AttentionDesc(cache_desc(**dict(cache)), 2, 4, 6, 3, 4, 0, 0, 0.125, FAKE, 256, 64, FAKE, 256, 64, FAKE, FAKE, FAKE, None, None, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    if size:
        return gba.lib().gba_q4_attend_workspace_size(ctypes.byref(d), ctypes.byref(ctypes.c_size_t()))
    return gba.lib().gba_q4_attend(ctypes.byref(d), None)


@pytest.mark.parametrize("size", [False, True], ids=["attend", "size"])
@pytest.mark.parametrize("kw,status", [(dict(cache=c), s) for c, s in BAD_CACHES] + [
    (dict(window=-1), EINVAL), (dict(sinks=-1), EINVAL), (dict(requests=-1), EINVAL), (dict(width=-1), EINVAL), (dict(tokens=-1), EINVAL),
    (dict(max_new=-1), EINVAL), (dict(q_heads=-4), EINVAL), (dict(q_heads=3), EINVAL), (dict(cache=dict(heads=0)), EINVAL), (dict(q=None), EINVAL),
    (dict(out=None), EINVAL), (dict(lens=None), EINVAL), (dict(offsets=None), EINVAL), (dict(table=None), EINVAL), (dict(workspace=FAKE + 16), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(q_token=260), EUNSUPPORTED), (dict(out_head=66), EUNSUPPORTED), (dict(q=FAKE + 8), EUNSUPPORTED),
    (dict(out=FAKE + 8), EUNSUPPORTED), (dict(table=FAKE + 2), EUNSUPPORTED), (dict(mask=FAKE + 4), EUNSUPPORTED), (dict(mask=FAKE, max_new=65), EUNSUPPORTED),
    (dict(requests=gba.GBA_MAX_REQUESTS + 1), EUNSUPPORTED), (dict(tokens=BIG), EUNSUPPORTED), (dict(width=2 ** 28), EUNSUPPORTED),
    (dict(tokens=0, q=None, out=None, lens=None, offsets=None, table=None), OK), (dict(max_new=0, q=None), OK)])
def test_attend_refusals(kw, status, size):
    assert attend(size=size, **kw) == status


def test_attend_refuses_null():
    assert gba.lib().gba_q4_attend(None, None) == EINVAL
    assert gba.lib().gba_q4_attend_workspace_size(None, ctypes.byref(ctypes.c_size_t())) == EINVAL


def sizes(window, sinks, requests=4, new=1, width=4096, q4=False):
    """Bytes of the workspace."""
    out = ctypes.c_size_t()
    if q4:
        d = gba.Q4AttentionDesc(cache_desc(num_blocks=65536), requests, width, requests * new, new, 8, window, sinks, 0.125, FAKE, 512, 64, FAKE, 512, 64,
                                FAKE, FAKE, FAKE, None, None, 0)
        assert gba.lib().gba_q4_attend_workspace_size(ctypes.byref(d), ctypes.byref(out)) == OK
    else:
        d = gba.AttentionDesc(C.cache_desc(num_blocks=65536), requests, width, requests * new, new, 8, 0.125, FAKE, 512, 64, FAKE, 512, 64,
                              FAKE, FAKE, FAKE, None, None, 0)
        assert gba.lib().gba_window_attention_workspace_size(ctypes.byref(d), window, sinks, ctypes.byref(out)) == OK
    return out.value


@pytest.mark.parametrize("q4", [False, True], ids=["16", "4"])
def test_workspaces_follow_the_window(q4):
    """A workspace has room for runs of what a window reaches, not of the text;
    windows past any text need no more than the text."""
    small, large, all_of_it, past = (sizes(w, 4, q4=q4) for w in (256, 8192, 2 ** 31, 2 ** 62))
    assert 0 < small <= large and all_of_it == past < 1 << 30
    assert sizes(100, 0, width=8, q4=q4) == 0  # (too short to be split)
    for window in (1, 1000, 2 ** 31 - 1, 2 ** 31, 2 ** 63 - 1):
        for sinks in (0, 2 ** 31, 2 ** 63 - 1):
            for requests, new, width in ((1, 1, 2 ** 27 - 1), (200, 1, 2 ** 20), (1, 5000, 2 ** 27 - 1), (1500, 3, 2 ** 16)):
                assert sizes(window, sinks, requests, new, width, q4) < 1 << 34


H = torch.float16


@pytest.mark.parametrize("odd", range(4))
def test_cache_refuses_tensors_of_different_gpus(odd):
    t = [V.Tensor(4, 2, 16, 32, dtype=torch.uint8), V.Tensor(4, 2, 16, 32, dtype=torch.uint8), V.Tensor(4, 2, 16, 1, 2, dtype=H), V.Tensor(4, 2, 16, 1, 2, dtype=H)]
    t[odd].device = torch.device("cuda", 1)
    with pytest.raises(ValueError, match="another device"):
        decode.Q4Cache(*t, dim=64)


def test_cache_refuses_cpu_tensors_and_wrong_types():
    k, s = torch.zeros((4, 2, 16, 32), dtype=torch.uint8), torch.zeros((4, 2, 16, 1, 2), dtype=H)
    with pytest.raises(TypeError):
        decode.Q4Cache(k, k, s, s, dim=64)
    for bad in (dict(dim=64, group=48), dict(dim=60), dict(dim=0), dict(dim=300)):
        with pytest.raises(ValueError):
            decode.Q4Cache(k, k, s, s, **bad)


@pytest.mark.skipif(not R._have_hipcc(), reason="hipcc not available")
@pytest.mark.parametrize("name,counts", [("window_attention", {"attention_kernel": 2 * (2 * 7 + 3)}), ("q4_attention", {"q4_attention_kernel": 2 * 8}),
                                         ("q4_cache", {"q4_store_kernel": 2 * 3 * 2 * 2, "q4_load_kernel": 2 * 3 * 2 * 2})])
def test_kernels_use_no_scratch(name, counts, tmp_path):
    seen = {}
    for (kernel, _, args), res in R.kernels(name, tmp_path).items():
        assert res["ScratchSize"] == 0, (kernel, args, res)
        seen[kernel] = seen.get(kernel, 0) + 1
        if kernel == "q4_attention_kernel":
            assert res["Occupancy"] >= (2 if args[0] <= 128 else 1), (args, res)
    for kernel, n in counts.items():
        assert seen.get(kernel) == n, (kernel, seen)
