"""The decoding entry points on the CPU: the mirrors of their structs, what
they refuse before anything is launched, and the binding's checks."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode, gba  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # a 256-byte aligned non-null address; never dereferenced here
OK, EINVAL, EUNSUPPORTED = gba.GBA_OK, gba.GBA_EINVAL, gba.GBA_EUNSUPPORTED
BIG = 2 ** 31


@pytest.mark.parametrize("struct,mirror", [("gba_q4_weight", gba.Q4WeightDesc), ("gba_block_tables", gba.BlockTablesDesc),
                                           ("gba_paged_cache", gba.PagedCacheDesc), ("gba_attention", gba.AttentionDesc)])
def test_structs_match_the_header(struct, mirror, tmp_path):
    names = [f[0] for f in mirror._fields_]
    prog = tmp_path / "s.c"
    prog.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"gba.h\"\nint main(void){\n"
                    f"printf(\"%zu\\n\", sizeof({struct}));\n" +
                    "".join(f"printf(\"%zu\\n\", offsetof({struct}, {n}));\n" for n in names) + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "s"), str(prog)], check=True)
    said = [int(v) for v in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()]
    assert said == [ctypes.sizeof(mirror)] + [getattr(mirror, n).offset for n in names]


def linear(weight=(), **kw):
    """gba_q4_linear on a valid request changed by kw; every case is refused
    or empty, so no pointer is used."""
    w = gba.Q4WeightDesc(gba.GBA_F16, 128, 256, 64, FAKE, FAKE, None)
    for k, v in dict(weight).items():
        setattr(w, k, v)
    a = dict(M=4, A=FAKE, lda=256, bias=None, act=0, C=FAKE, ldc=64)
    a.update(kw)
    return gba.lib().gba_q4_linear(ctypes.byref(w), a["M"], a["A"], a["lda"], a["bias"], a["act"], a["C"], a["ldc"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), EINVAL), (dict(lda=255), EINVAL), (dict(ldc=63), EINVAL), (dict(A=None), EINVAL), (dict(C=None), EINVAL),
    (dict(act=4), EINVAL), (dict(act=-1), EINVAL), (dict(weight=dict(dtype=2)), EINVAL), (dict(weight=dict(group=16)), EINVAL),
    (dict(weight=dict(group=0)), EINVAL), (dict(weight=dict(K=-1)), EINVAL), (dict(weight=dict(N=-1)), EINVAL),
    (dict(weight=dict(codes=None)), EINVAL), (dict(weight=dict(scales=None)), EINVAL),
    (dict(weight=dict(codes=FAKE + 8)), EUNSUPPORTED), (dict(weight=dict(scales=FAKE + 1)), EUNSUPPORTED),
    (dict(weight=dict(zeros=FAKE + 1)), EUNSUPPORTED), (dict(A=FAKE + 1), EUNSUPPORTED), (dict(C=FAKE + 1), EUNSUPPORTED),
    (dict(bias=FAKE + 1), EUNSUPPORTED), (dict(M=BIG), EUNSUPPORTED), (dict(M=64 * 65535 + 1), EUNSUPPORTED),
    (dict(weight=dict(K=BIG), lda=BIG), EUNSUPPORTED), (dict(weight=dict(N=BIG), ldc=BIG), EUNSUPPORTED),
    (dict(M=0, A=None, C=None), OK), (dict(weight=dict(N=0), C=None), OK)])
def test_linear_refusals(kw, status):
    assert linear(**kw) == status


def test_linear_and_pack_refuse_null():
    assert gba.lib().gba_q4_linear(None, 1, FAKE, 1, None, 0, FAKE, 1, None) == EINVAL
    pack = gba.lib().gba_q4_pack
    assert pack(-1, 4, FAKE, 4, FAKE, None) == EINVAL
    assert pack(4, 4, FAKE, 3, FAKE, None) == EINVAL
    assert pack(4, 4, None, 4, FAKE, None) == EINVAL
    assert pack(4, 4, FAKE, 4, None, None) == EINVAL
    assert pack(4, 4, FAKE, 4, FAKE + 4, None) == EUNSUPPORTED
    assert pack(BIG, 4, FAKE, 4, FAKE, None) == EUNSUPPORTED
    assert pack(0, 4, None, 4, None, None) == OK


def tables(desc=(), **kw):
    d = gba.BlockTablesDesc(4, 8, 32, 16, FAKE, FAKE, FAKE, FAKE, FAKE)
    for k, v in dict(desc).items():
        setattr(d, k, v)
    a = dict(lens=FAKE, count=FAKE, parents=None, tokens=16, offsets=FAKE, slots=FAKE, positions=FAKE, status=FAKE, mask=None)
    a.update(kw)
    return gba.lib().gba_tables_step(ctypes.byref(d), *a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=dict(requests=-1)), EINVAL), (dict(desc=dict(width=-1)), EINVAL), (dict(desc=dict(num_blocks=-1)), EINVAL),
    (dict(desc=dict(block_size=0)), EINVAL), (dict(tokens=-1), EINVAL), (dict(desc=dict(table=None)), EINVAL),
    (dict(desc=dict(held=None)), EINVAL), (dict(desc=dict(free_blocks=None)), EINVAL), (dict(desc=dict(free_count=None)), EINVAL), (dict(desc=dict(scratch=None)), EINVAL),
    (dict(desc=dict(scratch=FAKE + 4)), EUNSUPPORTED),
    (dict(lens=None), EINVAL), (dict(count=None), EINVAL), (dict(offsets=None), EINVAL), (dict(status=None), EINVAL),
    (dict(parents=FAKE), EINVAL), (dict(desc=dict(requests=gba.GBA_MAX_REQUESTS + 1)), EUNSUPPORTED),
    (dict(desc=dict(width=BIG)), EUNSUPPORTED), (dict(desc=dict(requests=4096, width=2 ** 20)), EUNSUPPORTED),
    (dict(desc=dict(num_blocks=2 ** 28)), EUNSUPPORTED), (dict(tokens=BIG), EUNSUPPORTED),
    (dict(desc=dict(table=FAKE + 2)), EUNSUPPORTED), (dict(lens=FAKE + 1), EUNSUPPORTED), (dict(slots=FAKE + 2), EUNSUPPORTED),
    (dict(parents=FAKE, mask=FAKE + 4), EUNSUPPORTED),
    (dict(desc=dict(requests=0, table=None, held=None, free_blocks=None, free_count=None), lens=None, offsets=None), OK)])
def test_tables_refusals(kw, status):
    assert tables(**kw) == status


def test_tables_refuse_null():
    assert gba.lib().gba_tables_step(None, FAKE, FAKE, None, 1, FAKE, FAKE, FAKE, FAKE, None, None) == EINVAL


def cache_desc(**kw):
    c = gba.PagedCacheDesc(gba.GBA_F16, 8, 16, 2, 64, FAKE, FAKE, 2048, 128, 64, 2048, 128, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def store(cache=(), **kw):
    a = dict(tokens=4, k=FAKE, kt=128, kh=64, v=FAKE, vt=128, vh=64, slots=FAKE)
    a.update(kw)
    return gba.lib().gba_cache_store(ctypes.byref(cache_desc(**dict(cache))), *a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(cache=dict(dtype=2)), EINVAL), (dict(cache=dict(num_blocks=-1)), EINVAL), (dict(cache=dict(block_size=0)), EINVAL),
    (dict(cache=dict(heads=-1)), EINVAL), (dict(cache=dict(dim=-1)), EINVAL), (dict(tokens=-1), EINVAL), (dict(k=None), EINVAL),
    (dict(v=None), EINVAL), (dict(slots=None), EINVAL), (dict(cache=dict(k=None)), EINVAL), (dict(cache=dict(v=None)), EINVAL),
    (dict(tokens=BIG), EUNSUPPORTED), (dict(cache=dict(num_blocks=2 ** 27)), EUNSUPPORTED), (dict(k=FAKE + 1), EUNSUPPORTED),
    (dict(cache=dict(v=FAKE + 1)), EUNSUPPORTED), (dict(slots=FAKE + 2), EUNSUPPORTED), (dict(tokens=0, k=None, v=None, slots=None), OK),
    (dict(cache=dict(num_blocks=0, k=None, v=None)), OK)])
def test_store_refusals(kw, status):
    assert store(**kw) == status


def attention(cache=(), call="gba_tree_attention", **kw):
    d = gba.AttentionDesc(cache_desc(**dict(cache)), 2, 4, 6, 3, 4, 0.125, FAKE, 256, 64, FAKE, 256, 64, FAKE, FAKE, FAKE, None, None, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    if call == "gba_tree_attention":
        return gba.lib().gba_tree_attention(ctypes.byref(d), None)
    return gba.lib().gba_tree_attention_workspace_size(ctypes.byref(d), ctypes.byref(ctypes.c_size_t()))


@pytest.mark.parametrize("call", ["gba_tree_attention", "gba_tree_attention_workspace_size"])
@pytest.mark.parametrize("kw,status", [
    (dict(cache=dict(dtype=3)), EINVAL), (dict(cache=dict(num_blocks=-1)), EINVAL), (dict(cache=dict(block_size=0)), EINVAL),
    (dict(requests=-1), EINVAL), (dict(width=-1), EINVAL), (dict(tokens=-1), EINVAL), (dict(max_new=-1), EINVAL),
    (dict(q_heads=-4), EINVAL), (dict(q_heads=3), EINVAL), (dict(cache=dict(heads=0)), EINVAL), (dict(q=None), EINVAL),
    (dict(out=None), EINVAL), (dict(lens=None), EINVAL), (dict(offsets=None), EINVAL), (dict(table=None), EINVAL),
    (dict(cache=dict(k=None)), EINVAL), (dict(cache=dict(v=None)), EINVAL), (dict(workspace=FAKE + 16), EINVAL),
    (dict(cache=dict(dim=60)), EUNSUPPORTED), (dict(cache=dict(dim=264)), EUNSUPPORTED), (dict(cache=dict(k_token=132)), EUNSUPPORTED),
    (dict(cache=dict(v_head=68)), EUNSUPPORTED), (dict(q_token=260), EUNSUPPORTED), (dict(out_head=66), EUNSUPPORTED),
    (dict(q=FAKE + 8), EUNSUPPORTED), (dict(out=FAKE + 8), EUNSUPPORTED), (dict(cache=dict(k=FAKE + 8)), EUNSUPPORTED),
    (dict(table=FAKE + 2), EUNSUPPORTED), (dict(mask=FAKE + 4), EUNSUPPORTED), (dict(mask=FAKE, max_new=65), EUNSUPPORTED),
    (dict(requests=gba.GBA_MAX_REQUESTS + 1), EUNSUPPORTED), (dict(tokens=BIG), EUNSUPPORTED), (dict(width=2 ** 28), EUNSUPPORTED),
    (dict(cache=dict(num_blocks=2 ** 27)), EUNSUPPORTED)])
def test_attention_refusals(kw, status, call):
    assert attention(call=call, **kw) == status


def test_attention_of_nothing():
    for kw in (dict(tokens=0), dict(requests=0), dict(max_new=0), dict(q_heads=0)):
        assert attention(q=None, out=None, lens=None, offsets=None, table=None, **kw) == OK
    assert gba.lib().gba_tree_attention(None, None) == EINVAL
    assert gba.lib().gba_tree_attention_workspace_size(None, ctypes.byref(ctypes.c_size_t())) == EINVAL


def test_binding_refuses_cpu_tensors_and_wrong_types():
    half = torch.zeros((1, 1, 16), dtype=torch.float16)
    codes = torch.zeros((1, 1, 64, 4), dtype=torch.int32)
    with pytest.raises(TypeError):
        decode.Q4Weight(codes, half, K=128, N=16)
    with pytest.raises(ValueError):
        decode.Q4Weight(codes, half, K=128, N=16, group=48)
    with pytest.raises(TypeError):
        decode.q4_pack(torch.zeros((128, 16), dtype=torch.uint8))
    with pytest.raises(TypeError):
        decode.PagedCache(torch.zeros((1, 1, 1, 8)), torch.zeros((1, 1, 1, 8)))
    i = torch.zeros((1, 1), dtype=torch.int32)
    with pytest.raises(TypeError):
        decode.BlockTables(i, i[0], i[0], i[0], 16, tokens=1)


def test_q4_groups_is_the_documented_layout():
    per_group = torch.arange(3 * 20, dtype=torch.float16).view(3, 20)
    out = decode.q4_groups(per_group)
    assert out.shape == (2, 3, 16) and out.is_contiguous()
    for g in range(3):
        for j in range(20):
            assert out[j // 16, g, j % 16] == per_group[g, j]


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_attention_refuses_a_scale_that_is_not_finite(scale):
    assert attention(scale=scale) == EINVAL
    assert attention(scale=scale, tokens=0) == EINVAL
