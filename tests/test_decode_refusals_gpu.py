"""What the decoding calls refuse of tensors on the GPU; nothing is launched,
and what was passed as an output stays as it is."""
import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode, gba  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


def gpu(*shape, dtype=HALF, fill=0):
    return torch.full(shape, fill, dtype=dtype, device="cuda")


def ints(*shape, fill=0):
    return gpu(*shape, dtype=torch.int32, fill=fill)


def weight():
    return decode.Q4Weight(ints(4, 2, 64, 4), gpu(4, 2, 16), K=256, N=60, group=128)


@pytest.mark.parametrize("change,error", [
    (dict(group=16), ValueError), (dict(K=384), ValueError), (dict(N=65), ValueError), (dict(codes="float"), TypeError),
    (dict(scales="cpu"), TypeError), (dict(scales="f32"), TypeError), (dict(scales="short"), ValueError), (dict(zeros="bf16"), TypeError),
    (dict(zeros="short"), ValueError)])
def test_weights(change, error):
    kinds = dict(cpu=lambda: torch.zeros(4, 2, 16, dtype=HALF), f32=lambda: gpu(4, 2, 16, dtype=torch.float32),
                 short=lambda: gpu(4, 1, 16), bf16=lambda: gpu(4, 2, 16, dtype=BF16), float=lambda: gpu(4, 2, 64, 4))
    a = dict(codes=ints(4, 2, 64, 4), scales=gpu(4, 2, 16), zeros=None, K=256, N=60, group=128)
    a.update({k: kinds[v]() if isinstance(v, str) else v for k, v in change.items()})
    with pytest.raises(error):
        decode.Q4Weight(a.pop("codes"), a.pop("scales"), a.pop("zeros"), **a)


@pytest.mark.parametrize("x,kw,error", [
    (lambda: torch.zeros(2, 256, dtype=HALF), {}, TypeError), (lambda: gpu(2, 256, dtype=BF16), {}, TypeError),
    (lambda: gpu(2, 255), {}, ValueError), (lambda: gpu(256), {}, ValueError), (lambda: gpu(256, 2).t(), {}, ValueError),
    (lambda: gpu(1, 256).expand(2, 256), {}, ValueError), (lambda: None, {}, TypeError),
    (lambda: gpu(2, 256), dict(act="gelu"), KeyError), (lambda: gpu(2, 256), dict(bias=lambda: gpu(64)), ValueError),
    (lambda: gpu(2, 256), dict(bias=lambda: gpu(60, dtype=BF16)), TypeError), (lambda: gpu(2, 256), dict(bias=lambda: gpu(120)[::2]), ValueError),
    (lambda: gpu(2, 256), dict(out=lambda: gpu(2, 64)), ValueError), (lambda: gpu(2, 256), dict(out=lambda: gpu(60, 2).t()), ValueError),
    (lambda: gpu(2, 256), dict(out=lambda: gpu(2, 60, dtype=torch.float32)), TypeError)])
def test_linear(x, kw, error):
    with pytest.raises(error):
        decode.q4_linear(x(), weight(), **{k: v() if callable(v) else v for k, v in kw.items()})


@pytest.mark.parametrize("args,error", [
    (lambda: (ints(4), ints(3)), ValueError), (lambda: (ints(5), ints(5)), ValueError), (lambda: (gpu(4), ints(4)), TypeError),
    (lambda: (torch.zeros(4, dtype=torch.int32), ints(4)), TypeError), (lambda: (ints(8)[::2], ints(4)), ValueError),
    (lambda: (ints(4), ints(4), ints(16)), ValueError), (lambda: (ints(4), [0] * 4), TypeError)])
def test_step(args, error):
    tables = decode.BlockTables.empty(4, 8, 16, 16, tokens=16)
    with pytest.raises(error):
        tables.step(*args())
    assert (tables.table == -1).all() and tables.free_count.item() == 16


def test_step_of_a_tree_and_its_outputs():
    tables = decode.BlockTables.empty(4, 8, 16, 16, tokens=16, tree=True)
    lens, new = ints(4), ints(4, fill=2)
    for parents, error in ((None, ValueError), (ints(15), ValueError), (gpu(16), TypeError)):
        with pytest.raises(error):
            tables.step(lens, new, parents)
    maps = tables.maps()
    for out, error in ((maps._replace(slots=ints(15)), ValueError), (maps._replace(mask=None), TypeError), (maps[:4], TypeError),
                       (maps._replace(mask=ints(16, 1)), TypeError), (list(maps), TypeError)):
        with pytest.raises(error):
            tables.step(lens, new, ints(16, fill=-1), out=out)
    assert (tables.table == -1).all() and tables.free_count.item() == 16
    with pytest.raises(ValueError):
        decode.BlockTables.empty(4, 8, 16, 0, tokens=16)
    with pytest.raises(TypeError):
        decode.BlockTables(gpu(4, 8), ints(4), ints(16), ints(1), 16, tokens=1)
    with pytest.raises(gba.GbaError):  # more requests than a step takes
        decode.BlockTables.empty(gba.GBA_MAX_REQUESTS + 1, 1, 1, 16, tokens=1).step(ints(gba.GBA_MAX_REQUESTS + 1), ints(gba.GBA_MAX_REQUESTS + 1))


@pytest.mark.parametrize("k,v,error", [
    (lambda: gpu(4, 16, 2, 64), lambda: gpu(4, 16, 2, 32), ValueError), (lambda: gpu(4, 16, 2, 64), lambda: gpu(4, 16, 2, 64, dtype=BF16), TypeError),
    (lambda: gpu(4, 16, 128), lambda: gpu(4, 16, 128), ValueError), (lambda: gpu(4, 16, 64, 2).transpose(2, 3), lambda: gpu(4, 16, 2, 64), ValueError),
    (lambda: torch.zeros(4, 16, 2, 64, dtype=HALF), lambda: gpu(4, 16, 2, 64), TypeError),
    (lambda: gpu(4, 16, 2, 64, dtype=torch.float32), lambda: gpu(4, 16, 2, 64, dtype=torch.float32), TypeError)])
def test_cache(k, v, error):
    with pytest.raises(error):
        decode.PagedCache(k(), v())


def cache():
    return decode.PagedCache(gpu(4, 16, 2, 64), gpu(4, 16, 2, 64))


@pytest.mark.parametrize("k,slots,error", [
    (lambda: gpu(3, 2, 32), lambda: ints(3), ValueError), (lambda: gpu(2, 2, 64), lambda: ints(3), ValueError),
    (lambda: gpu(3, 2, 64, dtype=BF16), lambda: ints(3), TypeError), (lambda: gpu(3, 2, 64), lambda: ints(3).long(), TypeError),
    (lambda: gpu(3, 2, 64), lambda: ints(6)[::2], ValueError), (lambda: gpu(3, 64, 2).transpose(1, 2), lambda: ints(3), ValueError)])
def test_store(k, slots, error):
    c = cache()
    with pytest.raises(error):
        c.store(k(), gpu(3, 2, 64, fill=1), slots())
    with pytest.raises(error):
        c.store(gpu(3, 2, 64, fill=1), k(), slots())
    assert not c.v.any() and not c.k.any()


@pytest.mark.parametrize("change,error", [
    (dict(q=lambda: gpu(6, 3, 64)), ValueError), (dict(q=lambda: gpu(6, 4, 32)), ValueError), (dict(q=lambda: gpu(6, 4, 64, dtype=BF16)), TypeError),
    (dict(q=lambda: gpu(6, 64, 4).transpose(1, 2)), ValueError), (dict(q=lambda: gpu(6, 256)), ValueError), (dict(table=lambda: ints(3, 2).t()), ValueError),
    (dict(table=lambda: ints(2, 3).long()), TypeError), (dict(lens=lambda: ints(3)), ValueError), (dict(offsets=lambda: ints(2)), ValueError),
    (dict(offsets=lambda: torch.zeros(3, dtype=torch.int32)), TypeError), (dict(mask=lambda: gpu(5, dtype=torch.int64)), ValueError),
    (dict(mask=lambda: ints(6)), TypeError), (dict(out=lambda: gpu(6, 2, 64)), ValueError), (dict(out=lambda: gpu(6, 4, 64, dtype=BF16)), TypeError),
    (dict(workspace=lambda: gpu(16, dtype=torch.int32)), TypeError), (dict(workspace=lambda: gpu(1024, dtype=torch.uint8)[1:]), gba.GbaError),
    (dict(mask=lambda: gpu(6, dtype=torch.int64), max_new=65), gba.GbaError), (dict(max_new=-1), gba.GbaError), (dict(scale="one"), TypeError),
    (dict(q=lambda: gpu(6, 4, 68)[:, :, :64]), gba.GbaError)])
def test_attention(change, error):
    a = dict(q=lambda: gpu(6, 4, 64), table=lambda: ints(2, 3), lens=lambda: ints(2), offsets=lambda: ints(3), max_new=3, out=lambda: gpu(6, 4, 64, fill=5))
    a.update(change)
    a = {k: v() if callable(v) else v for k, v in a.items()}
    with pytest.raises(error):
        decode.tree_attention(a.pop("q"), cache(), a.pop("table"), a.pop("lens"), a.pop("offsets"), **a)
    torch.cuda.synchronize()
    assert (a["out"] == 5).all() or "out" in change


def test_a_workspace_is_not_allocated_in_a_capture():
    c = decode.PagedCache(gpu(64, 16, 2, 64), gpu(64, 16, 2, 64))
    q, table, lens, offsets = gpu(2, 4, 64), ints(2, 64), ints(2), ints(3)
    stream = torch.cuda.Stream()
    decode._scratch.pop((0, stream.cuda_stream), None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(RuntimeError, match="workspace"):
                decode.tree_attention(q, c, table, lens, offsets, max_new=1)
