"""The cache in 4 bits and attention over it against plain 64-bit arithmetic."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode, gba  # noqa: E402

import decode_util as D  # noqa: E402
import q4_cache_util as Q  # noqa: E402
from test_window_gpu import tree_masks  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gba.lib()
    yield


# ------------------------------------------------------------------ store, load

def rows_of(seed, tokens, heads, dim, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((tokens, heads, dim), generator=g) * torch.exp(3 * torch.randn((tokens, heads, 1), generator=g))
    return x.to(dtype)


def same(a, b):
    """Equal, and NaN in the same places."""
    return bool((a == b).logical_or_(a.isnan() & b.isnan()).all())


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,heads,dim,block", [(1, 1, 8, 16), (3, 2, 128, 16), (100, 3, 64, 48), (257, 4, 80, 16), (33, 5, 256, 64), (70, 1, 136, 32), (9, 2, 96, 16)])
def test_store_and_load(tokens, heads, dim, block, group, dtype):
    print("CASE q4 store", tokens, heads, dim, block, group, dtype, flush=True)
    blocks = -(-tokens // block) + 2
    g = torch.Generator().manual_seed(tokens)
    slots = torch.randperm(blocks * block, generator=g)[:tokens].int()
    slots[::7] = torch.tensor([-1, blocks * block, 2 ** 31 - 1, -2 ** 31])[torch.arange(len(slots[::7])) % 4].int() if tokens > 7 else slots[::7]
    # keys and values as slices of a projection, one of them of odd strides
    wide = rows_of(tokens + 1, tokens, 3 * heads, dim, dtype).cuda()
    k, v = wide[:, heads:2 * heads], rows_of(tokens + 2, tokens, heads, dim + 3, dtype).cuda()[:, :, 1:dim + 1]
    if tokens > 3:
        k[2, 0], v[1, 0] = 1.5, 0.0  # groups of one value
    cache = Q.empty(blocks, block, heads, dim, dtype, group)
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scales, cache.v_scales)]
    cache.store(k, v, slots.cuda())
    there = (slots >= 0) & (slots < blocks * block)
    at = slots[there].long()
    real = -(-dim // group)
    for keys, x, stored, scales in ((True, k, cache.k, cache.k_scales), (False, v, cache.v, cache.v_scales)):
        codes, scale, offset = Q.rounded(x[there.cuda()].cpu(), group)
        got = Q.codes_of(stored, dim, keys)[at // block, :, at % block]
        assert torch.equal(got, codes)
        pairs = scales.cpu()[at // block, :, at % block]
        assert same(pairs[:, :, :real, 0].double(), scale) and same(pairs[:, :, :real, 1].double(), offset)
        assert not pairs[:, :, real:].any()
    # nothing else is written
    untouched = torch.ones(blocks * block, dtype=torch.bool)
    untouched[at] = False
    other = untouched.nonzero().view(-1)
    for was, t in zip(before, (cache.k, cache.v, cache.k_scales, cache.v_scales)):
        pick = lambda x: x.cpu()[other // block, :, other % block]  # noqa: E731
        assert torch.equal(pick(was).view(torch.uint8), pick(t).view(torch.uint8))
    # back: rounded once, zeros for rows that are not there; into tensors of other strides
    out = torch.full((tokens, heads + 1, dim + 5), 9.0, dtype=dtype, device="cuda")
    got_k, got_v = cache.load(slots.cuda(), v=out[:, 1:, 3:dim + 3])
    assert got_v.data_ptr() == out[:, 1:, 3:].data_ptr()
    assert (out[:, 0] == 9).all() and (out[:, :, :3] == 9).all() and (out[:, :, dim + 3:] == 9).all()
    for keys, got, stored, scales in ((True, got_k, cache.k, cache.k_scales), (False, got_v, cache.v, cache.v_scales)):
        want, _ = Q.values(stored[:, :, :, :], scales, dim, group, keys)
        want = want[at // block, :, at % block]
        assert (got.cpu()[~there] == 0).all()
        # one fp32 rounding, then one to the type
        got = got.cpu()[there].double()
        err = (got - want).abs()
        assert torch.equal(got.isnan(), want.isnan())
        assert (want.isnan() | (err <= (D.U[dtype] + 2.0 ** -23) * want.abs() + 2.0 ** -24 * (1 if dtype == HALF else 0))).all()


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
def test_store_of_extremes(dtype):
    """The type's largest and smallest values, infinities, NaN."""
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    sub = tiny * torch.finfo(dtype).eps
    x = torch.zeros((12, 1, 64))
    x[0, 0, 3], x[0, 0, 40] = big, -big
    x[1, 0, :] = big
    x[2, 0, 0] = tiny
    x[3, 0, ::2] = sub
    x[4, 0, 5] = math.inf
    x[5, 0, 50] = -math.inf
    x[6, 0, 9] = math.nan
    x[7] = -big
    x[8, 0, :32], x[8, 0, 32:] = torch.linspace(-1, 1, 32), math.nan
    x[9, 0] = torch.arange(64) - 100.0
    x[10, 0, :] = -math.inf
    x[11, 0, 1] = -0.0
    x = x.to(dtype)
    for group in (32, 64):
        cache = Q.empty(1, 16, 1, 64, dtype, group)
        slots = torch.arange(12, dtype=torch.int32).cuda()
        print("CASE q4 extremes", dtype, group, flush=True)
        cache.store(x.cuda(), x.cuda(), slots)
        codes, scale, offset = Q.rounded(x, group)
        for keys, stored, scales in ((True, cache.k, cache.k_scales), (False, cache.v, cache.v_scales)):
            assert torch.equal(Q.codes_of(stored, 64, keys)[0, 0, :12], codes[:, 0])
            pair = scales.double().cpu()[0, 0, :12]
            assert same(pair[..., 0], scale[:, 0]) and same(pair[..., 1], offset[:, 0])
        k, _ = cache.load(slots)
        bad = ~x.view(12, 64 // group, group).isfinite().all(2)
        assert torch.equal(k.cpu().view(12, 64 // group, group).isnan().all(2), bad) and torch.equal(k.cpu().isfinite().view(12, 64 // group, group).all(2), ~bad)


def test_rounding_is_to_the_nearest():
    """No value is further from its element than half a step and what the
    rounding of scale and offset adds (a part in 2^11 of 15 and 8 steps, and of
    the offset)."""
    x = rows_of(3, 50, 2, 128, HALF)
    cache = Q.empty(4, 16, 2, 128, HALF, 32)
    slots = torch.arange(50, dtype=torch.int32).cuda()
    cache.store(x.cuda(), x.cuda(), slots)
    k, _ = cache.load(slots)
    _, scale, offset = Q.rounded(x, 32)
    each = lambda t: t.repeat_interleave(32, -1)  # noqa: E731
    err = (k.cpu().double() - x.double()).abs()
    bound = each(scale) * (0.5 + 16 * 2.0 ** -11) + 2 * 2.0 ** -11 * (each(offset).abs() + x.double().abs()) + 2.0 ** -24
    assert (err <= bound).all()


def test_store_and_load_nothing():
    cache = Q.empty(2, 16, 1, 64, HALF, 64)
    none = torch.empty((0, 1, 64), dtype=HALF, device="cuda")
    cache.store(none, none, torch.empty(0, dtype=torch.int32, device="cuda"))
    k, v = cache.load(torch.empty(0, dtype=torch.int32, device="cuda"))
    assert k.shape == v.shape == (0, 1, 64)
    empty = decode.Q4Cache.empty(0, 16, 2, 64, BF16)
    one = torch.ones((1, 2, 64), dtype=BF16, device="cuda")
    empty.store(one, one, torch.zeros(1, dtype=torch.int32, device="cuda"))
    k, v = empty.load(torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert not k.any() and not v.any()


# ------------------------------------------------------------------ attention

# heads, query heads a key head, dim, block, group
LAYOUTS = [(1, 1, 64, 16, 64), (2, 4, 128, 16, 64), (1, 8, 80, 48, 32), (2, 1, 8, 16, 32), (2, 3, 256, 32, 64), (1, 16, 96, 112, 32),
           (2, 2, 120, 64, 128), (1, 5, 136, 16, 32), (1, 2, 64, 16, 32), (3, 2, 128, 32, 32), (1, 1, 200, 16, 128), (1, 2, 64, 16, 128)]


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_single_tokens(layout, dtype):
    heads, share, dim, block, group = LAYOUTS[layout]
    lens = [0, 1, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 200, 333]
    print("CASE q4 token", LAYOUTS[layout], dtype, flush=True)
    b = Q.Batch(layout, lens, [1] * len(lens), heads=heads, share=share, dim=dim, block=block, dtype=dtype, group=group)
    b.check(b.attend())
    for window, sinks in [(1, 0), (40, 3), (64, 70)]:
        b.check(b.attend(window=window, sinks=sinks), window=window, sinks=sinks, what=(window, sinks))


@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_several_tokens(layout, tree):
    heads, share, dim, block, group = LAYOUTS[layout]
    rng = random.Random(layout)
    lens, counts = [0, 0, 1, 5, 64, 100, 300, 7], [1, 64, 0, 33, 17, 2, 5, 0]
    print("CASE q4 several", LAYOUTS[layout], tree, flush=True)
    b = Q.Batch(20 + layout, lens, counts, heads=heads, share=share, dim=dim, block=block, dtype=[HALF, BF16][layout % 2], group=group)
    masks = tree_masks(rng, counts) if tree else None
    b.check(b.attend(masks), masks)
    for window, sinks in [(1, 0), (2, 1), (100, 5)]:
        b.check(b.attend(masks, window=window, sinks=sinks), masks, window, sinks, what=(window, sinks))


def test_any_mask_and_empty_rows():
    rng = random.Random(9)
    lens, counts = [0, 0, 3, 40], [5, 64, 8, 20]
    for dtype in (HALF, BF16):
        print("CASE q4 any mask", dtype, flush=True)
        b = Q.Batch(31, lens, counts, heads=2, share=2, dim=64, block=16, dtype=dtype, group=64)
        masks = [0 if rng.random() < 0.3 else rng.getrandbits(64) for _ in range(sum(counts))]
        got = b.attend(masks)
        b.check(got, masks)
        empty = [i for i in range(5) if masks[i] & 31 == 0]
        assert empty and not got[empty].any()


@pytest.mark.parametrize("share,dim,group", [(1, 64, 32), (4, 128, 64), (3, 64, 64), (2, 256, 128)])
def test_prompts(share, dim, group):
    b = Q.Batch(41, [0, 37, 700, 64], [700, 401, 300, 1], heads=1, share=share, dim=dim, block=16, dtype=HALF, group=group)
    for window, sinks in [(None, 0), (33, 3), (257, 70)]:
        for workspace in ("auto", None):
            print("CASE q4 prompt", share, dim, window, workspace, flush=True)
            b.check(b.attend(window=window, sinks=sinks, workspace=workspace), None, window, sinks)


@pytest.mark.parametrize("share,dim,counts", [(1, 64, [1, 1]), (4, 128, [1, 3]), (4, 128, [40, 64]), (8, 64, [64, 5])])
def test_long_requests(share, dim, counts):
    rng = random.Random(share)
    b = Q.Batch(51 + dim, [9000, 30] if counts[0] > 1 else [20000, 70], counts, heads=1, share=share, dim=dim, block=16, dtype=BF16, group=64)
    masks = tree_masks(rng, counts)
    for workspace in ("auto", None):
        for window, sinks in [(None, 0), (4001, 100)]:
            print("CASE q4 long", share, dim, counts, workspace, window, flush=True)
            b.check(b.attend(masks, workspace=workspace, window=window, sinks=sinks), masks, window, sinks)


def test_many_requests():
    rng = random.Random(77)
    lens = [rng.choice([0, 1, rng.randint(0, 700)]) for _ in range(150)]
    counts = [rng.choice([0, 1, 1, 3]) for _ in lens]
    b = Q.Batch(61, lens, counts, heads=2, share=2, dim=64, block=16, dtype=HALF, group=64)
    print("CASE q4 many", flush=True)
    b.check(b.attend())


def test_large_scores():
    b = Q.Batch(71, [200, 1], [4, 1], heads=2, share=2, dim=128, block=16, dtype=HALF, group=64, q_scale=60.0)
    print("CASE q4 large scores", flush=True)
    # (a score of some hundreds is off by 2^-14 relative to 1 / 60: 60 times the bound's)
    k, v, scale = b.read()
    got = b.attend().double().cpu()
    import window_util as W
    ref, _ = W.attention(b.q, k, v, b.table, b.lens, b.counts, None, b.scale, 1 << 40, 0)
    size, _ = W.attention(b.q, k, v.abs() + 8 * scale, b.table, b.lens, b.counts, None, b.scale, 1 << 40, 0)
    assert ((got - ref).abs() <= D.U[HALF] * ref.abs() + 60 * 2.0 ** -13 * size).all()


def test_negative_and_zero_scale():
    b = Q.Batch(72, [100, 3], [3, 2], heads=1, share=2, dim=64, block=16, dtype=BF16, group=32)
    for scale in (-0.2, 0.0):
        print("CASE q4 scale", scale, flush=True)
        got = b.attend(scale=scale)
        b.scale = scale
        b.check(got)


@pytest.mark.parametrize("rows", [1, 2, 5, 20])
def test_a_group_that_is_not_finite(rows):
    """The rows that see a value of NaN are NaN in its group, or in all of the
    row where a key is; others are not touched."""
    b = Q.Batch(17, [100, 50, 90], [rows, rows, rows], heads=2, share=2, dim=128, block=16, dtype=BF16, group=64)
    place = lambda r, p: (int(b.table[r, p // 16]), p % 16)  # noqa: E731
    page, at = place(0, 100 + rows - 1)  # of the last token: only its own row sees it
    b.cache.v_scales[page, 1, at, 1, 1] = math.nan
    page, at = place(1, 20)
    b.cache.v_scales[page, 0, at, 0, 0] = math.nan
    page, at = place(2, 90 + rows - 1)
    b.cache.k_scales[page, 1, at, 0, 1] = math.nan
    page, at = place(2, 30)  # before the window
    b.cache.v_scales[page, :, at] = math.nan
    b.cache.k_scales[page, :, at] = math.nan
    print("CASE q4 not finite", rows, flush=True)
    got = b.attend(window=85, sinks=2)
    b.check(got, None, 85, 2)
    assert got.isnan().any() and got.isfinite().any()


def test_padding_and_missing_blocks():
    b = Q.Batch(81, [50, 20], [2, 3], heads=2, share=2, dim=64, block=16, dtype=HALF, pad=3, group=64)
    out = torch.full(b.q.shape, 5.0, dtype=HALF, device="cuda")
    print("CASE q4 padding", flush=True)
    got = b.attend(out=out)
    assert got.data_ptr() == out.data_ptr() and (got[5:] == 5).all()
    b.check(got)
    b.table[0, 1], b.table[1, 0] = -1, 10 ** 6
    b.check(b.attend())


def test_an_empty_cache():
    cache = decode.Q4Cache.empty(0, 16, 1, 64, BF16)
    q = torch.ones((2, 1, 64), dtype=BF16, device="cuda")
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    got = decode.tree_attention(q, cache, i(0, 0, 0).view(1, 3), i(20), i(0, 2), max_new=2)
    assert not got.any()


@pytest.mark.parametrize("heads,share,dim,lens,counts", [
    (16, 4, 64, [500, 3000, 0, 2100], [64, 64, 60, 64]), (16, 4, 128, [2000, 2010, 2000, 1984], [64, 1, 64, 33]),
    (8, 8, 64, [2100 - 64 * i for i in range(10)] + [17 * i for i in range(10)], [i % 41 for i in range(20)]),
    (4, 4, 64, [(997 * i) % 2100 for i in range(64)], [16] * 64)])
def test_many_rows_of_requests_of_different_lengths(heads, share, dim, lens, counts):
    b = Q.Batch(61, lens, counts, heads=heads, share=share, dim=dim, block=32, dtype=BF16, group=64)
    assert 1024 <= len(lens) * heads * -(-max(counts) * share // 16) <= 4096 and b.table.shape[1] * 32 >= 2048
    masks = tree_masks(random.Random(len(lens)), counts)
    for words, window in [(None, None), (masks, None), (masks, 2050)]:
        print("CASE q4 lengths", heads, share, dim, words is not None, window, flush=True)
        b.check(b.attend(words, window=window, sinks=3 if window else 0), words, window, 3 if window else 0)


def test_on_another_stream_and_in_a_graph():
    b = Q.Batch(91, [3000, 500, 9], [4, 4, 4], heads=2, share=4, dim=128, block=16, dtype=BF16, group=64)
    q, cache, table, lens, offsets = b.arguments()
    q = q.contiguous()
    k, v = (torch.randn((12, 2, 128), device="cuda").to(BF16) for _ in range(2))
    slots = torch.tensor([int(b.table[r, (n + i) // 16]) * 16 + (n + i) % 16 for r, n in enumerate(b.lens) for i in range(4)], dtype=torch.int32).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, ws = torch.empty_like(q), torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    back = [torch.empty_like(k) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.store(k, v, slots)
        cache.load(slots, *back)
        decode.tree_attention(q, cache, table, lens, offsets, max_new=4, window=1000, sinks=4, out=out, workspace=ws)
    for less in (0, 5, 400, 0):
        now = [max(0, n - less) for n in b.lens]
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        k.normal_()
        v.normal_()
        out.zero_()
        print("CASE q4 graph", less, flush=True)
        graph.replay()
        torch.cuda.synchronize()
        there = decode.tree_attention(q, cache, table, lens, offsets, max_new=4, window=1000, sinks=4, stream=side)
        loaded = cache.load(slots, stream=side)
        side.synchronize()
        assert torch.equal(out, there) and torch.equal(loaded[0], back[0]) and torch.equal(loaded[1], back[1])
        b.check(out, None, 1000, 4, lens=now)
    assert not ws[: 1 << 18].any()


def test_a_step_with_tables_and_a_window():
    """Block tables, the store and attention with a window, step after step, with
    blocks that pass from request to request."""
    heads, share, dim, block, requests = 2, 2, 64, 16, 3
    tables = decode.BlockTables.empty(requests, 20, 40, block, tokens=requests * 40, tree=False)
    cache = Q.empty(40, block, heads, dim, HALF, 32)
    b = Q.Batch.__new__(Q.Batch)
    b.cache, b.dim, b.group, b.dtype, b.scale = cache, dim, 32, HALF, dim ** -0.5
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, rng = [0, 0, 0], random.Random(4)
    for step in range(8):
        new = [rng.choice([1, 1, 7, 40]) for _ in range(requests)]
        if step == 5:
            lens[1] = 0  # one ends and another begins in its place
        lens = [n if n + c <= 20 * block else 0 for n, c in zip(lens, new)]
        maps = tables.step(i(lens), i(new))
        rows = torch.randn((requests * 40, (share + 2) * heads, dim), device="cuda").to(HALF)
        cache.store(rows[:, share * heads:(share + 1) * heads], rows[:, (share + 1) * heads:], maps.slots)
        print("CASE q4 step", step, lens, new, flush=True)
        got = decode.tree_attention(rows[:, :share * heads], cache, tables.table, i(lens), maps.offsets, max_new=40, window=50, sinks=4)
        assert not maps.status.any()
        b.q, b.table, b.lens, b.counts = rows[:, :share * heads].cpu(), tables.table.cpu(), lens, new
        b.check(got, None, 50, 4)
        lens = [n + c for n, c in zip(lens, new)]


def test_refusals():
    H = dict(dtype=torch.uint8, device="cuda")
    k = torch.zeros((2, 1, 16, 32), **H)
    s = torch.zeros((2, 1, 16, 1, 2), dtype=HALF, device="cuda")
    decode.Q4Cache(k, k.clone(), s, s.clone(), dim=64)
    for bad in (dict(dim=60), dict(dim=264), dict(dim=0), dict(dim=128), dict(dim=64, group=32), dict(dim=64, group=48)):
        with pytest.raises(ValueError):
            decode.Q4Cache(k, k.clone(), s, s.clone(), **bad)
    with pytest.raises(ValueError):
        decode.Q4Cache(k[:, :, :8], k[:, :, :8], s, s, dim=64)
    with pytest.raises(TypeError):
        decode.Q4Cache(k.int(), k, s, s, dim=64)
    with pytest.raises(TypeError):
        decode.Q4Cache(k, k, s.float(), s, dim=64)
    with pytest.raises(TypeError):
        decode.Q4Cache(k, k, s, s.to(BF16), dim=64)
    b = Q.Batch(1, [5], [1], heads=1, share=1, dim=64, block=16, dtype=HALF, group=64)
    for kw in (dict(window=0), dict(window=-3), dict(window=4, sinks=-1)):
        with pytest.raises(gba.GbaError):
            b.attend(**kw)
    rows, slots = torch.zeros((1, 1, 64), dtype=HALF, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        b.cache.store(rows.float(), rows, slots)
    with pytest.raises(ValueError):
        b.cache.store(rows[:, :, :32], rows, slots)
    with pytest.raises(TypeError):
        b.cache.load(slots.long())
    with pytest.raises(ValueError):
        b.cache.load(slots, rows[:0])
