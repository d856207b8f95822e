"""The operators of a decoding step against plain 64-bit implementations."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import decode, gba  # noqa: E402

import decode_util as D  # noqa: E402

pytestmark = pytest.mark.gpu
HALF, BF16 = torch.float16, torch.bfloat16


def announce(*what):
    print("CASE", *what, flush=True)


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gba.lib()
    yield


# ------------------------------------------------------------------ linear

def weight(g, K, N, group, dtype, zeros, exact):
    """A random weight on the GPU and what it stands for in 64 bits.  exact:
    scales that are powers of two and whole zero points."""
    G = -(-K // group)
    codes = torch.randint(0, 16, (K, N), generator=g, dtype=torch.uint8)
    scales = 2.0 ** torch.randint(-4, -1, (G, N), generator=g) if exact else (torch.rand((G, N), generator=g) + 0.5) / (4.8 * math.sqrt(max(K, 1)))
    z = torch.randint(0, 16, (G, N), generator=g).float() if zeros else None
    scales = scales.to(dtype)
    z = None if z is None else z.to(dtype)
    w = decode.Q4Weight(decode.q4_pack(codes.cuda()), decode.q4_groups(scales.cuda()),
                        None if z is None else decode.q4_groups(z.cuda()), K=K, N=N, group=group)
    return w, D.dequantized(codes, scales, z, group)


SHAPES = [(1, 128, 16), (1, 1, 1), (3, 31, 17), (5, 127, 33), (16, 1000, 48), (17, 129, 15), (31, 257, 100), (33, 640, 64),
          (64, 1024, 40), (65, 136, 20), (130, 300, 35), (2, 2049, 16), (1, 8192, 7), (8, 8200, 19), (4, 4096, 1024)]


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_linear_whole_numbers(group, zeros, dtype):
    """Small whole inputs and scales that are powers of two: every fp32 sum is
    exact, so the result is the 64-bit one rounded once."""
    for i, (M, K, N) in enumerate(SHAPES):
        announce("linear exact", M, K, N, group, zeros, dtype)
        g = torch.Generator().manual_seed(100 + i)
        w, ref = weight(g, K, N, group, dtype, zeros, True)
        x = torch.randint(-4, 5, (M, K), generator=g).to(dtype)
        bias = torch.randint(-8, 9, (N,), generator=g).to(dtype) if i % 2 else None
        want = x.double() @ ref + (0 if bias is None else bias.double())
        for act in ("none", "relu"):
            got = decode.q4_linear(x.cuda(), w, None if bias is None else bias.cuda(), act=act)
            assert torch.equal(got.cpu(), D.activated(want, act).to(dtype)), (M, K, N, act)


# Every way a request may run: 1, 2 and 4 column blocks a workgroup (from 512 and
# 1024 of them on), 8 and 16 waves (from 16 chunks of K on), 16, 32 and 64 rows,
# rows that are copied straight to LDS and rows that are not.
WAYS = [(3, 300, 1000), (3, 2100, 1000), (2, 300, 8200), (2, 2100, 8200), (2, 140, 16400), (2, 2100, 16400), (20, 520, 100), (20, 520, 8200),
        (50, 520, 100), (50, 520, 8200), (20, 519, 8200), (50, 519, 100)]


@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_linear_every_way(way, group, zeros):
    M, K, N = WAYS[way]
    announce("linear way", M, K, N, group, zeros)
    g = torch.Generator().manual_seed(way)
    w, ref = weight(g, K, N, group, (HALF, BF16)[way % 2], zeros, True)
    x = torch.randint(-3, 4, (M, K), generator=g).to(w.dtype)
    want = (x.double().cuda() @ ref.cuda()).to(w.dtype)
    assert torch.equal(decode.q4_linear(x.cuda(), w), want)


@pytest.mark.parametrize("act", ["none", "relu", "sigmoid", "tanh"])
@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
def test_linear_rounding(dtype, act):
    """One rounding of the result, and fp32 sums: at most 280 additions of a
    group's terms (31 and 24 times an input and a scale) and of the groups, of
    which the errors add up like a random walk (16.7 steps; four deviations)."""
    for M, K, N, group, zeros in ((1, 1024, 1024, 128, False), (7, 1001, 203, 32, True), (64, 512, 72, 64, True)):
        announce("linear rounding", M, K, N, dtype, act)
        g = torch.Generator().manual_seed(7 + M)
        w, ref = weight(g, K, N, group, dtype, zeros, False)
        x, bias = torch.randn((M, K), generator=g).to(dtype), torch.randn((N,), generator=g).to(dtype)
        want = D.activated(x.double() @ ref + bias.double(), act)
        scale = float(w.scales.float().max())
        got = decode.q4_linear(x.cuda(), w, bias.cuda(), act=act).double().cpu()
        sums = 64 * 2.0 ** -24 * 55 * scale * x.double().abs().sum(1, keepdim=True)
        # sigmoid and tanh: a slope of at most 1 and an approximation of 2^-20
        assert ((got - want).abs() <= D.U[dtype] * want.abs() + sums + 2.0 ** -20).all()


def test_linear_strides_and_alignment():
    """Rows of x and out inside wider matrices, at addresses of 2 bytes."""
    g = torch.Generator().manual_seed(3)
    for M, K, N in ((5, 200, 50), (20, 333, 64)):
        for lead in (0, 1, 3):
            announce("linear strides", M, K, N, lead)
            w, ref = weight(g, K, N, 64, HALF, False, True)
            x = torch.randint(-3, 4, (M, K + 7), generator=g).half()
            out = torch.full((M, N + 9), 77.0, dtype=HALF, device="cuda")
            xs = x.cuda()[:, lead:lead + K]
            decode.q4_linear(xs, w, out=out[:, lead:lead + N])
            want = x[:, lead:lead + K].double() @ ref
            assert torch.equal(out[:, lead:lead + N].cpu(), want.half())
            left = torch.ones(N + 9, dtype=torch.bool)
            left[lead:lead + N] = False
            assert (out[:, left.cuda()] == 77).all()  # nothing beside the result is written


def test_linear_empty():
    w, _ = weight(torch.Generator().manual_seed(1), 64, 32, 32, HALF, False, True)
    assert decode.q4_linear(torch.empty((0, 64), dtype=HALF, device="cuda"), w).shape == (0, 32)
    w0 = decode.Q4Weight(torch.empty((2, 0, 64, 4), dtype=torch.int32, device="cuda"), torch.empty((2, 0, 16), dtype=HALF, device="cuda"), K=0, N=32)
    bias = torch.arange(-16, 16, dtype=HALF, device="cuda")
    got = decode.q4_linear(torch.empty((3, 0), dtype=HALF, device="cuda"), w0, bias, act="relu")
    assert torch.equal(got, bias.clamp_min(0).expand(3, 32))


def test_linear_padding_is_not_used():
    """Codes beyond K and N, whatever they are, change nothing."""
    g = torch.Generator().manual_seed(5)
    for K, N, group in ((100, 20, 32), (130, 5, 128), (33, 33, 64)):
        announce("linear padding", K, N, group)
        w, ref = weight(g, K, N, group, BF16, True, True)
        codes = decode.q4_pack(torch.full((-(-K // 128) * 128, -(-N // 16) * 16), 15, dtype=torch.uint8, device="cuda"))
        inside = decode.q4_pack(torch.full((K, N), 15, dtype=torch.uint8, device="cuda"))
        w.codes.copy_(w.codes | (codes & ~inside))
        x = torch.randint(-3, 4, (4, K), generator=g).to(BF16)
        assert torch.equal(decode.q4_linear(x.cuda(), w).cpu(), (x.double() @ ref).to(BF16))


def test_pack_is_the_documented_layout():
    g = torch.Generator().manual_seed(11)
    K, N = 300, 37
    codes = torch.randint(0, 256, (K, N + 3), generator=g, dtype=torch.uint8)  # high bits are not read
    packed = decode.q4_pack(codes.cuda()[:, :N]).cpu()
    for k, j in [(0, 0), (1, 0), (7, 15), (8, 16), (31, 36), (32, 3), (127, 5), (128, 9), (299, 36), (200, 20)]:
        word = int(packed[j // 16, k // 128, 16 * (k % 32 // 8) + j % 16, k % 128 // 32]) & 0xFFFFFFFF
        e = k % 8
        assert (word >> (4 * (e // 2) + 16 * (e % 2))) & 15 == int(codes[k, j]) & 15, (k, j)


# ------------------------------------------------------------------ tables

def same_step(tables, model, lens, new, parents):
    R, T = len(lens), tables.tokens
    i32 = dict(dtype=torch.int32, device="cuda")
    maps = tables.step(torch.tensor(lens, **i32), torch.tensor(new, **i32), None if parents is None else torch.tensor(parents, **i32))
    offsets, slots, positions, status, mask = model.step(lens, new, parents, T)
    assert maps.offsets.tolist() == offsets
    assert maps.status.tolist() == status
    assert maps.slots.tolist() == slots
    assert maps.positions.tolist() == positions
    if parents is not None:
        assert maps.mask.view(-1).tolist() == mask
    assert tables.held.tolist() == model.held
    assert int(tables.free_count) == len(model.free)
    assert tables.free_blocks[: len(model.free)].tolist() == model.free
    assert tables.table.tolist() == model.table
    return status


def random_parents(rng, T, wild):
    return [rng.randint(-3, 70) if wild and rng.random() < 0.1 else rng.randint(-1, 6) for _ in range(T)]


@pytest.mark.parametrize("requests,block,tree", [(1, 16, False), (4, 16, True), (63, 1, True), (65, 7, False), (300, 16, True),
                                                 (1023, 32, False), (1025, 16, True), (4096, 16, False), (4096, 64, True)])
def test_tables_follow_the_model(requests, block, tree):
    """Random steps with ended requests, rolled back drafts, too few blocks,
    requests too long for the table, and buffers too small for the tokens."""
    rng = random.Random(requests + block)
    width, most = 12, 70 if tree else 2 * block + 3
    blocks = max(1, requests * width // 3)
    tokens = max(8, requests * 12)
    tables = decode.BlockTables.empty(requests, width, blocks, block, tokens=tokens, tree=tree)
    model = D.TableModel(requests, width, blocks, block)
    lens, seen = [0] * requests, set()
    for step in range(8 if requests > 1000 else 20):
        announce("tables", requests, block, tree, step)
        new = [rng.choice([0, 1, 1, rng.randint(0, 9), rng.randint(0, most) if rng.random() < 0.2 else 2]) for _ in lens]
        asked = [-5 if rng.random() < 0.02 else n for n in lens]
        new = [-1 if rng.random() < 0.02 else c for c in new]
        parents = random_parents(rng, tokens, True) if tree else None
        status = same_step(tables, model, asked, new, parents)
        seen.update(status)
        # those that got room keep some of their tokens; others end now and then
        lens = [rng.choice([0, n]) if s else 0 if rng.random() < 0.1 else max(0, n) + rng.randint(0, max(0, c))
                for n, c, s in zip(asked, new, status)]
        lens = [min(n, h * block) for n, h in zip(lens, model.held)]
    assert 0 in seen


def test_tables_run_out_and_recover():
    tables, model = decode.BlockTables.empty(4, 8, 10, 16, tokens=64), D.TableModel(4, 8, 10, 16)
    announce("tables run out")
    assert same_step(tables, model, [0, 0, 0, 0], [16, 16, 1, 16], None) == [0, 0, 0, 0]
    # 10 - 4 left: 3 + 3 for the first two, nothing for the others -- but the third's block has room
    assert same_step(tables, model, [64, 64, 1, 16], [0, 0, 1, 1], None) == [0, 0, 0, 1]
    assert same_step(tables, model, [64, 0, 2, 16], [0, 0, 1, 1], None) == [0, 0, 0, 0]  # what the second gave back
    assert same_step(tables, model, [200, 0, 0, 0], [1, 0, 0, 0], None) == [2, 0, 0, 0]
    assert same_step(tables, model, [0, 0, 0, 0], [0, 60, 5, 5], None) == [0, 0, 3, 3]
    assert same_step(tables, model, [0, 0, 0, 0], [0, 0, 0, 0], None) == [0, 0, 0, 0]
    assert int(tables.free_count) == 10


def test_tables_blocks_pass_from_request_to_request():
    """One request ends and another takes its blocks in the same step."""
    tables, model = decode.BlockTables.empty(3, 600, 600, 4, tokens=8), D.TableModel(3, 600, 600, 4)
    announce("tables pass on")
    same_step(tables, model, [2000, 0, 100], [4, 0, 0], None)
    same_step(tables, model, [0, 2200, 90], [0, 3, 2], None)
    same_step(tables, model, [2300, 0, 0], [1, 0, 1], None)


def test_tables_graph():
    """A captured step replays on new lengths in the same buffers."""
    R, T = 40, 40 * 8
    tables, model = decode.BlockTables.empty(R, 16, 400, 8, tokens=T, tree=True), D.TableModel(R, 16, 400, 8)
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, new, parents = torch.zeros(R, **i32), torch.zeros(R, **i32), torch.full((T,), -1, **i32)
    out = tables.maps()
    announce("tables graph")
    tables.step(lens, new, parents, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tables.step(lens, new, parents, out=out)
    rng = random.Random(4)
    kept = [0] * R
    for _ in range(6):
        count = [rng.randint(0, 8) for _ in range(R)]
        par = random_parents(rng, T, False)
        lens.copy_(torch.tensor(kept))
        new.copy_(torch.tensor(count))
        parents.copy_(torch.tensor(par))
        graph.replay()
        torch.cuda.synchronize()
        offsets, slots, positions, status, mask = model.step(kept, count, par, T)
        assert (out.offsets.tolist(), out.slots.tolist(), out.positions.tolist(), out.status.tolist(), out.mask.view(-1).tolist()) == \
            (offsets, slots, positions, status, mask)
        assert tables.table.tolist() == model.table
        kept = [n + rng.randint(0, c) if s == 0 else 0 for n, c, s in zip(kept, count, status)]


# ------------------------------------------------------------------- store

@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("tokens,heads,dim,block", [(1, 1, 8, 1), (3, 2, 128, 16), (100, 3, 5, 7), (257, 4, 80, 16), (1, 16, 256, 64), (5000, 2, 64, 16)])
def test_store(tokens, heads, dim, block, dtype):
    g = torch.Generator().manual_seed(tokens + dim)
    blocks = 2 * (tokens // block + 1)
    for head_major, odd in ((False, 0), (True, 0), (False, 1)):
        announce("store", tokens, heads, dim, block, head_major, odd)
        caches = []
        for _ in range(2):
            c = torch.randn((blocks, heads, block, dim + odd) if head_major else (blocks, block, heads, dim + odd), generator=g).to(dtype).cuda()
            caches.append((c.permute(0, 2, 1, 3) if head_major else c)[..., odd:])
        qkv = torch.randn((tokens, 3 * heads, dim + odd), generator=g).to(dtype).cuda()[..., odd:]
        slots = torch.randperm(blocks * block, generator=g)[:tokens].to(torch.int32)
        # left out: negative, at the end, far away
        slots[1::5] = torch.tensor([-1, blocks * block, 2 ** 31 - 1, -2 ** 31])[torch.arange(len(slots[1::5])) % 4].to(torch.int32)
        want = [c.clone() for c in caches]
        for t, slot in enumerate(slots.tolist()):
            if 0 <= slot < blocks * block:
                want[0][slot // block, slot % block] = qkv[t, heads:2 * heads]
                want[1][slot // block, slot % block] = qkv[t, 2 * heads:]
        decode.PagedCache(*caches).store(qkv[:, heads:2 * heads], qkv[:, 2 * heads:], slots.cuda())
        assert torch.equal(caches[0], want[0]) and torch.equal(caches[1], want[1])


def test_store_nothing():
    k = torch.zeros((2, 4, 1, 8), dtype=HALF, device="cuda")
    none = torch.empty((0, 1, 8), dtype=HALF, device="cuda")
    decode.PagedCache(k, k.clone()).store(none, none, torch.empty((0,), dtype=torch.int32, device="cuda"))
    assert not k.any()


# --------------------------------------------------------------- attention

def attend(b, mask=None, max_new=None, **kw):
    cache = decode.PagedCache(b.k.cuda(), b.v.cuda())
    wide = torch.empty((b.q.shape[0], b.q.shape[1] + 3, b.q.shape[2]), dtype=b.dtype, device="cuda")
    q = wide[:, : b.q.shape[1]]
    q.copy_(b.q)
    return decode.tree_attention(q, cache, b.table.cuda(), torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda(),
                                 max_new=max(b.counts) if max_new is None else max_new,
                                 mask=None if mask is None else D.signed(mask).cuda(), **kw)


def tree_masks(rng, counts):
    masks = []
    for c in counts:
        mine = []
        for i in range(c):
            p = rng.randint(-1, i - 1)
            mine.append(1 << i | (mine[p] if p >= 0 else 0))
        masks += mine
    return masks


# heads, query heads a key head, head size, block size
LAYOUTS = [(1, 1, 64, 16), (2, 4, 128, 16), (1, 8, 80, 7), (3, 1, 8, 1), (2, 3, 256, 32), (1, 16, 96, 100), (2, 2, 120, 64), (1, 5, 136, 16)]


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_attention_single_tokens(layout, dtype):
    heads, share, dim, block = LAYOUTS[layout]
    lens = [0, 1, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 200, 333]
    announce("attention token", LAYOUTS[layout], dtype)
    b = D.Batch(layout, lens, [1] * len(lens), heads=heads, share=share, dim=dim, block=block, dtype=dtype, head_major=layout % 2 == 1)
    ref, spread = b.reference()
    D.check_attention(attend(b), ref, spread, dtype)


@pytest.mark.parametrize("dtype", [HALF, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_attention_trees(layout, dtype):
    """Trees of 0 to 64 drafts after 0 to 300 cached tokens."""
    heads, share, dim, block = LAYOUTS[layout]
    rng = random.Random(layout)
    lens, counts = [0, 0, 1, 5, 64, 100, 300, 7], [1, 64, 0, 33, 17, 2, 5, 0]
    announce("attention tree", LAYOUTS[layout], dtype)
    b = D.Batch(20 + layout, lens, counts, heads=heads, share=share, dim=dim, block=block, dtype=dtype, head_major=layout % 2 == 0)
    masks = tree_masks(rng, counts)
    ref, spread = b.reference(masks)
    D.check_attention(attend(b, masks), ref, spread, dtype)


def test_attention_any_mask_and_empty_rows():
    """Masks that no tree has: bits of later tokens, of none, and bits past
    the request's tokens, which mean nothing.  A token that sees nothing gets
    zeros."""
    rng = random.Random(9)
    lens, counts = [0, 0, 3, 40], [5, 64, 8, 20]
    announce("attention any mask")
    for dtype in (HALF, BF16):
        b = D.Batch(31, lens, counts, heads=2, share=2, dim=64, block=16, dtype=dtype)
        masks = [0 if rng.random() < 0.3 else rng.getrandbits(64) for _ in range(sum(counts))]
        ref, spread = b.reference(masks)
        got = attend(b, masks)
        D.check_attention(got, ref, spread, dtype)
        empty = [i for i in range(5) if masks[i] & 31 == 0]
        assert empty and not got[empty].any()


def test_attention_chain_of_many():
    """A chain longer than a mask has bits: a chunk of a prompt."""
    announce("attention chain")
    b = D.Batch(41, [0, 37, 64], [150, 70, 1], heads=1, share=2, dim=64, block=16, dtype=HALF)
    ref, spread = b.reference()
    D.check_attention(attend(b), ref, spread, HALF)


@pytest.mark.parametrize("share,dim,counts", [(1, 64, [1, 1]), (4, 128, [1, 3]), (4, 128, [40, 64]), (8, 64, [64, 5])])
def test_attention_long_requests(share, dim, counts):
    """Requests that are split across workgroups, and one that is not, with
    and without the room for it."""
    rng = random.Random(share)
    b = D.Batch(51 + dim, [9000, 30] if counts[0] > 1 else [30000, 70], counts, heads=1, share=share, dim=dim, block=16, dtype=BF16)
    masks = tree_masks(rng, counts)
    ref, spread = b.reference(masks)
    for workspace in ("auto", None):
        announce("attention long", share, dim, counts, workspace)
        D.check_attention(attend(b, masks, workspace=workspace), ref, spread, BF16)


def test_attention_many_requests():
    rng = random.Random(77)
    lens = [rng.choice([0, 1, rng.randint(0, 700)]) for _ in range(150)]
    counts = [rng.choice([0, 1, 1, 3]) for _ in lens]
    announce("attention many")
    b = D.Batch(61, lens, counts, heads=2, share=2, dim=64, block=16, dtype=HALF)
    ref, spread = b.reference()
    D.check_attention(attend(b), ref, spread, HALF)


def test_attention_large_scores():
    """Scores far apart: the weights of most keys vanish, and one key's value
    comes out as it is."""
    announce("attention large scores")
    b = D.Batch(71, [200, 1], [4, 1], heads=2, share=2, dim=128, block=16, dtype=HALF, q_scale=60.0)
    ref, spread = b.reference()
    D.check_attention(attend(b), ref, spread, HALF)


def test_attention_padding_and_missing_blocks():
    """Rows past the last request are left as they were; positions whose block
    is not in the cache count as not seen."""
    announce("attention padding")
    b = D.Batch(81, [50, 20], [2, 3], heads=2, share=2, dim=64, block=16, dtype=HALF, pad=3)
    out = torch.full(b.q.shape, 5.0, dtype=HALF, device="cuda")
    ref, spread = b.reference()
    got = attend(b, out=out)
    assert got.data_ptr() == out.data_ptr()
    D.check_attention(got[:5], ref, spread, HALF)
    assert (got[5:] == 5).all()
    b.table[0, 1], b.table[1, 0] = -1, 10 ** 6
    ref, spread = b.reference()
    D.check_attention(attend(b)[:5], ref, spread, HALF)


def test_attention_on_another_stream_and_in_a_graph():
    announce("attention graph")
    b = D.Batch(91, [3000, 500, 9], [4, 4, 4], heads=2, share=4, dim=128, block=16, dtype=BF16)
    masks = tree_masks(random.Random(2), b.counts)
    ref, spread = b.reference(masks)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = attend(b, masks, stream=None)
    cache = decode.PagedCache(b.k.cuda(), b.v.cuda())
    args = (b.q.cuda().contiguous(), cache, b.table.cuda(), torch.tensor(b.lens, dtype=torch.int32).cuda(), b.offsets.cuda())
    mask = D.signed(masks).cuda()
    torch.cuda.synchronize()
    there = decode.tree_attention(*args, max_new=4, mask=mask, stream=side)
    side.synchronize()
    assert torch.equal(got, there)
    out, ws = torch.empty_like(got), torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode.tree_attention(*args, max_new=4, mask=mask, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws[1 << 18:].fill_(255)  # all but the counters
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, got)
        assert not ws[: 1 << 18].any()
    D.check_attention(out, ref, spread, BF16)
