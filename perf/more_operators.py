"""The work that attention over bounded and compact caches is measured on.

Three kinds of case, for a decoding step over long texts:

  "window"  attention of each request's new tokens over a paged cache, each
            token seeing the last `window` ones of its text and a few first
            ones (sinks)
  "store"   new keys and values rounded to 4 bits in a paged cache, then read
            back from it
  "compact" attention over the cache in 4 bits: over all of it, or with a
            window

`own` says whether run() makes the calls of paper_2006_12645_amd.decode or
computes the same in elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}

# What no drawn case exceeds: the listed ones' largest number of cached elements
# (keys) of a rectangular batch, of scores, and of elements to store.
MOST_CACHED = 4 * 131072 * 8 * 128
MOST_SCORES = 1 << 28
MOST_STORED = 16384 * 1024


def _window(requests, new, shortest, longest, window, sinks, heads, share, dim, block, dtype, tree, mix):
    return {"kind": "window", "requests": requests, "new": new, "shortest": shortest, "longest": longest,
            "window": window, "sinks": sinks, "heads": heads, "share": share, "dim": dim, "block": block,
            "dtype": dtype, "tree": tree, "mix": mix}


def _store(tokens, heads, dim, group, block, dtype, mix):
    return {"kind": "store", "tokens": tokens, "heads": heads, "dim": dim, "group": group, "block": block,
            "dtype": dtype, "mix": mix}


def _compact(requests, new, shortest, longest, heads, share, dim, group, block, dtype, tree, mix, window=0, sinks=0):
    """window 0: there is none."""
    return dict(_window(requests, new, shortest, longest, window, sinks, heads, share, dim, block, dtype, tree, mix),
                kind="compact", group=group)


def listed():
    cases = [
        # one request, one token, a short window: latency of the call
        ("window_token", _window(1, 1, 6000, 6000, 1024, 4, 8, 4, 128, 16, "f16", False, 11)),
        # a full batch of long texts, one token each, in a window of 4096
        ("window_batch", _window(64, 1, 1000, 32768, 4096, 16, 8, 4, 128, 16, "bf16", False, 12)),
        # trees of up to 64 drafts, a window that ends inside pages
        ("window_trees", _window(16, 64, 500, 8192, 2000, 5, 8, 4, 128, 16, "f16", True, 13)),
        # the next 8192 tokens of a prompt after some thousand cached ones
        ("window_prompt", _window(1, 8192, 2500, 2500, 1024, 4, 8, 4, 128, 16, "bf16", False, 14)),
        # the new rows of eight requests, written and read back
        ("store_tokens", _store(8, 8, 128, 64, 16, "f16", 15)),
        # prompts of 16384 tokens in all, the finest groups
        ("store_prompts", _store(16384, 8, 128, 32, 16, "bf16", 16)),
        # one request, one token
        ("compact_token", _compact(1, 1, 1000, 1000, 8, 4, 128, 64, 16, "f16", False, 17)),
        # 64 requests of very different lengths, one token each
        ("compact_batch", _compact(64, 1, 16, 8192, 8, 4, 128, 64, 16, "bf16", False, 18)),
        # trees of up to 64 drafts: 256 query rows share each key
        ("compact_trees", _compact(16, 64, 500, 4096, 8, 4, 128, 64, 16, "bf16", True, 19)),
        # four very long requests, eight query heads a key head
        ("compact_long", _compact(4, 1, 60000, 131071, 8, 8, 128, 128, 64, "f16", False, 20)),
        # many long texts, small drafts, in a window over the cache in 4 bits
        ("compact_window", _compact(128, 4, 1000, 65536, 4, 4, 64, 32, 32, "bf16", False, 21, 4096, 8)),
    ]
    return [dict(case, name=name) for name, case in cases]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _some(rng, lo, hi):
    """lo to hi, over their logarithm: a power of two, or any."""
    v = _spread(rng, lo, hi)
    return max(lo, min(hi, 1 << round(math.log2(v)))) if rng.random() < 0.4 else v


def draw(rng):
    """One more case: 1 to 128 requests of 1 to 131072 cached tokens (windows:
    16 to 8192, up to 64 sinks) with one token, chains or trees of up to 64
    drafts, or prompts of up to 8192 tokens; head sizes 64 to 256, 1 to 8 query
    heads a key head, pages of 16 to 128 tokens; 1 to 16384 tokens to store;
    groups of 32, 64 or 128."""
    kind = rng.choice(["window", "store", "compact", "window", "compact"])
    dtype, mix = rng.choice(["f16", "bf16"]), rng.randrange(1 << 20)
    block, group = rng.choice([16, 16, 32, 64, 128]), rng.choice([32, 64, 64, 128])
    if kind == "store":
        heads, dim = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 96, 128, 256])
        return _store(min(_spread(rng, 1, 16384), MOST_STORED // (heads * dim)), heads, dim, group, block, dtype, mix)
    while True:
        requests, longest = _spread(rng, 1, 128), _spread(rng, 1, 131072)
        new = rng.choice([1, 1, _spread(rng, 2, 64), _spread(rng, 64, 8192) if kind == "window" else 1])
        heads, share = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 8])
        dim = rng.choice([64, 80, 128, 128, 256] if kind == "window" else [64, 96, 128, 128, 256])
        shortest = max(1, _spread(rng, longest / 32, longest)) if longest > 32 else 1
        tree = 1 < new <= 64 and rng.random() < 0.7
        windowed = kind == "window" or rng.random() < 0.4
        window, sinks = (_some(rng, 16, 8192), rng.choice([0, 4, rng.randint(1, 64)])) if windowed else (0, 0)
        case = _window(requests, new, shortest, longest, window, sinks, heads, share, dim, block, dtype, tree, mix)
        if kind == "compact":
            case.update(kind=kind, group=group)
        chunk, chunks, keys = _chunks(case)
        rows = requests * chunks * heads
        pool = requests * (longest + new) * heads * dim
        if pool <= MOST_CACHED and rows * keys * dim <= MOST_CACHED and rows * keys * share * chunk <= MOST_SCORES:
            return case


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _normal(g, std, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(std)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _lengths(case):
    """Cached and new tokens of every request: they are part of the case, since
    the work depends on them.  Cached lengths are spread over their logarithm;
    one request has the longest.  A tree has at least half of its tokens."""
    rng = random.Random(case["mix"])
    lo, hi, new = case["shortest"], case["longest"], case["new"]
    lens = [hi] + [_spread(rng, lo, hi) for _ in range(case["requests"] - 1)]
    rng.shuffle(lens)
    count = [rng.randint((new + 1) // 2, new) if case["tree"] else new for _ in lens]
    return lens, count


def _offsets(count):
    at = [0]
    for c in count:
        at.append(at[-1] + c)
    return at


def _masks(rng, count):
    """Bit j of a token's word: it is token j of its request, or descends from
    it, in a random tree: most tokens hang from one of the last few."""
    words, first = [], 0
    for c in count:
        for t in range(c):
            p = max(-1, t - 1 - int(rng.expovariate(0.7))) if t else -1
            words.append((1 << t) | (words[first + p] if p >= 0 else 0))
        first += c
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64).view(-1, 1).cuda()


def _width(dim):
    """Elements of a stored row: dim, padded."""
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def _stored(case, blocks):
    """Shapes of the codes (two in a byte) and of the scales and offsets."""
    width = _width(case["dim"])
    lead = (blocks, case["heads"], case["block"])
    return (*lead, width // 2), (*lead, max(1, width // case["group"]), 2)


def prepare(case, seed):
    """The tensors a program holds before the step, in the stored forms that
    the entry points document; the cache is wrapped in the package's handle
    where its kernels are to run."""
    s = _tensors(case, seed)
    if own:
        from paper_2006_12645_amd import decode
        if case["kind"] == "window":
            s["cache"] = decode.PagedCache(s["k_cache"], s["v_cache"])
        else:
            s["cache"] = decode.Q4Cache(s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"], dim=case["dim"],
                                        group=case["group"])
    return s


def _tensors(case, seed):
    g, rng, kind = _generator(seed), random.Random(seed), case["kind"]
    dtype, heads, dim, block = _TYPES[case["dtype"]], case["heads"], case["dim"], case["block"]
    if kind == "store":
        # the cache holds twice the tokens; runs of a block's slots, blocks in any order, every 16th row a padded one
        tokens = case["tokens"]
        blocks = 2 * (-(-tokens // block) + 1)
        at = torch.arange(tokens, device="cuda") + case["mix"] % block
        order = torch.randperm(blocks, generator=g, device="cuda")
        slots = order[at // block] * block + at % block
        slots[15::16] = -1
        qkv = _normal(g, 1.0, (tokens, 3 * heads, dim), dtype)
        codes, scales = _stored(case, blocks)
        empty = lambda: torch.zeros(codes, dtype=torch.uint8, device="cuda")                        # noqa: E731
        return {"case": case, "k": qkv[:, heads:2 * heads], "v": qkv[:, 2 * heads:], "slots": slots.to(torch.int32),
                "k_codes": empty(), "v_codes": empty(), "k_scales": torch.zeros(scales, dtype=dtype, device="cuda"),
                "v_scales": torch.zeros(scales, dtype=dtype, device="cuda")}
    lens, count = _lengths(case)
    need = [-(-(n + c) // block) for n, c in zip(lens, count)]
    blocks, width = sum(need) + 3, max(need)
    owner = torch.arange(width, device="cuda") < _ints(need).view(-1, 1)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    table[owner] = torch.randperm(blocks, generator=g, device="cuda", dtype=torch.int32)[: sum(need)]
    s = {"case": case, "q": _normal(g, 1.0, (sum(count), heads * case["share"], dim), dtype), "table": table,
         "lens": _ints(lens), "offsets": _ints(_offsets(count)), "mask": _masks(rng, count) if case["tree"] else None}
    if kind == "window":
        return {**s, "k_cache": _normal(g, 1.5, (blocks, block, heads, dim), dtype),
                "v_cache": _normal(g, 1.0, (blocks, block, heads, dim), dtype)}
    codes, scales = _stored(case, blocks)
    # any byte is two codes: uniform ones, as rounding between a group's ends leaves them about.  A code's deviation is
    # 4.6: keys of about 1.5, values of about 1, a middle that is off zero
    some = lambda: torch.randint(0, 256, codes, generator=g, device="cuda", dtype=torch.uint8)      # noqa: E731
    pair = lambda size: torch.stack([                                                               # noqa: E731
        (torch.rand(scales[:-1], generator=g, device="cuda") + 0.5) * (size / 4.8),
        torch.randn(scales[:-1], generator=g, device="cuda") * (0.2 * size)], -1).to(dtype)
    return {**s, "k_codes": some(), "v_codes": some(), "k_scales": pair(1.5), "v_scales": pair(1.0)}


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2006_12645_amd import decode
    case = s["case"]
    if case["kind"] == "store":
        s["cache"].store(s["k"], s["v"], s["slots"])
        return list(s["cache"].load(s["slots"]))
    return decode.tree_attention(s["q"], s["cache"], s["table"], s["lens"], s["offsets"], max_new=case["new"],
                                 mask=s["mask"], window=case["window"] or None, sinks=case["sinks"])


def _run_plain(s):
    return _plain_store(s) if s["case"]["kind"] == "store" else _plain_attend(s)


def _values(codes, scales, case, keys):
    """Rows of stored codes and their scales and offsets as 32-bit values: code
    2 i of a byte row in the low half of byte i.  The words of eight codes of a
    key's row stand transposed, word 4 s + g at place (width / 32) g + s."""
    width, lead = 2 * codes.shape[-1], codes.shape[:-1]
    if keys:
        codes = codes.view(*lead, 4, width // 32, 4).transpose(-3, -2).reshape(*lead, width // 2)
    q = torch.stack([codes & 15, codes >> 4], -1).view(*lead, scales.shape[-2], -1)
    scales = scales.float()
    v = (q.float() - 8.0) * scales[..., :1] + scales[..., 1:]
    return v.view(*lead, width)[..., : case["dim"]]


def _plain_store(s):
    case = s["case"]
    slots, block, dim, group, width = s["slots"], case["block"], case["dim"], case["group"], _width(case["dim"])
    # a padded row writes the last real row once more, at that row's slot
    t = torch.arange(len(slots), device=slots.device)
    real = slots >= 0
    row = torch.where(real, t, torch.where(real, t, 0).max())
    at = slots[row].long()
    there = torch.arange(width, device=slots.device).view(-1, min(group, width)) < dim

    def put(x, codes, scales, keys):
        x = x[row].float()
        x = torch.cat([x, x.new_zeros((*x.shape[:2], width - dim))], 2).view(*x.shape[:2], *there.shape)
        hi = torch.where(there, x, -math.inf).amax(3).clamp_min(-3e38)
        lo = torch.where(there, x, math.inf).amin(3).clamp_max(3e38)
        used = there.any(1)
        scale = torch.where(used, (0.5 * hi - 0.5 * lo) * (2.0 / 15.0), 0.0).to(scales.dtype).float()
        offset = torch.where(used, lo + 8.0 * scale, 0.0).to(scales.dtype).float()
        inverse = torch.where(scale > 0, 1.0 / scale, 0.0)
        q = (((x - offset.unsqueeze(3)) * inverse.unsqueeze(3)).round() + 8.0).clamp(0.0, 15.0)
        q = torch.where(there, q, 8.0).to(torch.uint8).view(*x.shape[:2], width // 2, 2)
        q = q[..., 0] | q[..., 1] << 4
        if keys:
            q = q.view(*q.shape[:2], width // 32, 4, 4).transpose(2, 3).reshape(*q.shape[:2], width // 2)
        codes[at // block, :, at % block] = q
        scales[at // block, :, at % block] = torch.stack([scale, offset], -1).to(scales.dtype)
        got = _values(codes[at // block, :, at % block], scales[at // block, :, at % block], case, keys)
        return torch.where(real.view(-1, 1, 1), got, 0.0).to(scales.dtype)

    return [put(s["k"], s["k_codes"], s["k_scales"], True), put(s["v"], s["v_codes"], s["v_scales"], False)]


def _chunks(case):
    """The plain form takes the new tokens of a request `chunk` at a time: as
    many chunks, each with `keys` keys at most (sinks and window)."""
    chunk = min(case["new"], 256)
    window = case["window"] or case["longest"] + case["new"]
    return chunk, -(-case["new"] // chunk), min(case["sinks"] + window + chunk, case["longest"] + case["new"])


def _plain_attend(s):
    case, q, mask = s["case"], s["q"], s["mask"]
    H, g, D, block, S = case["heads"], case["share"], case["dim"], case["block"], case["sinks"]
    W = case["window"] or case["longest"] + case["new"]
    C, n, X = _chunks(case)
    dev = q.device
    # each chunk is a request of its own, that of (request, chunk): what is before it is cached
    offsets, t0 = s["offsets"].long(), torch.arange(n, device=dev) * C
    count = ((offsets[1:] - offsets[:-1]).view(-1, 1) - t0).clamp(0, C).view(-1, 1)                # (R, 1)
    kept = (s["lens"].long().view(-1, 1) + t0).view(-1, 1)
    first = (offsets[:-1].view(-1, 1) + t0).view(-1, 1)
    table = s["table"].long().repeat_interleave(n, 0)
    R = len(kept)
    # its keys: the first S positions and those from the window of its first token on
    j = torch.arange(X, device=dev)
    pos = torch.where(j < S, j, j - S + (kept - W).clamp_min(S))                                   # (R, X)
    page = table.gather(1, (pos // block).clamp_max(table.shape[1] - 1))
    page, at = page.clamp_min(0).view(-1), (pos % block).view(-1)
    if case["kind"] == "window":
        rows = lambda c: c[page, at].float()                                                       # noqa: E731
        k, v = rows(s["k_cache"]), rows(s["v_cache"])
    else:
        k = _values(s["k_codes"][page, :, at], s["k_scales"][page, :, at], case, True)
        v = _values(s["v_codes"][page, :, at], s["v_scales"][page, :, at], case, False)
    k = k.view(R, X, H, D).permute(0, 2, 1, 3).contiguous()
    v = v.view(R, X, H, D).permute(0, 2, 1, 3).contiguous()
    # which of them each token sees
    i = torch.arange(C, device=dev)
    token = (first + i).clamp_max(len(q) - 1)                                                      # (R, C)
    p = pos.view(R, 1, X)
    if mask is None:
        last = (kept + i).view(R, C, 1)
        sees = (p <= last) & ((p > last - W) | (p < S))
    else:
        # a token's text: the cached tokens, then those of its mask in their order
        bits = (mask[token] >> torch.arange(64, device=dev)) & 1                                   # (R, C, 64)
        bits = torch.where(torch.arange(64, device=dev) < count.view(R, 1, 1), bits, 0)
        place = kept.view(R, 1, 1) + bits.cumsum(2) - bits
        begin = kept.view(R, 1, 1) + bits.sum(2, keepdim=True) - W                                 # of its window
        drafts = (bits > 0) & ((place >= begin) | (place < S))
        draft = p - kept.view(R, 1, 1)
        of_draft = drafts.gather(2, draft.clamp(0, 63).expand(R, C, X))
        sees = torch.where(draft < 0, (p >= begin) | (p < S), of_draft & (draft < 64))
    sees = (sees & (p < (kept + count).view(R, 1, 1))).view(R, 1, C, 1, X)
    # queries, (R, H, C g, D)
    x = q[token].float().view(R, C, H, g, D).permute(0, 2, 1, 3, 4).reshape(R, H, C * g, D)
    sc = (x @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(R, H, C, g, X)
    sc = torch.where(sees, sc, -math.inf)
    top = sc.amax(4, keepdim=True).clamp_min(-3e38)
    w = torch.exp(sc.sub_(top))
    total = w.sum(4, keepdim=True)
    o = (w.view(R, H, C * g, X) @ v).view(R, H, C, g, D) / total.clamp_min(1e-30)
    o = o.permute(0, 2, 1, 3, 4).reshape(R * C, H * g, D)
    t = torch.arange(len(q), device=dev)
    r = torch.searchsorted(offsets[1:].contiguous(), t, right=True).clamp_max(len(offsets) - 2)
    i = t - offsets[r]
    return o[(r * n + i // C) * C + i % C].to(q.dtype)


# ---------------------------------------------------------------- what it takes

def _row_bytes(case):
    """Of one head's key or value in the cache."""
    if case["kind"] == "window":
        return 2 * case["dim"]
    return case["dim"] / 2 + 4 * -(-case["dim"] // case["group"])


def work(case):
    """Inputs read once and outputs written once; two operations for every
    term of a product."""
    H, D = case["heads"], case["dim"]
    if case["kind"] == "store":
        # rows in, the stored form out, that in again, and rows out
        return {"bytes": 2 * case["tokens"] * H * (2 * D + 2 * _row_bytes(case) + 2 * D) + 8 * case["tokens"], "flops": 0}
    lens, count = _lengths(case)
    g = case["share"]
    W = case["window"] or case["longest"] + case["new"]
    S = case["sinks"] if case["window"] else 0
    # keys of a request that any of its tokens sees, and those that each one sees (a tree's token: with one of its request)
    some = [min(n + c, S + W + c - 1) for n, c in zip(lens, count)]
    pairs = sum(sum(min(n + 1 + (0 if case["tree"] else i), S + W) for i in range(c)) for n, c in zip(lens, count))
    pages = sum(-(-k // case["block"]) for k in some)
    return {"bytes": 2 * sum(some) * H * _row_bytes(case) + 4 * sum(count) * H * g * D + 4 * pages + 8 * len(lens) +
            (8 * sum(count) if case["tree"] else 0), "flops": 4 * H * g * D * pairs}


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in 64 bits."""
    s = _tensors(case, seed)
    if case["kind"] == "store":
        return _exact_store(case, s)
    lens, at, (H, g, D, block) = s["lens"].tolist(), s["offsets"].tolist(), (case["heads"], case["share"], case["dim"], case["block"])
    words = None if s["mask"] is None else [w & (1 << 64) - 1 for w in s["mask"].view(-1).tolist()]
    window, sinks = case["window"] or 1 << 40, case["sinks"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for r, n in enumerate(lens):
        c = at[r + 1] - at[r]
        for a in range(0, c, 512):
            b = min(a + 512, c)
            # the positions that any of tokens a .. b - 1 sees, and what each of them does not
            lowest = max(0, n + (a if words is None else 0) - window)
            near = torch.arange(max(lowest, sinks), n + (c if words is not None else b))
            pos = torch.cat([torch.arange(min(sinks, n + c)), near])
            if words is None:
                own_place = torch.arange(n + a, n + b).view(-1, 1)
                hidden = ~((pos <= own_place) & ((pos < sinks) | (own_place - pos < window)))
            else:
                hidden = torch.ones((b - a, len(pos)), dtype=torch.bool)
                for t in range(a, b):
                    text = [d for d in range(c) if words[at[r] + t] >> d & 1]
                    length = n + len(text)
                    seen = (pos < n) & ((pos < sinks) | (pos >= length - window))
                    for place, d in enumerate(text):
                        if n + place < sinks or n + place >= length - window:
                            seen |= pos == n + d
                    hidden[t - a] = ~seen
            hidden = hidden.cuda().repeat_interleave(g, 0)
            pos = pos.cuda()
            page, within = s["table"][r, pos // block].long(), pos % block
            for h in range(H):
                if case["kind"] == "window":
                    k, v = s["k_cache"][page, within, h].double(), s["v_cache"][page, within, h].double()
                else:
                    k = _exact_values(case, s["k_codes"][page, h, within], s["k_scales"][page, h, within], True)
                    v = _exact_values(case, s["v_codes"][page, h, within], s["v_scales"][page, h, within], False)
                x = s["q"][at[r] + a:at[r] + b, h * g:(h + 1) * g].double().reshape((b - a) * g, -1)
                score = (x @ k.t().contiguous() * D ** -0.5).masked_fill_(hidden, -math.inf)
                out[at[r] + a:at[r] + b, h * g:(h + 1) * g] = (torch.softmax(score, 1) @ v).view(b - a, g, -1)
    return out


def _exact_values(case, codes, scales, keys):
    """value = scale (code - 8) + offset, element by element of dim."""
    d = torch.arange(case["dim"], device=codes.device)
    word, width = d // 8, 2 * codes.shape[-1]
    if keys:
        word = word % 4 * (width // 32) + word // 4
    byte = codes[..., word * 4 + d % 8 // 2].long()
    code = torch.where(d % 2 == 1, byte // 16, byte % 16).double()
    of = scales[..., d // case["group"], :].double()
    return of[..., 0] * (code - 8) + of[..., 1]


def _exact_store(case, s):
    """Each step of the rounding in 64 bits, rounded to the 32 bits (scale and
    offset: to the cache's type) that the definition gives it; the value that
    the code stands for in 64."""
    dtype, dim = _TYPES[case["dtype"]], case["dim"]
    real = (s["slots"] >= 0).view(-1, 1, 1)
    single = lambda v: v.float().double()                                                           # noqa: E731
    fifteenth = float(torch.tensor(2 / 15))  # in 32 bits, of half the range
    outs = []
    for x in (s["k"], s["v"]):
        out = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        for d in range(0, dim, case["group"]):
            y = x[:, :, d:d + case["group"]].double()
            low, high = y.min(2, keepdim=True).values, y.max(2, keepdim=True).values
            scale = single(single(high / 2 - low / 2) * fifteenth).to(dtype).double()
            offset = single(low + 8 * scale).to(dtype).double()
            steps = single(single(y - offset) * single(1 / scale))
            code = (torch.round(steps) + 8).clamp(0, 15)
            value = torch.where(scale > 0, scale * (code - 8), 0.0) + offset
            out[:, :, d:d + case["group"]] = torch.where(real, value, 0.0)
        outs.append(out)
    return outs
