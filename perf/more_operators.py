"""Positions of queries and keys, and many requests over one cached prefix: what is measured of them, and their plain forms.

Operators: ``rotate`` norms the rows of queries and keys (where weights are given) and turns them by their positions, which have one
axis or several; ``append`` does so for a serving step and writes its keys and values into a key/value cache held in 4 bits, read back
here as the values it then stands for; ``shared`` attends over such a cache where the requests of a group share a prefix and have keys
of their own behind it.

The cache is made of pages of ``page`` tokens: codes ``[pages, KV heads, page, d/2]`` and scales ``[pages, KV heads, page, d/32]``,
bytes, for K and for V.  Elements are E2M1 (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign; element 2i in the low half of byte i), blocks of
32 elements of a row share a power of two (byte e stands for 2^(e - 127)).
"""
import math
import random

import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6
# (query heads, KV heads, head_dim) of the repository's configurations and tests
HEADS = [(2, 1, 64), (8, 2, 64), (16, 2, 128), (28, 4, 128), (8, 8, 128)]
PAGES = [16, 32, 64, 128]
# how the pairs of a row go with the axes of the positions: all with one; an eighth (or so) with time, the others with height and
# width, in runs; the three in turn
AXES = ["text", "runs", "turns"]


def listed():
    return [
        # one token of the smallest configuration; a short prompt with partial rotation of neighbouring elements
        dict(name="rotate-token", op="rotate", tokens=1, hq=2, hkv=1, d=64, rot=64, axes="text", adjacent=False, norm=True, fused=True),
        dict(name="rotate-prompt", op="rotate", tokens=333, hq=8, hkv=2, d=64, rot=32, axes="text", adjacent=True, norm=False, fused=False),
        # a host's block of a video, out of the projection's joint output; a longer block with norms
        dict(name="rotate-block", op="rotate", tokens=16384, hq=16, hkv=2, d=128, rot=128, axes="runs", adjacent=False, norm=False, fused=True),
        dict(name="rotate-frames", op="rotate", tokens=32768, hq=28, hkv=4, d=128, rot=128, axes="turns", adjacent=False, norm=True, fused=True),
        # a decoding step: of one request, of a server's batch; a video's block going straight into the cache
        dict(name="append-token", op="append", tokens=1, hq=2, hkv=1, d=64, page=16, rot=64, axes="text", adjacent=False, norm=False, skip=0),
        dict(name="append-step", op="append", tokens=64, hq=28, hkv=4, d=128, page=64, rot=128, axes="runs", adjacent=False, norm=True, skip=3),
        dict(name="append-block", op="append", tokens=16384, hq=16, hkv=2, d=128, page=64, rot=128, axes="turns", adjacent=False, norm=True, skip=333),
        # two requests behind a short prefix; 64 questions about one long video; a server's batch behind a long system prompt;
        # questions about several videos; the questions themselves, chunks of many tokens, before they are answered
        dict(name="shared-tiny", op="shared", n=2, groups=1, hq=2, hkv=1, d=64, page=16, p_lo=700, p_hi=700, q_lo=1, q_hi=1, k_lo=3, k_hi=40, lse=False),
        dict(name="shared-video", op="shared", n=64, groups=1, hq=16, hkv=2, d=128, page=64, p_lo=133120, p_hi=133120, q_lo=1, q_hi=1, k_lo=16, k_hi=512, lse=False),
        dict(name="shared-batch", op="shared", n=256, groups=1, hq=28, hkv=4, d=128, page=64, p_lo=32768, p_hi=32768, q_lo=1, q_hi=1, k_lo=65, k_hi=2048, lse=False),
        dict(name="shared-videos", op="shared", n=48, groups=7, hq=8, hkv=2, d=64, page=32, p_lo=1500, p_hi=16384, q_lo=1, q_hi=1, k_lo=5, k_hi=1000, lse=True),
        dict(name="shared-questions", op="shared", n=16, groups=1, hq=28, hkv=4, d=128, page=64, p_lo=40000, p_hi=40000, q_lo=7, q_hi=48, k_lo=48, k_hi=300, lse=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotate", "rotate", "append", "append", "shared", "shared", "shared", "shared"])
    hq, hkv, d = rng.choice(HEADS)
    if op in ("rotate", "append"):
        most = (1 << 20) // (hq + hkv) if op == "rotate" else (1 << 18) // (hq + hkv)
        c = dict(op=op, tokens=_log_int(rng, 1, most), hq=hq, hkv=hkv, d=d, rot=rng.choice([d, d, d, d // 2]), axes=rng.choice(AXES),
                 adjacent=rng.random() < 0.25, norm=rng.random() < 0.5)
        if op == "rotate":
            c.update(fused=rng.random() < 0.5)
        else:
            c.update(page=rng.choice(PAGES), skip=rng.choice([0, c["tokens"] // 7]))
        return c
    c = dict(op=op, n=1, groups=1, hq=hq, hkv=hkv, d=d, page=rng.choice(PAGES), q_lo=1, q_hi=1, lse=rng.random() < 0.5)
    kind = rng.choice(["video", "video", "videos", "questions"])
    if kind == "video":
        n = _log_int(rng, 2, 256)
        k = _log_int(rng, 16, 2048)
        p = _log_int(rng, 256, min(160000, 200000000 // (n * hq)))
        c.update(n=n, p_lo=p, p_hi=p, k_lo=rng.randint(1, k), k_hi=k)
    elif kind == "videos":
        n = rng.randint(8, 96)
        k = _log_int(rng, 16, 2048)
        p = _log_int(rng, 256, 24000)
        c.update(n=n, groups=rng.randint(2, 8), p_lo=rng.randint(64, p), p_hi=p, k_lo=rng.randint(1, k), k_hi=k)
    else:
        q = rng.randint(4, 64)
        k = _log_int(rng, 64, 600)
        p = _log_int(rng, 1024, 32768)
        c.update(n=rng.randint(2, 12), q_hi=q, p_lo=p, p_hi=p, k_lo=rng.randint(64, k), k_hi=k)
    return c


# ---- sizes: the case gives them all, the seed only their order and the values

def _spread(rng, n, lo, hi):
    """n whole numbers between lo and hi, both ends among them, spread over their logarithm."""
    if n == 1:
        return [hi]
    return [lo, hi] + [_log_int(rng, lo, hi) for _ in range(n - 2)]


def _requests(case):
    """Of a ``shared`` case: queries and own keys of every request, the prefix of every group, and how many requests it has."""
    c = case
    rng = random.Random(str([c[k] for k in sorted(c) if k != "name"]))
    keys = _spread(rng, c["n"], c["k_lo"], c["k_hi"])
    queries = _spread(rng, c["n"], c["q_lo"], c["q_hi"])
    prefixes = _spread(rng, c["groups"], c["p_lo"], c["p_hi"])
    cuts = sorted(rng.sample(range(1, c["n"]), c["groups"] - 1))
    sizes = [b - a for a, b in zip([0] + cuts, cuts + [c["n"]])]
    return [(min(q, k), k) for q, k in zip(queries, keys)], prefixes, sizes


def _ceil(a, b):
    return -(-a // b)


def _n_axes(case):
    return 1 if case["axes"] == "text" else 3


def work(case):
    c = case
    if c["op"] == "shared":
        requests, prefixes, sizes = _requests(c)
        rows, at, pairs = sum(q for q, _ in requests), 0, 0
        for p, n in zip(prefixes, sizes):
            pairs += p * sum(q for q, _ in requests[at:at + n])
            at += n
        pairs += sum(q * k - q * (q - 1) // 2 for q, k in requests)
        lengths = prefixes + [k for _, k in requests]
        held = 2 * c["hkv"] * (c["d"] // 2 + c["d"] // 32)
        nbytes = sum(lengths) * held + 4 * sum(_ceil(x, c["page"]) for x in lengths) + 4 * rows * c["hq"] * c["d"] + (4 * rows * c["hq"] if c["lse"] else 0)
        return {"bytes": nbytes, "flops": 4 * c["d"] * pairs * c["hq"]}
    per = 10 if c["norm"] else 6                                    # operations a pair
    small = c["tokens"] * 4 * _n_axes(c) + 2 * c["rot"] + (4 * c["d"] if c["norm"] else 0)
    if c["op"] == "rotate":
        elements = c["tokens"] * (c["hq"] + c["hkv"]) * c["d"]
        return {"bytes": 4 * elements + small, "flops": per * elements // 2}
    live = c["tokens"] - c["skip"]
    wide, held = 4 * c["hkv"] * c["d"], 2 * c["hkv"] * (c["d"] // 2 + c["d"] // 32)
    nbytes = 4 * c["tokens"] * c["hq"] * c["d"] + small + 8 * c["tokens"] + live * (wide + 2 * held) + c["tokens"] * wide
    return {"bytes": nbytes, "flops": per * (c["tokens"] * c["hq"] + live * c["hkv"]) * c["d"] // 2 + 4 * live * c["hkv"] * c["d"]}


# ---- the format

def _encode(x):
    """float [..., d] -> codes uint8 [..., d/2], scale bytes uint8 [..., d/32]."""
    b = x.unflatten(-1, (-1, 32))
    m = b.abs().amax(-1, keepdim=True)
    frac, exp = torch.frexp(m)                                     # m = frac * 2^exp, frac in [.5, 1)
    e = (exp - 3 + (frac > 0.875)).clamp(-125, 125)
    e = torch.where(m == 0, torch.full_like(e, -125), e)
    y = torch.ldexp(b, -e)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(a.dtype)
    a = (torch.round(a / step) * step).clamp(max=6.0)              # torch.round: halves to even, which is the even code here
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8).flatten(-2)


def _decode(codes, scales):
    """The float32 values that codes and scales stand for."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float32, device=codes.device)
    x = grid[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (x.unflatten(-1, (-1, 32)) * torch.exp2(scales.float() - 127.0)[..., None]).flatten(-2)


# ---- inputs

def _rows(g, n, heads, d, strong):
    """Rows of unit normal values; keys have a few strong channels."""
    x = torch.randn((n, heads, d), generator=g, device="cuda")
    if strong:
        x[..., :: d // 4] *= 4.0
    return x.bfloat16()


def _cache(g, n_pages, hkv, page, d):
    """A cache whose every slot holds a row."""
    c = dict(k_codes=(d // 2,), v_codes=(d // 2,), k_scales=(d // 32,), v_scales=(d // 32,))
    c = {name: torch.empty((n_pages, hkv, page) + tail, dtype=torch.uint8, device="cuda") for name, tail in c.items()}
    step = max(1, 4194304 // (page * hkv))
    for p in range(0, n_pages, step):
        e = min(n_pages, p + step)
        for x in "kv":
            codes, scales = _encode(_rows(g, (e - p) * page, hkv, d, x == "k").float())
            c[x + "_codes"][p:e] = codes.view(e - p, page, hkv, -1).transpose(1, 2)
            c[x + "_scales"][p:e] = scales.view(e - p, page, hkv, -1).transpose(1, 2)
    return c


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _positions(case, rng):
    """[axes, tokens]: text counts up from somewhere; a video has a time per frame and places in it, rows of 18 behind one another."""
    c = case
    first = rng.randrange(200000)
    t = torch.arange(c["tokens"], device="cuda", dtype=torch.int32)
    if c["axes"] == "text":
        return (first + t)[None].contiguous()
    return torch.stack((first + t // 252, first + t // 18 % 14, first + t % 18)).contiguous()


def _axis_of(case):
    """The axis that each pair goes with."""
    pairs = case["rot"] // 2
    if case["axes"] == "text":
        return [0] * pairs
    if case["axes"] == "turns":
        return [i % 3 for i in range(pairs)]
    a, b = pairs // 4, pairs // 4 + (pairs - pairs // 4) // 2
    return [0 if i < a else 1 if i < b else 2 for i in range(pairs)]


def _table(pool, at, lengths, page):
    """Pages of `pool` from entry `at` on for rows of these lengths; and the next entry."""
    blocks = [_ceil(x, page) for x in lengths]
    rows = []
    for b in blocks:
        rows.append(pool[at:at + b] + [0] * (max(blocks) - b))
        at += b
    return _ints(rows), at


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    s = dict(case=c)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    empty = lambda shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")
    if own:
        import paper_2601_21444_amd as apbv
        s["apbv"] = apbv
    if c["op"] in ("rotate", "append"):
        n = c["tokens"]
        joint = torch.cat((_rows(g, n, hq, d, False), _rows(g, n, hkv, d, True), _rows(g, n, hkv, d, False)), 1)
        s["q"], s["k"], s["v"] = joint[:, :hq], joint[:, hq:hq + hkv], joint[:, hq + hkv:]
        if c["op"] == "rotate" and not c["fused"]:
            s["q"], s["k"] = s["q"].contiguous(), s["k"].contiguous()
        s["positions"] = _positions(c, rng)
        s["inv_freq"] = (1e6 ** (-torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) / (c["rot"] // 2))).float()
        s["axis"] = _axis_of(c)
        s["wq"], s["wk"] = ((1.0 + 0.25 * torch.randn(d, generator=g, device="cuda")).bfloat16() if c["norm"] else None for _ in range(2))
        if c["op"] == "append":
            page = c["page"]
            n_pages = _ceil(n, page) + 5
            s["cache"] = _cache(g, n_pages, hkv, page, d)
            # consecutive tokens fill pages of a scattered order; skipped ones are padding
            order = torch.tensor(rng.sample(range(n_pages), n_pages), device="cuda")
            at = torch.arange(n, device="cuda") + rng.randrange(page)
            slots = order[at // page] * page + at % page
            slots[torch.randperm(n, generator=g, device="cuda")[:c["skip"]]] = -1
            s["slots"] = slots.int()
        if own:
            s["rotation"] = apbv.ApbvRotation(s["inv_freq"], d, axis=s["axis"], adjacent=c["adjacent"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS)
            s["out"] = dict(q_out=empty((n, hq, d)))
            if c["op"] == "rotate":
                s["out"]["k_out"] = empty((n, hkv, d))
            else:
                s["handle"] = apbv.ApbvCache(**s["cache"])
                s["loaded"] = dict(k_out=empty((n, hkv, d)), v_out=empty((n, hkv, d)))
        return s
    requests, prefixes, sizes = _requests(c)
    page, n, groups = c["page"], c["n"], c["groups"]
    rng.shuffle(requests)
    order = rng.sample(range(groups), groups)
    prefixes, sizes = [prefixes[i] for i in order], [sizes[i] for i in order]
    lengths = [k for _, k in requests]
    n_pages = sum(_ceil(x, page) for x in prefixes + lengths) + 3
    s["cache"] = _cache(g, n_pages, hkv, page, d)
    pool = rng.sample(range(n_pages), n_pages)
    s["prefix_table"], at = _table(pool, 0, prefixes, page)
    s["table"], at = _table(pool, at, lengths, page)
    starts = [sum(q for q, _ in requests[:i]) for i in range(n + 1)]
    members = [sum(sizes[:i]) for i in range(groups + 1)]
    rows = starts[-1]
    s.update(q=torch.randn((rows, hq, d), generator=g, device="cuda").bfloat16(), prefix_lengths=_ints(prefixes), lengths=_ints(lengths),
             starts=_ints(starts), members=_ints(members), max_q=max(q for q, _ in requests),
             max_group=max(starts[b] - starts[a] for a, b in zip(members, members[1:])), scale=1.0 / math.sqrt(d))
    if own:
        s["handle"] = apbv.ApbvCache(**s["cache"])
        nbytes = apbv.apbv_cache_shared_attention_workspace_bytes(groups, n, rows, hq, hkv, d, s["max_q"])
        s["out"] = dict(out=empty((rows, hq, d)), workspace=empty(max(nbytes, 256), torch.uint8))
        if c["lse"]:
            s["out"]["lse_out"] = empty((hq, rows), torch.float32)
    return s


# ---- one pass

def _turned(x, weight, cos, sin, case):
    """Rows [tokens, heads, d] of cos's type, normed and turned."""
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.to(x.dtype)
    rot, half = case["rot"], case["rot"] // 2
    cos, sin = cos[:, None], sin[:, None]
    y = x.clone()
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if case["adjacent"] else (slice(0, half), slice(half, rot))
    y[..., one] = x[..., one] * cos - x[..., two] * sin
    y[..., two] = x[..., two] * cos + x[..., one] * sin
    return y


def _angles(s):
    axis = torch.tensor(s["axis"], device="cuda")
    a = s["positions"][axis].T.double() * s["inv_freq"].double()
    return torch.cos(a), torch.sin(a)


def _rotate(s):
    cos, sin = (x.float() for x in _angles(s))
    return tuple(_turned(x.float(), w, cos, sin, s["case"]).bfloat16() for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])))


def _append(s):
    """The keys in 64 bits up to their codes: which side of a border between two codes a value lies on is for its exact value to say."""
    c, cache, slots = s["case"], s["cache"], s["slots"]
    cos, sin = _angles(s)
    q = _turned(s["q"].float(), s["wq"], cos.float(), sin.float(), c).bfloat16()
    live = slots >= 0
    where = slots.clamp(min=0).long()
    kept = torch.nonzero(live)[:, 0]
    at = where[kept]
    for name, x in (("k", _turned(s["k"].double(), s["wk"], cos, sin, c)), ("v", s["v"].float())):
        codes, scales = _encode(x[kept])
        cache[name + "_codes"][at // c["page"], :, at % c["page"]] = codes
        cache[name + "_scales"][at // c["page"], :, at % c["page"]] = scales
    out = [q]
    for name in "kv":
        x = _decode(cache[name + "_codes"][where // c["page"], :, where % c["page"]], cache[name + "_scales"][where // c["page"], :, where % c["page"]])
        out.append(torch.where(live[:, None, None], x, torch.zeros_like(x)).bfloat16())
    return tuple(out)


def _keys(cache, table):
    """K transposed, [n * KV heads, d, keys], and V [n * KV heads, keys, d], of the tables' rows."""
    k, v = (_decode(cache[x + "_codes"][table.long()], cache[x + "_scales"][table.long()]).transpose(1, 2).flatten(2, 3).flatten(0, 1) for x in "kv")
    return k.transpose(1, 2).contiguous(), v.contiguous()


def _part(s, table, lengths, starts, most, causal):
    """Attention of the rows starts[b] .. starts[b + 1] - 1 over the keys of table row b: O, maxima and sums of the exponentials,
    [rows, query heads, ...]."""
    c, q = s["case"], s["q"]
    n, hkv, d, group = table.shape[0], c["hkv"], c["d"], c["hq"] // c["hkv"]
    k, v = _keys(s["cache"], table)
    i = torch.arange(most, device="cuda")
    row = (starts[:-1, None] + i).clamp(max=q.shape[0] - 1).long()
    x = q[row].float().view(n, most, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(n * hkv, group * most, d)
    sc = (torch.matmul(x, k) * s["scale"]).view(n, hkv, group, most, -1)
    last = lengths[:, None] - (starts[1:] - starts[:-1])[:, None] + i if causal else (lengths[:, None] - 1).expand(n, most)
    seen = torch.arange(sc.shape[-1], device="cuda") <= last[..., None]
    sc = torch.where(seen[:, None, None], sc, float("-inf"))
    top = sc.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(sc - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n * hkv, group * most, -1), v).view(n, hkv, group, most, d)
    # back to rows
    r = torch.arange(q.shape[0], dtype=torch.int32, device="cuda")
    b = torch.searchsorted(starts, r, right=True) - 1
    at = (r - starts[b]).long()
    return [y.permute(0, 3, 1, 2, 4)[b, at].flatten(1, 2) for y in (o, top, total)]


def _attend(s):
    c = s["case"]
    o1, m1, l1 = _part(s, s["prefix_table"], s["prefix_lengths"], s["starts"][s["members"].long()], s["max_group"], False)
    o2, m2, l2 = _part(s, s["table"], s["lengths"], s["starts"], s["max_q"], True)
    m = torch.maximum(m1, m2)
    w1, w2 = torch.exp(m1 - m), torch.exp(m2 - m)
    total = w1 * l1 + w2 * l2
    out = ((w1 * o1 + w2 * o2) / total).bfloat16()
    return (out, (m + torch.log(total))[..., 0].T.contiguous()) if c["lse"] else (out,)


def run(state):
    s = state
    c = s["case"]
    if own:
        apbv = s["apbv"]
        if c["op"] == "rotate":
            return apbv.apbv_rotate(s["q"], s["k"], s["positions"], s["rotation"], **s["out"])
        if c["op"] == "append":
            q = apbv.apbv_cache_append(s["handle"], s["q"], s["k"], s["v"], s["slots"], s["positions"], s["rotation"], **s["out"])
            return (q,) + tuple(apbv.apbv_cache_load(s["handle"], s["slots"], **s["loaded"]))
        r = apbv.apbv_cache_shared_attention(s["q"], s["handle"], s["prefix_table"], s["prefix_lengths"], s["table"], s["lengths"], s["scale"],
                                             group_starts=s["members"], q_starts=s["starts"], max_q=s["max_q"], return_lse=c["lse"], **s["out"])
        return r if c["lse"] else (r,)
    if c["op"] == "rotate":
        return _rotate(s)
    if c["op"] == "append":
        return _append(s)
    return _attend(s)


# ---- the definition in 64 bits, apart from the plain forms

def _values64(codes, scales):
    """Sign, exponent and fraction of E2M1 spelled out, in float64."""
    x = torch.empty(codes.shape[:-1] + (codes.shape[-1] * 2,), dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        n = (codes >> (4 * half)) & 15
        exp, frac = ((n >> 1) & 3).double(), (n & 1).double()
        mag = torch.where(exp == 0, frac * 0.5, (1.0 + frac * 0.5) * 2.0 ** (exp - 1.0))
        x[..., half::2] = torch.where(n >= 8, -mag, mag)
    return x * torch.pow(2.0, scales.double() - 127.0).repeat_interleave(32, -1)


def _nearest64(x):
    """The value that each element of float rows is held as."""
    b = x.double().reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    big = b.abs().max(-1, keepdim=True).values
    e = torch.floor(torch.log2(big.clamp(min=2.0 ** -140))) - 2.0
    e = torch.where(big > 7.0 * 2.0 ** e, e + 1.0, e).clamp(-125.0, 125.0)
    y = b / 2.0 ** e
    index = torch.zeros(y.shape, dtype=torch.int64, device=x.device)
    for i in range(7):                                 # a half goes to the even code
        mid = (GRID[i] + GRID[i + 1]) / 2
        index += (y.abs() >= mid) if i % 2 else (y.abs() > mid)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    return (torch.sign(y) * grid[index] * 2.0 ** e).reshape(x.shape)


def _rotated64(s, x, weight):
    """Each pair as a complex number, multiplied by e^(i angle)."""
    c = s["case"]
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / c["d"] + EPS) * weight.double()
    half = c["rot"] // 2
    angle = torch.stack([s["positions"][a].double() * s["inv_freq"][i].double() for i, a in enumerate(s["axis"])], -1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    front, rest = x[..., :c["rot"]], x[..., c["rot"]:]
    if c["adjacent"]:
        pairs = torch.view_as_complex(front.reshape(front.shape[:-1] + (half, 2)).contiguous())
        front = torch.view_as_real(pairs * turn).flatten(-2)
    else:
        pairs = torch.complex(front[..., :half].contiguous(), front[..., half:].contiguous()) * turn
        front = torch.cat((pairs.real, pairs.imag), -1)
    return torch.cat((front, rest), -1)


def exact(case, seed):
    global own
    c, kept = case, own
    own = False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if c["op"] == "rotate":
        return _rotated64(s, s["q"], s["wq"]), _rotated64(s, s["k"], s["wk"])
    if c["op"] == "append":
        out = [_rotated64(s, s["q"], s["wq"])]
        for x in (_rotated64(s, s["k"], s["wk"]), s["v"]):
            y = _nearest64(x)
            y[s["slots"] < 0] = 0.0
            out.append(y)
        return tuple(out)
    page, hkv, d, group, cache, q = c["page"], c["hkv"], c["d"], c["hq"] // c["hkv"], s["cache"], s["q"]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty((c["hq"], q.shape[0]), dtype=torch.float64, device="cuda")
    starts, members, lengths, prefixes = (s[x].tolist() for x in ("starts", "members", "lengths", "prefix_lengths"))

    def keys(name, table, length, h):
        pages = table.long()[:_ceil(length, page)]
        return _values64(cache[name + "_codes"][pages, h], cache[name + "_scales"][pages, h]).reshape(-1, d)[:length]

    for g in range(c["groups"]):
        for h in range(hkv):
            pk, pv = (keys(x, s["prefix_table"][g], prefixes[g], h) for x in "kv")
            for b in range(members[g], members[g + 1]):
                lo, hi = starts[b], starts[b + 1]
                k, v = (torch.cat((p, keys(x, s["table"][b], lengths[b], h))) for x, p in (("k", pk), ("v", pv)))
                z = (q[lo:hi, h * group:(h + 1) * group].double().reshape(-1, d) @ k.T).view(hi - lo, group, -1) / math.sqrt(d)
                last = prefixes[g] + lengths[b] - (hi - lo) + torch.arange(hi - lo, device="cuda")       # the last key each query sees
                z.masked_fill_((torch.arange(k.shape[0], device="cuda") > last[:, None])[:, None], float("-inf"))
                lse[h * group:(h + 1) * group, lo:hi] = torch.logsumexp(z, -1).T
                out[lo:hi, h * group:(h + 1) * group] = (torch.softmax(z, -1).view(-1, k.shape[0]) @ v).view(hi - lo, group, d)
    return (out, lse) if c["lse"] else (out,)
