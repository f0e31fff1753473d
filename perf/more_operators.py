"""Streams over the paged cache: positions with several axes, a sliding window with first tokens that stay visible, and
keys that get new positions.

``axes`` rotates queries and keys at positions with several axes (time, height, width) and appends K and V to the paged
blocks; ``sink`` is attention of the new tokens with a sliding window and a few first tokens (sinks) that every row
sees; ``received`` accumulates, by the same rule, the attention that each cached token received; ``shift`` turns keys
that lie in the cache by a difference of positions.

Each runs in its plain form (elementary torch operations in 32 bits, angles in 64) or through the framework's calls
(``own``).  A case's structure (lengths, which keys a shift leaves alone) is a function of the case alone; contents,
positions and block tables come from the seed.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
FP8_MAX = 448.0        # the largest value of the 8-bit cache's type
POOL_FACTOR = 1.25     # paged blocks per live block


def _case(name, op, requests, new, past, **more):
    """``new`` tokens of each request over ``past`` tokens that the cache holds already."""
    c = {"name": name, "op": op, "requests": requests, "new": new, "past": past, "lengths": "equal", "q_heads": 32,
         "heads": 8, "dim": 128, "dtype": "bf16", "cache": "bf16", "block": 16, "layout": "kv_first"}
    if op == "axes":
        c.update(sections="16,24,24", order="sections", interleaved=False)
    if op in ("sink", "received"):
        c.update(window=1024, sink=4)
    if op == "received":
        c["decay"] = 1.0
    if op == "shift":
        c.update(layers=32, rot=128, interleaved=False, kind="chunk")
    c.update(more)
    return c


def listed():
    return [
        # one request decodes one token after text and images: the smallest call, all latency
        _case("axes-1x1", "axes", 1, 1, 1000),
        # the uncached halves of 16 prompts of 4,096 tokens, text with images between
        _case("axes-16x2048", "axes", 16, 2048, 2048),
        # ragged prompts in an 8-bit cache: a part of the head, neighbouring pairs, which take two axes in turn
        _case("axes-lognormal-fp8", "axes", 64, 700, 1400, lengths="lognormal", q_heads=16, heads=4, dim=80,
              cache="fp8", layout="block_first", sections="12,8", order="interleaved", interleaved=True),
        # one stream decodes one token
        _case("sink-1x1-of-1001", "sink", 1, 1, 1000, window=512),
        # 64 streams of 8,192 tokens decode with a window of 4,096
        _case("sink-64x1-of-8192", "sink", 64, 1, 8191, window=4096),
        # four prompts of 4,096 tokens with a window of 1,024
        _case("sink-4x4096", "sink", 4, 4096, 0),
        # decoding streams and chunks of prompts in one ragged batch, head size 80, 8-bit cache
        _case("sink-mixed-d80-fp8", "sink", 32, 300, 2500, lengths="mixed", q_heads=16, heads=4, dim=80, dtype="f16",
              cache="fp8", block=32, layout="block_first", window=700, sink=64),
        # what each cached token received from the tokens that 64 streams decode
        _case("received-64x1-of-8192", "received", 64, 1, 8191, window=2048),
        # and from chunks of 2,000 tokens of four prompts, older attention fading
        _case("received-4x2000-of-6000", "received", 4, 2000, 4000, decay=0.9),
        # a stream moves on: its four first tokens follow its window
        _case("shift-sink", "shift", 1, 0, 4, kind="sink"),
        # the 256-token chunks of eight documents of 2,048 tokens are used at another place
        _case("shift-chunk-8x2048", "shift", 8, 0, 2048),
        # eight ragged requests of an 8-bit cache after an eviction: each head's tokens get their new positions
        _case("shift-evicted-fp8", "shift", 8, 0, 2000, lengths="lognormal", cache="fp8", kind="evicted"),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _split(rng, total, parts):
    """``total`` cut into ``parts`` numbers of at least 1."""
    cuts = sorted(rng.sample(range(1, total), parts - 1))
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [total]))


def draw(rng):
    op = rng.choice(["axes", "axes", "sink", "sink", "sink", "sink", "received", "received", "shift", "shift"])
    heads = rng.choice([1, 2, 4, 8, 8])
    c = _case("", op, 1, 1, 1, heads=heads, q_heads=heads * rng.choice([1, 2, 4, 4, 4, 8]),
              dim=rng.choice([64, 80, 96, 128, 128, 128]), dtype=rng.choice(["bf16", "bf16", "f16"]),
              block=rng.choice([16, 16, 16, 32]), layout=rng.choice(["kv_first", "block_first"]),
              lengths=rng.choice(["equal", "lognormal", "mixed"]))
    del c["name"]
    c["cache"] = rng.choice([c["dtype"], c["dtype"], "fp8"])
    if op == "axes":
        c.update(sections=_split(rng, rng.randint(4, c["dim"] // 2), rng.choice([2, 3, 3, 4])),
                 order=rng.choice(["sections", "interleaved"]), interleaved=rng.choice([False, True]))
    if op == "received":
        c["decay"] = rng.choice([0.0, 0.9, 1.0])
    if op == "shift":
        c.update(layers=rng.choice([24, 32, 40, 48]), rot=2 * rng.randint(4, c["dim"] // 2),
                 interleaved=rng.choice([False, True]), kind=rng.choice(["sink", "chunk", "evicted", "evicted"]),
                 lengths=rng.choice(["equal", "lognormal"]), new=0)
    most = [work(k) for k in listed() if k["op"] == op]
    single = op in ("sink", "received") and rng.random() < 0.4
    while True:
        c["requests"] = _log_between(rng, 1, 64)
        c["past"] = _log_between(rng, 4, 64) if c.get("kind") == "sink" else _log_between(rng, 16, 32768)
        if op != "shift":
            c["new"] = 1 if single else _log_between(rng, 1, 4096)
        if op in ("sink", "received"):
            c["window"] = _log_between(rng, 16, 8192)
            c["sink"] = rng.choice([1, 4, 4, _log_between(rng, 1, 256)])
        w = work(c)
        if all(w[x] <= max(m[x] for m in most) for x in w) and _held(c) <= 1 << 31:
            return c


# ---------------------------------------------------------------------------
# structure of a case: a function of the case alone
# ---------------------------------------------------------------------------

def _lengths(c):
    """(new, total) tokens of each request.  Lognormal lengths have sigma 0.8
    around the case's mean, up to four times it; in a mixed batch every other
    request decodes one token."""
    R = c["requests"]
    new, past = np.full(R, c["new"], np.int64), np.full(R, c["past"], np.int64)
    if c["lengths"] != "equal":
        rng = np.random.default_rng([R, c["new"], c["past"]])
        f = np.minimum(rng.lognormal(-0.32, 0.8, (2, R)), 4.0)
        past = np.maximum(1, (past * f[0]).astype(np.int64))
        if c["new"]:
            new = np.maximum(1, (new * f[1]).astype(np.int64))
    if c["lengths"] == "mixed":
        new[::2] = 1
    return new, past + new


def _sections(c):
    return [int(x) for x in c["sections"].split(",")]


def _pairs(c):
    """Visible (query, key) pairs of all requests, for one query head."""
    new, total = _lengths(c)
    n = 0
    for a, t in zip(new.tolist(), total.tolist()):
        seen = np.arange(t - a, t) + 1
        n += int((np.minimum(seen, c["window"]) + np.minimum(np.maximum(seen - c["window"], 0), c["sink"])).sum())
    return n


def _held(c):
    """The largest tensor of a state or of the plain form, in elements: twice the keys that the cache holds, or the
    scores of all requests, padded to the longest."""
    new, total = _lengths(c)
    keys = 2 * int(total.sum()) * c["heads"] * c["dim"] * c.get("layers", 1)
    if c["op"] not in ("sink", "received"):
        return keys
    return max(keys, c["requests"] * c["q_heads"] * int(new.max()) * int(total.max()))


def _read_keys(c):
    """Keys that some query of their request sees."""
    new, total = _lengths(c)
    first = np.maximum(0, total - new - c["window"] + 1)
    return int((total - first + np.minimum(first, c["sink"])).sum())


KEPT_IN_PLACE = 4      # tokens of an evicted request whose position stays


def _turned(c):
    """(keys that a shift turns, shifts read) in all."""
    _, total = _lengths(c)
    n, every = int(total.sum()), c["layers"] * c["heads"]
    if c["kind"] == "evicted":
        return int(np.maximum(0, total - KEPT_IN_PLACE).sum()) * every, n * every
    return n * every, n


def work(case):
    c = case
    new, total = _lengths(c)
    e, ec = 2, 1 if c["cache"] == "fp8" else 2
    n, hq, h, d = int(new.sum()), c["q_heads"], c["heads"], c["dim"]
    if c["op"] == "axes":
        s = _sections(c)
        return {"bytes": n * d * (2 * hq * e + 2 * h * (e + ec)) + 4 * n * len(s), "flops": n * (hq + h) * sum(s) * 6}
    if c["op"] == "sink":
        return {"bytes": n * hq * (2 * d * e + 4) + 2 * _read_keys(c) * h * d * ec, "flops": 4 * _pairs(c) * hq * d}
    if c["op"] == "received":
        # sums of keys that nothing reaches stay as they are when nothing fades
        sums = {0.0: int(total.sum()), 1.0: 2 * _read_keys(c)}.get(c["decay"], 2 * int(total.sum()))
        return {"bytes": n * hq * (d * e + 4) + _read_keys(c) * h * d * ec + 4 * sums * h,
                "flops": 2 * _pairs(c) * hq * d}
    keys, shifts = _turned(c)
    return {"bytes": 2 * keys * c["rot"] * ec + 4 * shifts, "flops": keys * (c["rot"] // 2) * 6}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _frequencies(half):
    """Radians per position of each rotated pair, base 10,000."""
    return 10000.0 ** (-np.arange(half, dtype=np.float64) / half)


def _axis(c):
    """Axis of each pair: one axis's pairs after another's, or the axes in turn as long as they have pairs left."""
    s = _sections(c)
    if c["order"] == "sections":
        return np.repeat(np.arange(len(s)), s)
    return np.array([a for k in range(max(s)) for a in range(len(s)) if k < s[a]])


def _grid_positions(c, seed):
    """int32 [axes, rows] of the new tokens: 64 tokens of text, whose axes are alike, and an image of 16 x 24 patches
    in turn.  An image has one time; its last axes count rows and columns; text goes on after its largest."""
    new, total = _lengths(c)
    axes = len(_sections(c))
    rng = np.random.default_rng(seed)
    index = np.concatenate([np.arange(t - a, t) for a, t in zip(new.tolist(), total.tolist())])
    start = np.repeat(rng.integers(0, 64, c["requests"]), new)
    turn, at = np.divmod(index, 64 + 16 * 24)
    base = start + turn * (64 + 24)
    patch = np.maximum(at - 64, 0)
    text = base + np.minimum(at, 64)
    pos = np.repeat(text[None], axes, 0)
    pos[axes - 1] += np.where(at >= 64, patch % 24, 0)
    pos[axes - 2] += np.where(at >= 64, patch // 24, 0)
    return pos.astype(np.int32)


def prepare(case, seed):
    c = dict(case)
    new, total = _lengths(c)
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    R, hq, h, d, B = c["requests"], c["q_heads"], c["heads"], c["dim"], c["block"]
    L = c.get("layers", 1)
    n = int(new.sum())
    need = -(-total // B)
    nb = max(int(math.ceil(POOL_FACTOR * total.sum() / B)), int(need.sum()))
    bt = np.full((R, int(need.max())), -1, np.int32)
    perm = np.random.default_rng(seed).permutation(nb).astype(np.int32)
    at = 0
    for r in range(R):
        bt[r, :need[r]] = perm[at:at + need[r]]
        at += int(need[r])

    def rand(*shape):
        return torch.randn(shape, device=dev, dtype=torch.bfloat16, generator=gen)

    cache = DTYPES[c["cache"]]
    pool = torch.empty((L, 2, nb, B, h, d) if c["layout"] == "kv_first" else (L, nb, 2, B, h, d), dtype=cache,
                       device=dev)
    for layer in pool:
        layer.copy_(rand(*layer.shape))
    q_off = np.concatenate([[0], np.cumsum(new)])
    s = {"c": c, "pool": pool, "bt": torch.from_numpy(bt).to(dev), "q_off": torch.from_numpy(q_off).to(dev),
         "kv_len": torch.from_numpy(total.astype(np.int32)).to(dev), "n": n, "max_q": int(new.max()),
         "max_kv": int(total.max()), "k_scale": None, "v_scale": None}
    if c["cache"] == "fp8" and c["op"] != "shift":
        s["k_scale"] = torch.rand(h, device=dev, generator=gen) * 0.5 + 0.75
        s["v_scale"] = torch.rand(h, device=dev, generator=gen) * 0.5 + 0.75
    dt = DTYPES[c["dtype"]]
    if c["op"] == "axes":
        # q, k and v lie side by side, as one projection leaves them
        qkv = rand(n, hq + 2 * h, d).to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + h], qkv[:, hq + h:]
        s["freqs"] = torch.from_numpy(_frequencies(sum(_sections(c)))).to(dev)
        s["axis"] = torch.from_numpy(_axis(c)).to(dev)
        s["positions"] = torch.from_numpy(_grid_positions(c, seed)).to(dev)
        s["q_out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
    if c["op"] in ("sink", "received"):
        s["q"] = (1.5 * rand(n, hq, d)).to(dt)
        s["scale"] = d ** -0.5
        s["out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
        s["lse"] = torch.empty((n, hq), device=dev)
    if c["op"] == "received":
        s["lse"].copy_(_plain_scores(s)[1])
        s["weights"] = torch.rand((R, h, s["max_kv"]), device=dev, generator=gen)
    if c["op"] == "shift":
        s["freqs"] = torch.from_numpy(_frequencies(c["rot"] // 2)).to(dev)
        T = s["max_kv"]
        if c["kind"] == "evicted":
            # the first tokens stay; behind them every token moves up by what was evicted before it, at least one
            gone = torch.randint(0, 3, (L, R, h, T), device=dev, generator=gen)
            gone[..., :KEPT_IN_PLACE + 1] = 0
            shift = -(1 + gone.cumsum(-1))
            shift[..., :KEPT_IN_PLACE] = 0
        else:
            # one difference for a request's tokens, forwards or (a chunk) backwards
            by = torch.randint(1, 30000 if c["kind"] == "chunk" else 64, (1, R, 1, 1), device=dev, generator=gen)
            if c["kind"] == "chunk":
                by = torch.where(torch.rand((1, R, 1, 1), device=dev, generator=gen) < 0.5, by, -by)
            shift = by.expand(1, R, 1, T)
        s["shift"] = shift.int().contiguous()
    if own:
        import paper_2609_35065_amd as kv
        seg = B * h * d * pool.element_size()
        strides = (nb * seg, seg) if c["layout"] == "kv_first" else (seg, 2 * seg)
        s["layout"] = kv.make_layout(L, h, d, pool.element_size(), B, B, nb, 1, *strides)
        s["layers"] = list(pool)
        if c["op"] != "shift":
            s["batch"] = kv.make_batch(s["q_off"], s["kv_len"], s["bt"], n, s["max_q"], s["max_kv"])
        if c["op"] == "axes":
            s["axes"] = kv.kv_rope_axes(_sections(c), interleaved=c["order"] == "interleaved")
        if c["op"] in ("sink", "received"):
            size = (kv.kv_sink_attention_workspace if c["op"] == "sink" else kv.kv_sink_weights_workspace)(
                s["layout"], s["batch"], hq, c["window"], c["sink"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device=dev)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2609_35065_amd as kv
    c = s["c"]
    if c["op"] == "axes":
        kv.kv_rope_append_axes(s["layout"], s["layers"][0], s["batch"], s["q"], s["k"], s["v"], s["freqs"], s["axes"],
                               s["positions"], q_out=s["q_out"], interleaved=c["interleaved"], k_scale=s["k_scale"],
                               v_scale=s["v_scale"])
        return {"q": s["q_out"], "cache": s["pool"]}
    if c["op"] == "sink":
        kv.kv_sink_attention(s["layout"], s["layers"][0], s["batch"], s["q"], s["out"], s["scale"], c["window"],
                             c["sink"], lse=s["lse"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                             workspace=s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "received":
        kv.kv_sink_weights(s["layout"], s["layers"][0], s["batch"], s["q"], s["lse"], s["weights"], s["scale"],
                           c["window"], c["sink"], decay=c["decay"], k_scale=s["k_scale"], workspace=s["workspace"])
        return {"weights": s["weights"]}
    kv.kv_rope_shift(s["layout"], s["layers"], s["bt"], s["kv_len"], s["max_kv"], s["shift"], s["freqs"],
                     interleaved=c["interleaved"])
    return {"cache": s["pool"]}


def _planes(s):
    """K and V of all layers' pools, each [layers, blocks, B, H, D]."""
    p = s["pool"]
    return (p[:, 0], p[:, 1]) if s["c"]["layout"] == "kv_first" else (p[:, :, 0], p[:, :, 1])


def _tokens(s):
    """Request and place among its new tokens, of every row of q."""
    row = torch.arange(s["n"], device="cuda")
    req = torch.searchsorted(s["q_off"], row, right=True) - 1
    return req, row - s["q_off"][req]


def _run_plain(s):
    return {"axes": _plain_axes, "sink": _plain_sink, "received": _plain_received, "shift": _plain_shift}[s["c"]["op"]](s)


def _plain_keys(s, plane, scale):
    """A plane's rows [R, H, T, D] in 32 bits, by block table (missing blocks are masked later)."""
    x = plane[0][s["bt"].long().clamp(min=0)].float()                    # [R, blocks, B, H, D]
    x = x.flatten(1, 2)[:, :s["max_kv"]].transpose(1, 2).contiguous()
    return x if scale is None else x.mul_(scale[None, :, None, None])


def _plain_scores(s):
    """Masked scores [R, H, G, Tq, T] and their log-sum-exp in the rows' order [n, heads]."""
    c = s["c"]
    R, h, d = c["requests"], c["heads"], c["dim"]
    g, tq, t = c["q_heads"] // h, s["max_q"], s["max_kv"]
    new = s["q_off"][1:] - s["q_off"][:-1]
    i = torch.arange(tq, device="cuda")
    q = s["q"][(s["q_off"][:-1, None] + i).clamp(max=s["n"] - 1)].float()   # [R, Tq, heads, D]
    q = q.view(R, tq, h, g, d).permute(0, 2, 3, 1, 4).reshape(R, h, g * tq, d)
    k = _plain_keys(s, _planes(s)[0], s["k_scale"])
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(R, h, g, tq, t)
    j = torch.arange(t, device="cuda")
    pos = (s["kv_len"][:, None] - new[:, None] + i)[..., None]              # [R, Tq, 1]
    see = (j <= pos) & ((j > pos - c["window"]) | (j < c["sink"])) & (i[:, None] < new[:, None, None])
    x.masked_fill_(~see[:, None, None], -math.inf)
    req, at = _tokens(s)
    lse = torch.logsumexp(x, -1).view(R, h * g, tq)
    return x, lse[req, :, at]


def _plain_weights(s, x, lse):
    """exp(scores - lse) in place, with nothing for padded rows."""
    c = s["c"]
    i = torch.arange(s["max_q"], device="cuda")
    new = s["q_off"][1:] - s["q_off"][:-1]
    rows = lse[(s["q_off"][:-1, None] + i).clamp(max=s["n"] - 1)]            # [R, Tq, heads]
    rows = rows.view(c["requests"], s["max_q"], c["heads"], -1).permute(0, 2, 3, 1)
    rows = rows.masked_fill((i >= new[:, None])[:, None, None], 0.0)
    return x.sub_(rows[..., None]).exp_()


def _plain_sink(s):
    c = s["c"]
    x, lse = _plain_scores(s)
    R, h, tq = c["requests"], c["heads"], s["max_q"]
    p = _plain_weights(s, x, lse).view(R, h, -1, s["max_kv"])
    v = _plain_keys(s, _planes(s)[1], s["v_scale"])
    o = torch.matmul(p, v).view(R, c["q_heads"], tq, c["dim"])
    req, at = _tokens(s)
    return {"out": o[req, :, at].to(DTYPES[c["dtype"]]), "lse": lse}


def _plain_received(s):
    c = s["c"]
    x, _ = _plain_scores(s)
    got = _plain_weights(s, x, s["lse"]).sum((2, 3))
    inside = torch.arange(s["max_kv"], device="cuda") < s["kv_len"][:, None, None]
    old = s["weights"]
    s["weights"] = torch.where(inside, old * c["decay"] + got, old)
    return {"weights": s["weights"]}


def _plain_turn(x, angle, interleaved):
    """Rows [..., D] in 32 bits whose first pairs are turned by angles [..., half] in 64 bits: a position times a
    frequency needs more than 32 before whole turns are taken off."""
    angle = torch.remainder(angle, 2 * math.pi).float()
    cos, sin = angle.cos(), angle.sin()
    x = x.float()
    rot = 2 * angle.shape[-1]
    y, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y.chunk(2, -1)
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, rest], -1)


def _plain_axes(s):
    c = s["c"]
    req, at = _tokens(s)
    index = s["kv_len"][req] - (s["q_off"][1:] - s["q_off"][:-1])[req] + at
    angle = (s["positions"][s["axis"]].double() * s["freqs"][:, None]).t()[:, None]     # [n, 1, half]

    def put(plane, x, scale):
        if scale is not None:
            x = (x / scale[None, :, None]).clamp(-FP8_MAX, FP8_MAX)
        x = x.to(plane.dtype)
        if plane.dtype == torch.float8_e4m3fn:
            plane, x = plane.view(torch.uint8), x.view(torch.uint8)
        plane[0, s["bt"][req, (index // c["block"])].long(), index % c["block"]] = x

    kp, vp = _planes(s)
    put(kp, _plain_turn(s["k"], angle, c["interleaved"]), s["k_scale"])
    put(vp, s["v"].float(), s["v_scale"])
    return {"q": _plain_turn(s["q"], angle, c["interleaved"]).to(s["q"].dtype), "cache": s["pool"]}


def _plain_shift(s):
    c = s["c"]
    t = torch.arange(s["max_kv"], device="cuda")
    req, index = (t < s["kv_len"][:, None]).nonzero(as_tuple=True)          # every cached token
    blk, row = s["bt"][req, index // c["block"]].long(), index % c["block"]
    plane = _planes(s)[0]
    fp8 = c["cache"] == "fp8"
    raw = plane.view(torch.uint8) if fp8 else plane
    old = raw[:, blk, row]                                                  # [L, tokens, H, D]
    shift = s["shift"][:, req, :, index].transpose(0, 1)                    # [L or 1, tokens, H or 1]
    x = _plain_turn(old.view(plane.dtype), shift[..., None].double() * s["freqs"], c["interleaved"])
    x = x.clamp(-FP8_MAX, FP8_MAX).to(plane.dtype).view(torch.uint8) if fp8 else x.to(plane.dtype)
    raw[:, blk, row] = torch.where(shift[..., None] == 0, old, x)
    return {"cache": s["pool"]}


# ---------------------------------------------------------------------------
# the definition in 64 bits, request by request
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"axes": _exact_axes, "sink": _exact_sink, "received": _exact_received, "shift": _exact_shift}[case["op"]](s)


def _exact_rows(s, r, plane, scale):
    """Rows of request r of a layer's plane, [T, H, D]."""
    t = int(s["kv_len"][r])
    B = s["c"]["block"]
    rows = torch.cat([plane[0][int(b)] for b in s["bt"][r, :-(-t // B)].tolist()])[:t].double()
    return rows if scale is None else rows * scale.double()[None, :, None]


def _exact_visible(s, r):
    c = s["c"]
    a, b, t = int(s["q_off"][r]), int(s["q_off"][r + 1]), int(s["kv_len"][r])
    see = torch.zeros((b - a, t), dtype=torch.bool, device="cuda")
    back = torch.arange(t - (b - a), t, device="cuda")[:, None] - torch.arange(t, device="cuda")   # how far back
    see |= (back >= 0) & (back < c["window"])
    see[:, :c["sink"]] |= back[:, :c["sink"]] >= 0
    return a, b, t, see


def _exact_sink(s):
    c = s["c"]
    g = c["q_heads"] // c["heads"]
    out = torch.zeros((s["n"], c["q_heads"], c["dim"]), dtype=torch.float64, device="cuda")
    lse = torch.zeros((s["n"], c["q_heads"]), dtype=torch.float64, device="cuda")
    for r in range(c["requests"]):
        a, b, t, see = _exact_visible(s, r)
        k, v = (_exact_rows(s, r, p, x) for p, x in zip(_planes(s), (s["k_scale"], s["v_scale"])))
        for head in range(c["q_heads"]):
            x = s["q"][a:b, head].double() @ k[:, head // g].t() * s["scale"]
            x = torch.where(see, x, -math.inf)
            top = x.amax(-1, keepdim=True)
            e = torch.exp(x - top)
            total = e.sum(-1, keepdim=True)
            out[a:b, head] = (e @ v[:, head // g]) / total
            lse[a:b, head] = (top + total.log())[:, 0]
    return {"out": out, "lse": lse}


def _exact_received(s):
    c = s["c"]
    g = c["q_heads"] // c["heads"]
    out = s["weights"].double()
    for r in range(c["requests"]):
        a, b, t, see = _exact_visible(s, r)
        k = _exact_rows(s, r, _planes(s)[0], s["k_scale"])
        for h in range(c["heads"]):
            got = 0
            for head in range(h * g, (h + 1) * g):
                x = s["q"][a:b, head].double() @ k[:, h].t() * s["scale"] - s["lse"][a:b, head, None].double()
                got = got + torch.where(see, x.exp(), 0.0).sum(0)
            out[r, h, :t] = c["decay"] * out[r, h, :t] + got
    return {"weights": out}


def _exact_turn(x, turn, interleaved):
    """Rows in 64 bits, their pairs as complex numbers times ``turn``."""
    half = turn.shape[-1]
    first = torch.arange(half, device="cuda") * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    x = x.double().clone()
    z = torch.complex(x[..., first], x[..., second]) * turn
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_axes(s):
    c = s["c"]
    s_ = _sections(c)
    left, axis = list(s_), []
    while len(axis) < sum(s_):       # pair by pair: the next axis in turn, or the first that has pairs left
        if c["order"] == "sections":
            axis.append(next(a for a, n in enumerate(left) if n))
        else:
            last = axis[-1] if axis else -1
            turn = [(last + 1 + a) % len(s_) for a in range(len(s_))]
            axis.append(next(a for a in turn if left[a]))
        left[axis[-1]] -= 1
    where = np.concatenate([np.arange(int(t) - int(b - a), int(t)) for a, b, t in
                            zip(s["q_off"].tolist(), s["q_off"].tolist()[1:], s["kv_len"].tolist())])
    req = np.repeat(np.arange(c["requests"]), np.diff(s["q_off"].cpu().numpy()))
    angle = torch.stack([s["positions"][a].double() * float(f) for a, f in zip(axis, s["freqs"])], -1)
    turn = torch.exp(1j * angle)[:, None]
    pool = s["pool"].double()
    blocks = s["bt"].cpu().numpy()[req, where // c["block"]]
    blk, row = (torch.from_numpy(np.asarray(x, np.int64)).cuda() for x in (blocks, where % c["block"]))
    for plane, x, scale in ((0, _exact_turn(s["k"], turn, c["interleaved"]), s["k_scale"]),
                            (1, s["v"].double(), s["v_scale"])):
        if scale is not None:
            x = (x / scale.double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        if c["layout"] == "kv_first":
            pool[0, plane, blk, row] = x
        else:
            pool[0, blk, plane, row] = x
    return {"q": _exact_turn(s["q"], turn, c["interleaved"]), "cache": pool}


def _exact_shift(s):
    c = s["c"]
    B = c["block"]
    pool = s["pool"].double()
    for l in range(c["layers"]):
        for r in range(c["requests"]):
            n = int(s["kv_len"][r])
            by = s["shift"][l % s["shift"].shape[0], r, :, :n].t().double()      # [n, H or 1]
            turn = torch.exp(1j * by[..., None] * s["freqs"])
            blk = s["bt"][r].long().repeat_interleave(B)[:n]
            row = torch.arange(n, device="cuda") % B
            plane = pool[l, 0] if c["layout"] == "kv_first" else pool[l, :, 0]
            plane[blk, row] = _exact_turn(plane[blk, row], turn, c["interleaved"]).clamp(
                *((-FP8_MAX, FP8_MAX) if c["cache"] == "fp8" else (-math.inf, math.inf)))
    return {"cache": pool}
