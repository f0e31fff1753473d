"""Operators over the paged cache: what fills it, reads it and shrinks it.

``rope`` rotates the queries and keys of new tokens and writes their K and V
into the paged blocks; ``attn`` is attention of those tokens over the cache;
``weights`` accumulates, for each cached token, the attention it received;
``evict`` keeps the tokens that received most and moves them to the front of
their request's blocks.

Each runs in its plain form (elementary torch operations in 32 bits) or
through the framework's calls (``own``).  A case's structure (lengths) is a
function of the case alone; contents and block tables come from the seed.
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
    if op in ("attn", "weights"):
        c["window"] = 0
    if op == "rope":
        c.update(rot=128, interleaved=False, scaling="none")
    if op == "weights":
        c["decay"] = 1.0
    if op == "evict":
        c.update(layers=32, keep=0.5, shared=False)
    c.update(more)
    return c


def listed():
    return [
        # one request decodes one token: the smallest call, all latency
        _case("rope-1x1", "rope", 1, 1, 1000),
        # the uncached halves of 16 prompts of 4,096 tokens
        _case("rope-16x2048", "rope", 16, 2048, 2048),
        # ragged prompts, 8-bit cache, neighbouring pairs in a part of the head, scaled for long contexts
        _case("rope-lognormal-fp8", "rope", 64, 700, 1400, lengths="lognormal", q_heads=16, heads=4, dim=80,
              cache="fp8", layout="block_first", rot=40, interleaved=True, scaling="ramp"),
        # one request decodes one token over a prompt of odd length
        _case("attn-1x1-of-1001", "attn", 1, 1, 1000),
        # the benchmark batch decodes: 64 requests of 4,096 tokens
        _case("attn-64x1-of-4096", "attn", 64, 1, 4095),
        # eight long documents in an 8-bit cache
        _case("attn-8x1-of-32768-fp8", "attn", 8, 1, 32767, cache="fp8"),
        # the uncached halves of 8 prompts of 4,096 tokens over prefix and suffix
        _case("attn-8x2048-of-4096", "attn", 8, 2048, 2048),
        # decoding requests and chunks of prompts in one ragged batch, head size 80, sliding window
        _case("attn-mixed-d80", "attn", 32, 300, 2048, lengths="mixed", q_heads=16, heads=4, dim=80, dtype="f16",
              cache="f16", block=32, layout="block_first", window=1024),
        # what each cached token received from the decoded tokens of the benchmark batch
        _case("weights-64x1-of-4096", "weights", 64, 1, 4095),
        # and from the chunks of four prompts, older attention fading
        _case("weights-4x1000-of-4000", "weights", 4, 1000, 3000, decay=0.9),
        # one request of the 32-layer shape gives up half of its cache
        _case("evict-1x1001", "evict", 1, 0, 1001),
        # eight ragged requests are cut to a quarter of the mean length
        _case("evict-8x4096", "evict", 8, 0, 4096, lengths="lognormal", keep=0.25),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "attn", "attn", "attn", "attn", "weights", "weights", "evict", "evict"])
    heads = rng.choice([1, 2, 4, 8, 8])
    c = _case("", op, 1, 1, 1, heads=heads, q_heads=heads * rng.choice([1, 2, 4, 4, 4, 8]),
              dim=rng.choice([64, 80, 96, 128, 128, 128]), dtype=rng.choice(["bf16", "bf16", "f16"]),
              block=rng.choice([16, 16, 16, 32]), layout=rng.choice(["kv_first", "block_first"]),
              lengths=rng.choice(["equal", "lognormal", "mixed"]))
    del c["name"]
    c["cache"] = rng.choice([c["dtype"], c["dtype"], "fp8"])
    if op == "evict":
        c.update(lengths=rng.choice(["equal", "lognormal"]), layers=rng.choice([24, 32, 40, 48]),
                 keep=round(rng.uniform(0.1, 0.9), 2), shared=rng.choice([False, False, True]), new=0)
    if op == "rope":
        c.update(rot=2 * rng.randint(4, c["dim"] // 2), interleaved=rng.choice([False, True]),
                 scaling=rng.choice(["none", "linear", "ramp"]))
    if op in ("attn", "weights"):
        c["window"] = rng.choice([0, 0, 0, rng.randint(16, 4096)])
    if op == "weights":
        c["decay"] = rng.choice([0.0, 0.9, 1.0])
    top = {k["op"]: work(k) for k in listed() if k["name"] in ("rope-16x2048", "attn-8x2048-of-4096",
                                                              "weights-4x1000-of-4000", "evict-8x4096")}[op]
    single = op in ("attn", "weights") and rng.random() < 0.4
    while True:
        c["requests"] = _log_between(rng, 1, 64)
        c["past"] = _log_between(rng, 16, 32768)
        if op != "evict":
            c["new"] = 1 if single else _log_between(rng, 1, 2048)
        w = work(c)
        if w["bytes"] <= (256 << 20 if op == "weights" else 1 << 30 if op == "attn" else top["bytes"]) \
                and w["flops"] <= max(top["flops"], 1) and _padded(c) <= 1 << 31:
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
        past = (past * f[0]).astype(np.int64)
        if c["new"]:
            new = np.maximum(1, (new * f[1]).astype(np.int64))
    if c["lengths"] == "mixed":
        new[::2] = 1
    return new, past + new


def _pairs(c):
    """Visible (query, key) pairs of all requests, for one query head."""
    new, total = _lengths(c)
    n = 0
    for a, t in zip(new.tolist(), total.tolist()):
        pos = np.arange(t - a, t) + 1
        n += int((np.minimum(pos, c["window"]) if c["window"] else pos).sum())
    return n


def _padded(c):
    """Scores of the plain form, which pads every request to the longest."""
    if c["op"] not in ("attn", "weights"):
        return 0
    new, total = _lengths(c)
    return c["requests"] * c["q_heads"] * int(new.max()) * int(total.max())


def _read_keys(c):
    """Keys that some query of their request sees."""
    new, total = _lengths(c)
    return int((np.minimum(total, c["window"] + new - 1) if c["window"] else total).sum())


def _budget(c):
    return max(2, int(c["past"] * c["keep"]))


def work(case):
    c = case
    new, total = _lengths(c)
    e, ec = 2, 1 if c["cache"] == "fp8" else 2
    n, hq, h, d = int(new.sum()), c["q_heads"], c["heads"], c["dim"]
    if c["op"] == "rope":
        return {"bytes": n * d * (2 * hq * e + 2 * h * (e + ec)), "flops": n * (hq + h) * (c["rot"] // 2) * 6}
    if c["op"] == "attn":
        return {"bytes": n * hq * (2 * d * e + 4) + 2 * _read_keys(c) * h * d * ec, "flops": 4 * _pairs(c) * hq * d}
    if c["op"] == "weights":
        back = 2 if c["decay"] else 1
        return {"bytes": n * hq * (d * e + 4) + _read_keys(c) * h * d * ec + back * 4 * int(total.sum()) * h,
                "flops": 2 * _pairs(c) * hq * d}
    g = 1 if c["shared"] else h
    kept = int(np.minimum(total, _budget(c)).sum())
    # weights are read once, kept ids written and read, kept rows and weights moved
    return {"bytes": c["layers"] * (4 * g * int(total.sum()) + 8 * g * kept + 8 * g * kept + 4 * kept * h * d * ec),
            "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _frequencies(c):
    """Frequency of each rotated pair, and the factor on rotated values: base
    10,000, original context 4,096, factor 8 (positions divided, or, by ramp,
    only those of pairs that turn less than 32 times in the original context)."""
    half = c["rot"] // 2
    f = 10000.0 ** (-np.arange(half, dtype=np.float64) / half)
    if c["scaling"] == "linear":
        return f / 8, 1.0
    if c["scaling"] == "ramp":
        keep = np.clip((4096 * f / (2 * math.pi) - 1) / (32 - 1), 0, 1)
        return f * keep + f / 8 * (1 - keep), 0.1 * math.log(8) + 1
    return f, 1.0


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
         "max_kv": int(total.max()), "q_scale": None, "k_scale": None, "v_scale": None}
    if c["cache"] == "fp8":
        s["k_scale"] = torch.rand(h, device=dev, generator=gen) * 0.5 + 0.75
        s["v_scale"] = torch.rand(h, device=dev, generator=gen) * 0.5 + 0.75
    dt = DTYPES[c["dtype"]]
    if c["op"] == "rope":
        # q, k and v lie side by side, as one projection leaves them
        qkv = rand(n, hq + 2 * h, d).to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + h], qkv[:, hq + h:]
        f, s["magnitude"] = _frequencies(c)
        s["freqs"] = torch.from_numpy(f).to(dev)
        s["q_out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
    if c["op"] in ("attn", "weights"):
        s["q"] = (1.5 * rand(n, hq, d)).to(dt)
        s["scale"] = d ** -0.5
        s["out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
        s["lse"] = torch.empty((n, hq), device=dev)
    if c["op"] == "weights":
        s["lse"].copy_(_plain_scores(s)[1])
        s["weights"] = torch.rand((R, h, s["max_kv"]), device=dev, generator=gen)
    if c["op"] == "evict":
        # accumulated attention: a long tail, and tokens that never received any
        w = torch.rand((L, R, 1 if c["shared"] else h, s["max_kv"]), device=dev, generator=gen)
        s["weights"] = torch.where(w < 0.1, torch.zeros_like(w), w ** 4)
        s["budget"] = _budget(c)
        s["sink"], s["recent"] = min(4, s["budget"] // 4), s["budget"] // 4
        s["keep"] = torch.empty((*w.shape[:3], s["budget"]), dtype=torch.int32, device=dev)
        s["new_len"] = torch.empty(R, dtype=torch.int32, device=dev)
    if own:
        import paper_2609_35065_amd as kv
        seg = B * h * d * pool.element_size()
        strides = (nb * seg, seg) if c["layout"] == "kv_first" else (seg, 2 * seg)
        s["layout"] = kv.make_layout(L, h, d, pool.element_size(), B, B, nb, 1, *strides)
        s["layers"] = list(pool)
        if c["op"] != "evict":
            s["batch"] = kv.make_batch(s["q_off"], s["kv_len"], s["bt"], n, s["max_q"], s["max_kv"])
        if c["op"] == "attn":
            size = kv.kv_paged_attention_workspace(s["layout"], s["batch"], hq, c["window"])
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
    if c["op"] == "rope":
        kv.kv_rope_append(s["layout"], s["layers"][0], s["batch"], s["q"], s["k"], s["v"], s["freqs"],
                          q_out=s["q_out"], interleaved=c["interleaved"], magnitude=s["magnitude"],
                          k_scale=s["k_scale"], v_scale=s["v_scale"])
        return {"q": s["q_out"], "cache": s["pool"]}
    if c["op"] == "attn":
        kv.kv_paged_attention(s["layout"], s["layers"][0], s["batch"], s["q"], s["out"], s["scale"],
                              window=c["window"], lse=s["lse"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                              workspace=s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "weights":
        kv.kv_attention_weights(s["layout"], s["layers"][0], s["batch"], s["q"], s["lse"], s["weights"], s["scale"],
                                window=c["window"], decay=c["decay"], k_scale=s["k_scale"])
        return {"weights": s["weights"]}
    kv.kv_evict_select(s["weights"], s["kv_len"], s["budget"], s["sink"], s["recent"], s["keep"], s["new_len"])
    kv.kv_evict_compact(s["layout"], s["layers"], s["bt"], s["keep"], s["new_len"], weights=s["weights"])
    return {"keep": s["keep"], "new_len": s["new_len"], "cache": s["pool"], "weights": s["weights"]}


def _planes(s, layer=0):
    """K and V of a layer's pool, each [blocks, B, H, D]."""
    p = s["pool"][layer]
    return (p[0], p[1]) if s["c"]["layout"] == "kv_first" else (p[:, 0], p[:, 1])


def _tokens(s):
    """Request and place among its new tokens, of every row of q."""
    row = torch.arange(s["n"], device="cuda")
    req = torch.searchsorted(s["q_off"], row, right=True) - 1
    return req, row - s["q_off"][req]


def _plain_keys(s, plane, scale):
    """A plane's rows [R, H, T, D] in 32 bits, by block table (missing blocks are masked later)."""
    c = s["c"]
    x = plane[s["bt"].long().clamp(min=0)].float()                       # [R, blocks, B, H, D]
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
    pos = s["kv_len"][:, None] - new[:, None] + i                           # [R, Tq]
    hide = (j > pos[..., None]) | (i[:, None] >= new[:, None, None])
    if c["window"]:
        hide |= j <= pos[..., None] - c["window"]
    x.masked_fill_(hide[:, None, None], -math.inf)
    req, at = _tokens(s)
    lse = torch.logsumexp(x, -1).view(R, h * g, tq)
    return x, lse[req, :, at]


def _plain_weights(s, x, lse):
    """exp(scores - lse) in place, with nothing for padded and empty rows."""
    c = s["c"]
    i = torch.arange(s["max_q"], device="cuda")
    new = s["q_off"][1:] - s["q_off"][:-1]
    rows = lse[(s["q_off"][:-1, None] + i).clamp(max=s["n"] - 1)]            # [R, Tq, heads]
    rows = rows.view(c["requests"], s["max_q"], c["heads"], -1).permute(0, 2, 3, 1)
    rows = rows.masked_fill((i >= new[:, None])[:, None, None], 0.0).clamp(min=-1e30)
    return x.sub_(rows[..., None]).exp_()


def _run_plain(s):
    c = s["c"]
    if c["op"] == "rope":
        return _plain_rope(s)
    if c["op"] == "evict":
        return _plain_evict(s)
    x, lse = _plain_scores(s)
    R, h, tq = c["requests"], c["heads"], s["max_q"]
    if c["op"] == "attn":
        p = _plain_weights(s, x, lse).view(R, h, -1, s["max_kv"])
        v = _plain_keys(s, _planes(s)[1], s["v_scale"])
        o = torch.matmul(p, v).view(R, c["q_heads"], tq, c["dim"])
        req, at = _tokens(s)
        return {"out": o[req, :, at].to(DTYPES[c["dtype"]]), "lse": lse}
    got = _plain_weights(s, x, s["lse"]).sum((2, 3))
    inside = torch.arange(s["max_kv"], device="cuda") < s["kv_len"][:, None, None]
    old = s["weights"]
    s["weights"] = torch.where(inside, old * c["decay"] + got, old)
    return {"weights": s["weights"]}


def _plain_rope(s):
    c = s["c"]
    req, at = _tokens(s)
    index = s["kv_len"][req] - (s["q_off"][1:] - s["q_off"][:-1])[req] + at
    # the angle alone needs more than 32 bits: a position times a frequency, modulo a turn
    angle = torch.remainder(index.double()[:, None] * s["freqs"], 2 * math.pi).float()
    cos, sin = angle.cos()[:, None] * s["magnitude"], angle.sin()[:, None] * s["magnitude"]

    def turn(x):
        x = x.float()
        y, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        if c["interleaved"]:
            a, b = y[..., 0::2], y[..., 1::2]
            y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = y.chunk(2, -1)
            y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([y, rest], -1)

    def put(plane, x, scale):
        if scale is not None:
            x = (x / scale[None, :, None]).clamp(-FP8_MAX, FP8_MAX)
        x = x.to(plane.dtype)
        if plane.dtype == torch.float8_e4m3fn:
            plane, x = plane.view(torch.uint8), x.view(torch.uint8)
        plane[s["bt"][req, (index // c["block"])].long(), index % c["block"]] = x

    kp, vp = _planes(s)
    put(kp, turn(s["k"]), s["k_scale"])
    put(vp, s["v"].float(), s["v_scale"])
    return {"q": turn(s["q"]).to(s["q"].dtype), "cache": s["pool"]}


def _plain_evict(s):
    c = s["c"]
    w, t, n = s["weights"], s["max_kv"], s["budget"]
    j = torch.arange(t, device="cuda")
    size = s["kv_len"][None, :, None, None]
    order = torch.where((j < s["sink"]) | (j >= size - s["recent"]), math.inf, w)
    order = torch.where(j < size, order, -math.inf)
    got = torch.sort(order, dim=-1, descending=True, stable=True).indices[..., :n]    # ties: lowest index first
    got = torch.where(got < size, got, t).sort(-1).values                         # [L, R, heads, budget]
    if t < n:
        got = torch.nn.functional.pad(got, (0, n - t), value=t)
    keep = torch.where(got < size, got, -1).int()
    new_len = s["kv_len"].clamp(max=n)
    # a row that is not kept moves onto itself
    i = torch.arange(n, device="cuda").expand(got.shape)
    there = keep >= 0
    src = torch.where(there, got, 0)
    dst = torch.where(there, i, 0)
    src = torch.where(there, src, src[..., :1])
    L, R, g, _ = got.shape
    l = torch.arange(L, device="cuda")[:, None, None, None]
    r = torch.arange(R, device="cuda")[None, :, None, None]
    hs = torch.arange(c["heads"], device="cuda")[None, None, :, None]
    moved = w.gather(-1, src)
    back = w.clone()
    s["weights"] = back.scatter_(-1, dst, moved)
    pool = s["pool"].view(torch.uint8) if c["cache"] == "fp8" else s["pool"]
    pool = pool if c["layout"] == "kv_first" else pool.transpose(1, 2)            # [L, 2, blocks, B, H, D]
    bt = s["bt"].long()
    two = torch.arange(2, device="cuda")[:, None, None, None, None]
    a = (l, two, bt[r, src // c["block"]], src % c["block"], hs)
    b = (l, two, bt[r, dst // c["block"]], dst % c["block"], hs)
    pool[b] = pool[a]
    return {"keep": keep, "new_len": new_len, "cache": s["pool"], "weights": s["weights"]}


# ---------------------------------------------------------------------------
# the definition in 64 bits, request by request
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "weights": _exact_weights, "evict": _exact_evict}[case["op"]](s)


def _exact_rows(s, r, plane, scale):
    """Rows of request r of a plane, [T, H, D]."""
    t = int(s["kv_len"][r])
    B = s["c"]["block"]
    rows = torch.cat([plane[int(b)] for b in s["bt"][r, :-(-t // B)].tolist()])[:t].double()
    return rows if scale is None else rows * scale.double()[None, :, None]


def _exact_visible(s, r):
    a, b, t = int(s["q_off"][r]), int(s["q_off"][r + 1]), int(s["kv_len"][r])
    pos = torch.arange(t - (b - a), t, device="cuda")[:, None]
    j = torch.arange(t, device="cuda")[None]
    see = j <= pos
    if s["c"]["window"]:
        see = see & (pos - j < s["c"]["window"])
    return a, b, t, see


def _exact_attn(s):
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


def _exact_weights(s):
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


def _exact_rope(s):
    c = s["c"]
    half = c["rot"] // 2
    where = np.concatenate([np.arange(int(t) - int(b - a), int(t)) for a, b, t in
                            zip(s["q_off"].tolist(), s["q_off"].tolist()[1:], s["kv_len"].tolist())])
    req = np.repeat(np.arange(c["requests"]), np.diff(s["q_off"].cpu().numpy()))
    turn = torch.exp(1j * torch.from_numpy(where).cuda()[:, None] * s["freqs"]) * s["magnitude"]
    first = torch.arange(half, device="cuda") * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else half)

    def rotated(x):
        x = x.double().clone()
        z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
        x[..., first], x[..., second] = z.real, z.imag
        return x

    pool = s["pool"].double()
    blocks = s["bt"].cpu().numpy()[req, where // c["block"]]
    blk, row = (torch.from_numpy(np.asarray(x, np.int64)).cuda() for x in (blocks, where % c["block"]))
    for plane, x, scale in ((0, rotated(s["k"]), s["k_scale"]), (1, s["v"].double(), s["v_scale"])):
        if scale is not None:
            x = (x / scale.double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        if c["layout"] == "kv_first":
            pool[0, plane, blk, row] = x
        else:
            pool[0, blk, plane, row] = x
    return {"q": rotated(s["q"]), "cache": pool}


def _exact_evict(s):
    """Rows are moved as they are, so only the whole numbers and the moved weights are worked out: the cache is left to
    the comparison of both forms."""
    c = s["c"]
    w = s["weights"].cpu().numpy().astype(np.float64)
    L, R, g, t = w.shape
    out = w.copy()
    size = s["kv_len"].tolist()
    keep = np.full((L, R, g, s["budget"]), -1, np.int32)
    for l in range(L):
        for r in range(R):
            for h in range(g):
                n = size[r]
                ids = np.arange(n)
                if n > s["budget"]:
                    safe = (ids < s["sink"]) | (ids >= n - s["recent"])
                    rest = ids[~safe]
                    rest = rest[np.lexsort((rest, -w[l, r, h, rest]))][:s["budget"] - int(safe.sum())]
                    ids = np.sort(np.concatenate([ids[safe], rest]))
                keep[l, r, h, :ids.size] = ids
                out[l, r, h, :ids.size] = w[l, r, h, ids]
    return {"keep": torch.from_numpy(keep), "new_len": torch.tensor([min(n, s["budget"]) for n in size]).int(),
            "cache": None, "weights": torch.from_numpy(out)}
