"""kv_evict_select and kv_evict_compact against plain sorting and indexing:
whole numbers and moved bytes, so every comparison is exact."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv

pytestmark = pytest.mark.gpu


def _choose(w, n, budget, sink, recent):
    ids = np.arange(n)
    if n <= budget:
        return ids
    safe = (ids < sink) | (ids >= n - recent)
    rest = ids[~safe]
    x = w[rest].astype(np.float64)
    below = np.isnan(x)
    x[below] = 0
    rest = rest[np.lexsort((rest, -x, below))][:budget - int(safe.sum())]
    return np.sort(np.concatenate([ids[safe], rest]))


def _expected(w, lengths, budget, sink, recent):
    L, R, G, W = w.shape
    keep = np.full((L, R, G, budget), -1, np.int32)
    for l in range(L):
        for r in range(R):
            for g in range(G):
                k = _choose(w[l, r, g], min(int(lengths[r]), W), budget, sink, recent)
                keep[l, r, g, :k.size] = k
    return keep


def _select(w, lengths, budget, sink, recent):
    L, R, G, W = w.shape
    keep = torch.full((L, R, G, budget), 77, dtype=torch.int32, device="cuda")
    new = torch.full((R,), 77, dtype=torch.int32, device="cuda")
    kv.kv_evict_select(torch.from_numpy(w).cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), budget, sink,
                       recent, keep, new)
    torch.cuda.synchronize()
    return keep, new


def _weights(kind, shape, rng):
    if kind == "tail":
        return (rng.random(shape) ** 6).astype(np.float32)
    if kind == "ties":
        return rng.integers(0, 4, shape).astype(np.float32)
    if kind == "equal":
        return np.full(shape, 0.25, np.float32)
    if kind == "signs":
        return np.where(rng.random(shape) < 0.3, np.float32(-0.0), rng.normal(size=shape).astype(np.float32).round(1))
    if kind == "bits":   # any pattern: subnormal numbers, infinities, NaN of both signs
        return rng.integers(0, 2 ** 32, shape, dtype=np.uint32).view(np.float32)
    w = rng.random(shape).astype(np.float32)
    w[rng.random(shape) < 0.2] = math.nan
    w[rng.random(shape) < 0.1] = math.inf
    w[rng.random(shape) < 0.1] = -math.inf
    return w


@pytest.mark.parametrize("kind", ["tail", "ties", "equal", "signs", "bits", "special"])
@pytest.mark.parametrize("budget,sink,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (16, 4, 4), (100, 0, 100), (100, 100, 0),
                                                (255, 3, 17), (256, 0, 0), (300, 100, 200), (1000, 4, 250)])
def test_selection(kind, budget, sink, recent):
    rng = np.random.default_rng(budget + len(kind))
    lengths = [0, 1, 2, budget, budget + 1, 255, 256, 257, 1000]
    w = _weights(kind, (2, len(lengths), 3, 1000), rng)
    lengths = [min(n, 1000) for n in lengths]
    keep, new = _select(w, lengths, budget, sink, recent)
    assert np.array_equal(keep.cpu().numpy(), _expected(w, lengths, budget, sink, recent))
    assert new.cpu().tolist() == [min(n, budget) for n in lengths]


@pytest.mark.parametrize("n", [4096, 8191, 20000, 70001])
def test_long_rows(n):
    rng = np.random.default_rng(n)
    for kind in ("tail", "ties"):
        w = _weights(kind, (1, 2, 2, n), rng)
        keep, new = _select(w, [n, n - 1], n // 3, 4, n // 10)
        assert np.array_equal(keep.cpu().numpy(), _expected(w, [n, n - 1], n // 3, 4, n // 10))


def test_lengths_outside_the_row():
    rng = np.random.default_rng(0)
    w = _weights("tail", (1, 3, 1, 50), rng)
    keep, new = _select(w, [70, -3, 50], 20, 2, 2)
    assert np.array_equal(keep.cpu().numpy(), _expected(w, [50, 0, 50], 20, 2, 2))
    assert new.cpu().tolist() == [20, 0, 20]


def _compact(c, keep, new, w=None):
    c.device()
    dw = None if w is None else torch.from_numpy(w).cuda()
    kv.kv_evict_compact(c.layout, c.d_pool, c.d_bt, torch.from_numpy(keep).cuda(), torch.tensor(new, dtype=torch.int32).cuda(),
                        weights=dw)
    torch.cuda.synchronize()
    return dw


def _move(c, keep, new):
    """The pools after the moves, on the host."""
    L, R, G, n = keep.shape
    want = [p.clone() for p in c.pool]
    old = c.pool
    for l in range(L):
        for plane in (0, 1):
            src = c.view(plane, l).view(torch.uint8) if c.elem == 1 else c.view(plane, l)
            c.pool = want
            dst = c.view(plane, l).view(torch.uint8) if c.elem == 1 else c.view(plane, l)
            c.pool = old
            for r in range(R):
                for g in range(G):
                    hs = slice(None) if G == 1 else slice(g, g + 1)
                    for i in range(new[r]):
                        s = int(keep[l, r, g, i])
                        if s < 0 or s // c.block >= c.bt.shape[1] or i // c.block >= c.bt.shape[1]:
                            continue
                        a, b = int(c.bt[r, s // c.block]), int(c.bt[r, i // c.block])
                        if 0 <= a < c.num_blocks and 0 <= b < c.num_blocks:
                            dst[b, i % c.block, hs] = src[a, s % c.block, hs]
    return want


def _same(c, want):
    for got, x in zip(c.d_pool, want):
        assert torch.equal(got.cpu().view(torch.uint8), x.view(torch.uint8))


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dtype,dim,block,layout,pad", [
    (torch.bfloat16, 64, 16, "kv_first", 0), (torch.bfloat16, 80, 32, "block_first", 48), (torch.float16, 8, 5, "kv_first", 16),
    (torch.float8_e4m3fn, 80, 16, "block_first", 0), (torch.float32, 128, 1, "kv_first", 0), (torch.bfloat16, 256, 128, "kv_first", 0)])
def test_moves(shared, dtype, dim, block, layout, pad):
    rng = np.random.default_rng(dim + block)
    lengths = [0, 1, 40, 300, 129]
    c = ref.Cache(lengths, heads=2, dim=dim, dtype=dtype, block=block, layout=layout, pad=pad, layers=2, seed=dim)
    budget = 100
    G = 1 if shared else 2
    w = _weights("tail", (2, len(lengths), G, 300), rng)
    keep = _expected(w, lengths, budget, 4, 10)
    new = [min(n, budget) for n in lengths]
    want = _move(c, keep, new)
    dw = _compact(c, keep, new, w)
    _same(c, want)
    exp = w.copy()
    for l in range(2):
        for r in range(len(lengths)):
            for g in range(G):
                exp[l, r, g, :new[r]] = w[l, r, g, keep[l, r, g, :new[r]]]
    assert np.array_equal(dw.cpu().numpy(), exp)


def test_missing_blocks_and_odd_indices():
    """Moves out of or into a missing block are skipped, as are indices past the table, negative ones and -1."""
    c = ref.Cache([200, 64], heads=2, dim=64, layers=1, seed=3)
    c.bt[0, 0] = -1
    c.bt[0, 7] = c.num_blocks + 5
    c.bt = np.ascontiguousarray(c.bt[:, :12])
    keep = np.full((1, 2, 2, 60), -1, np.int32)
    keep[0, 0, :, :50] = np.arange(0, 200, 4)
    keep[0, 1, :, :30] = np.arange(34, 64)
    keep[0, 1, 1, 29] = 2 ** 31 - 1
    new = [60, 200]
    want = _move(c, keep, [60, 60])
    _compact(c, keep, new)
    _same(c, want)


def test_long_in_order_moves():
    """Many tiles whose sources lie just behind their destinations."""
    c = ref.Cache([5000], heads=1, dim=64, layers=1, seed=4)
    for gap in (1, 2, 63, 64, 65, 2000):
        keep = np.concatenate([np.arange(10), np.arange(10 + gap, 10 + gap + 2900)]).astype(np.int32)[None, None, None]
        want = _move(c, keep, [2910])
        _compact(c, keep, [2910])
        _same(c, want)


def test_select_then_compact_in_a_graph():
    rng = np.random.default_rng(5)
    c = ref.Cache([700, 90], heads=2, dim=64, layers=2, seed=6).device()
    w = _weights("tail", (2, 2, 2, 700), rng)
    d_w, d_len = torch.from_numpy(w).cuda(), c.d_len
    keep = torch.empty(2, 2, 2, 128, dtype=torch.int32, device="cuda")
    new = torch.empty(2, dtype=torch.int32, device="cuda")

    def go():
        kv.kv_evict_select(d_w, d_len, 128, 4, 32, keep, new)
        kv.kv_evict_compact(c.layout, c.d_pool, c.d_bt, keep, new, weights=d_w)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    for x in range(3):
        fresh = _weights("tail", w.shape, rng)
        outs = []
        for run in (go, g.replay):
            d_w.copy_(torch.from_numpy(fresh))
            for d, h in zip(c.d_pool, c.pool):
                d.copy_(h)
            run()
            torch.cuda.synchronize()
            outs.append([t.clone() for t in (keep, new, d_w, *c.d_pool)])
        for a, b in zip(*outs):
            assert torch.equal(a, b), x
