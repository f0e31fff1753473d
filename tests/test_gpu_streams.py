"""ServedCache over streams: positions with several axes, a window with sinks, accumulated weights, evictions, and kept
tokens that get new positions, in turn."""
import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
import stream_ref
from paper_2609_35065_amd.serving import ServedCache

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
FREQS, _ = kv.kv_rope_frequencies(64, 10000.0)


def _at(c, l):
    """The cache with its layer l as the only one."""
    view = ref.Cache.__new__(ref.Cache)
    view.__dict__.update(c.__dict__)
    view.rows = lambda r, plane, layer=0: c.rows(r, plane, l)
    return view


def _kept(w, n, budget, sink, recent):
    """Cache indices that a head of n tokens keeps, by their weights."""
    if n <= budget:
        return np.arange(n)
    mid = np.arange(sink, n - recent)
    mid = mid[np.lexsort((mid, -w[mid]))][:budget - sink - recent]
    return np.sort(np.concatenate([np.arange(sink), mid, np.arange(n - recent, n)]))


@pytest.mark.parametrize("renumber", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, F8], ids=["bf16", "f16", "f8"])
def test_windows_sinks_evictions(dtype, renumber):
    """Keys are followed from their projection: at every step each cached key is the one of its token, turned to the
    position that it has by then."""
    L, H, HQ, D, window, sink = 2, 2, 4, 64, 12, 3
    total = [120, 160, 60]
    c = ref.Cache(total, heads=H, dim=D, dtype=dtype, layers=L, seed=17, scaled=False).device()
    s = ServedCache(c.layout, c.d_pool, c.d_bt, [0, 0, 0], HQ, torch.from_numpy(FREQS).cuda(), decay=0.5, window=window, sink=sink,
                    renumber=renumber)
    u = 2.0 ** -4 if dtype == F8 else ref.UNIT[c.q_dtype]
    # of each layer, request and head: unrotated keys, their positions, and how often they were rounded
    raw = [[[np.zeros((0, D)) for _ in range(H)] for _ in total] for _ in range(L)]
    pos = [[[np.zeros(0, int) for _ in range(H)] for _ in total] for _ in range(L)]
    times = [[[np.zeros(0, int) for _ in range(H)] for _ in total] for _ in range(L)]
    lengths, nxt = np.zeros(3, int), np.zeros(3, int)
    weights = torch.zeros(L, 3, H, s.capacity, dtype=torch.float64)
    recent = 0 if renumber else window - 1
    for new in ([70, 90, 9], [1, 1, 1], "evict", [1, 0, 1], [20, 3, 1], "evict", [1, 1, 1], "evict", [1, 30, 2]):
        if new == "evict":
            w = s.weights.cpu().numpy()
            s.evict(24, sink=sink, recent=recent)
            torch.cuda.synchronize()
            kept = np.minimum(lengths, 24)
            weights.zero_()
            for l in range(L):
                c.pool[l] = c.d_pool[l].cpu()
                for r in range(3):
                    for h in range(H):
                        ids = _kept(w[l, r, h], int(lengths[r]), 24, sink, recent)
                        raw[l][r][h], at, k = raw[l][r][h][ids], pos[l][r][h][ids], times[l][r][h][ids]
                        if renumber:
                            now = np.arange(ids.size)
                            pos[l][r][h], times[l][r][h] = now, k + (now != ids)
                        else:
                            pos[l][r][h], times[l][r][h] = at, k
                        weights[l, r, h, :ids.size] = torch.from_numpy(w[l, r, h, ids]).double()
                assert torch.equal(s.weights[l].cpu().double(), weights[l])
            lengths = kept
            if renumber:
                nxt = kept.copy()
            assert s.lengths.tolist() == kept.tolist() and s.positions.tolist() == nxt.tolist()
        else:
            s.begin(new)
            lengths, n = lengths + new, sum(new)
            c.lengths = lengths
            for l in range(L):
                q, k, v = (ref.rows_of(n, heads, D, c.q_dtype, c.gen) for heads in (HQ, H, H))
                a = 0
                for r, m in enumerate(new):
                    for h in range(H):
                        raw[l][r][h] = np.concatenate([raw[l][r][h], k[a:a + m, h].double().numpy()])
                        pos[l][r][h] = np.concatenate([pos[l][r][h], np.arange(nxt[r], nxt[r] + m)])
                        times[l][r][h] = np.concatenate([times[l][r][h], np.ones(m, int)])
                    a += m
                dq, out = q.cuda(), torch.empty(n, HQ, D, dtype=c.q_dtype, device="cuda")
                s.attend(l, dq, k.cuda(), v.cuda(), out)
                torch.cuda.synchronize()
                c.pool[l] = c.d_pool[l].cpu()
                at = _at(c, l)
                want, tol, wl, lt = stream_ref.attention(at, new, dq.cpu(), D ** -0.5, True, window, sink)
                ref.assert_within(out, want, tol, "out")
                ref.assert_within(s._lse, wl, lt, "lse")
                want, tol = stream_ref.weights(at, new, dq.cpu(), s._lse.cpu(), D ** -0.5, weights[l], 0.5, True, window, sink)
                ref.assert_within(s.weights[l], want, tol, "weights")
                weights[l] = s.weights[l].cpu().double()
            nxt = nxt + new
            assert s.positions.tolist() == nxt.tolist()
        c.lengths = lengths
        for l in range(L):
            for r in range(3):
                got, _ = c.rows(r, 0, l)
                for h in range(H):
                    x = torch.from_numpy(raw[l][r][h])
                    want, err = stream_ref.turn(x, pos[l][r][h][:, None], FREQS, False)
                    # a rounding is of a value no larger than the pair's two together, and later turns carry it to both
                    size = (x[:, :32].abs() + x[:, 32:].abs()).repeat(1, 2)
                    k = torch.from_numpy(times[l][r][h])[:, None]
                    tol = k * (u * 1.2 * size * 2 ** 0.5 + 2.0 ** -9 * (dtype == F8) + 2.0 ** -20 + err)
                    ref.assert_within(got[:, h], want, tol, f"keys of layer {l} request {r} head {h}")


def test_text_and_images():
    """Prompts of text, an image's patches and text again, then single tokens: positions as given, then on from the
    largest; the same keys as kv_rope_append_axes by itself leaves."""
    H, HQ, D, sections = 2, 4, 64, [8, 12, 12]
    lengths = [70, 55, 12]
    c = ref.Cache(lengths, heads=H, dim=D, seed=3, layers=1).device()
    axes = kv.kv_rope_axes(sections, interleaved=True)
    s = ServedCache(c.layout, c.d_pool, c.d_bt, [0, 0, 4], HQ, torch.from_numpy(FREQS).cuda(), axes=axes, window=30, sink=2)
    text = np.tile(np.arange(5), (3, 1))
    patch = np.stack([np.zeros(24, int), np.arange(24) // 6, np.arange(24) % 6])
    prompt = np.concatenate([text, 5 + patch, 5 + 6 + text], 1)               # next: 16
    given = np.concatenate([prompt, 100 + patch, 4 + text[:, :1]], 1)
    steps = [([34, 24, 1], given, [16, 106, 5]), ([1, 1, 0], None, [17, 107, 5]), ([2, 0, 3], None, [19, 107, 8]), ([0, 0, 0], None, [19, 107, 8]),
             ([0, 24, 0], 200 + patch, [19, 206, 8])]
    held, nxt = np.array([0, 0, 4]), [0, 0, 4]
    for new, positions, after in steps:
        n = sum(new)
        s.begin(new, positions)
        if positions is None:
            positions = np.tile(np.concatenate([np.arange(p, p + m) for p, m in zip(nxt, new)]), (3, 1))
        held, nxt = held + new, after
        assert s.positions.tolist() == after and s.lengths.tolist() == held.tolist()
        q, k, v = (ref.rows_of(n, heads, D, torch.bfloat16, c.gen) for heads in (HQ, H, H))
        dq, out = q.cuda(), torch.empty(n, HQ, D, dtype=torch.bfloat16, device="cuda")
        s.attend(0, dq, k.cuda(), v.cuda(), out)
        torch.cuda.synchronize()
        c.pool[0], c.lengths = c.d_pool[0].cpu(), held
        want, err = stream_ref.turn(q, positions[axes].T[:, None], FREQS, False)
        ref.assert_within(dq, want, 2.0 ** -8 * want.abs() * 1.001 + err + 2.0 ** -24, "q")
        want, err = stream_ref.turn(k, positions[axes].T[:, None], FREQS, False)
        got = torch.cat([c.rows(r, 0)[0][int(held[r]) - m:] for r, m in enumerate(new)])
        ref.assert_within(got, want, 2.0 ** -8 * want.abs() * 1.001 + err + 2.0 ** -24, "k")
        want, tol, _, _ = stream_ref.attention(c, new, dq.cpu(), D ** -0.5, True, 30, 2)
        ref.assert_within(out, want, tol, "out")


def test_a_stream_on_several_streams_of_the_gpu():
    """Steps and a renumbering eviction whose calls come on two streams: the same results as on one."""
    got = []
    for streams in (1, 2):
        c = ref.Cache([900, 300], heads=2, dim=64, layers=2, seed=5).device()
        s = ServedCache(c.layout, c.d_pool, c.d_bt, [100, 7], 4, torch.from_numpy(FREQS).cuda(), window=16, sink=4, renumber=True)
        side = [torch.cuda.Stream() for _ in range(streams)]
        x = torch.zeros(8192, 8192, device="cuda")
        rows = [[ref.rows_of(700, h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2)] for _ in range(4)]
        outs = [torch.empty_like(q) for q, _, _ in rows]
        torch.cuda.synchronize()
        for step in range(2):
            with torch.cuda.stream(side[0]):
                torch.mm(x, x, out=x)
                s.begin([600, 100] if step == 0 else [500, 200])
                s.attend(0, *rows[2 * step], outs[2 * step])
            with torch.cuda.stream(side[-1]):
                s.attend(1, *rows[2 * step + 1], outs[2 * step + 1])
                s.evict(64, sink=4, recent=8)
        torch.cuda.synchronize()
        got.append([t.cpu() for t in (*outs, s.weights, *c.d_pool)])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_a_captured_layer_of_a_stream():
    c = ref.Cache([900, 134], heads=2, dim=64, seed=6).device()
    s = ServedCache(c.layout, c.d_pool, c.d_bt, [100, 100], 4, torch.from_numpy(FREQS).cuda(), window=16, sink=4,
                    axes=kv.kv_rope_axes([8, 24]))
    q, k, v = (ref.rows_of(702, h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2))
    out, graph = torch.empty_like(q), torch.cuda.CUDAGraph()
    s.begin([700, 2])
    assert s._workspace is not None
    before = [s.weights.clone(), c.d_pool[0].clone(), q.clone()]

    def restore():
        for t, was in zip((s.weights, c.d_pool[0], q), before):
            t.copy_(was)

    s.attend(0, q, k, v, out)
    want = [t.clone() for t in (out, s.weights, c.d_pool[0], q)]
    restore()
    with torch.cuda.graph(graph):
        s.attend(0, q, k, v, out)
    for _ in range(3):
        restore()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, s.weights, c.d_pool[0], q), want):
            assert torch.equal(a, b)
