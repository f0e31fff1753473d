"""ServedCache with a sliding window: a window is one of positions, also after evictions, where cache indices are closer
together than the tokens' positions.  What the index window cannot express is refused."""
import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
from paper_2609_35065_amd.serving import ServedCache

FREQS, _ = kv.kv_rope_frequencies(64, 10000.0)


def _host_cache(lengths, **kw):
    layout = kv.make_layout(1, 2, 64, 2, 16, 16, 8, 1, 8 * 4096, 4096)
    return ServedCache(layout, [torch.empty(8 * 4096)], torch.zeros(2, 8, dtype=torch.int32), lengths, 4,
                       torch.from_numpy(FREQS), **kw)


@pytest.mark.parametrize("window,recent", [(8, 6), (8, 0), (100, 20), (22, 20)])
def test_refuses_an_eviction_inside_the_window(window, recent):
    s = _host_cache([100, 3], window=window)
    with pytest.raises(ValueError, match="window"):
        s.evict(24, recent=recent)
    assert s.lengths.tolist() == [100, 3] and s.positions.tolist() == [100, 3]


@pytest.mark.gpu
@pytest.mark.parametrize("window,recent", [(8, 6), (0, 0), (1, 0), (8, 7), (1 << 30, 0)])
def test_evictions_that_the_window_allows(window, recent):
    """Nobody is cut, there is no window, or the last tokens that it reaches all stay."""
    cut = window != 8 or recent >= 7
    c = ref.Cache([50, 20], heads=2, dim=64, seed=3).device()
    s = ServedCache(c.layout, c.d_pool, c.d_bt, [50, 20], 4, torch.from_numpy(FREQS).cuda(), window=window)
    assert s.evict(24 if cut else 50, recent=recent) == ([2, 2] if cut else [4, 2])
    torch.cuda.synchronize()


def _by_position(c, new, q, window, positions):
    """out, and the bound on its error, of new tokens at the end of each request; positions[r][h] are the positions of
    the keys that head h holds.  Row by row and head by head: a row's mask is then one on keys."""
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    g = q.shape[1] // c.heads
    row = 0
    for r, n in enumerate(new):
        keys = [c.rows(r, plane)[0] for plane in (0, 1)]
        for i in range(n):
            last = int(c.lengths[r]) - n + i
            for h in range(c.heads):
                at = torch.from_numpy(positions[r][h][:last + 1])
                one = ref.Cache.__new__(ref.Cache)
                one.__dict__.update(c.__dict__)
                one.lengths, one.heads = [last + 1], 1
                one.rows = lambda _, plane, layer=0: (keys[plane][:last + 1, h:h + 1], at > at[-1] - window)
                o, t, _, _ = ref.attention(one, [1], q[row:row + 1, h * g:(h + 1) * g], 0.125)
                out[row, h * g:(h + 1) * g], tol[row, h * g:(h + 1) * g] = o[0], t[0]
            row += 1
    return out, tol


@pytest.mark.gpu
@pytest.mark.parametrize("window", [1, 8, 20])
def test_steps_after_evictions_see_the_window_of_positions(window):
    H, HQ, D = 2, 4, 64
    c = ref.Cache([100, 60, 40], heads=H, dim=D, seed=window).device()
    lengths = np.array([80, 9, 30])
    s = ServedCache(c.layout, c.d_pool, c.d_bt, lengths, HQ, torch.from_numpy(FREQS).cuda(), window=window, scale=0.125)
    at = [[np.arange(n) for _ in range(H)] for n in lengths]
    nxt = lengths.copy()
    for new in ("evict", [1, 1, 1], [9, 30, 2], "evict", [1, 0, 1], [12, 3, 0], "evict", [1, 1, 1]):
        if new == "evict":
            w, budget = s.weights[0].cpu().numpy(), 32
            s.evict(budget, sink=2, recent=window - 1)
            for r, n in enumerate(lengths):
                for h in range(H):
                    ids = np.arange(n)
                    if n > budget:
                        mid = np.arange(2, n - window + 1)
                        mid = mid[np.lexsort((mid, -w[r, h, mid]))][:budget - 1 - window]
                        ids = np.sort(np.concatenate([[0, 1], mid, np.arange(n - window + 1, n)]))
                    at[r][h] = at[r][h][ids]
            lengths = np.minimum(lengths, budget)
            continue
        s.begin(new)
        for r, n in enumerate(new):
            for h in range(H):
                at[r][h] = np.concatenate([at[r][h], np.arange(nxt[r], nxt[r] + n)])
        nxt, lengths = nxt + new, lengths + new
        q, k, v = (ref.rows_of(sum(new), heads, D, torch.bfloat16, c.gen).cuda() for heads in (HQ, H, H))
        out = torch.empty_like(q)
        s.attend(0, q, k, v, out)
        torch.cuda.synchronize()
        c.pool[0], c.lengths = c.d_pool[0].cpu(), lengths
        want, tol = _by_position(c, new, q.cpu(), window, at)
        ref.assert_within(out, want, tol, "out")
