"""ServedCache: chunks, single tokens and evictions in turn, against the definition in 64 bits on the rows that the
cache holds at each step."""
import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
from paper_2609_35065_amd.serving import ServedCache

F8 = torch.float8_e4m3fn
FREQS, _ = kv.kv_rope_frequencies(64, 10000.0)


def _key_rows(k, pos):
    """Keys [n, H, 64] turned at their positions, half layout, in 64 bits."""
    u = torch.from_numpy(np.asarray(pos, np.float64)[:, None] * FREQS)[:, None]
    a, b = k.double().chunk(2, -1)
    return torch.cat([a * u.cos() - b * u.sin(), a * u.sin() + b * u.cos()], -1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, F8], ids=["bf16", "f16", "f8"])
def test_steps_and_evictions(dtype):
    L, H, HQ, D = 2, 2, 4, 64
    total = [90, 140, 33]
    c = ref.Cache(total, heads=H, dim=D, dtype=dtype, layers=L, seed=17, scaled=False).device()
    s = ServedCache(c.layout, c.d_pool, c.d_bt, [40, 0, 9], HQ, torch.from_numpy(FREQS).cuda(), decay=0.5)
    lengths, position = np.array([40, 0, 9]), np.array([40, 0, 9])
    weights = torch.zeros(L, 3, H, s.capacity, dtype=torch.float64)
    for new in ([30, 60, 0], [1, 1, 1], "evict", [1, 0, 1], [2, 3, 1], "evict", [1, 1, 1]):
        if new == "evict":
            before = [p.cpu().clone() for p in c.d_pool]
            w = s.weights.cpu().numpy()
            blocks = s.evict(24, sink=2, recent=6)
            torch.cuda.synchronize()
            kept = np.minimum(lengths, 24)
            assert blocks == [-(-int(n) // 16) for n in kept] and s.lengths.tolist() == kept.tolist()
            weights.zero_()
            for l in range(L):
                c.pool[l] = c.d_pool[l].cpu()
                was = ref.Cache.__new__(ref.Cache)
                was.__dict__.update(c.__dict__)
                was.pool = before
                was.lengths, c.lengths = lengths, kept
                for r in range(3):
                    n, m = int(lengths[r]), int(kept[r])
                    for h in range(H):
                        ids = np.arange(n)
                        if n > 24:
                            mid = np.arange(2, n - 6)
                            mid = mid[np.lexsort((mid, -w[l, r, h, mid]))][:24 - 8]
                            ids = np.sort(np.concatenate([[0, 1], mid, np.arange(n - 6, n)]))
                        for plane in (0, 1):
                            old, now = was.rows(r, plane, l)[0], c.rows(r, plane, l)[0]
                            assert torch.equal(now[:, h], old[ids, h])
                        weights[l, r, h, :m] = torch.from_numpy(w[l, r, h, ids]).double()
                assert torch.equal(s.weights[l].cpu().double(), weights[l])
            lengths = kept
            continue
        s.begin(new)
        lengths = lengths + new
        c.lengths = lengths
        n = sum(new)
        pos = np.concatenate([np.arange(p, p + a) for p, a in zip(position, new)])
        for l in range(L):
            q, k, v = (ref.rows_of(n, heads, D, c.q_dtype, c.gen) for heads in (HQ, H, H))
            dq, out = q.cuda(), torch.empty(n, HQ, D, dtype=c.q_dtype, device="cuda")
            s.attend(l, dq, k.cuda(), v.cuda(), out)
            torch.cuda.synchronize()
            c.pool[l] = c.d_pool[l].cpu()
            u = ref.UNIT[c.q_dtype]
            for x, got, unit in ((q, dq.cpu(), u), (k, None, 2.0 ** -4 if dtype == F8 else u)):
                want = _key_rows(x, pos)
                if got is None:      # the cache's last rows of each request
                    got = torch.cat([c.rows(r, 0, l)[0][int(lengths[r]) - a:] for r, a in enumerate(new)])
                err = 2.0 ** -20 * x.double().abs().amax(-1, keepdim=True) * 2 + (2.0 ** -10 if unit > u else 2.0 ** -24)
                ref.assert_within(got, want, unit * want.abs() * 1.001 + err, "rotated rows")
            want, tol, wl, lt = ref.attention(c, new, dq.cpu(), D ** -0.5, layer=l)
            ref.assert_within(out, want, tol, "out")
            ref.assert_within(s._lse, wl, lt, "lse")
            view = ref.Cache.__new__(ref.Cache)
            view.__dict__.update(c.__dict__)
            view.rows = lambda r, plane: c.rows(r, plane, l)
            want, tol = ref.weights(view, new, dq.cpu(), s._lse.cpu(), D ** -0.5, weights[l], 0.5)
            ref.assert_within(s.weights[l], want, tol, "weights")
            weights[l] = s.weights[l].cpu().double()
        position = position + new


def _host_cache(lengths, **kw):
    layout = kv.make_layout(1, 2, 64, 2, 16, 16, 8, 1, 8 * 4096, 4096)
    return ServedCache(layout, [torch.empty(8 * 4096)], torch.zeros(2, 3, dtype=torch.int32), lengths, 4,
                       torch.from_numpy(FREQS), **kw)


def test_refuses_what_does_not_fit():
    for bad in ([1], [1, 49], [-1, 0]):
        with pytest.raises(ValueError):
            _host_cache(bad)
    s = _host_cache([40, 0], decay=None)
    for bad in ([9, 0], [0, -1], [1], [1, 1, 1]):
        with pytest.raises(ValueError):
            s.begin(bad)
    assert s.lengths.tolist() == [40, 0]
    with pytest.raises(ValueError):
        s.evict(8)
