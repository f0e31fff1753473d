"""ServedCache: where a request goes on after positions that the caller gave, axes that no pair takes, and layers given by
their addresses."""
import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
import stream_ref
from paper_2609_35065_amd.serving import ServedCache

pytestmark = pytest.mark.gpu
FREQS, _ = kv.kv_rope_frequencies(64, 10000.0)


def _served(lengths, room=64, layers=1, seed=0, **kw):
    c = ref.Cache([n + room for n in lengths], heads=2, dim=64, layers=layers, seed=seed).device()
    return c, ServedCache(c.layout, c.d_pool, c.d_bt, lengths, 4, torch.from_numpy(FREQS).cuda(), **kw)


def test_a_request_goes_on_after_its_largest_position():
    """Given positions below earlier ones do not move a request back."""
    c, s = _served([40, 7, 3], axes=kv.kv_rope_axes([8, 12, 12]))
    s.begin([2, 1, 0], np.array([[5, 6, 50], [5, 90, 2], [5, 6, 2]]))
    assert s.positions.tolist() == [91, 51, 3]
    s.begin([1, 2, 1], np.array([[60, 20, 70, 0], [61, 3, 3, 1], [60, 3, 3, 2]]))
    assert s.positions.tolist() == [91, 71, 3]
    s.begin([1, 1, 1])
    torch.cuda.synchronize()
    assert s.positions.tolist() == [92, 72, 4]
    assert s._positions.cpu().tolist() == [[91, 71, 3]] * 3
    # where the held tokens have other positions than 0, 1, ..., the caller says where a request goes on
    c, s = _served([40], axes=kv.kv_rope_axes([8, 12, 12]))
    s.positions[0] = 12
    s.begin([1], np.array([[12], [20], [14]]))
    assert s.positions.tolist() == [21]


@pytest.mark.parametrize("sections", [[16, 16, 0], [0, 32, 0, 0], [32, 0]])
def test_axes_that_no_pair_takes(sections):
    c, s = _served([0, 4], seed=1, axes=kv.kv_rope_axes(sections), decay=None)
    new, n = [20, 3], 23
    given = np.random.default_rng(0).integers(0, 500, (len(sections), n))
    s.begin(new, given)
    assert s.positions.tolist() == [max(0, given[:, :20].max() + 1), max(4, given[:, 20:].max() + 1)]
    q, k, v = (ref.rows_of(n, h, 64, torch.bfloat16, c.gen) for h in (4, 2, 2))
    dq, out = q.cuda(), torch.empty(n, 4, 64, dtype=torch.bfloat16, device="cuda")
    s.attend(0, dq, k.cuda(), v.cuda(), out)
    torch.cuda.synchronize()
    want, err = stream_ref.turn(q, given[kv.kv_rope_axes(sections)].T[:, None], FREQS, False)
    ref.assert_within(dq, want, 2.0 ** -8 * want.abs() * 1.001 + err + 2.0 ** -24, "q")
    for more in (0, kv.KV_MAX_AXES + 1):
        with pytest.raises(ValueError, match="positions"):
            s.begin([1, 1], np.zeros((more, 2), int))


@pytest.mark.parametrize("renumber", [False, True])
def test_layers_given_by_their_addresses(renumber):
    got = []
    for by_address in (False, True):
        c = ref.Cache([300, 90], heads=2, dim=64, layers=2, seed=5).device()
        s = ServedCache(c.layout, [t.data_ptr() for t in c.d_pool] if by_address else c.d_pool, c.d_bt, [0, 0], 4,
                        torch.from_numpy(FREQS).cuda(), renumber=renumber)
        for new in ([200, 60], [1, 1]):
            s.begin(new)
            for l in range(2):
                q, k, v = (ref.rows_of(sum(new), h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2))
                s.attend(l, q, k, v, torch.empty_like(q))
            s.evict(50, sink=2, recent=4)
        torch.cuda.synchronize()
        got.append([t.cpu() for t in (s.weights, *c.d_pool)])
    for a, b in zip(*got):
        assert torch.equal(a, b)
