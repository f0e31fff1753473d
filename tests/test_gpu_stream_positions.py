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
