"""ServedCache between its calls: a step that is refused leaves it as it was."""
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
from paper_2609_35065_amd.serving import ServedCache

pytestmark = pytest.mark.gpu
FREQS, _ = kv.kv_rope_frequencies(64, 10000.0)


def _served(lengths, room=64, q_heads=4, layers=1, seed=0, **kw):
    c = ref.Cache([n + room for n in lengths], heads=2, dim=64, layers=layers, seed=seed).device()
    return c, ServedCache(c.layout, c.d_pool, c.d_bt, lengths, q_heads, torch.from_numpy(FREQS).cuda(), **kw)


def test_a_refused_step_changes_nothing():
    c, s = _served([40, 7], q_heads=1 << 30)          # more rows than the operators count
    for _ in range(2):
        with pytest.raises(kv.KvError):
            s.begin([1, 2])
        assert s.lengths.tolist() == [40, 7] and s.positions.tolist() == [40, 7] and s.batch is None
