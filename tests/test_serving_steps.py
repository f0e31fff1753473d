"""ServedCache between its calls: a step that is refused leaves it as it was, and the
host does not wait for the GPU."""
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


def _busy(x, n):
    """Work of the GPU's that lasts some hundred milliseconds: n products of 8,192 a side in 32 bits."""
    for _ in range(n):
        torch.mm(x, x, out=x)


def test_the_host_does_not_wait_for_the_gpu():
    c, s = _served([40, 7], room=200)
    x = torch.zeros(8192, 8192, device="cuda")
    q, k, v = (ref.rows_of(2, h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2))
    out = torch.empty_like(q)

    def steps():
        for _ in range(3):
            s.begin([1, 1])
            s.attend(0, q, k, v, out)
        return s.evict(40, sink=2, recent=4)

    _busy(x, 1)
    steps()
    torch.cuda.synchronize()
    _busy(x, 20)
    done = torch.cuda.Event()
    done.record()
    assert steps() == [3, 1]
    assert not done.query(), "the host waited"
    torch.cuda.synchronize()
