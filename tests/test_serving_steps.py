"""ServedCache between its calls: a step that is refused leaves it as it was, the host
does not wait for the GPU, and calls on several streams keep their order."""
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


def test_layers_on_several_streams_keep_their_order():
    """Each layer's call comes on another stream, behind work that takes long on the first: the same results as on
    one stream."""
    got = []
    for streams in (1, 2):
        c, s = _served([500, 70], layers=2, seed=5)
        side = [torch.cuda.Stream() for _ in range(streams)]
        x = torch.zeros(8192, 8192, device="cuda")
        rows = [[ref.rows_of(3, h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2)] for _ in range(4)]
        outs = [torch.empty_like(q) for q, _, _ in rows]
        torch.cuda.synchronize()
        for step in range(2):
            with torch.cuda.stream(side[0]):
                _busy(x, 4)
                s.begin([1, 2])
                s.attend(0, *rows[2 * step], outs[2 * step])
            with torch.cuda.stream(side[-1]):
                s.attend(1, *rows[2 * step + 1], outs[2 * step + 1])
        with torch.cuda.stream(side[0]):
            s.evict(64, sink=1, recent=8)
        torch.cuda.synchronize()
        got.append([t.cpu() for t in (*outs, s.weights, *c.d_pool)])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_a_captured_layer():
    """A step's layer as a graph: captured on a stream of the graph's own, replayed against the eager call."""
    c, s = _served([500, 70], seed=6)
    q, k, v = (ref.rows_of(2, h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2))
    out, graph = torch.empty_like(q), torch.cuda.CUDAGraph()
    s.begin([1, 1])
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


def test_a_step_has_to_begin_after_an_eviction():
    c, s = _served([40, 7])
    q, k, v = (ref.rows_of(2, h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2))
    with pytest.raises(ValueError, match="begin"):
        s.attend(0, q, k, v, torch.empty_like(q))
    s.begin([1, 1])
    s.attend(0, q, k, v, torch.empty_like(q))
    s.evict(16, sink=2, recent=4)
    with pytest.raises(ValueError, match="begin"):
        s.attend(0, q, k, v, torch.empty_like(q))
    s.begin([1, 1])
    s.attend(0, q, k, v, torch.empty_like(q))
    torch.cuda.synchronize()


def test_another_default_type():
    """A program may have torch make bfloat16 tensors by default: sums stay in 32 bits."""
    c = ref.Cache([104, 71], heads=2, dim=64).device()
    freqs = torch.from_numpy(FREQS).cuda()
    q, k, v = (ref.rows_of(2, h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2))
    torch.set_default_dtype(torch.bfloat16)
    try:
        s = ServedCache(c.layout, c.d_pool, c.d_bt, [40, 7], 4, freqs)
        s.begin([1, 1])
        s.attend(0, q, k, v, torch.empty_like(q))
        assert s.weights.dtype == torch.float32
        s.evict(16, recent=4)
    finally:
        torch.set_default_dtype(torch.float32)
    torch.cuda.synchronize()
