"""kv_sink_weights against the definition in 64 bits: sinks whose rows are cut into parts or not, keys that no row sees,
which only fade, and the variants of few and many rows and of shared keys."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
import stream_ref
from test_gpu_attention_weights import BATCHES
from test_gpu_operator_paths import WIDE, _some_heads

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f8": F8}


def _run(c, new, q, lse, scale, window, sink, causal, decay, old, max_kv=None, max_q=None):
    c.device()
    b = c.batch(new, max_kv=max_kv, max_q=max_q)
    w = old.cuda()
    size = kv.kv_sink_weights_workspace(c.layout, b, q.shape[1], window, sink)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda") if size else None
    kv.kv_sink_weights(c.layout, c.d_pool[0], b, q.cuda(), lse.cuda(), w, scale, window, sink, causal=causal, decay=decay,
                       k_scale=c.d_scales[0], workspace=ws)
    torch.cuda.synchronize()
    return w, size


def _check(c, new, q, scale, window, sink, causal=True, decay=1.0, old=None, width=None, lse_edit=None, **hints):
    lse = stream_ref.attention(c, new, q, scale, causal, window, sink)[2].float()
    if lse_edit:
        lse_edit(lse)
    width = int(c.lengths.max(initial=1)) if width is None else width
    if old is None:
        old = torch.rand(len(new), c.heads, width, generator=c.gen)
    w, size = _run(c, new, q, lse, scale, window, sink, causal, decay, old, **hints)
    want, wt = stream_ref.weights(c, new, q, lse, scale, old, decay, causal, window, sink)
    ref.assert_within(w, want, wt, "weights")
    for r, n in enumerate(c.lengths):   # nothing past the length is touched
        assert torch.equal(w[r, :, n:].cpu().view(torch.int32), old[r, :, n:].contiguous().view(torch.int32))
    again, _ = _run(c, new, q, lse, scale, window, sink, causal, decay, old, **hints)
    assert torch.equal(w.nan_to_num(), again.nan_to_num())
    return w, size


@pytest.mark.parametrize("name", sorted(BATCHES))
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_batches(name, dtype):
    lengths, new = BATCHES[name]
    c = ref.Cache(lengths, heads=2, dim=128, dtype=DTYPES[dtype], seed=len(name))
    q = ref.rows_of(sum(new), 8, 128, c.q_dtype, c.gen, 1.5).contiguous()
    _check(c, new, q, 128 ** -0.5, 100, 4)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("decay", [1.0, 0.25, 0.0])
@pytest.mark.parametrize("new", [[1, 1, 1], [220, 1, 29]], ids=["decode", "chunk"])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (7, 4), (64, 63), (64, 64), (100, 65), (200, 180), (30, 300),
                                         (5, 10000), (10000, 4), (0, 9), (40, (1 << 31) - 1)])
def test_windows_sinks_and_decay(window, sink, new, decay, causal):
    c = ref.Cache([400, 129, 33], heads=2, dim=64, seed=window % 1000 + sink % 1000)
    q = ref.rows_of(sum(new), 4, 64, torch.bfloat16, c.gen).contiguous()
    _check(c, new, q, 0.125, window, sink, causal, decay)


@pytest.mark.parametrize("dim", [8, 40, 64, 80, 96, 128, 136, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f8"])
@pytest.mark.parametrize("new", [[1, 1], [70, 10]], ids=["decode", "chunk"])
def test_head_sizes(dim, dtype, new):
    if dtype == "f8" and dim % 16:
        pytest.skip("rows of an 8-bit cache are whole 16-byte units")
    c = ref.Cache([300, 75], heads=2, dim=dim, dtype=DTYPES[dtype], seed=dim, layout="block_first", pad=16)
    q = ref.rows_of(sum(new), 4, dim, c.q_dtype, c.gen, 1.5).contiguous()
    _check(c, new, q, dim ** -0.5, 50, 5)


@pytest.mark.parametrize("window,sink,new,lengths", [
    (16, 4, [700, 5, 300], [900, 300, 300]),        # three parts
    (1, 130, [600, 1], [700, 500]),                 # and three tiles of sinks
    (20, 1000, [900, 40], [1500, 90]),              # sixteen tiles
    (20, 1030, [900, 40], [1500, 90]),              # too many to be cut
    (250, 4, [2100], [2100])])
def test_sinks_in_parts(window, sink, new, lengths):
    c = ref.Cache(lengths, heads=2, dim=64, seed=sink)
    q = ref.rows_of(sum(new), 4, 64, torch.bfloat16, c.gen).contiguous()
    _, size = _check(c, new, q, 0.125, window, sink, decay=0.5)
    assert (size > 0) == (sink <= 1024)
    _check(c, new, q, 0.125, window, sink, causal=False)


@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (80, "f16"), (128, "f8"), (256, "bf16")])
@pytest.mark.parametrize("window,sink,causal", [(50, 4, True), (130, 70, True), (60, 30, False)])
def test_keys_that_no_waves_share(dim, dtype, window, sink, causal):
    """Many heads: tiles of 256 keys beside the sinks'."""
    c = ref.Cache(WIDE["lengths"], heads=128, dim=dim, dtype=DTYPES[dtype], seed=dim)
    new = WIDE["new"]
    q = ref.rows_of(sum(new), 256, dim, c.q_dtype, c.gen, 1.5).contiguous()
    heads = [0, 125]
    of_q = [2 * h + x for h in heads for x in (0, 1)]
    some = _some_heads(c, heads)
    lse = torch.zeros(sum(new), 256)
    lse[:, of_q] = stream_ref.attention(some, new, q[:, of_q], dim ** -0.5, causal, window, sink)[2].float()
    old = torch.rand(len(new), 128, 700, generator=c.gen)
    w, _ = _run(c, new, q, lse, dim ** -0.5, window, sink, causal, 0.5, old)
    want, tol = stream_ref.weights(some, new, q[:, of_q], lse[:, of_q], dim ** -0.5, old[:, heads], 0.5, causal, window, sink)
    ref.assert_within(w[:, heads], want, tol, "weights")


def test_no_decay_reads_nothing_old_and_full_decay_changes_nothing_unseen():
    c = ref.Cache([500, 40], heads=2, dim=64, seed=1)
    for new in ([1, 1], [30, 1]):
        q = ref.rows_of(sum(new), 4, 64, torch.bfloat16, c.gen).contiguous()
        w, _ = _check(c, new, q, 0.125, 20, 3, decay=0.0, old=torch.full((2, 2, 500), math.nan))
        assert bool(w[0].isfinite().all()) and bool((w[0, :, 3:500 - new[0] - 19] == 0).all())
        old = torch.full((2, 2, 500), math.nan)
        w, _ = _check(c, new, q, 0.125, 20, 3, decay=1.0, old=old)
        assert bool(w[0].isnan().all())


def test_missing_blocks_and_values_out_of_sight():
    for new in ([1, 1, 1, 1], [60, 1, 5, 2]):
        c = ref.Cache([300, 96, 40, 500], heads=2, dim=64, seed=5)
        x = c.view(0)
        used = set(c.bt.ravel().tolist())
        for b in range(c.num_blocks):
            if b not in used:
                x[b] = math.nan
        x[int(c.bt[2, -1]), 40 % 16:] = math.inf
        for t in range(7, 300 - new[0] - 30):
            x[int(c.bt[0, t // 16]), t % 16] = math.nan
        c.bt[0, 16] = -1
        c.bt[0, 5:9] = c.num_blocks
        c.bt[1, :] = -7
        c.bt[2, 0] = -1
        c.bt = np.ascontiguousarray(c.bt[:, :18])
        q = ref.rows_of(sum(new), 4, 64, torch.bfloat16, c.gen).contiguous()
        _check(c, new, q, 0.125, 30, 7)
        _check(c, new, q, 0.125, 30, 7, decay=0.5)


def test_narrow_weights_and_hints():
    c = ref.Cache([300, 20], heads=2, dim=64, seed=6)
    for new in ([1, 1], [40, 1]):
        q = ref.rows_of(sum(new), 4, 64, torch.bfloat16, c.gen).contiguous()
        for width in (2, 131, 290, 777):
            _check(c, new, q, 0.125, 25, 6, width=width, decay=0.5)
        for hint in (0, 5, 1 << 22):
            _check(c, new, q, 0.125, 25, 6, max_kv=hint)
        for hint in (0, 1, 3000, 1 << 20):
            _check(c, new, q, 0.125, 25, 6, max_q=hint)


def test_rows_without_a_sum_add_nothing():
    c = ref.Cache([100], heads=1, dim=64, seed=7)
    for n in (2, 20):
        q = ref.rows_of(n, 2, 64, torch.bfloat16, c.gen).contiguous()

        def edit(lse):
            lse[n // 2:n // 2 + 3] = -math.inf
        _check(c, [n], q, 0.125, 30, 4, lse_edit=edit)


def test_without_sinks_and_a_window_the_same_as_kv_attention_weights():
    c = ref.Cache([300, 20], heads=2, dim=64, seed=8)
    for new in ([1, 1], [40, 1]):
        q = ref.rows_of(sum(new), 4, 64, torch.bfloat16, c.gen).contiguous()
        lse = ref.attention(c, new, q, 0.125)[2].float()
        old = torch.rand(2, 2, 300, generator=c.gen)
        w, _ = _run(c, new, q, lse, 0.125, 0, 5, True, 0.5, old)
        plain = old.cuda()
        kv.kv_attention_weights(c.layout, c.d_pool[0], c.batch(new), q.cuda(), lse.cuda(), plain, 0.125, decay=0.5)
        assert torch.equal(w, plain)


def test_graph_replays():
    c = ref.Cache([900, 300], heads=2, dim=64, seed=9).device()
    new = [700, 5]
    b = c.batch(new)
    q = ref.rows_of(705, 4, 64, torch.bfloat16, c.gen).contiguous().cuda()
    out, lse, w = torch.empty_like(q), torch.empty(705, 4, device="cuda"), torch.zeros(2, 2, 900, device="cuda")
    ws = torch.empty(max(kv.kv_sink_attention_workspace(c.layout, b, 4, 16, 4), kv.kv_sink_weights_workspace(c.layout, b, 4, 16, 4)),
                     dtype=torch.uint8, device="cuda")

    def step():
        kv.kv_sink_attention(c.layout, c.d_pool[0], b, q, out, 0.125, 16, 4, lse=lse, workspace=ws)
        kv.kv_sink_weights(c.layout, c.d_pool[0], b, q, lse, w, 0.125, 16, 4, decay=0.5, workspace=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    kept = torch.zeros_like(w)
    for x in range(4):
        q.mul_(-1.1)
        w.copy_(kept)
        step()
        torch.cuda.synchronize()
        want = w.clone()
        w.copy_(kept)
        lse.zero_()
        ws.fill_(0xff)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, want), x
        kept = want


@pytest.mark.parametrize("value", [math.inf, math.nan], ids=["inf", "nan"])
def test_rows_whose_sum_is_not_finite(value):
    """A row of infinite lse adds 0 to finite scores, one of NaN adds NaN to what it sees; with and without sinks."""
    c = ref.Cache([300], heads=1, dim=64, seed=7).device()
    for n in (2, 60):
        q = ref.rows_of(n, 2, 64, torch.bfloat16, c.gen).contiguous()

        def edit(lse):
            lse[n // 2] = value
        w, _ = _check(c, [n], q, 0.125, 30, 4, lse_edit=edit)
        assert bool(w.isnan().any()) == math.isnan(value)
        lse = ref.attention(c, [n], q, 0.125)[2].float()
        edit(lse)
        old = torch.rand(1, 1, 300, generator=c.gen)
        plain = old.cuda()
        kv.kv_attention_weights(c.layout, c.d_pool[0], c.batch([n]), q.cuda(), lse.cuda(), plain, 0.125)
        want, tol = stream_ref.weights(c, [n], q, lse, 0.125, old, 1.0)
        ref.assert_within(plain, want, tol, "weights")
