"""Variants of the accumulated weights that only some batches take, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
import stream_ref
from test_gpu_operator_paths import _some_heads
from test_gpu_sink_weights import _check, _run

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f8": F8}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("decay", [1.0, 0.5, 0.0])
@pytest.mark.parametrize("window,new,lengths", [(16, [700, 5, 300], [900, 300, 300]), (1, [300], [300]), (100, [2000, 1], [2500, 400])])
def test_long_chunks_without_sinks(window, new, lengths, decay, causal):
    """A window alone, over chunks that are longer than its rows: nothing is cut into parts, and no workspace is needed."""
    c = ref.Cache(lengths, heads=2, dim=64, seed=window)
    q = ref.rows_of(sum(new), 4, 64, torch.bfloat16, c.gen).contiguous()
    _, size = _check(c, new, q, 0.125, window, 0, causal, decay)
    assert size == 0


@pytest.mark.parametrize("hint", [None, 1 << 17], ids=["shared", "unshared"])
@pytest.mark.parametrize("new", [[5, 9, 1, 40], [8, 9, 16, 24], [33, 32, 31, 1], [64, 65, 128, 7]])
def test_requests_of_a_few_rows_beside_many(new, hint):
    """Four rows a token: requests that fill one group of 32 rows, a part of it, or several, whether waves share keys or
    not."""
    c = ref.Cache([n + 150 for n in new], heads=2, dim=64, seed=sum(new))
    q = ref.rows_of(sum(new), 8, 64, torch.bfloat16, c.gen).contiguous()
    for window, sink in ((0, 0), (60, 4), (60, 0)):
        _check(c, new, q, 0.125, window, sink, decay=0.5, max_kv=hint)


# so many heads that the waves of a workgroup pass a request's keys tile after tile, 0 to 6 tiles each
TILES = dict(heads=64, lengths=[1, 255, 257, 513, 769, 1025, 1500, 300], new=[1] * 8)


def _check_some(c, new, q, scale, window, sink, decay, causal=True, **hints):
    """kv_sink_weights, or kv_attention_weights (sink None), for two of many heads."""
    group = q.shape[1] // c.heads
    heads = [0, c.heads - 3]
    of_q = [group * h + x for h in heads for x in range(group)]
    some = _some_heads(c, heads)
    lse = torch.zeros(sum(new), q.shape[1])
    lse[:, of_q] = stream_ref.attention(some, new, q[:, of_q], scale, causal, window, sink or 0)[2].float()
    width = int(c.lengths.max())
    old = torch.rand(len(new), c.heads, width, generator=c.gen)
    if sink is None:
        w = old.cuda()
        kv.kv_attention_weights(c.layout, c.d_pool[0], c.batch(new, **hints), q.cuda(), lse.cuda(), w, scale, causal=causal,
                                window=window, decay=decay, k_scale=c.d_scales[0])
        torch.cuda.synchronize()
    else:
        w, _ = _run(c, new, q, lse, scale, window, sink, causal, decay, old, **hints)
    want, tol = stream_ref.weights(some, new, q[:, of_q], lse[:, of_q], scale, old[:, heads], decay, causal, window, sink or 0)
    ref.assert_within(w[:, heads], want, tol, "weights")
    for r, n in enumerate(c.lengths):   # nothing past the length is touched
        assert torch.equal(w[r, :, n:].cpu(), old[r, :, n:])


@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (64, "f8"), (80, "f16"), (80, "f8"), (128, "bf16"), (128, "f8"), (256, "bf16"),
                                       (256, "f8")])
def test_waves_that_pass_several_tiles(dim, dtype):
    c = ref.Cache(TILES["lengths"], heads=TILES["heads"], dim=dim, dtype=DTYPES[dtype], seed=dim).device()
    q = ref.rows_of(8, 128, dim, c.q_dtype, c.gen, 1.5).contiguous()
    for window, sink in ((0, None), (300, None), (1200, 4), (300, 70), (1200, 0)):
        for decay in (0.0, 0.5, 1.0):
            _check_some(c, TILES["new"], q, dim ** -0.5, window, sink, decay)
    _check_some(c, TILES["new"], q, dim ** -0.5, 300, 70, 0.5, causal=False)


@pytest.mark.parametrize("dim,dtype", [(64, "f16"), (80, "bf16"), (128, "bf16"), (256, "f8")])
def test_few_tiles_and_more_rows_than_the_host_knows_of(dim, dtype):
    """Hints that are too small: one workgroup a head for all keys, sixteen rows after sixteen; with and without the next
    tile on its way."""
    for heads, lengths, new, hint in ((2, [1500, 700, 20], [20, 1, 9], 1), (64, TILES["lengths"], [1, 2, 30, 1, 9, 8, 17, 1], None)):
        c = ref.Cache(lengths, heads=heads, dim=dim, dtype=DTYPES[dtype], seed=dim).device()
        q = ref.rows_of(sum(new), heads * 2, dim, c.q_dtype, c.gen, 1.5).contiguous()
        for window, sink in ((0, None), (300, 70)):
            _check_some(c, new, q, dim ** -0.5, window, sink, 0.5, max_q=1, max_kv=hint)


@pytest.mark.parametrize("dtype", ["bf16", "f8"])
def test_missing_blocks_in_several_tiles(dtype):
    c = ref.Cache(TILES["lengths"], heads=TILES["heads"], dim=64, dtype=DTYPES[dtype], seed=3)
    x = c.view(0)
    if dtype == "bf16":
        x[int(c.bt[6, 30])] = math.nan                     # out of every window's sight
    c.bt[6, 70:75] = -1
    c.bt[5, 20] = c.num_blocks
    c.bt[4, :] = -7
    c.bt = np.ascontiguousarray(c.bt[:, :90])
    c.device()
    q = ref.rows_of(8, 128, 64, torch.bfloat16, c.gen, 1.5).contiguous()
    for window, sink in ((300, None), (700, 4), (300, 70)):
        _check_some(c, TILES["new"], q, 0.125, window, sink, 0.5)


# tiles of 128 keys, each half of them two waves that share the rows; in the second the sinks' rows are cut into parts
PAIRS = [dict(heads=64, lengths=[1000, 800], new=[200, 150], window=500), dict(heads=64, lengths=[900, 700], new=[660, 500], window=100)]


@pytest.mark.parametrize("dim,dtype", [(64, "f16"), (80, "bf16"), (80, "f8"), (128, "bf16"), (128, "f8"), (256, "bf16"), (256, "f8")])
@pytest.mark.parametrize("at", [0, 1])
def test_tiles_of_128_keys(at, dim, dtype):
    t = PAIRS[at]
    c = ref.Cache(t["lengths"], heads=64, dim=dim, dtype=DTYPES[dtype], seed=dim).device()
    q = ref.rows_of(sum(t["new"]), 128, dim, c.q_dtype, c.gen, 1.5).contiguous()
    for sink, decay, causal in ((4, 1.0, True), (70, 0.5, True), (0, 0.0, True), (4, 0.5, False)):
        _check_some(c, t["new"], q, dim ** -0.5, t["window"], sink, decay, causal)
