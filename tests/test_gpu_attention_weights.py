"""kv_attention_weights against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def _check(c, new, q, scale, causal=True, window=0, decay=1.0, old=None, width=None, max_kv=None, lse_edit=None):
    c.device()
    b = c.batch(new, max_kv=max_kv)
    out, tol, lse, lt = ref.attention(c, new, q, scale, causal, window)
    lse = lse.float()
    if lse_edit:
        lse_edit(lse)
    width = int(c.lengths.max(initial=1)) if width is None else width
    if old is None:
        old = torch.rand(len(new), c.heads, width, generator=c.gen)
    w = old.cuda()
    kv.kv_attention_weights(c.layout, c.d_pool[0], b, q.cuda(), lse.cuda(), w, scale, causal=causal, window=window,
                            decay=decay, k_scale=c.d_scales[0])
    torch.cuda.synchronize()
    want, wt = ref.weights(c, new, q, lse, scale, old, decay, causal, window)
    ref.assert_within(w, want, wt, "weights")
    for r, n in enumerate(c.lengths):   # nothing past the length is touched
        assert torch.equal(w[r, :, n:].cpu().view(torch.int32), old[r, :, n:].contiguous().view(torch.int32))
    return w


BATCHES = {"one": ([1], [1]), "decode": ([1001], [1]), "decode-ragged": ([1, 31, 32, 33, 127, 128, 129, 500], [1] * 8),
           "none-new": ([40, 0, 33], [0, 0, 5]), "all-new": ([77], [77]), "chunks": ([130, 257, 64], [65, 257, 1]),
           "more-new-than-cache": ([5], [9]), "long": ([2500, 30], [130, 1])}


@pytest.mark.parametrize("name", sorted(BATCHES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, F8], ids=["bf16", "f16", "f8"])
def test_batches(name, dtype):
    lengths, new = BATCHES[name]
    c = ref.Cache(lengths, heads=2, dim=128, dtype=dtype, seed=len(name))
    q = ref.rows_of(sum(new), 8, 128, c.q_dtype, c.gen, 1.5).contiguous()
    _check(c, new, q, 128 ** -0.5)


@pytest.mark.parametrize("dim", [8, 40, 64, 80, 96, 112, 128, 136, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, F8], ids=["bf16", "f8"])
def test_head_sizes(dim, dtype):
    if dtype == F8 and dim % 16:
        pytest.skip("rows of an 8-bit cache are whole 16-byte units")
    c = ref.Cache([200, 75], heads=2, dim=dim, dtype=dtype, seed=dim, layout="block_first", pad=16)
    q = ref.rows_of(80, 4, dim, c.q_dtype, c.gen, 1.5).contiguous()
    _check(c, [70, 10], q, dim ** -0.5)


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 71), (3, 3), (2, 6), (8, 4), (1, 32)])
def test_groups(heads, group):
    c = ref.Cache([150, 90], heads=heads, dim=64, dtype=torch.float16, seed=heads * 100 + group, block=20)
    q = ref.rows_of(53, heads * group, 64, torch.float16, c.gen, 2.0).contiguous()
    _check(c, [50, 3], q, 0.125)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 7, 64, 10000])
@pytest.mark.parametrize("decay", [1.0, 0.25])
def test_windows_and_decay(causal, window, decay):
    c = ref.Cache([400, 129, 33], heads=2, dim=64, seed=window)
    q = ref.rows_of(250, 4, 64, torch.bfloat16, c.gen).contiguous()
    _check(c, [220, 1, 29], q, 0.125, causal=causal, window=window, decay=decay)


def test_no_decay_reads_nothing_old():
    c = ref.Cache([100, 40], heads=2, dim=64, seed=1)
    q = ref.rows_of(31, 4, 64, torch.bfloat16, c.gen).contiguous()
    w = _check(c, [30, 1], q, 0.125, decay=0.0, old=torch.full((2, 2, 100), math.nan))
    assert bool(w[0].isfinite().all())


def test_missing_blocks_and_values_out_of_sight():
    c = ref.Cache([300, 96, 40], heads=2, dim=64, seed=5)
    x = c.view(0)
    used = set(c.bt.ravel().tolist())
    for b in range(c.num_blocks):
        if b not in used:
            x[b] = math.nan
    x[int(c.bt[2, -1]), 40 % 16:] = math.inf
    c.bt[0, 2] = -1
    c.bt[0, 5:9] = c.num_blocks
    c.bt[1, :] = -7
    c.bt = np.ascontiguousarray(c.bt[:, :17])
    q = ref.rows_of(66, 4, 64, torch.bfloat16, c.gen).contiguous()
    _check(c, [60, 1, 5], q, 0.125)


def test_narrow_weights_and_hints():
    c = ref.Cache([300, 20], heads=2, dim=64, seed=6)
    q = ref.rows_of(41, 4, 64, torch.bfloat16, c.gen).contiguous()
    _check(c, [40, 1], q, 0.125, width=131)
    _check(c, [40, 1], q, 0.125, width=777)
    for hint in (0, 5, 1 << 22):
        _check(c, [40, 1], q, 0.125, max_kv=hint)


def test_rows_without_a_sum_add_nothing():
    c = ref.Cache([100], heads=1, dim=64, seed=7)
    q = ref.rows_of(20, 2, 64, torch.bfloat16, c.gen).contiguous()

    def edit(lse):
        lse[3:9] = -math.inf
    _check(c, [20], q, 0.125, lse_edit=edit)


def test_sum_over_keys_is_the_number_of_rows():
    """Each row hands out a weight of one: with the lse of kv_paged_attention the weights add up to the rows."""
    c = ref.Cache([700, 90], heads=2, dim=128, seed=8).device()
    new = [300, 90]
    b = c.batch(new)
    q = ref.rows_of(390, 8, 128, torch.bfloat16, c.gen, 1.5).cuda()
    out, lse = torch.empty_like(q), torch.empty(390, 8, device="cuda")
    size = kv.kv_paged_attention_workspace(c.layout, b, 8)
    kv.kv_paged_attention(c.layout, c.d_pool[0], b, q, out, 0.1, lse=lse,
                          workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if size else None)
    w = torch.zeros(2, 2, 700, device="cuda")
    kv.kv_attention_weights(c.layout, c.d_pool[0], b, q, lse, w, 0.1)
    again = torch.zeros_like(w)
    kv.kv_attention_weights(c.layout, c.d_pool[0], b, q, lse, again, 0.1)
    assert torch.equal(w, again)
    total = w.double().sum(-1).cpu()
    # 4 heads of a group hand out n each; every weight is good to about 2^-17 (scores of 128 terms)
    assert bool(((total - torch.tensor([[1200.0] * 2, [360.0] * 2])).abs() <= 1200 * 2.0 ** -15).all())
