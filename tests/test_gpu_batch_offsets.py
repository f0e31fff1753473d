"""A batch whose first offset is not 0: the rows before it belong to no request, and reach no request's cache."""
import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", [1, 5, 70])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn], ids=["bf16", "f8"])
def test_rows_before_the_first_request_are_not_appended(first, dtype):
    new, lengths = [3, 0, 20], [90, 40, 33]
    c = ref.Cache(lengths, heads=2, dim=64, dtype=dtype, seed=first).device()
    n = first + sum(new)
    q, k, v = (ref.rows_of(n, h, 64, torch.bfloat16, c.gen).cuda() for h in (4, 2, 2))
    off = torch.from_numpy(first + np.concatenate([[0], np.cumsum(new)]).astype(np.int64)).cuda()
    f = torch.from_numpy(kv.kv_rope_frequencies(64)[0]).cuda()
    kw = dict(k_scale=c.d_scales[0], v_scale=c.d_scales[1])

    want_pool, want = c.d_pool[0].clone(), torch.empty_like(q[first:])
    kv.kv_rope_append(c.layout, want_pool, c.batch(new), q[first:], k[first:], v[first:], f, q_out=want, **kw)
    out = torch.empty_like(q)
    b = kv.make_batch(off, c.d_len, c.d_bt, n, max(new), max(lengths))
    kv.kv_rope_append(c.layout, c.d_pool[0], b, q, k, v, f, q_out=out, **kw)
    torch.cuda.synchronize()
    assert torch.equal(c.d_pool[0].view(torch.uint8), want_pool.view(torch.uint8))
    assert torch.equal(out[first:], want)


@pytest.mark.parametrize("new,lengths,cut", [([3, 0, 20], [90, 40, 33], True), ([1, 1, 1], [90, 40, 33], False),
                                             ([1, 1, 1], [900, 400, 330], True), ([300, 1, 90], [400, 9, 90], True)])
def test_the_other_operators_leave_them_alone(new, lengths, cut):
    """With keys cut into parts, and without."""
    first = 5
    c = ref.Cache(lengths, heads=2, dim=64, seed=2).device()
    n = first + sum(new)
    q = ref.rows_of(n, 4, 64, torch.bfloat16, c.gen).cuda().contiguous()
    off = torch.from_numpy(first + np.concatenate([[0], np.cumsum(new)]).astype(np.int64)).cuda()
    got = []
    for rows, b in ((q[first:], c.batch(new)), (q, kv.make_batch(off, c.d_len, c.d_bt, n, max(new), max(lengths)))):
        out, lse = torch.full_like(rows, 7.0), torch.full((rows.shape[0], 4), 7.0, device="cuda")
        size = kv.kv_paged_attention_workspace(c.layout, b, 4)
        assert (size > 0) == cut
        kv.kv_paged_attention(c.layout, c.d_pool[0], b, rows, out, 0.125, lse=lse,
                              workspace=torch.zeros(size, dtype=torch.uint8, device="cuda") if size else None)
        w = torch.zeros(3, 2, max(lengths), device="cuda")
        kv.kv_attention_weights(c.layout, c.d_pool[0], b, rows, lse, w, 0.125)
        got.append((out, lse, w))
    torch.cuda.synchronize()
    assert bool((got[1][0][:first] == 7.0).all()) and bool((got[1][1][:first] == 7.0).all())
    for a, b in zip(got[0][:2], got[1][:2]):
        assert torch.equal(a, b[first:])
    assert torch.equal(got[0][2], got[1][2])
