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
