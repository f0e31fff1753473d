"""Rotary appends whose rows pass the caches by: 256 MiB and more of whole cache lines."""
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
from test_gpu_rope_axes import _case

pytestmark = pytest.mark.gpu
STREAMED = 1 << 28


@pytest.mark.parametrize("kw", [dict(), dict(in_place=True, dtype=torch.float16), dict(inverse=True, gap=0, magnitude=1.3)], ids=str)
def test_several_axes(kw):
    new = [1000, 1, 0, 1050]
    assert sum(new) * 4 * 128 * (248 + 2 * 4) >= STREAMED
    _case(new, [1003, 30, 5, 1050], [16, 24, 24], hq=248, heads=4, dim=128, seed=9, **kw)


@pytest.mark.parametrize("dim,heads", [(128, 248), (256, 124)])
def test_one_axis_on_parts_and_on_the_whole(dim, heads):
    """On the whole batch, which is streamed, the results of calls on its parts, which are not."""
    c = ref.Cache([1100, 1000], heads=4, dim=dim, seed=2).device()
    n = 2060
    assert n * 4 * dim * (heads + 8) >= STREAMED > 1090 * 4 * dim * (heads + 8)
    q, k, v = (torch.randn(n, h, dim, device="cuda").bfloat16() for h in (heads, 4, 4))
    freqs = torch.from_numpy(kv.kv_rope_frequencies(dim)[0]).cuda()
    whole, start = torch.empty_like(q), c.d_pool[0].clone()
    kv.kv_rope_append(c.layout, c.d_pool[0], c.batch([1090, 970]), q, k, v, freqs, q_out=whole)
    want = c.d_pool[0].clone()
    c.d_pool[0].copy_(start)
    parts = torch.empty_like(q)
    at = 0
    for r, m in enumerate([1090, 970]):
        b = kv.make_batch(torch.tensor([0, m], device="cuda"), c.d_len[r:r + 1].clone(), c.d_bt[r:r + 1].contiguous(), m, m, 1100)
        kv.kv_rope_append(c.layout, c.d_pool[0], b, q[at:at + m], k[at:at + m], v[at:at + m], freqs, q_out=parts[at:at + m])
        at += m
    torch.cuda.synchronize()
    assert torch.equal(whole, parts) and torch.equal(c.d_pool[0], want)
