"""A cache tensor whose element type is not the one it would be read as is refused; memory of no type of its own (the
bytes of the copies' pools) is taken as before."""
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def _calls(c, pool, cache_dtype=None):
    """The three operators over a pool, each as a call without arguments."""
    b = c.batch([1, 3])
    q, k, v = (ref.rows_of(4, h, 64, c.q_dtype, c.gen).cuda() for h in (4, 2, 2))
    out, lse, w = torch.empty_like(q), torch.zeros(4, 4, device="cuda"), torch.zeros(2, 2, 40, device="cuda")
    f = torch.zeros(0, dtype=torch.float64, device="cuda")
    kw = {"cache_dtype": cache_dtype}
    return [lambda: kv.kv_rope_append(c.layout, pool, b, q, k, v, f, **kw),
            lambda: kv.kv_paged_attention(c.layout, pool, b, q, out, 0.1, lse=lse, **kw) or (out, lse),
            lambda: kv.kv_attention_weights(c.layout, pool, b, q, lse, w, 0.1, **kw) or w]


@pytest.mark.parametrize("dtype,q,other", [
    (torch.float16, torch.bfloat16, torch.float16), (torch.bfloat16, torch.float16, torch.bfloat16),
    (F8, torch.bfloat16, torch.float8_e5m2), (F8, torch.float16, torch.float8_e4m3fnuz)])
def test_another_type_is_refused(dtype, q, other):
    c = ref.Cache([20, 40], heads=2, dim=64, dtype=dtype, q_dtype=q).device()
    pool = c.d_pool[0].view(torch.uint8).view(other)
    for call in _calls(c, pool):
        with pytest.raises(ValueError, match="cache"):
            call()


@pytest.mark.parametrize("given", [torch.bfloat16, torch.float16])
def test_a_given_type_must_be_the_tensors(given):
    have = torch.float16 if given == torch.bfloat16 else torch.bfloat16
    c = ref.Cache([20, 40], heads=2, dim=64, dtype=have, q_dtype=given).device()
    for call in _calls(c, c.d_pool[0], given):
        with pytest.raises(ValueError, match="cache"):
            call()


@pytest.mark.parametrize("dtype", [torch.bfloat16, F8])
def test_bytes_and_addresses_are_taken(dtype):
    c = ref.Cache([20, 40], heads=2, dim=64, dtype=dtype).device()
    pool = c.d_pool[0]
    c.gen.manual_seed(1)
    want = [x.clone() for x in _calls(c, pool)[1]()]
    for other in (pool.view(torch.uint8), pool.view(torch.uint8).view(torch.int16), pool.data_ptr()):
        c.gen.manual_seed(1)
        for a, b in zip(_calls(c, other)[1](), want):
            assert torch.equal(a, b)
    torch.cuda.synchronize()


def test_rotation_alone_reads_no_cache():
    c = ref.Cache([20, 40], heads=2, dim=64, dtype=torch.float16, q_dtype=torch.bfloat16).device()
    q = ref.rows_of(4, 4, 64, torch.bfloat16, c.gen).cuda()
    kv.kv_rope_append(c.layout, c.d_pool[0], c.batch([1, 3]), q, None, None,
                      torch.from_numpy(kv.kv_rope_frequencies(64)[0]).cuda())
    torch.cuda.synchronize()
