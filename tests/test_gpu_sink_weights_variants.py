"""Variants of the accumulated weights that only some batches take, against the definition in 64 bits."""
import pytest
import torch

import paged_ref as ref
from test_gpu_sink_weights import _check

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
