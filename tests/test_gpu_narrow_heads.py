"""Attention over an 8-bit cache at head sizes between 64 and 96, in 96 columns and, where no request fills a tile and keys
are not cut into parts, in 128."""
import math

import pytest
import torch

import paged_ref as ref
import stream_ref
from test_gpu_paged_attention import _check, _run
from test_gpu_sink_attention import _run as run_sinks

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.mark.parametrize("hint", [1, None], ids=["whole", "parts"])
@pytest.mark.parametrize("dim", [80, 96])
@pytest.mark.parametrize("q_dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("new", [[20, 1, 30, 0], [31, 31, 5, 8], [32, 40, 1, 64]])
def test_chunks(new, q_dtype, dim, hint):
    c = ref.Cache([700, 31, 64, 200], heads=2, dim=dim, dtype=F8, q_dtype=q_dtype, seed=dim, pad=16)
    q = ref.rows_of(sum(new), 8, dim, q_dtype, c.gen, 1.5)
    for causal, window in ((True, 0), (False, 0), (True, 50)):
        _check(c, new, q, dim ** -0.5, causal=causal, window=window, max_kv=hint)
    out, lse = run_sinks(c, new, q, dim ** -0.5, 50, 5, max_kv=hint)
    want, tol, wl, lt = stream_ref.attention(c, new, q, dim ** -0.5, True, 50, 5)
    ref.assert_within(out, want, tol, "out")
    ref.assert_within(lse, wl, lt, "lse")


@pytest.mark.parametrize("hint", [1, None], ids=["whole", "parts"])
def test_values_out_of_sight(hint):
    c = ref.Cache([300, 40], heads=2, dim=80, dtype=F8, seed=2)
    x = c.view(1)
    x[int(c.bt[0, 290 // 16]), 290 % 16, :, 3:7] = math.nan          # seen by the last rows alone
    x[int(c.bt[1, 2]), 40 % 16:] = math.nan
    c.bt[0, 3] = -1
    q = ref.rows_of(27, 8, 80, torch.bfloat16, c.gen)
    out, _ = _run(c, [25, 2], q, 0.125, max_kv=hint)
    want, tol, _, _ = ref.attention(c, [25, 2], q, 0.125)
    ref.assert_within(out, want, tol, "out")
    assert bool(out[:15].isfinite().all()) and bool(out[15:25, :, 3:7].isnan().all())
