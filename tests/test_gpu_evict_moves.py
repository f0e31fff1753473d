"""Compaction: weights stay with their rows where a move is skipped, and the moves of many heads, whose workgroups take
whole rows."""
import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
from test_gpu_evict import _compact, _expected, _move, _same, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", [False, True])
def test_weights_stay_where_a_move_is_skipped(shared):
    c = ref.Cache([200, 64], heads=2, dim=64, layers=1, seed=3)
    c.bt[0, 0] = -1
    c.bt[0, 7] = c.num_blocks + 5
    c.bt = np.ascontiguousarray(c.bt[:, :12])          # index 192 on of the first request lies past the table
    G = 1 if shared else 2
    keep = np.full((1, 2, G, 60), -1, np.int32)
    keep[0, 0, :, :50] = np.arange(0, 200, 4)
    keep[0, 1, :, :30] = np.arange(34, 64)
    new = [60, 60]
    w = _weights("tail", (1, 2, G, 200), np.random.default_rng(1))
    want = _move(c, keep, new)
    dw = _compact(c, keep, new, w)
    _same(c, want)
    exp = w.copy()
    for r in range(2):
        for g in range(G):
            for i, s in enumerate(keep[0, r, g]):
                at = [c.bt[r, x // 16] if x // 16 < c.bt.shape[1] else -1 for x in (int(s), i)]
                if s > i and all(0 <= b < c.num_blocks for b in at):
                    exp[0, r, g, i] = w[0, r, g, s]
    assert np.array_equal(dw.cpu().numpy(), exp)


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.bfloat16, 256), (torch.float8_e4m3fn, 128)])
def test_moves_of_many_heads(dtype, dim):
    rng = np.random.default_rng(dim)
    lengths = [150, 130, 40, 127, 64, 91, 33, 1]
    c = ref.Cache(lengths, heads=8, dim=dim, dtype=dtype, layers=8, seed=dim)
    w = _weights("tail", (8, 8, 8, 150), rng)
    keep = _expected(w, lengths, 60, 2, 10)
    new = [min(n, 60) for n in lengths]
    want = _move(c, keep, new)
    dw = _compact(c, keep, new, w)
    _same(c, want)
    exp = w.copy()
    for l in range(8):
        for r in range(8):
            for g in range(8):
                exp[l, r, g, :new[r]] = w[l, r, g, keep[l, r, g, :new[r]]]
    assert np.array_equal(dw.cpu().numpy(), exp)
