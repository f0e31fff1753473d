"""Refusals of the operators over the paged cache, and rotary frequencies: no
call here reaches a kernel launch."""
import ctypes as ct
import math

import numpy as np
import pytest

import paper_2609_35065_amd as kv

A = 1 << 20   # a 16-byte aligned address; nothing reads it


def _layout(**over):
    d = dict(num_layers=1, kv_heads=2, head_dim=64, elem_bytes=2, block_size=16, chunk_tokens=16, num_blocks=20, num_slots=1,
             paged_kv_stride=20 * 4096, paged_block_stride=4096)
    d.update(over)
    if "paged_block_stride" not in over:
        seg = d["block_size"] * d["kv_heads"] * d["head_dim"] * d["elem_bytes"]
        d.update(paged_block_stride=seg, paged_kv_stride=seg * d["num_blocks"])
    return kv.make_layout(**d)


def _batch(**over):
    d = dict(num_reqs=1, bt_stride=4, num_q=1, max_q_len=1, max_kv_len=10, d_q_off=A, d_kv_len=A, d_block_tables=A)
    d.update(over)
    return kv.KvBatch(*[d[k] for k, _ in kv.KvBatch._fields_])


def _rows(heads=4, dtype=kv.KV_BF16, data=A, ts=None, hs=64):
    return kv.KvRows(data, heads * 64 if ts is None else ts, hs, heads, dtype)


def _p(x):
    return None if x is None else ct.addressof(x)


LAYOUTS = [(dict(num_layers=0), kv.KV_EINVAL), (dict(elem_bytes=4), kv.KV_EINVAL), (dict(elem_bytes=1), kv.KV_EINVAL),
           (dict(head_dim=264), kv.KV_ELIMIT), (dict(head_dim=68), kv.KV_EALIGN),
           (dict(num_blocks=1 << 24, paged_block_stride=8192, paged_kv_stride=4096), kv.KV_ELIMIT)]
BATCHES = [(dict(num_reqs=-1), kv.KV_EINVAL), (dict(bt_stride=0), kv.KV_EINVAL), (dict(num_q=-1), kv.KV_EINVAL),
           (dict(max_q_len=-1), kv.KV_EINVAL), (dict(max_kv_len=-5), kv.KV_EINVAL), (dict(d_q_off=0), kv.KV_EINVAL),
           (dict(d_kv_len=0), kv.KV_EINVAL), (dict(d_block_tables=0), kv.KV_EINVAL), (dict(num_reqs=0), kv.KV_EINVAL),
           (dict(d_q_off=A + 4), kv.KV_EALIGN), (dict(d_kv_len=A + 2), kv.KV_EALIGN), (dict(d_block_tables=A + 1), kv.KV_EALIGN)]
ROWS = [(dict(heads=0), kv.KV_EINVAL), (dict(dtype=2), kv.KV_EINVAL), (dict(data=0), kv.KV_EINVAL), (dict(ts=-256), kv.KV_EINVAL),
        (dict(hs=-8), kv.KV_EINVAL), (dict(data=A + 8), kv.KV_EALIGN), (dict(ts=257), kv.KV_EALIGN), (dict(hs=68), kv.KV_EALIGN)]


def _attention(lo=None, b=None, q=None, out=None, scale=0.1, window=0, cache=kv.KV_BF16, layer=A, lse=A, ws=None, size=0):
    lo, b, q, out = lo or _layout(), b or _batch(), q or _rows(), out or _rows()
    return kv.lib().kv_paged_attention(_p(lo), layer, _p(b), _p(q), _p(out), scale, 1, window, cache, None, None, lse, ws, size,
                                       None)


def _weights(lo=None, b=None, q=None, scale=0.1, window=0, cache=kv.KV_BF16, layer=A, lse=A, w=A, n=10, decay=1.0):
    lo, b, q = lo or _layout(), b or _batch(), q or _rows()
    return kv.lib().kv_attention_weights(_p(lo), layer, _p(b), _p(q), lse, scale, 1, window, cache, None, decay, w, n, None)


_SAME = object()


def _rope(lo=None, b=None, q=_SAME, out=_SAME, k=_SAME, v=_SAME, freqs=A, rot=64, flags=0, pos=None, cache=kv.KV_BF16, layer=A):
    lo, b = lo or _layout(), b or _batch()
    q, out = (_rows() if x is _SAME else x for x in (q, out))
    k, v = (_rows(2) if x is _SAME else x for x in (k, v))
    return kv.lib().kv_rope_append(_p(lo), layer, _p(b), _p(q), _p(out), _p(k), _p(v), freqs, rot, flags, 1.0, pos, cache, None,
                                   None, None)


@pytest.mark.parametrize("call", [_attention, _weights, _rope], ids=["attention", "weights", "rope"])
@pytest.mark.parametrize("over,code", LAYOUTS)
def test_layouts(call, over, code):
    assert call(lo=_layout(**over)) == code


@pytest.mark.parametrize("call", [_attention, _weights, _rope], ids=["attention", "weights", "rope"])
@pytest.mark.parametrize("over,code", BATCHES)
def test_batches(call, over, code):
    assert call(b=_batch(**over)) == code


@pytest.mark.parametrize("call", [_attention, _weights, _rope], ids=["attention", "weights", "rope"])
@pytest.mark.parametrize("over,code", ROWS)
def test_rows(call, over, code):
    assert call(q=_rows(**over)) == code


def test_attention_refuses():
    L = kv.lib()
    lo, b, q = _layout(), _batch(), _rows()
    assert L.kv_paged_attention(None, A, _p(b), _p(q), _p(q), 0.1, 1, 0, 0, None, None, None, None, 0, None) == kv.KV_EINVAL
    assert L.kv_paged_attention(_p(lo), A, None, _p(q), _p(q), 0.1, 1, 0, 0, None, None, None, None, 0, None) == kv.KV_EINVAL
    assert L.kv_paged_attention(_p(lo), A, _p(b), None, _p(q), 0.1, 1, 0, 0, None, None, None, None, 0, None) == kv.KV_EINVAL
    assert _attention(layer=None) == kv.KV_EINVAL and _attention(layer=A + 8) == kv.KV_EALIGN
    assert _attention(lse=A + 2) == kv.KV_EALIGN
    assert _attention(out=_rows(8)) == kv.KV_EINVAL                       # heads differ
    assert _attention(out=_rows(dtype=kv.KV_F16)) == kv.KV_EINVAL
    assert _attention(q=_rows(3), out=_rows(3)) == kv.KV_EINVAL           # not a multiple of the KV heads
    assert _attention(b=_batch(num_q=2), out=_rows(ts=0)) == kv.KV_EINVAL    # rows on one another
    assert _attention(out=_rows(hs=32)) == kv.KV_EINVAL
    assert _attention(cache=kv.KV_F16) == kv.KV_EINVAL and _attention(cache=7) == kv.KV_EINVAL
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert _attention(scale=scale) == kv.KV_EINVAL
    assert _attention(window=-1) == kv.KV_EINVAL
    long = _batch(max_kv_len=5000, bt_stride=400)
    need = kv.kv_paged_attention_workspace(_layout(), long, 4)
    assert need > 0
    assert _attention(b=long) == kv.KV_EINVAL                             # no workspace
    assert _attention(b=long, ws=A + 8, size=need) == kv.KV_EALIGN
    assert _attention(b=long, ws=A, size=need - 1) == kv.KV_ELIMIT
    none = _batch(num_q=0, num_reqs=0, d_q_off=0, d_kv_len=0, d_block_tables=0)
    assert _attention(b=none, q=_rows(data=0), out=_rows(data=0)) == kv.KV_OK


def test_weights_refuses():
    assert _weights(q=_rows(3)) == kv.KV_EINVAL and _weights(cache=kv.KV_F16) == kv.KV_EINVAL
    assert _weights(layer=None) == kv.KV_EINVAL and _weights(w=None) == kv.KV_EINVAL and _weights(lse=None) == kv.KV_EINVAL
    assert _weights(n=-1) == kv.KV_EINVAL and _weights(window=-1) == kv.KV_EINVAL
    assert _weights(scale=0.0) == kv.KV_EINVAL and _weights(decay=math.nan) == kv.KV_EINVAL
    assert _weights(layer=A + 8) == kv.KV_EALIGN and _weights(lse=A + 1) == kv.KV_EALIGN and _weights(w=A + 2) == kv.KV_EALIGN
    assert _weights(n=0, w=None) == kv.KV_OK
    none = _batch(num_q=0, num_reqs=0, d_q_off=0, d_kv_len=0, d_block_tables=0)
    assert _weights(b=none, q=_rows(data=0), lse=None, w=None) == kv.KV_OK


def test_rope_refuses():
    assert _rope(q=None, out=None, k=None, v=None) == kv.KV_EINVAL
    assert _rope(out=None) == kv.KV_EINVAL and _rope(q=None) == kv.KV_EINVAL
    assert _rope(v=None) == kv.KV_EINVAL and _rope(k=None) == kv.KV_EINVAL
    assert _rope(layer=None) == kv.KV_EINVAL and _rope(layer=A + 4) == kv.KV_EALIGN
    assert _rope(out=_rows(8)) == kv.KV_EINVAL and _rope(out=_rows(dtype=kv.KV_F16)) == kv.KV_EINVAL
    assert _rope(k=_rows(4)) == kv.KV_EINVAL and _rope(v=_rows(1)) == kv.KV_EINVAL
    assert _rope(k=_rows(2, dtype=kv.KV_F16)) == kv.KV_EINVAL
    assert _rope(cache=kv.KV_F16) == kv.KV_EINVAL
    for rot in (-2, 7, 66):
        assert _rope(rot=rot) == kv.KV_EINVAL
    assert _rope(freqs=None) == kv.KV_EINVAL and _rope(freqs=A + 4) == kv.KV_EALIGN
    assert _rope(flags=4) == kv.KV_EINVAL and _rope(pos=A + 2) == kv.KV_EALIGN
    none = _batch(num_q=0, num_reqs=0, d_q_off=0, d_kv_len=0, d_block_tables=0)
    assert _rope(b=none) == kv.KV_OK


def test_workspace_refuses():
    L = kv.host_lib()
    n = ct.c_int64(0)
    lo, b = _layout(), _batch()
    assert L.kv_paged_attention_workspace(ct.byref(lo), ct.byref(b), 4, 0, None) == kv.KV_EINVAL
    assert L.kv_paged_attention_workspace(None, ct.byref(b), 4, 0, ct.byref(n)) == kv.KV_EINVAL
    assert L.kv_paged_attention_workspace(ct.byref(lo), None, 4, 0, ct.byref(n)) == kv.KV_EINVAL
    for heads in (0, -2, 3):
        assert L.kv_paged_attention_workspace(ct.byref(lo), ct.byref(b), heads, 0, ct.byref(n)) == kv.KV_EINVAL
    assert L.kv_paged_attention_workspace(ct.byref(lo), ct.byref(b), 4, -1, ct.byref(n)) == kv.KV_EINVAL
    big = _batch(num_q=1 << 39, num_reqs=1)
    assert L.kv_paged_attention_workspace(ct.byref(lo), ct.byref(big), 4, 0, ct.byref(n)) == kv.KV_ELIMIT


def _select(w=A, n=10, lens=A, layers=1, reqs=1, heads=2, budget=4, sink=1, recent=1, keep=A, new=A):
    return kv.lib().kv_evict_select(w, n, lens, layers, reqs, heads, budget, sink, recent, keep, new, None)


def test_select_refuses():
    for bad in (dict(w=None), dict(lens=None), dict(keep=None), dict(new=None), dict(layers=0), dict(reqs=-1), dict(heads=0),
                dict(budget=0), dict(sink=-1), dict(recent=-1), dict(sink=3, recent=2), dict(n=-1), dict(n=1 << 31)):
        assert _select(**bad) == kv.KV_EINVAL, bad
    for bad in (dict(w=A + 2), dict(lens=A + 1), dict(keep=A + 2), dict(new=A + 3)):
        assert _select(**bad) == kv.KV_EALIGN, bad
    assert _select(layers=1 << 16, reqs=1 << 14) == kv.KV_ELIMIT
    assert _select(reqs=0, w=None, lens=None, keep=None, new=None) == kv.KV_OK


def test_select_refuses_rows_past_its_indices():
    assert _select(n=(1 << 30) + 1) == kv.KV_ELIMIT


def _compact(lo=None, layers=(A,), bt=A, stride=4, reqs=1, heads=2, keep=A, budget=4, new=A, w=None, n=0):
    lo = lo or _layout()
    arr = (ct.c_void_p * len(layers))(*layers) if layers is not None else None
    return kv.lib().kv_evict_compact(_p(lo), arr, bt, stride, reqs, heads, keep, budget, new, w, n, None)


def test_compact_refuses():
    for bad in (dict(layers=None), dict(layers=(None,)), dict(bt=None), dict(stride=0), dict(reqs=-1), dict(heads=3), dict(keep=None),
                dict(budget=0), dict(new=None), dict(w=A, n=-1), dict(lo=_layout(block_size=0))):
        assert _compact(**bad) == kv.KV_EINVAL, bad
    for bad in (dict(layers=(A + 8,)), dict(bt=A + 2), dict(keep=A + 1), dict(new=A + 2), dict(w=A + 2, n=4),
                dict(lo=_layout(head_dim=4, kv_heads=2))):
        assert _compact(**bad) == kv.KV_EALIGN, bad
    assert _compact(lo=_layout(num_blocks=1 << 24, paged_block_stride=8192, paged_kv_stride=4096)) == kv.KV_ELIMIT
    assert _compact(reqs=0, bt=None, keep=None, new=None) == kv.KV_OK


# ---------------------------------------------------------------------------
# frequencies
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("rot", [0, 2, 18, 64, 128])
def test_plain_and_linear_frequencies(rot):
    f, m = kv.kv_rope_frequencies(rot, 500000.0)
    want = [500000.0 ** (-2 * i / rot) for i in range(rot // 2)]
    assert m == 1.0 and f.size == rot // 2 and np.allclose(f, want, rtol=1e-14, atol=0)
    g, m = kv.kv_rope_frequencies(rot, 500000.0, kv.KV_ROPE_LINEAR, 4.0)
    assert m == 1.0 and np.array_equal(g, f / 4)


def test_base_scaling_stretches_the_slowest_pair_by_the_factor():
    f, _ = kv.kv_rope_frequencies(64)
    g, m = kv.kv_rope_frequencies(64, scaling=kv.KV_ROPE_BASE, factor=8.0)
    assert m == 1.0 and g[0] == f[0] == 1.0 and math.isclose(g[-1], f[-1] / 8, rel_tol=1e-12)
    assert (np.diff(f / g) > 0).all()


def test_ramp_keeps_fast_pairs_and_interpolates_slow_ones():
    f, _ = kv.kv_rope_frequencies(128)
    g, m = kv.kv_rope_frequencies(128, scaling=kv.KV_ROPE_RAMP, factor=16.0, context=4096.0, low=1.0, high=32.0)
    assert math.isclose(m, 0.1 * math.log(16.0) + 1, rel_tol=1e-6)
    turns = 4096 * f / (2 * math.pi)
    assert np.array_equal(g[turns >= 32], f[turns >= 32])
    assert np.allclose(g[turns <= 1], f[turns <= 1] / 16, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    y = (turns[mid] - 1) / 31
    assert mid.any() and np.allclose(g[mid], f[mid] * (y + (1 - y) / 16), rtol=1e-12)
    one, m1 = kv.kv_rope_frequencies(128, scaling=kv.KV_ROPE_RAMP, factor=1.0, context=4096.0)
    assert m1 == 1.0 and np.allclose(one, f, rtol=1e-15)


def test_frequencies_refuse():
    L = kv.host_lib()
    out, m = np.zeros(64), ct.c_float(0)

    def call(rot=64, base=1e4, scaling=0, factor=2.0, context=4096.0, low=1.0, high=32.0, h=out.ctypes.data, mag=ct.byref(m)):
        return L.kv_rope_frequencies(rot, base, scaling, factor, context, low, high, h, mag)

    assert call() == kv.KV_OK and call(rot=0, h=None) == kv.KV_OK
    for bad in (dict(rot=-2), dict(rot=3), dict(h=None), dict(mag=None), dict(base=1.0), dict(base=math.inf), dict(base=math.nan),
                dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.nan),
                dict(scaling=2, rot=2), dict(scaling=3, context=0.0), dict(scaling=3, low=5.0, high=5.0),
                dict(scaling=3, low=math.nan), dict(scaling=3, high=math.inf)):
        assert call(**bad) == kv.KV_EINVAL, bad
