"""Refusals of the operators for streams, the axes of pairs, and workspaces: no call here reaches a kernel launch."""
import ctypes as ct
import math

import numpy as np
import pytest
import torch

import paper_2609_35065_amd as kv
from paper_2609_35065_amd.serving import ServedCache
from test_paged_refusals import A, BATCHES, LAYOUTS, ROWS, _batch, _layout, _p, _rows

_SAME = object()


def _attention(lo=None, b=None, q=None, out=None, scale=0.1, window=20, sink=4, cache=kv.KV_BF16, layer=A, lse=A, ws=None, size=0):
    lo, b, q, out = lo or _layout(), b or _batch(), q or _rows(), out or _rows()
    return kv.lib().kv_sink_attention(_p(lo), layer, _p(b), _p(q), _p(out), scale, 1, window, sink, cache, None, None, lse, ws, size,
                                      None)


def _weights(lo=None, b=None, q=None, scale=0.1, window=20, sink=4, cache=kv.KV_BF16, layer=A, lse=A, w=A, n=10, decay=1.0, ws=None,
             size=0):
    lo, b, q = lo or _layout(), b or _batch(), q or _rows()
    return kv.lib().kv_sink_weights(_p(lo), layer, _p(b), _p(q), lse, scale, 1, window, sink, cache, None, decay, w, n, ws, size, None)


def _axes(lo=None, b=None, q=_SAME, out=_SAME, k=_SAME, v=_SAME, freqs=A, rot=64, flags=0, pos=A, apart=1, axes=3, axis=_SAME,
          cache=kv.KV_BF16, layer=A):
    lo, b = lo or _layout(), b or _batch()
    q, out = (_rows() if x is _SAME else x for x in (q, out))
    k, v = (_rows(2) if x is _SAME else x for x in (k, v))
    axis = np.zeros(32, np.uint8) if axis is _SAME else axis
    return kv.lib().kv_rope_append_axes(_p(lo), layer, _p(b), _p(q), _p(out), _p(k), _p(v), freqs, rot, flags, 1.0, pos, apart, axes,
                                        None if axis is None else axis.ctypes.data, cache, None, None, None)


def _shift(lo=None, layers=(A,), bt=A, stride=4, reqs=1, lens=A, max_len=10, nl=1, heads=2, shift=A, n=10, freqs=A, rot=64, flags=0,
           cache=kv.KV_BF16):
    lo = lo or _layout()
    arr = (ct.c_void_p * len(layers))(*layers) if layers is not None else None
    return kv.lib().kv_rope_shift(_p(lo), arr, bt, stride, reqs, lens, max_len, nl, heads, shift, n, freqs, rot, flags, cache, None)


ROW_CALLS = pytest.mark.parametrize("call", [_attention, _weights, _axes], ids=["attention", "weights", "axes"])


@pytest.mark.parametrize("call", [_attention, _weights, _axes, _shift], ids=["attention", "weights", "axes", "shift"])
@pytest.mark.parametrize("over,code", LAYOUTS)
def test_layouts(call, over, code):
    assert call(lo=_layout(**over)) == code


@ROW_CALLS
@pytest.mark.parametrize("over,code", BATCHES)
def test_batches(call, over, code):
    assert call(b=_batch(**over)) == code


@ROW_CALLS
@pytest.mark.parametrize("over,code", ROWS)
def test_rows(call, over, code):
    assert call(q=_rows(**over)) == code


def test_attention_refuses():
    assert _attention(layer=None) == kv.KV_EINVAL and _attention(layer=A + 8) == kv.KV_EALIGN
    assert _attention(window=-1) == kv.KV_EINVAL and _attention(sink=-1) == kv.KV_EINVAL
    assert _attention(lse=A + 2) == kv.KV_EALIGN and _attention(out=_rows(8)) == kv.KV_EINVAL
    assert _attention(q=_rows(3), out=_rows(3)) == kv.KV_EINVAL and _attention(cache=kv.KV_F16) == kv.KV_EINVAL
    assert _attention(b=_batch(num_q=2), out=_rows(ts=0)) == kv.KV_EINVAL
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert _attention(scale=scale) == kv.KV_EINVAL
    long = _batch(max_kv_len=5000, bt_stride=400)
    need = kv.kv_sink_attention_workspace(_layout(), long, 4, 3000, 4)
    assert 0 < need <= kv.kv_paged_attention_workspace(_layout(), long, 4)
    assert _attention(b=long, window=3000) == kv.KV_EINVAL                # no workspace
    assert _attention(b=long, window=3000, ws=A + 8, size=need) == kv.KV_EALIGN
    assert _attention(b=long, window=3000, ws=A, size=need - 1) == kv.KV_ELIMIT
    assert kv.kv_sink_attention_workspace(_layout(), long, 4, 100, 4) == 0  # no more keys than a step has
    none = _batch(num_q=0, num_reqs=0, d_q_off=0, d_kv_len=0, d_block_tables=0)
    assert _attention(b=none, q=_rows(data=0), out=_rows(data=0)) == kv.KV_OK


def test_weights_refuses():
    assert _weights(q=_rows(3)) == kv.KV_EINVAL and _weights(cache=kv.KV_F16) == kv.KV_EINVAL
    assert _weights(layer=None) == kv.KV_EINVAL and _weights(w=None) == kv.KV_EINVAL and _weights(lse=None) == kv.KV_EINVAL
    assert _weights(n=-1) == kv.KV_EINVAL and _weights(window=-1) == kv.KV_EINVAL and _weights(sink=-1) == kv.KV_EINVAL
    assert _weights(scale=0.0) == kv.KV_EINVAL and _weights(decay=math.nan) == kv.KV_EINVAL
    assert _weights(layer=A + 8) == kv.KV_EALIGN and _weights(lse=A + 1) == kv.KV_EALIGN and _weights(w=A + 2) == kv.KV_EALIGN
    assert _weights(ws=A + 8, size=64) == kv.KV_EALIGN
    chunk = _batch(max_q_len=5000, num_q=5000, max_kv_len=5000, bt_stride=400)
    need = kv.kv_sink_weights_workspace(_layout(), chunk, 4, 100, 4)
    assert need > 0 and need % (2 * 64 * 4) == 0
    assert _weights(b=chunk, window=100) == kv.KV_EINVAL
    assert _weights(b=chunk, window=100, ws=A, size=need - 1) == kv.KV_ELIMIT
    assert _weights(n=0, w=None) == kv.KV_OK
    none = _batch(num_q=0, num_reqs=0, d_q_off=0, d_kv_len=0, d_block_tables=0)
    assert _weights(b=none, q=_rows(data=0), lse=None, w=None) == kv.KV_OK


def test_workspaces_refuse_and_vanish():
    L = kv.host_lib()
    n = ct.c_int64(0)
    lo, b = _layout(), _batch()
    for call in (L.kv_sink_attention_workspace, L.kv_sink_weights_workspace):
        assert call(ct.byref(lo), ct.byref(b), 4, 20, 4, None) == kv.KV_EINVAL
        assert call(None, ct.byref(b), 4, 20, 4, ct.byref(n)) == kv.KV_EINVAL
        assert call(ct.byref(lo), None, 4, 20, 4, ct.byref(n)) == kv.KV_EINVAL
        for heads, window, sink in ((0, 20, 4), (-2, 20, 4), (3, 20, 4), (4, -1, 4), (4, 20, -1)):
            assert call(ct.byref(lo), ct.byref(b), heads, window, sink, ct.byref(n)) == kv.KV_EINVAL
        big = _batch(num_q=1 << 39, num_reqs=1)
        assert call(ct.byref(lo), ct.byref(big), 4, 20, 4, ct.byref(n)) == kv.KV_ELIMIT
        assert call(ct.byref(lo), ct.byref(b), 4, (1 << 31) - 1, (1 << 31) - 1, ct.byref(n)) == kv.KV_OK
    chunk = _batch(max_q_len=5000, num_q=5000, max_kv_len=5000, bt_stride=400)
    # nothing is cut: no sinks, no window, a window as long as the chunk, single tokens, more sinks than are cut
    for window, sink, batch in ((100, 0, chunk), (0, 4, chunk), (5000, 4, chunk), (100, 4, b), (100, 1025, chunk)):
        assert kv.kv_sink_weights_workspace(lo, batch, 4, window, sink) == 0


def test_axes_refuses():
    assert _axes(q=None, out=None, k=None, v=None) == kv.KV_EINVAL and _axes(out=None) == kv.KV_EINVAL
    assert _axes(v=None) == kv.KV_EINVAL and _axes(layer=None) == kv.KV_EINVAL and _axes(layer=A + 4) == kv.KV_EALIGN
    for rot in (-2, 7, 66):
        assert _axes(rot=rot) == kv.KV_EINVAL
    assert _axes(flags=4) == kv.KV_EINVAL and _axes(freqs=None) == kv.KV_EINVAL
    assert _axes(pos=A + 2) == kv.KV_EALIGN and _axes(pos=None) == kv.KV_EINVAL
    for axes in (0, -1, kv.KV_MAX_AXES + 1):
        assert _axes(axes=axes) == kv.KV_EINVAL
    assert _axes(axis=None) == kv.KV_EINVAL
    for bad in (3, 255):
        axis = np.zeros(32, np.uint8)
        axis[31] = bad
        assert _axes(axis=axis) == kv.KV_EINVAL
    assert _axes(b=_batch(num_q=5), apart=4, q=_rows(), out=_rows()) == kv.KV_EINVAL     # axes that lie on one another
    none = _batch(num_q=0, num_reqs=0, d_q_off=0, d_kv_len=0, d_block_tables=0)
    assert _axes(b=none, pos=None, apart=0) == kv.KV_OK


def test_shift_refuses():
    for bad in (dict(layers=None), dict(layers=(None,)), dict(bt=None), dict(stride=0), dict(reqs=-1), dict(lens=None), dict(max_len=-1),
                dict(nl=2), dict(nl=0), dict(heads=3), dict(shift=None), dict(n=-1), dict(freqs=None), dict(rot=66), dict(rot=3),
                dict(rot=-2), dict(flags=4), dict(cache=kv.KV_F8E4M3), dict(cache=5)):
        assert _shift(**bad) == kv.KV_EINVAL, bad
    for bad in (dict(layers=(A + 8,)), dict(bt=A + 2), dict(lens=A + 1), dict(shift=A + 2), dict(freqs=A + 4)):
        assert _shift(**bad) == kv.KV_EALIGN, bad
    assert _shift(reqs=1 << 30, lo=_layout(num_layers=2), layers=(A, A), nl=2) == kv.KV_ELIMIT
    assert _shift(reqs=0, bt=None, lens=None, shift=None) == kv.KV_OK
    assert _shift(n=0, shift=None) == kv.KV_OK and _shift(rot=0, freqs=None) == kv.KV_OK


@pytest.mark.parametrize("sections,in_turn,want", [
    ([2, 3, 1], False, [0, 0, 1, 1, 1, 2]), ([2, 3, 1], True, [0, 1, 2, 0, 1, 1]), ([0, 2], True, [1, 1]), ([0, 2], False, [1, 1]),
    ([4], True, [0] * 4), ([], False, None), ([0], False, []), ([1] * 8, True, list(range(8))), ([1] * 9, True, None),
    ([-1, 3], False, None), ([100, 29], False, None), ([64, 64], True, [0, 1] * 64)])
def test_axes_of_pairs(sections, in_turn, want):
    if want is None:
        with pytest.raises(kv.KvError):
            kv.kv_rope_axes(sections, in_turn)
    else:
        got = kv.kv_rope_axes(sections, in_turn)
        assert got.dtype == np.uint8 and got.tolist() == want
    s, out = np.ones(2, np.int32), np.zeros(4, np.uint8)
    L = kv.host_lib()
    assert L.kv_rope_axes(2, s.ctypes.data, 2, out.ctypes.data) == kv.KV_EINVAL
    assert L.kv_rope_axes(2, s.ctypes.data, 0, None) == kv.KV_EINVAL and L.kv_rope_axes(2, None, 0, out.ctypes.data) == kv.KV_EINVAL


def _host_cache(lengths, heads=2, **kw):
    layout = kv.make_layout(1, heads, 64, 2, 16, 16, 8, 1, 8 * 4096, 4096)
    return ServedCache(layout, [kw.pop("pool", torch.empty(8 * 4096))], torch.zeros(2, 8, dtype=torch.int32), lengths, 4,
                       torch.from_numpy(kv.kv_rope_frequencies(64)[0]), **kw)


def test_served_cache_refuses():
    with pytest.raises(ValueError, match="sink"):
        _host_cache([1, 1], sink=-1)
    axes = kv.kv_rope_axes([8, 12, 12])
    with pytest.raises(ValueError, match="axis"):
        _host_cache([1, 1], axes=axes, renumber=True)
    s = _host_cache([100, 3], window=8, sink=4)
    for sink, recent in ((3, 7), (0, 7), (4, 6)):
        with pytest.raises(ValueError, match="leave the"):
            s.evict(24, sink=sink, recent=recent)
    assert s.lengths.tolist() == [100, 3] and s.positions.tolist() == [100, 3]
    with pytest.raises(ValueError, match="first 4"):
        _host_cache([100, 3], window=8, sink=4, renumber=True).evict(24, sink=1)
    with pytest.raises(ValueError, match="type of the keys"):
        _host_cache([100, 3], renumber=True, pool=torch.empty(8 * 8192, dtype=torch.uint8)).evict(24)
    with pytest.raises(ValueError, match="axes"):
        _host_cache([100, 3]).begin([1, 1], positions=np.zeros((1, 2), np.int64))
    s = _host_cache([100, 3], axes=axes)
    for bad in (np.zeros((2, 2), int), np.zeros((3, 3), int), np.zeros((3, 2)), np.full((3, 2), 1 << 31), np.zeros(2, int)):
        with pytest.raises(ValueError, match="positions"):
            s.begin([1, 1], positions=bad)
    assert s.lengths.tolist() == [100, 3] and s.positions.tolist() == [100, 3]


@pytest.mark.parametrize("axes", [None, kv.kv_rope_axes([8, 12, 12])])
def test_served_cache_refuses_positions_beyond_31_bits(axes):
    s = _host_cache([100, 3], axes=axes)
    s.positions[1] = (1 << 31) - 1                     # the last one: it may still be taken, no request goes on after it
    with pytest.raises(ValueError, match="2\\^31"):
        s.begin([1, 2])
    assert s.lengths.tolist() == [100, 3] and s.positions.tolist() == [100, (1 << 31) - 1]


def test_workspaces_of_no_requests():
    none = _batch(num_q=0, num_reqs=0, d_q_off=0, d_kv_len=0, d_block_tables=0)
    for hint in (0, 5000):
        empty = _batch(num_q=0, num_reqs=0, max_q_len=hint, max_kv_len=hint, d_q_off=0, d_kv_len=0, d_block_tables=0)
        for b in (none, empty):
            assert kv.kv_sink_attention_workspace(_layout(), b, 4, 20, 4) == 0
            assert kv.kv_sink_weights_workspace(_layout(), b, 4, 20, 4) == 0
