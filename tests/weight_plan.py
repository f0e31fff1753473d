"""The launch plan of the accumulated weights, from the host's code built by itself: which variant a batch takes."""
import collections
import ctypes as ct
import functools
import os
import subprocess
import tempfile

import paper_2609_35065_amd as kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_35065_amd", "csrc")
Plan = collections.namedtuple("Plan", "windowed few ahead keys tiles sink_tiles parts workspace")


@functools.lru_cache(None)
def _build():
    with tempfile.TemporaryDirectory() as d:
        so = os.path.join(d, "weight_plan.so")
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", so,
                               os.path.join(ROOT, "tests", "native", "weight_plan.cpp"), os.path.join(CSRC, "host.cpp")])
        return ct.CDLL(so)


def weight_plan(lengths, new, heads, group, window=0, sink=-1, dim=64, max_q=None, max_kv=None):
    """The Plan of a batch whose requests hold ``lengths`` tokens, ``new`` of them new (sink -1: kv_attention_weights)."""
    seg = 16 * heads * dim * 2
    layout = kv.make_layout(1, heads, dim, 2, 16, 16, 64, 1, 64 * seg, seg)
    b = kv.KvBatch(len(lengths), 1, sum(new), max(new) if max_q is None else max_q, max(lengths) if max_kv is None else max_kv,
                   0, 0, 0)
    out = (ct.c_int64 * 8)()
    rc = _build().weight_plan(ct.byref(layout), ct.byref(b), heads * group, window, sink, out)
    assert rc == kv.KV_OK, rc
    return Plan(*out)
