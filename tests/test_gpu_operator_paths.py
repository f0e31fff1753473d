"""The variants of the operators that only large batches take, against the definition in 64 bits: tiles of 256 rows,
several tokens a workgroup of the rotary append, weights of keys that no waves share; and pools of which no 32-bit
count of bytes reaches the end."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
from test_gpu_attention_weights import _check as check_weights
from test_gpu_paged_attention import _run as run_attention
from test_gpu_rope import _case as check_rope

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f8": F8}


# tiles of 256 rows are taken where there are 1,024 workgroups of them: many heads need the fewest rows for it
WIDE = dict(heads=128, lengths=[700, 40, 301, 500], new=[600, 1, 200, 240])


def _some_heads(c, heads):
    """The cache as far as some of its KV heads go."""
    one = ref.Cache.__new__(ref.Cache)
    one.__dict__.update(c.__dict__)
    one.heads = len(heads)

    def rows(r, plane, layer=0):
        x, there = c.rows(r, plane, layer)
        return x[:, heads], there
    one.rows = rows
    return one


def _check_wide(c, new, q, scale, **kw):
    assert sum(new) * 2 // 256 * c.heads >= 1024
    out, lse = run_attention(c, new, q, scale, **kw)
    heads = [0, c.heads - 3]
    of_q = [2 * h + x for h in heads for x in (0, 1)]
    want, tol, wl, lt = ref.attention(_some_heads(c, heads), new, q[:, of_q], scale, kw.get("causal", True), kw.get("window", 0))
    ref.assert_within(out[:, of_q], want, tol, "out")
    ref.assert_within(lse[:, of_q], wl, lt, "lse")
    return out


@pytest.mark.parametrize("dim", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_tiles_of_256_rows(dim, dtype):
    c = ref.Cache(WIDE["lengths"], heads=128, dim=dim, dtype=TYPES[dtype], seed=dim, layout="block_first" if dim == 80 else "kv_first")
    q = ref.rows_of(sum(WIDE["new"]), 256, dim, c.q_dtype, c.gen, 1.5, gap=2)
    _check_wide(c, WIDE["new"], q, dim ** -0.5)


@pytest.mark.parametrize("causal,window", [(True, 50), (False, 0), (False, 200)])
def test_tiles_of_256_rows_windows(causal, window):
    c = ref.Cache(WIDE["lengths"], heads=128, dim=64, seed=window, block=20)
    q = ref.rows_of(sum(WIDE["new"]), 256, 64, torch.bfloat16, c.gen)
    _check_wide(c, WIDE["new"], q, 0.125, causal=causal, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_tiles_of_256_rows_out_of_sight(dtype, bad):
    """Missing blocks, and values that are not finite where some rows do not see them."""
    c = ref.Cache(WIDE["lengths"], heads=128, dim=64, dtype=TYPES[dtype], seed=9)
    used = set(c.bt.ravel().tolist())
    for p in (0, 1):
        x = c.view(p)
        for b in range(c.num_blocks):
            if b not in used:
                x[b] = bad
        x[int(c.bt[2, 18]), 301 % 16:] = bad
    v = c.view(1)
    for t in (350, 698):                                   # seen by the rows from t on
        v[int(c.bt[0, t // 16]), t % 16, :, 5:9] = bad
    c.bt[0, 2] = -1
    c.bt[3, 5:9] = c.num_blocks
    c.bt[1, :] = -7
    q = ref.rows_of(sum(WIDE["new"]), 256, 64, TYPES[dtype], c.gen)
    out = _check_wide(c, WIDE["new"], q, 0.125)
    assert bool((out[600] == 0).all())


# two, three and four tokens a workgroup, the last one part-filled
@pytest.mark.parametrize("rows", [2049, 3333, 4099])
@pytest.mark.parametrize("rot,interleaved", [(64, False), (40, True), (36, False), (0, False)], ids=["half", "interleaved", "odd", "none"])
@pytest.mark.parametrize("kind", ["bf16", "in-place", "f8"])
def test_rotary_append_of_many_tokens(rows, rot, interleaved, kind):
    rng = np.random.default_rng(rows)
    new = rng.multinomial(rows, np.ones(60) / 60)
    new[7] += new[8]
    new[8] = 0
    lengths = new + rng.integers(0, 30, 60)
    check_rope(new.tolist(), lengths.tolist(), hq=3, heads=1, dim=64, rot=rot, interleaved=interleaved,
               in_place=kind == "in-place", cache=F8 if kind == "f8" else None, seed=rot, gap=1)


@pytest.mark.parametrize("dim", [64, 80, 96, 128, 136, 256])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_weights_of_keys_that_no_waves_share(dim, dtype):
    """A wave takes keys of its own where the host's hint promises enough of them."""
    if dtype == "f8" and dim % 16:
        pytest.skip("rows of an 8-bit cache are whole 16-byte units")
    c = ref.Cache([333, 75, 20], heads=2, dim=dim, dtype=TYPES[dtype], seed=dim)
    q = ref.rows_of(190, 8, dim, c.q_dtype, c.gen, 1.5).contiguous()
    _check = dict(max_kv=1 << 17)
    check_weights(c, [120, 70, 0], q, dim ** -0.5, **_check)
    check_weights(c, [120, 70, 0], q, dim ** -0.5, window=100, decay=0.5, **_check)


@pytest.mark.parametrize("dtype", ["bf16", "f8"])
def test_pools_past_32_bits(dtype):
    """The same blocks at the far end of a pool of 36 GiB: what an operator reads and writes there is what it reads and
    writes in a small one, bit for bit."""
    c = ref.Cache([333, 75, 20], heads=2, dim=128, dtype=TYPES[dtype], seed=4, layers=1).device()
    stride, far = 8 << 20, 4600
    seg = c.block * 2 * 128 * c.elem
    first = far - c.num_blocks                             # block b of the small pool is block first + b of the large
    layout = kv.make_layout(1, 2, 128, c.elem, c.block, c.block, far, 1, seg, stride)
    pool = torch.empty(far * stride, dtype=torch.uint8, device="cuda")
    ends = pool.view(far, stride)[first:, :2 * seg]
    small = torch.stack([c.d_pool[0].view(torch.uint8)[p * c.strides[0]:][:c.num_blocks * seg].view(-1, seg) for p in (0, 1)], 1)
    got = []
    for lo, p, bt in ((c.layout, c.d_pool[0], c.d_bt), (layout, pool, torch.where(c.d_bt >= 0, c.d_bt + first, -1))):
        if p is pool:
            ends.copy_(small.flatten(1))
        c.gen.manual_seed(1)
        for new in ([1, 1, 1], [100, 3, 20]):
            n = sum(new)
            off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)])).cuda()
            b = kv.make_batch(off, c.d_len, bt, n, max(new), 333)
            q, k, v = (ref.rows_of(n, h, 128, torch.bfloat16, c.gen).cuda() for h in (8, 2, 2))
            out, lse, w = torch.empty_like(q), torch.empty(n, 8, device="cuda"), torch.zeros(3, 2, 333, device="cuda")
            kw = dict(k_scale=c.d_scales[0], cache_dtype=TYPES[dtype])
            kv.kv_rope_append(lo, p, b, q, k, v, torch.from_numpy(kv.kv_rope_frequencies(128)[0]).cuda(),
                              v_scale=c.d_scales[1], **kw)
            size = kv.kv_paged_attention_workspace(lo, b, 8)
            kv.kv_paged_attention(lo, p, b, q, out, 0.1, lse=lse, v_scale=c.d_scales[1],
                                  workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if size else None, **kw)
            kv.kv_attention_weights(lo, p, b, q, lse, w, 0.1, **kw)
            got += [q, out, lse, w]
        keep = torch.empty(1, 3, 2, 40, dtype=torch.int32, device="cuda")
        left = torch.empty(3, dtype=torch.int32, device="cuda")
        kv.kv_evict_select(w[None], c.d_len, 40, 2, 8, keep, left)
        kv.kv_evict_compact(lo, [p], bt, keep, left, weights=w[None])
        got += [keep, left, w]
    torch.cuda.synchronize()
    half = len(got) // 2
    for x, (a, b) in enumerate(zip(got[:half], got[half:])):
        assert torch.equal(a, b), x
    small = torch.stack([c.d_pool[0].view(torch.uint8)[p * c.strides[0]:][:c.num_blocks * seg].view(-1, seg) for p in (0, 1)], 1)
    assert torch.equal(ends, small.flatten(1))
