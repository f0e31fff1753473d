"""kv_rope_shift against the definition in 64 bits: shifts shared by layers or heads or not, whole and partial rows of
every alignment, the 8-bit cache, missing blocks, and everything else as it was, bit by bit."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2609_35065_amd as kv
import stream_ref

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f8": F8}


def _case(lengths, heads=2, dim=64, dtype="bf16", rot=None, interleaved=False, inverse=False, layers=2, per_layer=True, per_head=True,
          top=5000, zeros=0.3, width=None, block=16, layout="kv_first", pad=0, seed=0, edit=None, max_len=None, spread=1.0, base=10000.0):
    rot = dim if rot is None else rot
    c = ref.Cache(lengths, heads=heads, dim=dim, dtype=DTYPES[dtype], block=block, layout=layout, pad=pad, layers=layers, seed=seed,
                  scaled=False)
    if spread != 1.0:
        c.pool = [(x.float() * spread).clamp(-448, 448).to(x.dtype) for x in c.pool]
    if edit:
        edit(c)
    freqs = kv.kv_rope_frequencies(rot, base)[0]
    T = int(max(lengths)) if width is None else width
    rng = np.random.default_rng(seed)
    shift = rng.integers(-top, top + 1, (layers if per_layer else 1, len(lengths), heads if per_head else 1, T))
    shift[rng.random(shift.shape) < zeros] = 0
    shift = shift.clip(-1 << 31, (1 << 31) - 1).astype(np.int32)
    c.device()
    kv.kv_rope_shift(c.layout, c.d_pool, c.d_bt, c.d_len, int(max(lengths)) if max_len is None else max_len,
                     torch.from_numpy(shift).cuda(), torch.from_numpy(freqs).cuda(), interleaved=interleaved, inverse=inverse)
    torch.cuda.synchronize()
    u = ref.UNIT[c.q_dtype]
    for l in range(layers):
        was = c.pool[l].clone()
        c.pool[l] = c.d_pool[l].cpu()
        old = ref.Cache.__new__(ref.Cache)
        old.__dict__.update(c.__dict__)
        old.pool = list(c.pool)
        old.pool[l] = was
        got, before = (y.view(0, l).view(torch.uint8) if c.elem == 1 else y.view(0, l) for y in (c, old))
        for r, n in enumerate(lengths):
            m = min(int(n), T)
            s = shift[l % shift.shape[0], r][:, :m].T                  # [m, heads or 1]
            x, there = old.rows(r, 0, l)
            y, _ = c.rows(r, 0, l)
            x, y = x[:m], y[:m]
            want, err = stream_ref.turn(x, s[..., None], freqs, interleaved, 1.0, inverse)
            if dtype == "f8":
                tol = want.clamp(-448, 448).abs() * 2.0 ** -4 + 2.0 ** -10 + err
                want = want.clamp(-448, 448)
            else:
                tol = u * want.abs() * 1.001 + err + 2.0 ** -24
            still = torch.from_numpy(np.broadcast_to(s == 0, (m, heads)).copy()) | ~there[:m, None]
            want = torch.where(still[..., None], x, want)
            tol = tol.masked_fill(still[..., None], 0.0)
            tol[..., rot:] = 0.0
            ref.assert_within(y[there[:m]], want[there[:m]], tol[there[:m]], f"layer {l} request {r}")
            for t in range(m):                                         # what turned is put back: all else has to be equal
                b = int(c.bt[r, t // block]) if t // block < c.bt.shape[1] else -1
                if 0 <= b < c.num_blocks:
                    on = ~still[t]
                    width_ = rot
                    got[b, t % block][on, :width_] = before[b, t % block][on, :width_]
        assert torch.equal(c.pool[l].view(torch.uint8), was.view(torch.uint8)), "other bytes changed"


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(64, 64), (64, 0), (64, 2), (64, 6), (64, 14), (64, 16), (64, 18), (80, 40), (96, 96), (128, 128),
                                     (128, 126), (16, 16), (48, 34), (256, 250), (256, 256)])
def test_head_and_rotated_sizes(dim, rot, interleaved, dtype):
    _case([70, 5, 130], dim=dim, rot=rot, interleaved=interleaved, dtype=dtype, seed=dim + rot)


def test_rows_of_one_unit():
    for inter in (False, True):
        _case([70, 5], dim=8, rot=8, interleaved=inter)
        _case([70, 5], dim=24, rot=22, interleaved=inter)


@pytest.mark.parametrize("per_layer", [False, True])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("heads", [1, 3, 8, 16, 17, 40])
def test_shared_shifts_and_heads(heads, per_head, per_layer):
    _case([100, 33], heads=heads, per_head=per_head, per_layer=per_layer, layers=3, seed=heads)


@pytest.mark.parametrize("block", [1, 3, 16, 20, 128])
@pytest.mark.parametrize("layout,pad", [("kv_first", 0), ("block_first", 0), ("kv_first", 48), ("block_first", 16)])
def test_blocks_and_layouts(block, layout, pad):
    _case([133, 28, 1], block=block, layout=layout, pad=pad, seed=block)


@pytest.mark.parametrize("kw", [dict(zeros=1.0), dict(zeros=0.0), dict(inverse=True), dict(width=40), dict(width=200), dict(max_len=0),
                                dict(max_len=1 << 30), dict(top=1 << 31), dict(top=1, zeros=0.0), dict(base=1e6)], ids=str)
@pytest.mark.parametrize("per_head", [False, True])
def test_forms(kw, per_head):
    _case([150, 64, 65, 1, 0], dtype="f16", seed=4, per_head=per_head, **kw)


def test_eight_bit_values_at_the_end_of_the_type():
    for inter in (False, True):
        _case([150, 64], dtype="f8", dim=80, rot=40, interleaved=inter, spread=300.0, seed=5)


def test_missing_blocks_and_values_that_are_not_finite():
    def edit(c):
        x = c.view(0)
        x[int(c.bt[2, 0]), 3, 1, 5] = math.inf
        x[int(c.bt[2, 0]), 4, 0, 37] = math.nan
        c.bt[0, 2] = -1
        c.bt[0, 5:7] = c.num_blocks
        c.bt[0, 8] = 2 ** 31 - 1
        c.bt[1, :] = -7
        c.bt = np.ascontiguousarray(c.bt[:, :9])
    for per_head in (False, True):
        # an infinity times a sine of 0 is NaN in the formula too: rows are shifted by odd numbers, whose sines are not 0
        _case([180, 30, 60], edit=edit, seed=7, per_head=per_head, zeros=0.0, top=1, layers=1)


def test_back_again():
    """A shift undone leaves keys within two roundings, and shifts add."""
    c = ref.Cache([300], heads=4, dim=128, seed=1, layers=1).device()
    freqs = torch.from_numpy(kv.kv_rope_frequencies(128)[0]).cuda()
    shift = torch.randint(1, 1000, (1, 1, 1, 300), generator=torch.Generator().manual_seed(1)).int().cuda()
    x = c.rows(0, 0)[0]
    for inverse in (False, True):
        kv.kv_rope_shift(c.layout, c.d_pool, c.d_bt, c.d_len, 300, shift, freqs, inverse=inverse)
    torch.cuda.synchronize()
    c.pool[0] = c.d_pool[0].cpu()
    size = (x[..., :64].abs() + x[..., 64:].abs()).repeat(1, 1, 2)
    # a rounding of each element of the turned pair reaches both of the pair that is turned back, and that is rounded again
    assert bool(((c.rows(0, 0)[0] - x).abs() <= size * (2 * 2.0 ** -8 + 2.0 ** -8 + 2.0 ** -18)).all())


def test_bytes_need_a_type():
    c = ref.Cache([30], heads=2, dim=64, layers=1).device()
    raw = [t.view(torch.uint8) for t in c.d_pool]
    freqs, shift = torch.zeros(32, dtype=torch.float64, device="cuda"), torch.ones(1, 1, 1, 30, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="cache_dtype"):
        kv.kv_rope_shift(c.layout, raw, c.d_bt, c.d_len, 30, shift, freqs)
    kv.kv_rope_shift(c.layout, raw, c.d_bt, c.d_len, 30, shift, freqs, cache_dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="read as"):
        kv.kv_rope_shift(c.layout, c.d_pool, c.d_bt, c.d_len, 30, shift, freqs, cache_dtype=torch.float16)
    torch.cuda.synchronize()
    assert torch.equal(c.d_pool[0].cpu(), c.pool[0])           # turned by nothing


def test_pools_past_32_bits_and_graph_replays():
    c = ref.Cache([75, 20], heads=2, dim=128, seed=4, layers=1).device()
    stride, far = 8 << 20, 4600
    seg = c.block * 2 * 128 * 2
    first = far - c.num_blocks
    layout = kv.make_layout(1, 2, 128, 2, c.block, c.block, far, 1, seg, stride)
    pool = torch.empty(far * stride, dtype=torch.uint8, device="cuda")
    ends = pool.view(far, stride)[first:, :2 * seg]
    small = c.d_pool[0].view(torch.uint8)
    planes = [small[p * c.strides[0]:][:c.num_blocks * seg].view(-1, seg) for p in (0, 1)]
    ends.copy_(torch.stack(planes, 1).flatten(1))
    bt = torch.where(c.d_bt >= 0, c.d_bt + first, -1).int()
    freqs = torch.from_numpy(kv.kv_rope_frequencies(128)[0]).cuda()
    shift = torch.zeros(1, 2, 2, 75, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kv.kv_rope_shift(layout, [pool], bt, c.d_len, 75, shift, freqs, cache_dtype=torch.bfloat16)
    for x in range(3):
        shift.random_(-99, 99, generator=torch.Generator("cuda").manual_seed(x))
        kv.kv_rope_shift(c.layout, c.d_pool, c.d_bt, c.d_len, 75, shift, freqs)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(ends, torch.stack(planes, 1).flatten(1)), x
