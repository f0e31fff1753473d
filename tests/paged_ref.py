"""Paged caches and plain references in 64 bits for the tests of the operators
over the cache.  The references are written from the definitions, request by
request, on the CPU."""
import math

import numpy as np
import torch

import paper_2609_35065_amd as kv

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # largest relative rounding error
F8_MAX = 448.0


class Cache:
    """A layer's pool (or several) with shuffled block tables on the host and on the GPU."""

    def __init__(self, lengths, heads=2, dim=64, dtype=torch.bfloat16, block=16, layout="kv_first", pad=0, layers=1,
                 seed=0, spare=3, table_pad=0, scaled=True, q_dtype=None):
        self.gen = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lengths = np.asarray(lengths, np.int64)
        self.heads, self.dim, self.dtype, self.block = heads, dim, dtype, block
        self.q_dtype = q_dtype or (torch.bfloat16 if dtype == torch.float8_e4m3fn else dtype)
        e = torch.empty(0, dtype=dtype).element_size()
        self.elem = e
        need = -(-self.lengths // block)
        nb = int(need.sum()) + spare
        seg = block * heads * dim * e
        row = seg + pad
        self.strides = (nb * row, row) if layout == "kv_first" else (row, 2 * row)
        self.num_blocks = nb
        self.layout = kv.make_layout(layers, heads, dim, e, block, block, nb, 1, *self.strides)
        # every byte of the pool holds a value, that of unused blocks and paddings included
        self.pool = [torch.randn(2 * nb * row // e, generator=self.gen).to(dtype) for _ in range(layers)]
        perm = rng.permutation(nb).astype(np.int32)
        self.bt = np.full((len(lengths), max(1, int(need.max()) if len(need) else 1) + table_pad), -1, np.int32)
        at = 0
        for r, n in enumerate(need):
            self.bt[r, :n] = perm[at:at + n]
            at += n
        self.scales = None
        if dtype == torch.float8_e4m3fn and scaled:
            self.scales = [torch.rand(heads, generator=self.gen) + 0.5 for _ in range(2)]

    def view(self, plane, layer=0):
        """[blocks, B, H, D] of a plane, of the host's pool."""
        e = self.elem
        shape = (self.num_blocks, self.block, self.heads, self.dim)
        strides = (self.strides[1] // e, self.heads * self.dim, self.dim, 1)
        return self.pool[layer].as_strided(shape, strides, plane * self.strides[0] // e)

    def rows(self, r, plane, layer=0, scaled=True):
        """(rows float64 [T, H, D], whether each is there [T]) of request r."""
        T = int(self.lengths[r])
        t = np.arange(T)
        b = t // self.block
        inside = b < self.bt.shape[1]
        blk = np.where(inside, self.bt[r, np.minimum(b, self.bt.shape[1] - 1)], -1)
        there = (blk >= 0) & (blk < self.num_blocks)
        x = self.view(plane, layer).view(torch.uint8) if self.elem == 1 else self.view(plane, layer)
        x = x[torch.from_numpy(np.where(there, blk, 0)).long(), torch.from_numpy(t % self.block)]
        x = (x.view(self.dtype) if self.elem == 1 else x).double()
        if scaled and self.scales is not None:
            x = x * self.scales[plane].double()[None, :, None]
        return x, torch.from_numpy(there)

    def device(self):
        self.d_pool = [t.cuda() for t in self.pool]
        self.d_bt = torch.from_numpy(self.bt).cuda()
        self.d_len = torch.from_numpy(self.lengths.astype(np.int32)).cuda()
        self.d_scales = [None, None] if self.scales is None else [s.cuda() for s in self.scales]
        return self

    def batch(self, new, max_q=None, max_kv=None):
        off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        self.d_off = torch.from_numpy(off).cuda()
        return kv.make_batch(self.d_off, self.d_len, self.d_bt, int(off[-1]),
                             int(max(new, default=0)) if max_q is None else max_q,
                             int(self.lengths.max(initial=0)) if max_kv is None else max_kv)


def rows_of(n, heads, dim, dtype, gen, spread=1.0, gap=0):
    """Rows [n, heads, dim] as a slice of wider rows (gap heads beside them)."""
    x = (spread * torch.randn(n, heads + gap, dim, generator=gen)).to(dtype)
    return x[:, :heads]


def sees(T, n, there, causal, window):
    """[n, T]: which key each of the last n tokens sees."""
    pos = torch.arange(T - n, T)[:, None]
    j = torch.arange(T)[None]
    see = there[None].expand(n, T).clone()
    if causal:
        see &= j <= pos
    if window:
        see &= j > pos - window
    return see


def attention(cache, new, q, scale, causal=True, window=0, layer=0):
    """out, lse, and a bound on the error of each that follows from the roundings of the method: the result's to its
    type and the weights' to the values' type (one unit each), 32-bit scores (a dot product of D terms), exponentials
    and sums."""
    hq = q.shape[1]
    g = hq // cache.heads
    u = UNIT[cache.q_dtype]
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    ltol = torch.zeros(q.shape[:2], dtype=torch.float64)
    a = 0
    for r, n in enumerate(new):
        n = int(n)
        T = int(cache.lengths[r])
        k, there = cache.rows(r, 0, layer)
        v, _ = cache.rows(r, 1, layer)
        see = sees(T, n, there, causal, window)
        for h in range(hq):
            x = q[a:a + n, h].double()
            s = x @ k[:, h // g].t() * scale
            slack = (x.abs() @ k[:, h // g].abs().t() * scale).where(see, torch.tensor(0.0, dtype=torch.float64))
            es = (slack.amax(-1) if T else torch.zeros(n).double()) * cache.dim * 2.0 ** -24 + 1e-6
            s = s.where(see, torch.tensor(-math.inf, dtype=torch.float64))
            some = see.any(-1)
            L = torch.logsumexp(s, -1) if T else torch.full((n,), -math.inf).double()
            p = torch.exp(s - L.where(some, torch.tensor(0.0, dtype=torch.float64))[:, None])
            p = p.where(see, torch.tensor(0.0, dtype=torch.float64))
            vh = v[:, h // g]
            # keys that a row does not see reach it in no way, not even as 0 times infinity
            o = torch.stack([(p[i, see[i]][:, None] * vh[see[i]]).sum(0) for i in range(n)]) if n else p @ vh
            mass = p @ vh.abs().nan_to_num(posinf=0.0, neginf=0.0)
            small = see.double() @ vh.abs().nan_to_num(posinf=0.0, neginf=0.0) * 2.0 ** -24
            out[a:a + n, h] = o
            tol[a:a + n, h] = u * o.abs() + (u + 2 * es[:, None] + 1e-5) * mass * 1.02 + small
            lse[a:a + n, h] = L
            ltol[a:a + n, h] = es + 2.0 ** -21 * (L.abs().nan_to_num(posinf=0.0) + 1)
        a += n
    return out, tol, lse, ltol


def weights(cache, new, q, lse, scale, old, decay, causal=True, window=0):
    """Accumulated weights [R, H, W], and a bound on their error (32-bit scores, exponentials and sums)."""
    g = q.shape[1] // cache.heads
    out = old.double().clone()
    tol = torch.zeros(out.shape, dtype=torch.float64)
    a = 0
    for r, n in enumerate(new):
        n, T = int(n), min(int(cache.lengths[r]), out.shape[2])
        k, there = cache.rows(r, 0)
        see = sees(int(cache.lengths[r]), n, there, causal, window)[:, :T]
        for h in range(cache.heads):
            got, err = torch.zeros(T).double(), torch.zeros(T).double()
            for head in range(h * g, (h + 1) * g):
                x, L = q[a:a + n, head].double(), lse[a:a + n, head].double()
                s = x @ k[:T, h].t() * scale
                es = x.abs() @ k[:T, h].abs().t() * scale * cache.dim * 2.0 ** -24 + (s.abs() + L.abs()[:, None]) * 2.0 ** -21
                p = torch.exp(s - L[:, None]).where(see & (L != -math.inf)[:, None], torch.tensor(0.0, dtype=torch.float64))
                got += p.sum(0)
                err += (p * (es.nan_to_num(posinf=0.0) + 2.0 ** -20)).sum(0)
            out[r, h, :T] = (decay * out[r, h, :T] if decay else 0.0) + got
            tol[r, h, :T] = err + 2.0 ** -21 * out[r, h, :T].abs() + 1e-12
        a += n
    return out, tol


def assert_within(got, want, tol, what):
    got = got.double().cpu()
    want_nan = want.isnan()
    assert torch.equal(got.isnan(), want_nan), f"{what}: NaN in other places"
    inf = want.isinf()
    assert torch.equal(got.isinf(), inf) and torch.equal(got[inf], want[inf]), f"{what}: infinities in other places"
    fine = ~(want_nan | inf)
    off = (got - want).abs()[fine]
    over = off > tol[fine]
    assert not over.any(), f"{what}: {int(over.sum())} of {over.numel()} off by up to {off[over].max():.3g}, bound " \
                           f"{tol[fine][over][off[over].argmax()]:.3g}"
