"""References in 64 bits for windows with sinks, and for turned rows: those of paged_ref with another rule of what a row
sees."""
import contextlib

import numpy as np
import torch

import paged_ref as ref


@contextlib.contextmanager
def _sinks(sink):
    """Let a row also see the first ``sink`` keys that are there, up to its own place if the rule is causal."""
    plain = ref.sees

    def sees(T, n, there, causal, window):
        return plain(T, n, there, causal, window) | (plain(T, n, there, causal, 0) & (torch.arange(T) < sink))
    ref.sees = sees
    try:
        yield
    finally:
        ref.sees = plain


def attention(cache, new, q, scale, causal=True, window=0, sink=0, layer=0):
    with _sinks(sink):
        return ref.attention(cache, new, q, scale, causal, window, layer)


def weights(cache, new, q, lse, scale, old, decay, causal=True, window=0, sink=0):
    """As ref.weights.  Its bound leaves a sum 2^-21; a lane adds 16 rows at a time, their sums, one for 32 rows, in turn,
    then at most 70 partial sums: an error of 2^-24 each."""
    with _sinks(sink):
        out, tol = ref.weights(cache, new, q, lse, scale, old, decay, causal, window)
    rows = max(new, default=0) * (q.shape[1] // cache.heads)
    return out, tol + (16 + rows / 32 + 70) * 2.0 ** -24 * out.abs()


def turn(x, pos, freqs, interleaved, magnitude=1.0, inverse=False):
    """(rows turned, bound on the error before rounding): ``pos`` has a position for each pair, [..., half], and each
    row of x."""
    x = x.double()
    half = freqs.size
    pos = torch.as_tensor(np.asarray(pos, np.float64))
    u = pos * torch.from_numpy(freqs) * (-1 if inverse else 1)
    first = torch.arange(half) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    out, err = x.clone(), torch.zeros_like(x)
    a, b = x[..., first], x[..., second]
    out[..., first] = (a * u.cos() - b * u.sin()) * magnitude
    out[..., second] = (a * u.sin() + b * u.cos()) * magnitude
    # an angle of 32 bits (2^-23.3 of a radian), sines of 2^-22.9, two products and a sum of 2^-24 each: below 2^-20; and
    # the rounding of the product in 64 bits, three of 2^-53 of the angle on either side
    err[..., first] = err[..., second] = (a.abs() + b.abs()) * magnitude * (2.0 ** -20 + u.abs() * 2.0 ** -50)
    return out, err
