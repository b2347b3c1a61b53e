"""Plain 64-bit forms of the operators of a serving step (norms of heads, plans, trees, kept paths), for the tests."""
import math

import torch

from paged_ref import HALF_STEP, rotate

D = 128
U = 2.0 ** -24


def normed(x, w, eps):
    """(r w x, n = r x, r) in float64; w [128] or [heads, 128]."""
    x = x.double()
    r = 1.0 / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps)
    return x * r * w.double(), x * r, r


def spread(x, freq, amp, layout):
    """What bounds each element of the rotated x: amp (|x1| + |x2|) of its pair, |x| past the rotary dimensions."""
    t = x.double().abs()
    if freq is None:
        return t
    n = freq.numel()
    i = torch.arange(n, device=x.device) * (2 if layout else 1)
    j = i + (1 if layout else n)
    y = t.clone()
    y[..., i] = y[..., j] = abs(amp) * (t[..., i] + t[..., j])
    return y


def turned(x, pos, freq, amp, layout, inverse=False):
    return x.double() if freq is None else rotate(x, pos, freq, amp, layout, inverse)


def norm_rope(x, w, eps, pos, freq, amp=1.0, layout=0, inverse=False):
    """(y, its tolerance).  The mean of 128 squares is off by 22 roundings (16 terms in a lane, three exchanges, products,
    eps), r by half of that and its own ulp (2 halves), n w by two products: 16 in all; the rotation by eight more
    (paged_ref.rotate_tolerance).  Then the output is rounded."""
    nw = normed(x, w, eps)[0]
    y = turned(nw, pos, freq, amp, layout, inverse)
    return y, HALF_STEP * y.abs() + 24 * U * spread(nw, freq, amp, layout) * (1 + HALF_STEP)


def norm_rope_gradients(x, w, eps, dy, pos, freq, amp=1.0, layout=0, inverse=False):
    """((dx, tolerance), (dw, tolerance)) from the formula.

    With G the bound of an element of g = R^T dy (off by 8 roundings of it) and M = mean(|w| G |n|): h = g w is off by 9
    |w| G, n by 15 |n| (above), the mean of h n by (9 + 15 + 22) M, n times it by 62 |n| M, the difference by one more of
    each, its product with r (13) by 14 more: r (24 |w| G + 77 |n| M), and the output is rounded.  A term of dw is off by
    8 + 15 + 1; the sums of N terms add up to N more (but no more than 300: chains of at most 256, then 64 bits)."""
    _, n, r = normed(x, w, eps)
    w = w.double()
    g = turned(dy, pos, freq, amp, layout, not inverse)
    G = spread(dy, freq, amp, layout)
    h = g * w
    dx = r * (h - n * (h * n).mean(-1, keepdim=True))
    M = (w.abs() * G * n.abs()).mean(-1, keepdim=True)
    tx = HALF_STEP * dx.abs() + U * r * (24 * w.abs() * G + 77 * n.abs() * M) * (1 + HALF_STEP)
    over = (0, 1) if w.dim() == 1 else (0,)
    terms = min(300, x.shape[0] * (x.shape[1] if w.dim() == 1 else 1))
    dw = (g * n).sum(over)
    tw = U * dw.abs() + (26 + terms) * U * (G * n.abs()).sum(over)
    return (dx, tx), (dw, tw)


def frequencies(rot, base=5e5, dev="cuda"):
    i = torch.arange(rot // 2, dtype=torch.float64, device=dev)
    return base ** (-2.0 * i / rot)
