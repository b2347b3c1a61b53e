"""Plain 64-bit forms of the paged-cache operators, and synthetic paged caches, for the tests."""
import math

import torch

D = 128
HALF_STEP = 2.0 ** -8  # of bf16, relative


def spaced(shape, gen, fused, dev="cuda", scale=1.0):
    """bf16 rows [tokens, heads, 128]: dense, or the middle heads of rows three times as wide."""
    t, h, d = shape
    x = scale * torch.randn((t, 3 * h if fused else h, d), generator=gen, device=dev)
    x = x.to(torch.bfloat16)
    return x[:, h:2 * h] if fused else x


def rotate(x, pos, freq, amp=1.0, layout=0, inverse=False):
    """[tokens, heads, 128] rotated, in float64."""
    x = x.double()
    n = freq.numel()
    a = pos.double()[:, None] * freq.double() * (-1.0 if inverse else 1.0)
    c, s = amp * torch.cos(a)[:, None], amp * torch.sin(a)[:, None]
    i = torch.arange(n, device=x.device) * (2 if layout else 1)
    j = i + (1 if layout else n)
    y = x.clone()
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def rotate_tolerance(x, ref, freq, amp=1.0, layout=0):
    """The output's rounding, and eight roundings of 2^-24 in products, sums, sines and the angle (its
    fp32 turns are off by 2^-25 of half a turn, 2^-24 pi < 4 x 2^-24 in radians)."""
    n = freq.numel()
    x = x.double().abs()
    i = torch.arange(n, device=x.device) * (2 if layout else 1)
    j = i + (1 if layout else n)
    t = torch.zeros_like(x)
    t[..., i] = t[..., j] = abs(amp) * (x[..., i] + x[..., j])
    return HALF_STEP * ref.abs() + 8 * 2.0 ** -24 * t * (1 + HALF_STEP)


class Cache:
    """A pool with a permuted page table; rows(s, h) gathers a sequence's rows."""

    def __init__(self, lens, kv, page, gen, order="heads", spare=3, dev="cuda", fill=None):
        used = [-(-max(n, 0) // page) for n in lens]
        total = sum(used) + spare
        perm = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
        self.page, self.kv, self.lens = page, kv, list(lens)
        self.table = torch.full((len(lens), max(max(used, default=0), 1) + 1), -1, dtype=torch.int32, device=dev)
        at = 0
        for s, n in enumerate(used):
            self.table[s, :n] = perm[at:at + n]
            at += n
        shape = (total, kv, page, D) if order == "heads" else (total, page, kv, D)
        make = lambda: torch.randn(shape, generator=gen, device=dev).to(torch.bfloat16)  # noqa: E731
        self.K, self.V = make(), make()
        if order != "heads":
            self.K, self.V = self.K.permute(0, 2, 1, 3), self.V.permute(0, 2, 1, 3)
        if fill is not None:  # everything that no sequence holds
            hold = torch.zeros(total, page, dtype=torch.bool, device=dev)
            for s, n in enumerate(self.lens):
                for r0 in range(0, n, page):
                    hold[int(self.table[s, r0 // page]), :min(page, n - r0)] = True
            for x in (self.K, self.V):
                x[(~hold)[:, None, :].expand(x.shape[:3])] = fill
        self.len = torch.tensor(self.lens, dtype=torch.int32, device=dev)

    def rows(self, pool, s, h):
        n = self.lens[s]
        p = self.table[s, :-(-n // self.page)].long()
        return pool[p, h].reshape(-1, D)[:n]


def attend(cache, q, news, hi=None, window=0, scale=None, weights_bits=16, seen=None):
    """(y, lse, tolerance of y, tolerance of lse) in float64; `seen(s)` masks rows with no page.

    Errors of the kernel's steps: a logit is a sum of 128 exact products in fp32 (any order): off by
    e = 128 2^-24 scale sum |q k|, doubled for the scale's and the subtraction's roundings; its weight is off by that
    and 2^-22 (exp2), a stored weight of `weights_bits` bits by 2^-weights_bits more; the sums of n weights
    add n 2^-24.  y is off by twice the weights' relative error (numerator and denominator) times
    sum w |v|, then rounded to bf16."""
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    T, Hq, _ = q.shape
    G = Hq // cache.kv
    y = torch.zeros((T, Hq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    ty, tl = torch.zeros_like(y), torch.zeros((T, Hq), dtype=torch.float64, device=q.device)
    t0 = 0
    for s, m in enumerate(news):
        n = cache.lens[s]
        for h in range(cache.kv if m and n > 0 else 0):
            k, v = cache.rows(cache.K, s, h).double(), cache.rows(cache.V, s, h).double()
            for j in range(m):
                t = t0 + j
                last = n - m + j if hi is None else min(int(hi[t]), n - 1)
                lo = max(0, last - window + 1) if window else 0
                i = torch.arange(lo, last + 1, device=q.device) if last >= lo else torch.zeros(0, dtype=torch.long, device=q.device)
                if seen is not None:
                    i = i[seen(s)[i]]
                if i.numel() == 0:
                    continue
                qs = q[t, h * G:(h + 1) * G].double()
                l = scale * qs @ k[i].t()
                z = torch.logsumexp(l, 1)
                w = torch.exp(l - z[:, None])
                e = 2 * 128 * 2.0 ** -24 * (scale * qs.abs() @ k[i].abs().t()).amax(1) + 2.0 ** -22 + i.numel() * 2.0 ** -24
                o = w @ v[i]
                y[t, h * G:(h + 1) * G], lse[t, h * G:(h + 1) * G] = o, z
                ty[t, h * G:(h + 1) * G] = HALF_STEP * o.abs() + (1 + HALF_STEP) * (
                    (2 * e + 2.0 ** -weights_bits)[:, None] * (w @ v[i].abs()))
                tl[t, h * G:(h + 1) * G] = e + 2.0 ** -22 * (z.abs() + 1)
        t0 += m
    return y, lse, ty, tl


def check(got, ref, tol, what=""):
    got, ref = got.double(), ref.double()
    same = (got == ref) | (got.isnan() & ref.isnan())
    off = torch.where(same, torch.zeros_like(ref), (got - ref).abs())
    bad = ~(off <= tol)
    assert not bool(bad.any()), "%s: %d off, worst %.3g against %.3g" % (
        what, int(bad.sum()), float((off - tol).nan_to_num(math.inf).max()), float(tol.max()))
