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


# ---- plans -------------------------------------------------------------------------------------

BAD_LAYOUT, BAD_PAGE = 16, 32


def plan(count, lens, table, page, ring, state, room, parent=None, words=0):
    """What ebd_plan_step makes of these (lists; the table a list of rows): a dict of lists, by the definition."""
    N, P = len(ring), len(table[0]) if table else 0
    lens, table, ring = list(lens), [list(r) for r in table], list(ring)
    head, free = state
    if not (0 <= head < N and 0 <= free <= N):
        head = free = 0
    known = lambda pg: 0 <= pg < N  # noqa: E731
    taken = back = 0
    off, slots, pos, masks, status = [0], [], [], [], [0] * len(count)
    for s, n in enumerate(count):
        first = max(lens[s], 0)
        if n < 0:
            for pg in table[s]:
                if known(pg):
                    if free + back < N:
                        ring[(head + free + back) % N] = pg
                    back += 1
            table[s] = [-1] * P
            lens[s] = 0
            off.append(off[-1])
            continue
        if n > 0 and first + n > 2 ** 30:
            n, status[s] = 0, BAD_LAYOUT
        if n > 0:
            for e in range(first // page, (first + n - 1) // page + 1):
                if e >= P:
                    status[s] |= BAD_PAGE
                    break
                if known(table[s][e]):
                    continue
                if taken < free:
                    table[s][e] = ring[(head + taken) % N]
                if not known(table[s][e]):
                    status[s] |= BAD_PAGE
                taken += 1
            lens[s] = first + n
        off.append(off[-1] + n)
        bits, depth = [], []
        for j in range(min(n, room - off[-2]) if n else 0):
            if j < 0:
                break
            row = first + j
            pg = table[s][row // page] if row // page < P else -1
            slots.append(pg * page + row % page if known(pg) else -1)
            if parent is None:
                pos.append(row)
                continue
            if j >= 64 * words:
                status[s] |= BAD_LAYOUT
                pos.append(-1)
                masks.append([0] * words)
                continue
            up = parent[off[-2] + j]
            if not -1 <= up < j:
                up = -1
                status[s] |= BAD_LAYOUT
            depth.append(0 if up < 0 else depth[up] + 1)
            bits.append((bits[up] if up >= 0 else 0) | 1 << j)
            pos.append(first + depth[j])
            masks.append([signed(bits[j] >> (64 * w) & (2 ** 64 - 1)) for w in range(words)])
        if n > 0 and off[-1] > room:
            status[s] |= BAD_LAYOUT
    pad = room - len(slots)
    got = min(taken, free)
    return {"len": lens, "table": table, "ring": ring, "state": [(head + got) % N, min(free - got + back, N)], "new_off": off,
            "slots": slots + [-1] * pad, "pos": pos + [-1] * pad, "mask": masks + [[0] * words for _ in range(pad)],
            "status": status}


def signed(word):
    return word - 2 ** 64 if word >> 63 else word


def tree(n, rng):
    """Parents of a tree of n drafted tokens."""
    return [rng.randrange(j + 1) - 1 for j in range(n)]


def chains(n, width):
    """... of `width` chains side by side."""
    return [j - width if j >= width else -1 for j in range(n)]


# ---- trees -------------------------------------------------------------------------------------

def masks_of(parents, words):
    """Mask words (signed) of a tree's tokens, and their depths."""
    bits, depth, out = [], [], []
    for j, up in enumerate(parents):
        bits.append((bits[up] if up >= 0 else 0) | 1 << j)
        depth.append(0 if up < 0 else depth[up] + 1)
        out.append([signed(bits[j] >> (64 * w) & (2 ** 64 - 1)) for w in range(words)])
    return out, depth


def sees(first, n, held, word_row, pos, window, limit=None):
    """Rows that a token sees by the definition: word_row its mask words, pos its position, n the rows of the sequence."""
    if pos < 0:
        return []
    lo = max(0, pos - window + 1) if window else 0
    rows = list(range(min(lo, max(first, 0)), max(first, 0)))
    for w, word in enumerate(word_row):
        rows += [first + 64 * w + i for i in range(64) if word >> i & 1]
    return [r for r in rows if 0 <= r < n and (limit is None or r < limit) and (held is None or held(r))]


def attend_row(cache, s, h, q, rows, scale=None, weights_bits=16):
    """(y, lse, tolerance of y, tolerance of lse) of query rows q [heads, 128] of KV head h of sequence s over these rows of
    it, in float64 (the tolerances of paged_ref.attend)."""
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    q = q.double()
    if not rows:
        z = torch.zeros(q.shape[0], dtype=torch.float64, device=q.device)
        return torch.zeros_like(q), z - math.inf, torch.zeros_like(q), z
    i = torch.tensor(rows, device=q.device)
    pg = cache.table[s][i // cache.page].long()
    k, v = (x[pg, h, i % cache.page].double() for x in (cache.K, cache.V))
    l = scale * q @ k.t()
    z = torch.logsumexp(l, 1)
    w = torch.exp(l - z[:, None])
    e = 2 * 128 * U * (scale * q.abs() @ k.abs().t()).amax(1) + 2.0 ** -22 + len(rows) * U
    y = w @ v
    ty = HALF_STEP * y.abs() + (1 + HALF_STEP) * ((2 * e + 2.0 ** -weights_bits)[:, None] * (w @ v.abs()))
    return y, z, ty, e + 2.0 ** -22 * (z.abs() + 1)
