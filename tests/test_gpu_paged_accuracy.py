"""How far the paged attention's outputs are off: by the bits that its weights hold, and by the norms of whole rows."""
import math

import pytest
import torch

import paged_ref as ref
from test_gpu_paged_edges import _attend, _gen, _picked

pytestmark = pytest.mark.gpu

# Query rows of a KV head (new tokens times query heads) up to which a weight holds 16 bits, a bf16 head and a bf16 tail
SIXTEEN_BITS_ROWS = 64


def _bits(rows):
    return 16 if rows <= SIXTEEN_BITS_ROWS else 8


def _sharp(c, q, m, G):
    """Keys that some query rows weigh far above the others: a query's own direction, at every 29th row."""
    for r in range(0, c.lens[0], 29):
        h = r // 29 % c.kv
        c.K[int(c.table[0, r // c.page]), h, r % c.page] = (q[r % m, h * G].float() * (1.0 + r % 3)).to(torch.bfloat16)


@pytest.mark.parametrize("m,G,n", [(1, 4, 33), (1, 1, 700), (1, 4, 4097), (4, 4, 300), (5, 4, 130), (8, 4, 2000), (9, 4, 90),
                                   (14, 4, 400), (8, 7, 5000), (16, 4, 1000), (64, 1, 700), (13, 5, 900), (40, 4, 500)])
@pytest.mark.parametrize("sharp", [False, True])
def test_weights_hold_their_bits(m, G, n, sharp):
    """Element by element: each weight rounded to 16 bits up to 64 query rows, to 8 beyond (see paged_ref.attend)."""
    print("weights", m, G, n, sharp, flush=True)
    c = ref.Cache([n], 2, 16, _gen(n + m))
    q = ref.spaced((m, 2 * G, 128), _gen(1), False)
    if sharp:
        _sharp(c, q, m, G)
    _, y, lse, _ = _attend(c, [m], G, q=q)
    ry, rl, ty, tl = ref.attend(c, q, [m], weights_bits=_bits(m * G))
    ref.check(y, ry, ty, "y")
    ref.check(lse, rl, tl, "lse")


def _norms(c, q, t, last, h, G):
    """Of one token and KV head: y [G, 128], and the norms that errors of the weights are measured by."""
    i = torch.arange(last + 1, device=q.device)
    k, v = (c.rows(x, 0, h)[i].double() for x in (c.K, c.V))
    qs = q[t, h * G:(h + 1) * G].double()
    l = qs @ k.t() / math.sqrt(128.0)
    w = torch.exp(l - torch.logsumexp(l, 1)[:, None])
    e = 2 * 128 * 2.0 ** -24 * (qs.abs() @ k.abs().t()).amax(1) / math.sqrt(128.0) + 2.0 ** -22 + i.numel() * 2.0 ** -24
    v2 = v.norm(dim=1)
    return w, v, w @ v, (w.square() @ v2.square()).sqrt(), 2 * e * (w @ v2)


@pytest.mark.parametrize("m,G,n,kv", [(1, 4, 300, 2), (7, 4, 400, 2), (14, 4, 400, 2), (70, 2, 350, 2), (40, 4, 400, 2),
                                      (500, 4, 9001, 8)])
def test_rows_by_their_norms(m, G, n, kv):
    """A row of y is off by its own rounding, 2^-8 |y|, and by the weights' roundings d_i: sum d_i w_i v_i.  The d_i come
    from the logits and have nothing to do with the values' directions, so that sum's square is sum d_i^2 w_i^2 |v_i|^2 but
    for its cross terms, each about 1 / sqrt(128) of its squares and of either sign.  With every |d_i| at its most, which is
    sqrt(3) times the mean of evenly spread ones, that is half a step times sqrt(sum w_i^2 |v_i|^2).

    The bound is narrow enough that one key of the mean weight 1 / n, left out of a few hundred, is seen: y moves by about
    sqrt(128) / n, and with logits from N(0, 1), whose weights have the mean square e / n^2, |y| and the root of the squares
    are about sqrt(128 e / n), the bound 2^-7 of that, smaller by 78 / sqrt(n)."""
    print("norms", m, G, n, kv, flush=True)
    c = ref.Cache([n], kv, 16, _gen(n + m))
    q, y, _, _ = _attend(c, [m], G)
    step = 2.0 ** -_bits(m * G)
    for t in _picked(m).tolist():
        last = n - m + t
        for h in range(kv):
            w, v, o, by, fp32 = _norms(c, q, t, last, h, G)
            bound = 2.0 ** -8 * o.norm(dim=1) + (1 + 2.0 ** -8) * (step * by + fp32)
            off = (y[t, h * G:(h + 1) * G].double() - o).norm(dim=1)
            assert bool((off <= bound).all()), (t, h, float((off / bound).max()))
            mean = torch.where(w >= 1.0 / (last + 1), w, 2.0).argmin(1)  # the formula without this key:
            wx = w.gather(1, mean[:, None])
            lacks = (o - wx * v[mean]) / (1 - wx)
            assert n > 1000 or bool(((lacks - o).norm(dim=1) > bound).all())


@pytest.mark.parametrize("m,G", [(5, 4), (8, 7)])
def test_many_short_chunks_over_more_rows_than_caches_hold(m, G):
    """17 to 64 query rows of each sequence, keys and values past 64 MB: the loads that leave no trace in the caches."""
    print("short chunks", m, G, flush=True)
    lens = [2500 - 97 * (i % 9) for i in range(16)]
    news = [m - (i % 3) for i in range(16)]
    c = ref.Cache(lens, 4, 16, _gen(m), fill=math.nan)
    q, y, lse, st = _attend(c, news, G)
    assert not bool(st.any())
    ry, rl, ty, tl = ref.attend(c, q, news, weights_bits=16)
    ref.check(y, ry, ty, "y")
    ref.check(lse, rl, tl, "lse")


@pytest.mark.parametrize("m,G,kv", [(1, 40, 2), (2, 130, 1), (3, 300, 1)])
def test_more_query_heads_than_a_block_has_rows(m, G, kv):
    print("wide groups", m, G, kv, flush=True)
    lens = [350, 41]
    c = ref.Cache(lens, kv, 32, _gen(G))
    q, y, lse, _ = _attend(c, [m, m], G)
    ry, rl, ty, tl = ref.attend(c, q, [m, m], weights_bits=_bits(m * G))
    ref.check(y, ry, ty, "y")
    ref.check(lse, rl, tl, "lse")
