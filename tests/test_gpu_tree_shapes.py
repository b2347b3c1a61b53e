"""Attention of drafted trees on the GPU by every shape of its kernels: values that are all alike, values and keys that are
not finite, rows without a page, bounds below the truth, tokens that see nothing."""
import math
import random

import pytest
import torch

import paged_ref as ref
import step_ref as step
import tree_shapes
from test_gpu_tree import _call

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _batch(name, **kw):
    """(cache, new tokens, heads of a KV head, mask words, positions, window) of a batch of trees."""
    news, held, kv, G, window, _, _ = tree_shapes.BATCHES[name]
    print("batch", name, flush=True)
    rng = random.Random(sum(news) + sum(held))
    c = ref.Cache([h + m for h, m in zip(held, news)], kv, 16, _gen(sum(held)), **kw)
    words = -(-max(news) // 64)
    mask, pos = [], []
    for h, m in zip(held, news):
        a, d = step.masks_of(step.tree(m, rng), words)
        mask += a
        pos += [h + x for x in d]
    return c, news, G, mask, pos, window


@pytest.mark.parametrize("name", tree_shapes.BATCHES)
def test_values_that_are_all_alike(name):
    """Weights sum to one in the products, too: where every value of a head is the same row u, y is u, to the bit.

    The quotient of the sums over rounded weights is off by fp32 roundings alone, fewer than 2^13 of them (a row of each
    key, one more a tile and a split), far from half a step of an output.  Logits of a standard deviation of 6 let few keys
    rule a row, whose one rounding would show in all of its elements."""
    c, news, G, mask, pos, window = _batch(name)
    g = _gen(5)
    # just below a power of two, where a step is smallest beside the value
    u = (torch.randint(0, 2, (c.kv, 128), generator=g, device="cuda") * 2 - 1) * (1.9921875 * 2.0 ** torch.randint(
        -3, 4, (c.kv, 128), generator=g, device="cuda"))
    c.V.copy_(u.to(BF)[None, :, None, :].expand(c.V.shape))
    c.K.mul_(6.0)
    _, y, _, st = _call(c, news, G, mask, pos, window=window)
    assert not bool(st.any())
    want = u.to(BF).repeat_interleave(G, 0)
    wrong = (y != want).any(-1)
    assert not bool(wrong.any()), "%d of %d rows, by up to %g" % (
        int(wrong.sum()), wrong.numel(), float(((y.double() - want.double()) / want.double()).abs().max()))


def _row(c, s, h, q, rows, eight):
    """step_ref.attend_row with the bound of weights that are divided by the sum of what they were rounded to: with weights
    w_i (1 + e_i), |e_i| <= 2^-8, over their sum, y' - y = sum w_i (1 + e_i) (v_i - y) / sum w_i (1 + e_i) =
    sum w_i e_i (v_i - y) / sum w_i (1 + e_i), since sum w_i (v_i - y) = 0: at most 2^-8 / (1 - 2^-8) of the weighted mean of
    |v - y|.  The other steps are as there (their sums' roundings, and the quotient's, are below 2^-16 of |v|)."""
    y, z, ty, tl = step.attend_row(c, s, h, q, rows, None, 16)
    if eight and rows:
        i = torch.tensor(rows, device=q.device)
        pg = c.table[s][i // c.page].long()
        k, v = (x[pg, h, i % c.page].double() for x in (c.K, c.V))
        w = torch.softmax(q.double() @ k.t() / math.sqrt(128), 1)
        away = torch.stack([w[a] @ (v - y[a]).abs() for a in range(q.shape[0])])
        ty = ty + (1 + ref.HALF_STEP) * 2.0 ** -8 / (1 - 2.0 ** -8) * away
    return y, z, ty, tl


def _check(c, name, mask, pos, q, y, lse, held=None, limit=None, max_new=None, few=10):
    """Some tokens and heads of each sequence against the formula; elements and rows that are not finite have to be the same."""
    news, _, kv, G, window, shape, _ = tree_shapes.BATCHES[name]
    t0 = 0
    for s, m in enumerate(news):
        first, shown = c.lens[s] - m, m if max_new is None else min(m, max_new)
        pick = sorted({0, 1, 31, 32, 63, 64, 65, shown - 2, shown - 1} | set(range(0, shown, max(1, shown // few))))
        for j in (j for j in pick if 0 <= j < shown):
            t = t0 + j
            rows = step.sees(first, c.lens[s], None if held is None else lambda r: held(s, r), mask[t], pos[t], window, limit)  # noqa: B023
            for h in sorted({0, kv // 2, kv - 1}):
                a = slice(h * G, h * G + G)
                ry, rl, ty, tl = _row(c, s, h, q[t, a], rows, shape[0] > 64)
                what = "sequence %d token %d head %d" % (s, j, h)
                odd = ~torch.isfinite(ry)
                assert torch.equal(y[t, a].double()[odd].nan_to_num(9.0), ry[odd].nan_to_num(9.0)), what
                ref.check(y[t, a][~odd], ry[~odd], ty[~odd], "y of " + what)
                if bool(rl.isnan().any()):
                    assert torch.equal(lse[t, a].isnan(), rl.isnan()), what
                else:
                    ref.check(lse[t, a], rl, tl, "lse of " + what)
        t0 += m


@pytest.mark.parametrize("name", tree_shapes.BATCHES)
def test_shapes(name):
    """With tokens that see nothing by their position, by their mask, and where nobody holds the rest of a page."""
    c, news, G, mask, pos, window = _batch(name, fill=math.nan)
    for s, m in enumerate(news):
        t0 = sum(news[:s])
        pos[t0 + m // 2] = -1
        mask[t0 + m - 1] = [0] * len(mask[0])
    q, y, lse, st = _call(c, news, G, mask, pos, window=window, pad=2)
    assert not bool(st.any())
    assert bool((y[sum(news):] == 7).all()) and bool((lse[sum(news):] == 7).all())
    _check(c, name, mask, pos, q, y, lse, few=20)
    _, y2, lse2, _ = _call(c, news, G, mask, pos, q=q, window=window, pad=2)
    assert torch.equal(y, y2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("name", tree_shapes.BATCHES)
def test_shapes_values_that_are_not_finite(name):
    c, news, G, mask, pos, window = _batch(name, fill=math.nan)
    for s, m in enumerate(news):
        first = c.lens[s] - m

        def put(pool, row, h, e, x, s=s):
            pool[int(c.table[s, row // 16]), h, row % 16, e] = x

        for h in (0, c.kv - 1):
            put(c.V, first + m - 1, h, 5, math.inf)
            put(c.V, first + 1, h, 5, -math.inf)
            put(c.V, first + m // 3, h, 77, math.nan)
        put(c.K, first + m // 2, 0, 9, math.nan)  # (in the first head alone)
        put(c.V, first // 2, c.kv - 1, 120, -math.inf)  # a held row, which all see without a window
        if window and first > 60:  # outside every window
            put(c.V, first - 50, slice(None), slice(None), math.nan)
            put(c.K, first - 50, slice(None), slice(None), math.inf)
    q, y, lse, st = _call(c, news, G, mask, pos, window=window)
    assert not bool(st.any())
    _check(c, name, mask, pos, q, y, lse, few=20)


@pytest.mark.parametrize("name", tree_shapes.BATCHES)
def test_shapes_rows_without_a_page(name):
    """Flagged only where a token sees such a row: a page of held rows in the first sequence, the last page in the last one, and
    one that a window hides, or the masks (of tokens that see nothing but held rows), in the second."""
    import paper_2607_21475_amd as ebd

    c, news, G, mask, pos, window = _batch(name)
    N = c.K.shape[0]
    gone = set()

    def lose(s, e, value):
        gone.add((s, e))
        c.table[s, e] = value

    firsts = [n - m for n, m in zip(c.lens, news)]
    lose(0, (firsts[0] - 1) // 16, N)
    last = len(news) - 1
    lose(last, (c.lens[last] - 1) // 16, -1)
    if last > 1:
        e = (c.lens[1] - 1) // 16
        lose(1, e, -2 ** 31)
        for j in range(news[1]):
            row = mask[news[0] + j]
            mask[news[0] + j] = [step.signed(w & sum(1 << i for i in range(64) if firsts[1] + 64 * k + i < 16 * e))
                                 for k, w in enumerate(row)]
    held = lambda s, r: (s, r // 16) not in gone  # noqa: E731
    q, y, lse, st = _call(c, news, G, mask, pos, window=window)
    want, t0 = [], 0
    for s, m in enumerate(news):
        seen = {r for j in range(m) for r in step.sees(firsts[s], c.lens[s], None, mask[t0 + j], pos[t0 + j], window)}
        want.append(ebd.EBD_ST_BAD_PAGE if any(not held(s, r) for r in seen) else 0)
        t0 += m
    assert st.tolist() == want and want[0] and (last < 2 or not want[1] or 16 * ((c.lens[1] - 1) // 16) < firsts[1])
    _check(c, name, mask, pos, q, y, lse, held=held)


@pytest.mark.parametrize("name", tree_shapes.BATCHES)
def test_shapes_bounds_below_the_truth(name):
    import paper_2607_21475_amd as ebd

    c, news, G, mask, pos, window = _batch(name)
    new, rows = tree_shapes.bounds(name)
    q, y, lse, st = _call(c, news, G, mask, pos, window=window, max_new=new)
    assert st.tolist() == [ebd.EBD_ST_BAD_LAYOUT if m > new else 0 for m in news]
    for s, m in enumerate(news):
        behind = slice(sum(news[:s]) + min(m, new), sum(news[:s + 1]))
        assert bool((y[behind] == 7).all()) and bool((lse[behind] == 7).all())
    _check(c, name, mask, pos, q, y, lse, max_new=new)
    q, y, lse, st = _call(c, news, G, mask, pos, window=window, max_rows=rows)
    assert st.tolist() == [ebd.EBD_ST_BAD_LAYOUT if n > rows else 0 for n in c.lens]
    _check(c, name, mask, pos, q, y, lse, limit=rows)
