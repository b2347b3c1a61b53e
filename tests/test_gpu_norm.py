"""Norms of heads with rotary positions, forward, backward and on the way into the paged cache, on the GPU."""
import math

import pytest
import torch

import paged_ref as ref
import step_ref as step

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
EPS = 1e-6


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _weights(g, heads, own):
    return 1.0 + 0.3 * torch.randn((heads, 128) if own else (128,), generator=g, device="cuda")


def _backward(x, dy, dx, norm, rot, pos, shape):
    import paper_2607_21475_amd as ebd

    p = ebd.norm_rope_backward_params(x, dy, dx, norm, rot, pos)
    dw = torch.full(shape, 7.0, device="cuda")
    ws = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_NORM_ROPE_BACKWARD, p))
    ws.fill_(255)
    ebd.ebd_norm_rope_backward(p, x, dy, dx, dw, ws)
    return dw


CASES = [
    # tokens, heads, rotary dimensions (0: none), layout, fused, weights of each head's own
    (1, 1, 128, 0, False, False), (1, 32, 128, 1, True, True), (7, 3, 64, 0, True, False), (130, 33, 96, 0, False, True),
    (5, 8, 2, 0, False, False), (5, 9, 2, 1, False, True), (64, 16, 34, 0, True, False), (33, 17, 34, 1, True, False),
    (9, 28, 126, 0, False, True), (3, 70, 112, 1, True, True), (6, 140, 50, 0, False, True), (3, 200, 128, 0, True, False),
    (1025, 5, 128, 0, False, False), (2000, 1, 128, 0, False, True), (40, 6, 0, 0, True, True), (3, 1, 0, 0, False, False),
    (1500, 40, 128, 0, True, True), (700, 130, 64, 1, False, False),
]


@pytest.mark.parametrize("tokens,heads,rot,layout,fused,own", CASES)
def test_norm_rope_and_its_gradients(tokens, heads, rot, layout, fused, own):
    import paper_2607_21475_amd as ebd

    print("norm", tokens, heads, rot, layout, fused, own, flush=True)
    g = _gen(tokens + heads + rot)
    x, dy = ref.spaced((tokens, heads, 128), g, fused), ref.spaced((tokens, heads, 128), g, not fused)
    pos = torch.randint(-1000, 1 << 20, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    w = _weights(g, heads, own)
    norm = ebd.head_norm(w, EPS)
    for amp, inverse in ((1.0, False), (1.3, True)):
        f = step.frequencies(rot) if rot else None
        r = ebd.rotary(f, layout, amp, inverse) if rot else None
        want, tol = step.norm_rope(x, w, EPS, pos, f, amp, layout, inverse)
        y = ref.spaced((tokens, heads, 128), g, not fused)
        ebd.ebd_norm_rope(ebd.norm_rope_params(x, y, norm, r, pos), x, y)
        ref.check(y, want, tol, "y")
        (dx, tx), (dw, tw) = step.norm_rope_gradients(x, w, EPS, dy, pos, f, amp, layout, inverse)
        gx = ref.spaced((tokens, heads, 128), g, fused)
        gw = _backward(x, dy, gx, norm, r, pos, w.shape)
        ref.check(gx, dx, tx, "dx")
        ref.check(gw, dw, tw, "dw")
        again = _backward(x, dy, gx, norm, r, pos, w.shape)
        assert torch.equal(gw, again)
        # in place: y over x, dx over dy, dx over x
        z = x.clone()
        ebd.ebd_norm_rope(ebd.norm_rope_params(z, z, norm, r, pos), z, z)
        assert torch.equal(z, y)
        z = dy.clone()
        _backward(x, z, z, norm, r, pos, w.shape)
        assert torch.equal(z, gx)
        z = x.clone()
        _backward(z, dy, z, norm, r, pos, w.shape)
        assert torch.equal(z, gx)


def test_gradients_against_differences():
    """<dx, u> and <dw, v> against central differences of sum(dy . y) in float64.  Steps of 2^-12 along directions of unit
    elements: a term's third derivative is below 100 |dy| (x of rows with mean square near 1), so a difference is off by
    2^-24 / 6 of that."""
    import paper_2607_21475_amd as ebd

    g = _gen(5)
    T, H, amp, layout = 19, 3, 0.8, 1
    x, dy = ref.spaced((T, H, 128), g, False), ref.spaced((T, H, 128), g, False)
    w, f = _weights(g, H, True), step.frequencies(96)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 977
    gx = torch.empty_like(x)
    gw = _backward(x, dy, gx, ebd.head_norm(w, EPS), ebd.rotary(f, layout, amp), pos, w.shape)
    (_, tx), (_, tw) = step.norm_rope_gradients(x, w, EPS, dy, pos, f, amp, layout)
    e = 2.0 ** -12
    slack = 100 * e * e / 6 * float(dy.double().abs().sum())

    def total(x, w):
        return float((dy.double() * step.norm_rope(x, w, EPS, pos, f, amp, layout)[0]).sum())

    for i in range(4):
        u = torch.randint(0, 2, x.shape, generator=g, device="cuda").double() * 2 - 1
        v = torch.randint(0, 2, w.shape, generator=g, device="cuda").double() * 2 - 1
        want = (total(x.double() + e * u, w) - total(x.double() - e * u, w)) / (2 * e)
        assert abs(float((gx.double() * u).sum()) - want) <= float(tx.sum()) + slack
        want = (total(x, w.double() + e * v) - total(x, w.double() - e * v)) / (2 * e)
        assert abs(float((gw.double() * v).sum()) - want) <= float(tw.sum()) + slack


def test_norm_rows_that_are_zero_large_or_not_finite():
    import paper_2607_21475_amd as ebd

    g = _gen(6)
    x = ref.spaced((8, 4, 128), g, False)
    x[0, 0] = 0
    x[1, 1] *= 2.0 ** 100
    x[2, 2] = 3e38
    x[3, 3] *= 2.0 ** -120
    x[4, 0, 7] = math.inf
    x[5, 1, 9] = math.nan
    x[6, 2, 100] = -math.inf
    dy = ref.spaced((8, 4, 128), g, False)
    pos = torch.arange(8, device="cuda", dtype=torch.int32)
    w, f = _weights(g, 4, True), step.frequencies(64)
    r, norm = ebd.rotary(f), ebd.head_norm(w, EPS)
    want, tol = step.norm_rope(x, w, EPS, pos, f)
    y, gx = torch.empty_like(x), torch.empty_like(x)
    ebd.ebd_norm_rope(ebd.norm_rope_params(x, y, norm, r, pos), x, y)
    (dx, tx), _ = step.norm_rope_gradients(x, w, EPS, dy, pos, f)
    _backward(x, dy, gx, norm, r, pos, w.shape)
    least = 2.0 ** -133  # (half a step of bf16 below its normal numbers, 2^-134, and what fp32 loses there)
    for got, ref64, t, what in ((y, want, tol, "y"), (gx, dx, tx, "dx")):
        assert torch.equal(got.isnan(), ref64.isnan()), what
        zero = torch.zeros((), dtype=torch.float64, device="cuda")
        nan = ref64.isnan()
        ref.check(torch.where(nan, zero, got.double()), torch.where(nan, zero, ref64), torch.where(nan, zero, t) + least, what)


def test_norm_without_tokens_and_around_the_rows():
    import paper_2607_21475_amd as ebd

    g = _gen(7)
    w = _weights(g, 5, False)
    e = torch.empty((0, 5, 128), dtype=BF, device="cuda")
    norm = ebd.head_norm(w, EPS)
    ebd.ebd_norm_rope(ebd.norm_rope_params(e, e, norm), e, e)
    assert bool((_backward(e, e, e, norm, None, None, w.shape) == 0).all())
    own = _weights(g, 5, True)
    assert bool((_backward(e, e, e, ebd.head_norm(own, EPS), None, None, own.shape) == 0).all())
    x = ref.spaced((6, 4, 128), g, True)
    whole = torch.full((6, 12, 128), 7.0, dtype=BF, device="cuda")
    ebd.ebd_norm_rope(ebd.norm_rope_params(x, whole[:, 4:8], norm), x, whole[:, 4:8])
    _backward(x, x, whole[:, 4:8], norm, None, None, w.shape)
    assert bool((whole[:, :4] == 7).all()) and bool((whole[:, 8:] == 7).all()) and bool((whole[:, 4:8] != 7).any())


def test_norm_offsets_past_32_bits():
    """Tokens 2^31 elements apart, and heads of a stride that is no row."""
    import paper_2607_21475_amd as ebd

    g = _gen(8)
    hold = torch.empty(2 * 2 ** 31 + 1024, dtype=BF, device="cuda")
    x = torch.as_strided(hold, (3, 2, 128), (2 ** 31, 136, 1))
    x.copy_(ref.spaced((3, 2, 128), g, False))
    w, f = _weights(g, 2, False), step.frequencies(34)
    pos = torch.tensor([0, 5, 2 ** 31 - 1], device="cuda", dtype=torch.int32)
    norm, r = ebd.head_norm(w, EPS), ebd.rotary(f)
    y = torch.empty((3, 2, 128), dtype=BF, device="cuda")
    ebd.ebd_norm_rope(ebd.norm_rope_params(x, y, norm, r, pos), x, y)
    ref.check(y, *step.norm_rope(x, w, EPS, pos, f), "y")
    dy, (dx, tx) = y.clone(), step.norm_rope_gradients(x, w, EPS, y, pos, f)[0]
    _backward(x, dy, x, norm, r, pos, w.shape)
    ref.check(x, dx, tx, "dx")


def test_norm_long_sums():
    """40000 rows into one row of weights: chains of many additions."""
    import paper_2607_21475_amd as ebd

    g = _gen(9)
    x = ref.spaced((40000, 1, 128), g, False) + 0.5
    dy = ref.spaced((40000, 1, 128), g, False) + 0.5
    w = _weights(g, 1, False)
    _, (dw, tw) = step.norm_rope_gradients(x, w, EPS, dy, None, None)
    ref.check(_backward(x, dy, torch.empty_like(x), ebd.head_norm(w, EPS), None, None, w.shape), dw, tw, "dw")


@pytest.mark.parametrize("tokens,heads,own", [(3000001, 1, False), (300001, 2, True)])
def test_norm_many_tokens(tokens, heads, own):
    """Work-groups of hundreds of tokens each, and a launch of millions of waves' shares."""
    import paper_2607_21475_amd as ebd

    g = _gen(10)
    x, dy = ref.spaced((tokens, heads, 128), g, False), ref.spaced((tokens, heads, 128), g, False)
    w, f = _weights(g, heads, own), step.frequencies(128)
    pos = torch.arange(tokens, device="cuda", dtype=torch.int32)
    norm, r = ebd.head_norm(w, EPS), ebd.rotary(f)
    y, gx = torch.empty_like(x), torch.empty_like(x)
    ebd.ebd_norm_rope(ebd.norm_rope_params(x, y, norm, r, pos), x, y)
    gw = _backward(x, dy, gx, norm, r, pos, w.shape)
    dw = tw = 0.0
    for a in range(0, tokens, 200000):
        b = slice(a, min(a + 200000, tokens))
        ref.check(y[b], *step.norm_rope(x[b], w, EPS, pos[b], f), "y")
        (dx, tx), (p, tp) = step.norm_rope_gradients(x[b], w, EPS, dy[b], pos[b], f)
        ref.check(gx[b], dx, tx, "dx")
        dw, tw = dw + p, tw + tp
    ref.check(gw, dw, tw, "dw")


# ---- append ------------------------------------------------------------------------------------

@pytest.mark.parametrize("lens,news,kv,heads,page,order,rot,layout,fused,given,own,which", [
    ([1], [1], 8, 32, 16, "heads", 128, 0, True, False, False, "kq"),
    ([40, 7, 300, 16], [40, 0, 33, 16], 4, 28, 32, "tokens", 128, 0, True, False, True, "kq"),
    ([5, 1000, 64], [1, 1, 1], 1, 1, 16, "heads", 64, 1, False, True, False, "k"),
    ([130, 129], [130, 65], 2, 6, 64, "tokens", 34, 0, False, True, True, "q"),
    ([33, 0, 12], [33, 0, 3], 3, 0, 256, "heads", 128, 1, True, False, False, "k"),
    ([70, 2], [9, 2], 5, 7, 16, "heads", 0, 0, False, False, True, "kq"),
    ([50, 31], [9, 3], 2, 140, 16, "heads", 18, 0, False, False, False, ""),
] + [([17 + s % 5 for s in range(150)], [s % 4 for s in range(150)], 2, 4, 16, "heads", 128, 0, False, False, False, "kq")])
@pytest.mark.parametrize("slots", [False, True])
def test_append_norm(lens, news, kv, heads, page, order, rot, layout, fused, given, own, which, slots):
    import paper_2607_21475_amd as ebd

    print("append_norm", lens[:4], news[:4], kv, heads, page, order, rot, layout, which, slots, flush=True)
    g = _gen(sum(lens) + page)
    c = ref.Cache(lens, kv, page, g, order)
    pad = 3  # tokens behind the last sequence
    T = sum(news) + pad
    k, v = ref.spaced((T, kv, 128), g, fused), ref.spaced((T, kv, 128), g, fused)
    q = ref.spaced((T, heads, 128), g, fused) if heads else None
    out = torch.full((T, heads, 128), 7.0, dtype=BF, device="cuda") if heads else None
    off = torch.tensor([0] + [sum(news[:i + 1]) for i in range(len(news))], device="cuda")
    row = torch.tensor([n - m + j for n, m in zip(lens, news) for j in range(m)] + [0] * pad, device="cuda")
    pos = (row * 3 + 100000 if given else row).to(torch.int32)
    f = step.frequencies(rot) if rot else None
    r = ebd.rotary(f, layout, 1.25) if rot else None
    wk, wq = _weights(g, kv, own), _weights(g, heads, own) if heads else None
    K0, V0 = c.K.clone(), c.V.clone()
    st = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    at = None
    if slots:
        seq = torch.tensor([s for s, m in enumerate(news) for _ in range(m)], device="cuda")
        at = torch.full((T,), -1, dtype=torch.int64, device="cuda")
        at[:-pad] = c.table[seq, row[:-pad] // page].long() * page + row[:-pad] % page
        at[-1] = c.K.shape[0] * page  # just outside the pool
    p = ebd.append_norm_params(ebd.pages(c.K, c.V, c.table), k, v, None if slots else off, None if slots else c.len,
                               k_norm=ebd.head_norm(wk, EPS) if "k" in which else None,
                               q_norm=ebd.head_norm(wq, EPS) if "q" in which else None, rot=r,
                               pos=pos if given or slots else None, q=q, q_out=out, slots=at)
    ebd.ebd_append_norm(p, k, v, c.K, c.V, q, out, status=st)
    assert not bool(st.any())

    def want(x, w, on):
        if on:
            return step.norm_rope(x, w, EPS, pos, f, 1.25, layout)
        if not rot:
            return x.double(), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        y = ref.rotate(x, pos, f, 1.25, layout)
        return y, ref.rotate_tolerance(x, y, f, 1.25, layout)

    ky, kt = want(k, wk, "k" in which)
    K1, V1, tk = K0.double(), V0.clone(), torch.zeros(K0.shape, dtype=torch.float64, device="cuda")
    t = 0
    for s, (n, m) in enumerate(zip(lens, news)):
        for i in range(n - m, n):
            pg = int(c.table[s, i // page])
            K1[pg, :, i % page], tk[pg, :, i % page], V1[pg, :, i % page] = ky[t], kt[t], v[t]
            t += 1
    ref.check(c.K, K1, tk, "K")
    assert torch.equal(c.V, V1)
    if heads:
        y, tol = want(q, wq, "q" in which)
        ref.check(out[:t], y[:t], tol[:t], "q")
        assert bool((out[t:] == 7).all())


def test_append_norm_rows_without_a_page():
    """As ebd_append_paged: a row without a page is flagged and not written, its query is."""
    import paper_2607_21475_amd as ebd

    g = _gen(9)
    c = ref.Cache([40, 40], 2, 16, g)
    c.table[0, 2] = -1
    c.len[1] = 2  # fewer rows than new tokens
    off = torch.tensor([0, 4, 8], device="cuda")
    k, v = ref.spaced((8, 2, 128), g, False), ref.spaced((8, 2, 128), g, False)
    q, out = ref.spaced((8, 3, 128), g, False), torch.zeros((8, 3, 128), dtype=BF, device="cuda")
    st = torch.full((2,), 64, dtype=torch.int32, device="cuda")
    w = _weights(g, 2, False)
    K0, V0 = c.K.clone(), c.V.clone()
    p = ebd.append_norm_params(ebd.pages(c.K, c.V, c.table), k, v, off, c.len, q_norm=ebd.head_norm(w, EPS), q=q, q_out=out)
    ebd.ebd_append_norm(p, k, v, c.K, c.V, q, out, status=st)
    assert st.tolist() == [96, 96]
    pg = int(c.table[1, 0])
    for x, new in ((K0, k), (V0, v)):
        x[pg, :, 0], x[pg, :, 1] = new[6], new[7]
    assert torch.equal(c.K, K0) and torch.equal(c.V, V0)
    ref.check(out, *step.norm_rope(q, w, EPS, None, None), "q")
