"""Paged-cache operators on the GPU where values are not finite, bounds are wrong or tokens are padding."""
import math

import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
INF = float("inf")


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _attend(c, news, G, q=None, seed=0, hi=None, window=0, max_rows=None):
    import paper_2607_21475_amd as ebd

    T = sum(news)
    if q is None:
        q = ref.spaced((T, c.kv * G, 128), _gen(seed + 1), False)
    y = torch.full((T, c.kv * G, 128), 7.0, dtype=BF, device="cuda")
    lse = torch.full((T, c.kv * G), 7.0, dtype=torch.float32, device="cuda")
    off = torch.tensor([0] + [sum(news[:i + 1]) for i in range(len(news))], device="cuda")
    st = torch.zeros(len(news), dtype=torch.int32, device="cuda")
    p = ebd.attend_paged_params(ebd.pages(c.K, c.V, c.table), q, y, off, c.len, max(news),
                                max(c.lens) if max_rows is None else max_rows, qpos=hi, window=window)
    ws = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, p))
    ws.fill_(255)
    ebd.ebd_attend_paged(p, q, c.K, c.V, y, ws, lse=lse, status=st)
    return q, y, lse, st


def _agree(got, want, tol, what):
    """As ref.check, with NaN where the formula has NaN and nowhere else."""
    got, want = got.double(), want.double()
    assert torch.equal(got.isnan(), want.isnan()), "%s: %d NaN, the formula has %d" % (
        what, int(got.isnan().sum()), int(want.isnan().sum()))
    zero = torch.zeros((), dtype=torch.float64, device=got.device)
    nan = want.isnan()
    ref.check(torch.where(nan, zero, got), torch.where(nan, zero, want), torch.where(nan, zero, tol), what)


# Query rows of a KV head and rows of the sequence: each kernel and shape, with the rows split and not.
SHAPES = [([1], 4, 33), ([1], 4, 4097), ([2], 3, 20001), ([3], 4, 20), ([5], 4, 130), ([6], 4, 3000), ([14], 4, 200),
          ([14], 4, 5000), ([70], 2, 150), ([40], 4, 2500), ([500], 4, 9001)]


def _picked(m):
    """Tokens that are compared with the formula: all of a few, every 41st and the last of many."""
    return torch.tensor(sorted(set(range(0, m, 1 if m < 100 else 41)) | {m - 1}), device="cuda")


def _against(c, q, y, lse, m, n, what, window=0):
    """The picked tokens against the formula (the others see nothing in the reference and are left out)."""
    pick = _picked(m)
    hi = torch.full((m,), -1, dtype=torch.int32, device="cuda")
    hi[pick] = (n - m + pick).to(torch.int32)
    ry, rl, ty, tl = ref.attend(c, q, [m], hi=hi, window=window, weights_bits=8)
    _agree(y[pick], ry[pick], ty[pick], what + ", y")
    _agree(lse[pick], rl[pick], tl[pick], what + ", lse")
    return ry[pick]


@pytest.mark.parametrize("news,G,n", SHAPES)
def test_a_query_that_holds_nan_gives_nan(news, G, n):
    """... and only there: the other rows of its block are what they were."""
    m, kv = news[0], 8 if n == 9001 else 2
    print("nan query", m, G, n, flush=True)
    c = ref.Cache([n], kv, 16, _gen(n + m))
    q = ref.spaced((m, kv * G, 128), _gen(1), False)
    for t, h in {(0, 0), (m - 1, kv * G - 1), (m // 2 // 41 * 41, G)}:
        q[t, h, 5] = math.nan
    _, y, lse, st = _attend(c, news, G, q=q)
    assert not bool(st.any())
    want = _against(c, q, y, lse, m, n, "nan query")
    assert bool(want.isnan().any()) and not bool(want.isnan().all())


@pytest.mark.parametrize("news,G,n", SHAPES)
def test_keys_that_hold_nan_give_nan_to_all_that_see_them(news, G, n):
    """One key, the last of all, a tile of 32, all: whichever wave, group or split they fall to."""
    m, kv = news[0], 8 if n == 9001 else 1
    print("nan keys", m, G, n, flush=True)
    c = ref.Cache([n], kv, 16, _gen(n + m))
    K0 = c.K.clone()
    for first, last in ((0, 1), (n - 1, n), (n // 2, n // 2 + 1), (n // 64 * 32, min(n, n // 64 * 32 + 32)), (0, n)):
        for r in range(first, last):
            c.K[int(c.table[0, r // 16]), 0, r % 16, 3] = math.nan
        q, y, lse, _ = _attend(c, news, G)
        want = _against(c, q, y, lse, m, n, "nan keys %d to %d" % (first, last))
        assert bool(want.isnan().any())
        c.K.copy_(K0)


@pytest.mark.parametrize("news,G,n", SHAPES)
def test_infinite_values_that_all_see(news, G, n):
    """An infinity times a positive weight is that infinity; of both signs, NaN."""
    m = news[0]
    kv = 8 if n == 9001 else 1
    print("infinite values", m, G, n, flush=True)
    c = ref.Cache([n], kv, 16, _gen(n + m))
    for r, e, x in ((0, 1, INF), (n // 3, 2, -INF), (0, 9, INF), (n // 5 + 1, 9, -INF)):
        c.V[int(c.table[0, r // 16]), 0, r % 16, e] = x
    q, y, lse, _ = _attend(c, news, G)
    want = _against(c, q, y, lse, m, n, "infinite values")
    assert bool((want == INF).any()) and bool((want == -INF).any()) and bool(want.isnan().any())


@pytest.mark.parametrize("news", [[2], [12], [30], [90]])
def test_rows_that_no_token_sees_raise_no_flag(news):
    """Windows apart from each other: the pages between them, and rows past the table, are seen by no token."""
    c = ref.Cache([700], 2, 16, _gen(8), fill=math.nan)
    m, window = news[0], 16
    hi = torch.full((m,), 30, dtype=torch.int32, device="cuda")
    hi[m // 2:] = 600
    keep = torch.zeros(c.table.shape[1], dtype=torch.bool, device="cuda")
    keep[0:2] = keep[36:38] = True
    held = ref.Cache([700], 2, 16, _gen(8), fill=math.nan)
    c.table[0, ~keep] = -1
    c.len[0] = 16 * c.table.shape[1] + 40
    q, y, lse, st = _attend(c, news, 4, hi=hi, window=window, max_rows=4000)
    held.K, held.V = c.K, c.V
    ry, rl, ty, tl = ref.attend(held, q, news, hi=hi, window=window, weights_bits=8)
    ref.check(y, ry, ty, "y")
    ref.check(lse, rl, tl, "lse")
    assert st.tolist() == [0]
    # one token that sees such a row is enough
    import paper_2607_21475_amd as ebd
    for at in (40, 592 + 16, 16 * c.table.shape[1] + 30):
        hi[m - 1] = at
        assert _attend(c, news, 4, hi=hi, window=window, max_rows=4000)[3].tolist() == [ebd.EBD_ST_BAD_PAGE], at


def _gather_params(c, off, max_rows):
    import paper_2607_21475_amd as ebd

    return ebd.gather_paged_params(ebd.pages(c.K, c.V, c.table), torch.tensor(off, device="cuda"), max_rows)


@pytest.mark.parametrize("first,short", [(0, 0), (0, 1), (0, 70), (0, 171), (0, 300), (-1, 0), (-70, 0), (-130, 5), (10, 0),
                                         (1 << 40, 0), (-(1 << 40), 0)])
def test_gather_writes_no_row_outside_its_outputs(first, short):
    """Units that seq_off places before, across and behind the ends of Ku and Vu, which lie between guard rows."""
    import paper_2607_21475_amd as ebd

    print("gather bounds", first, short, flush=True)
    lens, kv = [100, 50], 2
    c = ref.Cache(lens, kv, 16, _gen(6))
    off = [0, 100, 200, 250, 300]
    rows, guard = 300 - short, 400
    big = torch.full((2, guard + rows + guard, 128), 7.0, dtype=BF, device="cuda")
    Ku, Vu = big[0, guard:guard + rows], big[1, guard:guard + rows]
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    p = _gather_params(c, [o + first for o in off], 100)
    if rows == 0:  # outputs without memory, which the entry point refuses
        with pytest.raises(ebd.EbdError):
            ebd.ebd_gather_paged(p, c.K, c.V, Ku, Vu, status=st)
        return
    ebd.ebd_gather_paged(p, c.K, c.V, Ku, Vu, status=st)
    want = torch.full_like(big, 7.0)
    flags = []
    for u, (a, b) in enumerate(zip(off, off[1:])):
        lo, hi = max(a + first, 0), min(b + first, rows)
        flags.append(0 if (lo, hi) == (a + first, b + first) else ebd.EBD_ST_BAD_LAYOUT)
        if lo < hi:
            for x, pool in zip(want, (c.K, c.V)):
                x[guard + lo:guard + hi] = c.rows(pool, u // kv, u % kv)[lo - a - first:hi - a - first]
    assert torch.equal(big, want) and st.tolist() == flags


def test_gather_refuses_outputs_of_other_shapes():
    import paper_2607_21475_amd as ebd

    c = ref.Cache([20], 2, 16, _gen(6))
    p = _gather_params(c, [0, 20, 40], 20)
    x = torch.zeros((40, 128), dtype=BF, device="cuda")
    for Ku, Vu in ((x, x[:39]), (x[:39], x), (x.view(80, 64), x.view(80, 64)), (x.view(-1), x.view(-1)),
                   (x.view(20, 2, 128), x.view(20, 2, 128)), (x, None), (None, x)):
        with pytest.raises(ValueError):
            ebd.ebd_gather_paged(p, c.K, c.V, Ku, Vu)
    # the same parameters serve outputs of other sizes
    for rows in (40, 43, 40):
        Ku, Vu = (torch.full((rows, 128), 7.0, dtype=BF, device="cuda") for _ in range(2))
        ebd.ebd_gather_paged(p, c.K, c.V, Ku, Vu)
        assert torch.equal(Ku[:40], torch.cat([c.rows(c.K, 0, h) for h in range(2)])) and bool((Ku[40:] == 7).all())


def test_helpers_give_padding_tokens_zeros():
    """Outputs that the helpers allocate hold nothing of what that memory held before."""
    import paper_2607_21475_amd as ebd

    g = _gen(3)
    new, kv, G, T = [5, 0, 3], 2, 3, 14
    c = ebd.PagedCache.allocate([40, 8, 40], kv, page_size=16)
    c.K.normal_(generator=g), c.V.normal_(generator=g)
    c.len += torch.tensor([30, 0, 12], dtype=torch.int32, device="cuda")
    off = torch.tensor([2, 7, 7, 10], device="cuda")  # two tokens before the sequences and four behind
    k, v, q = (ref.spaced((T, h, 128), g, False) for h in (kv, kv, kv * G))
    freq, _ = ebd.rope_frequencies(128)
    pad = torch.ones(T, dtype=torch.bool, device="cuda")
    pad[2:10] = False

    def dirty():
        x = [torch.full(s, math.nan, dtype=t, device="cuda") for s, t in (((T, kv * G, 128), BF), ((T, kv * G), torch.float32))]
        del x

    dirty()
    qr = c.append(k, v, off, ebd.rotary(freq), q=q)
    assert not bool(qr[pad].any()) and bool(qr[~pad].any(-1).all())
    dirty()
    out = c.attend(qr, off, 5, 30)
    assert not bool(out["y"][pad].any()) and bool((out["lse"][pad] == -INF).all())
    assert bool(torch.isfinite(out["lse"][~pad]).all())
    dirty()
    short = c.attend(qr, off, 3, 30)  # new tokens past max_new get no output
    assert not bool(short["y"][5:7].any()) and bool((short["lse"][5:7] == -INF).all())
    assert torch.equal(short["lse"][7:10], out["lse"][7:10])


def test_append_of_the_most_tokens():
    """2^24 - 1 tokens of 128 rows, 2^34 threads; the tokens before the last three are padding, which reads one token."""
    import paper_2607_21475_amd as ebd

    T, kv = (1 << 24) - 1, 64
    g = _gen(2)
    c = ref.Cache([20], kv, 16, g)
    k, v = (ref.spaced((1, kv, 128), g, False).expand(T, kv, 128) for _ in range(2))
    K0, V0 = c.K.clone(), c.V.clone()
    for n in (3, 0):
        off = torch.tensor([T - n, T], device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        ebd.ebd_append_paged(ebd.append_paged_params(ebd.pages(c.K, c.V, c.table), k, v, off, c.len), k, v, c.K, c.V, status=st)
        torch.cuda.synchronize()
        print("appended", n, flush=True)
        for r in range(17, 20) if n else ():
            for x, new in ((K0, k), (V0, v)):
                x[int(c.table[0, r // 16]), :, r % 16] = new[0]
        assert torch.equal(c.K, K0) and torch.equal(c.V, V0) and not bool(st.any())


@pytest.mark.parametrize("news", [[130] + [17] * 12 + [16] * 5 + [0] * 230, [0] * 70 + [129, 0, 17, 16, 33] + [0] * 40 + [17, 140],
                                  [300] + [0] * 90])
def test_attend_chunks_among_sequences_without_new_tokens(news):
    """As many blocks of query rows as their tokens may make, and none for the sequences that have none."""
    print("attend idle", len(news), sum(news), flush=True)
    lens = [n + 40 + 13 * (i % 7) for i, n in enumerate(news)]
    c = ref.Cache(lens, 1, 16, _gen(5), fill=math.nan)
    for G in (1, 5):
        q, y, lse, st = _attend(c, news, G)
        assert not bool(st.any())
        ry, rl, ty, tl = ref.attend(c, q, news, weights_bits=8)
        ref.check(y, ry, ty, "y")
        ref.check(lse, rl, tl, "lse")


def test_outputs_of_every_second_head():
    """Rotated rows and results written to heads 0 and 2 of three: the heads between them stay as they were."""
    import paper_2607_21475_amd as ebd

    g = _gen(4)
    c = ref.Cache([40], 2, 16, g)
    x = ref.spaced((5, 2, 128), g, False)
    freq, _ = ebd.rope_frequencies(128)
    pos = torch.arange(5, device="cuda", dtype=torch.int32)
    off = torch.tensor([0, 5], device="cuda")
    whole = torch.full((2, 5, 3, 128), 7.0, dtype=BF, device="cuda")
    r, y = whole[0, :, ::2], whole[1, :, ::2]
    ebd.ebd_rope(ebd.rope_params(x, r, pos, ebd.rotary(freq)), x, r)
    p = ebd.attend_paged_params(ebd.pages(c.K, c.V, c.table), r, y, off, c.len, 5, 40)
    ebd.ebd_attend_paged(p, r, c.K, c.V, y, ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, p)))
    want = ref.rotate(x, pos, freq)
    ref.check(r, want, ref.rotate_tolerance(x, want, freq), "rotated")
    ry, _, ty, _ = ref.attend(c, r, [5], weights_bits=8)
    ref.check(y, ry, ty, "y")
    assert bool((whole[:, :, 1] == 7).all())
