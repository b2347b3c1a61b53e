"""Attention of drafted trees over the paged cache on the GPU, against the plain 64-bit form."""
import math
import random

import pytest
import torch

import paged_ref as ref
import step_ref as step

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
INF = math.inf


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _masks(kind, n, words, rng):
    """(mask words of n tokens, their depths)."""
    if kind == "tree":
        return step.masks_of(step.tree(n, rng), words)
    if kind == "chains":
        return step.masks_of(step.chains(n, 3), words)
    if kind == "none":
        return [[0] * words for _ in range(n)], [0] * n
    if kind == "all":  # bits behind the last token among them
        return [[-1] * words for _ in range(n)], [0] * n
    return [[step.signed(rng.getrandbits(64) & rng.getrandbits(64)) for _ in range(words)] for _ in range(n)], list(range(n))


def _call(c, news, G, mask, pos=None, q=None, window=0, scale=0.0, max_new=None, max_rows=None, pad=0, seed=0, fused=False):
    import paper_2607_21475_amd as ebd

    T = sum(news) + pad
    if q is None:
        q = ref.spaced((T, c.kv * G, 128), _gen(seed + 1), fused)
    y = torch.full((T, c.kv * G, 128), 7.0, dtype=BF, device="cuda")
    lse = torch.full((T, c.kv * G), 7.0, dtype=torch.float32, device="cuda")
    off = torch.tensor([0] + [sum(news[:i + 1]) for i in range(len(news))], device="cuda")
    st = torch.zeros(len(news), dtype=torch.int32, device="cuda")
    m = torch.tensor(mask + [[-1] * len(mask[0])] * pad, dtype=torch.int64, device="cuda")
    qpos = None if pos is None else torch.tensor(pos + [5] * pad, dtype=torch.int32, device="cuda")
    p = ebd.attend_tree_params(ebd.pages(c.K, c.V, c.table), q, y, off, c.len, max(news) if max_new is None else max_new,
                               max(c.lens) if max_rows is None else max_rows, m, qpos=qpos, window=window, scale=scale)
    ws = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_TREE, p))
    ws.fill_(255)
    ebd.ebd_attend_tree(p, q, c.K, c.V, y, ws, lse=lse, status=st)
    return q, y, lse, st


def _check(c, news, G, mask, pos, q, y, lse, window=0, scale=None, held=None, limit=None, few=24, max_new=None, bits=8):
    """The tokens of each sequence (some of many) against the formula."""
    t0 = 0
    for s, m in enumerate(news):
        first = c.lens[s] - m
        shown = m if max_new is None else min(m, max_new)
        pick = range(shown) if shown <= few else sorted({0, 1, 31, 32, 63, 64, 65, shown - 2, shown - 1} & set(range(shown)) |
                                                        set(range(0, shown, max(1, shown // few))))
        for j in pick:
            t = t0 + j
            at = first + j if pos is None else pos[t]
            rows = step.sees(first, c.lens[s], None if held is None else lambda r: held(s, r), mask[t], at, window, limit)  # noqa: B023
            for h in range(c.kv):
                a = slice(h * G, h * G + G)
                ry, rl, ty, tl = step.attend_row(c, s, h, q[t, a], rows, scale, bits)
                ref.check(y[t, a], ry, ty, "y of sequence %d token %d head %d" % (s, j, h))
                ref.check(lse[t, a], rl, tl, "lse of sequence %d token %d head %d" % (s, j, h))
        t0 += m


CASES = [
    # rows held before, new tokens, KV heads, group, page, order, window, masks, words, own positions
    ([0], [1], 1, 1, 16, "heads", 0, "tree", 1, True),
    ([0, 5, 31], [3, 2, 4], 2, 4, 16, "heads", 0, "tree", 1, False),
    ([4096], [8], 8, 1, 16, "heads", 0, "tree", 1, True),
    ([1000, 17, 64], [7, 3, 1], 2, 4, 64, "tokens", 300, "tree", 1, True),
    ([33, 500], [5, 6], 1, 5, 16, "heads", 0, "random", 2, True),
    ([100, 2000, 0], [16, 9, 12], 2, 4, 32, "heads", 0, "tree", 1, True),
    ([3000, 47], [13, 13], 1, 4, 16, "tokens", 64, "chains", 1, True),
    ([77, 1023], [60, 41], 2, 1, 64, "heads", 0, "tree", 1, True),
    ([500, 90, 0], [64, 25, 33], 2, 4, 16, "heads", 0, "tree", 1, True),
    ([700, 2049], [130, 66], 1, 7, 32, "tokens", 512, "tree", 3, True),
    ([10, 300], [300, 200], 2, 3, 64, "heads", 100, "chains", 5, False),
    ([1, 129], [257, 100], 1, 2, 16, "heads", 0, "random", 5, True),
    ([640, 100], [20, 40], 2, 4, 16, "heads", 0, "all", 2, True),
    ([640, 0], [20, 40], 2, 4, 16, "heads", 0, "none", 1, True),
    ([900, 33, 1500, 3, 256], [70, 1, 1, 2, 1], 2, 4, 16, "heads", 0, "tree", 2, True),
    ([9000], [500], 8, 4, 64, "heads", 0, "tree", 8, True),
    ([6000] * 4, [4] * 4, 8, 4, 64, "heads", 0, "tree", 1, True),
    ([6000] * 4, [8] * 4, 8, 4, 64, "heads", 0, "tree", 1, True),
    ([6000] * 4, [15] * 4, 8, 4, 64, "heads", 0, "tree", 1, True),
    ([600] * 24, [64] * 24, 8, 4, 64, "heads", 0, "tree", 1, True),   # (blocks of 256 query rows)
    ([300] * 64, [30] * 64, 8, 4, 16, "tokens", 0, "tree", 1, True),  # (two work-groups of 128 a CU)
]


@pytest.mark.parametrize("held,news,kv,G,page,order,window,kind,words,own", CASES)
def test_tree(held, news, kv, G, page, order, window, kind, words, own):
    print("tree", held[:3], news[:3], kv, G, page, order, window, kind, words, own, flush=True)
    rng = random.Random(sum(held) + 3 * sum(news))
    lens = [h + m for h, m in zip(held, news)]
    c = ref.Cache(lens, kv, page, _gen(sum(lens)), order, fill=math.nan)
    mask, pos = [], []
    for h, m in zip(held, news):
        a, d = _masks(kind, m, words, rng)
        mask += a
        pos += [h + x for x in d]
    if own and len(pos) > 3:
        pos[2] = -1  # a padding token inside a sequence sees nothing
    pos = pos if own else None
    many = len(news) * kv * G * max(news) > 3000 or sum(lens) > 5000
    q, y, lse, st = _call(c, news, G, mask, pos, window=window, pad=2, fused=len(news) > 1)
    assert not bool(st.any())
    assert bool((y[sum(news):] == 7).all()) and bool((lse[sum(news):] == 7).all())
    most = max(news) * G  # weights have 16 bits up to 64 query rows of a sequence
    _check(c, news, G, mask, pos, q, y, lse, window, few=6 if many else 24, bits=16 if most <= 64 else 8)
    q2, y2, lse2, _ = _call(c, news, G, mask, pos, q=q, window=window, pad=2)
    assert torch.equal(y, y2) and torch.equal(lse, lse2)


def test_tree_a_chain_is_the_causal_attention():
    import paper_2607_21475_amd as ebd

    for held, news, G in (([100, 31], [7, 3], 4), ([2000, 77], [40, 90], 4)):
        lens = [h + m for h, m in zip(held, news)]
        c = ref.Cache(lens, 2, 16, _gen(4))
        words = 2
        mask = [w for m in news for w in step.masks_of(step.chains(m, 1), words)[0]]
        q, y, lse, _ = _call(c, news, G, mask)
        off = torch.tensor([0, news[0], sum(news)], device="cuda")
        y2, lse2 = torch.empty_like(y), torch.empty_like(lse)
        p = ebd.attend_paged_params(ebd.pages(c.K, c.V, c.table), q, y2, off, c.len, max(news), max(lens))
        ebd.ebd_attend_paged(p, q, c.K, c.V, y2, ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, p)), lse=lse2)
        _, _, ty, tl = ref.attend(c, q, news, weights_bits=8)
        ref.check(y, y2.double(), 2 * ty, "y")
        ref.check(lse, lse2.double(), 2 * tl, "lse")


# New tokens of the one sequence and query heads of a KV head: each kernel
SHAPES = [(3, 4), (7, 4), (15, 4), (40, 4), (150, 2)]


@pytest.mark.parametrize("new,G", SHAPES)
@pytest.mark.parametrize("held", [37, 3001])
def test_tree_values_that_are_not_finite(new, G, held):
    """A key or value that a token does not see has no effect on it, infinities and NaN included; those that it sees do."""
    rng = random.Random(new)
    c = ref.Cache([held + new], 2, 16, _gen(new), fill=math.nan)
    words = -(-new // 64)
    parents = step.tree(new, rng)
    mask, depth = step.masks_of(parents, words)
    pos = [held + d for d in depth]
    at = lambda r: (int(c.table[0, r // 16]), r % 16)  # noqa: E731
    # a new token's value, or key (in a tree of three the middle one is token 1, and keeps its key)
    bad = {new - 1: (INF, None), new // 2: (None, math.nan), 1: (-INF, None)}
    lost = [i for i, (v, k) in bad.items() if k is not None]
    for i, (v, k) in bad.items():
        pg, slot = at(held + i)
        if v is not None:
            c.V[pg, 0, slot, 5] = v
        if k is not None:
            c.K[pg, 0, slot, 9] = k
    window = 20
    pg, slot = at(held - 30)  # outside every window
    c.V[pg, :, slot] = math.nan
    c.K[pg, :, slot] = INF
    q, y, lse, st = _call(c, [new], G, mask, pos, window=window)
    assert not bool(st.any())
    for j in range(new):
        rows = step.sees(held, held + new, None, mask[j], pos[j], window)
        for h in range(2):
            a = slice(h * G, h * G + G)
            ry, rl, ty, tl = step.attend_row(c, 0, h, q[j, a], rows, None, 8)
            if h == 0 and any(held + i in rows for i in lost):  # a key that is NaN
                assert bool(y[j, a].isnan().all()) and bool(lse[j, a].isnan().all())
                continue
            mixed = ry.isnan() | ry.isinf()
            assert torch.equal(y[j, a].double()[mixed].nan_to_num(9.0), ry[mixed].nan_to_num(9.0)), (j, h)
            ref.check(y[j, a][~mixed], ry[~mixed], ty[~mixed], "y %d" % j)
            ref.check(lse[j, a], rl, tl, "lse %d" % j)


@pytest.mark.parametrize("new,G", SHAPES)
def test_tree_rows_without_a_page(new, G):
    """A row without a page is not seen, and flagged only where a token sees it; so is one past the table."""
    import paper_2607_21475_amd as ebd

    rng = random.Random(new)
    held = [100, 100, 100, 100]
    lens = [h + new for h in held]
    words = -(-new // 64)
    c = ref.Cache(lens, 1, 16, _gen(3))
    trees = [step.masks_of(step.tree(new, rng), words)[0] for _ in lens]
    c.table[0, 2] = -1                       # held rows 32 .. 47: all see them
    last = (lens[1] - 1) // 16               # the last page of sequence 1: its tokens' rows from `cut` on
    cut = max(last * 16 - held[1], 0)
    c.table[1, last] = 1 << 20
    trees[2] = [[step.signed(w & (2 ** 64 - 1) & ~(((1 << new) - 1 ^ (1 << cut) - 1) >> (64 * i) & (2 ** 64 - 1)))
                 for i, w in enumerate(r)] for r in trees[2]]  # ... which no token of sequence 2 sees
    c.table[2, last] = -5
    mask = [r for t in trees for r in t]
    news = [new] * 4
    q, y, lse, st = _call(c, news, G, mask)
    bad = [True, any(step.sees(100, lens[1], lambda r: r >= last * 16, m, 0, 1) for m in trees[1]),
           last * 16 < held[2], False]  # (a short tree's last page has held rows, too, that all see)
    assert st.tolist() == [ebd.EBD_ST_BAD_PAGE if b else 0 for b in bad]
    known = lambda s, r: 0 <= int(c.table[s, r // 16]) < c.K.shape[0]  # noqa: E731
    _check(c, news, G, mask, None, q, y, lse, held=known, few=10)
    # sequence 3 is longer than the table: its last rows are nowhere
    short = ref.Cache([h for h in lens], 1, 16, _gen(3))
    short.table = short.table[:, :last].contiguous()
    q, y, lse, st = _call(short, news, G, mask)
    lost = [any(step.sees(100, lens[s], lambda r: r >= last * 16, m, 100, 0) for m in trees[s]) for s in range(4)]
    if last * 16 < 100:
        lost = [True] * 4
    assert st.tolist() == [ebd.EBD_ST_BAD_PAGE if b else 0 for b in lost]
    short.lens = lens
    grow = torch.cat([short.table, torch.zeros_like(short.table[:, :2])], 1)
    short.table = grow
    _check(short, news, G, mask, None, q, y, lse, held=lambda s, r: r < last * 16, few=10)


@pytest.mark.parametrize("new,G", SHAPES)
def test_tree_bounds_below_the_truth(new, G):
    """Tokens past max_new get no output, rows past max_rows are not seen, new tokens past the mask's words neither; and a
    sequence of fewer rows than new tokens."""
    import paper_2607_21475_amd as ebd

    rng = random.Random(new + 1)
    news, held = [new, new + 30], [60, 0]
    lens = [h + m for h, m in zip(held, news)]
    c = ref.Cache(lens, 2, 16, _gen(8))
    mask = [r for m in news for r in step.masks_of(step.tree(m, rng), 1)[0]]
    q, y, lse, st = _call(c, news, G, mask, max_new=new)
    assert st.tolist() == [0, ebd.EBD_ST_BAD_LAYOUT]
    assert bool((y[2 * new:] == 7).all()) and bool((lse[2 * new:] == 7).all())
    _check(c, news, G, mask, None, q, y, lse, few=10, max_new=new)
    q, y, lse, st = _call(c, news, G, mask, max_rows=20)
    assert st.tolist() == [ebd.EBD_ST_BAD_LAYOUT] * 2
    _check(c, news, G, mask, None, q, y, lse, few=10, limit=20)
    c.len[0] = new - 2  # two new tokens before the sequence's first row
    c.lens = [new - 2, lens[1]]
    q, y, lse, st = _call(c, news, G, mask, max_rows=max(lens))
    assert st.tolist() == [0, 0]
    _check(c, news, G, mask, None, q, y, lse, few=10)


def test_tree_offsets_past_32_bits():
    """A pool whose pages lie 2^31 elements apart."""
    g = _gen(12)
    c = ref.Cache([60], 2, 16, g)
    n = c.K.shape[0]
    far = []
    for x in (c.K, c.V):
        hold = torch.empty((n - 1) * 2 ** 31 // 4 + 4 * 4096, dtype=BF, device="cuda")
        v = torch.as_strided(hold, x.shape, (2 ** 31 // 4, 2048, 128, 1))
        v.copy_(x)
        far.append(v)
    c.K, c.V = far
    assert (n - 1) * 2 ** 29 > 2 ** 31
    mask, depth = step.masks_of(step.tree(20, random.Random(5)), 1)
    for G in (1, 4):
        q, y, lse, st = _call(c, [20], G, mask, [40 + d for d in depth])
        _check(c, [20], G, mask, [40 + d for d in depth], q, y, lse)


def test_tree_in_a_graph_and_on_two_streams():
    """A captured step replayed with other masks, lengths and queries, and the program's own work between."""
    import paper_2607_21475_amd as ebd

    g, rng = _gen(2), random.Random(2)
    news, G, kv = [9, 14], 4, 2
    c = ref.Cache([800, 350], kv, 16, g)
    off = torch.tensor([0, 9, 23], device="cuda")
    q = ref.spaced((23, 8, 128), g, False)
    y, lse = torch.empty_like(q), torch.empty((23, 8), device="cuda")
    mask = torch.zeros((23, 1), dtype=torch.int64, device="cuda")
    pos = torch.zeros(23, dtype=torch.int32, device="cuda")
    p = ebd.attend_tree_params(ebd.pages(c.K, c.V, c.table), q, y, off, c.len, 14, 800, mask, qpos=pos, window=300)
    ws = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_TREE, p))

    def renew(i):
        c.lens = [800 - 37 * i, 350 - 11 * i]
        c.len.copy_(torch.tensor(c.lens))
        words, at = [], []
        for n, m in zip(c.lens, news):
            a, d = step.masks_of(step.tree(m, rng), 1)
            words += a
            at += [n - m + x for x in d]
        mask.copy_(torch.tensor(words))
        pos.copy_(torch.tensor(at))
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        return words, at

    renew(0)
    ebd.ebd_attend_tree(p, q, c.K, c.V, y, ws, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ebd.ebd_attend_tree(p, q, c.K, c.V, y, ws, lse=lse)
    for i in range(1, 5):
        words, at = renew(i)
        y.fill_(7)
        ws.fill_(255)
        graph.replay()
        got = y.clone(), lse.clone()
        torch.cuda.synchronize()
        _check(c, news, G, words, at, q, y, lse, window=300)
        ebd.ebd_attend_tree(p, q, c.K, c.V, y, ws, lse=lse)
        assert torch.equal(got[0], y) and torch.equal(got[1], lse)
    outs = [(torch.empty_like(y), ebd.workspace(ws.numel()), torch.cuda.Stream()) for _ in range(2)]
    torch.cuda.synchronize()
    for o, w, s in outs * 5:
        with torch.cuda.stream(s):
            ebd.ebd_attend_tree(p, q, c.K, c.V, o, w)
    torch.cuda.synchronize()
    assert all(torch.equal(o, y) for o, _, _ in outs)


@pytest.mark.parametrize("held,news,kv,G,window", [
    ([70, 9, 300], [5, 0, 3], 2, 4, 0), ([500, 20], [3, 1], 1, 40, 0), ([64, 0, 17, 900], [0, 4, 0, 90], 1, 33, 50),
    ([3, 2000], [1, 40], 2, 17, 0), ([0] * 40, [s % 3 for s in range(40)], 2, 4, 0), ([10] * 3, [0, 0, 0], 2, 4, 0),
])
def test_tree_many_heads_and_sequences_without_tokens(held, news, kv, G, window):
    rng = random.Random(sum(held) + G)
    lens = [h + m for h, m in zip(held, news)]
    c = ref.Cache(lens, kv, 16, _gen(G))
    words = max(1, -(-max(news) // 64))
    mask, pos = [], []
    for h, m in zip(held, news):
        a, d = step.masks_of(step.tree(m, rng), words)
        mask += a
        pos += [h + x for x in d]
    if not mask:  # padding tokens alone
        q, y, lse, st = _none(c, news, G)
        assert bool((y == 7).all()) and bool((lse == 7).all()) and not bool(st.any())
        return
    q, y, lse, st = _call(c, news, G, mask, pos, window=window, pad=1)
    assert not bool(st.any())
    _check(c, news, G, mask, pos, q, y, lse, window, few=6)


def _none(c, news, G):
    import paper_2607_21475_amd as ebd

    q = ref.spaced((2, c.kv * G, 128), _gen(1), False)
    y, lse = torch.full_like(q, 7.0), torch.full((2, c.kv * G), 7.0, device="cuda")
    off = torch.zeros(len(news) + 1, dtype=torch.int64, device="cuda")
    st = torch.zeros(len(news), dtype=torch.int32, device="cuda")
    p = ebd.attend_tree_params(ebd.pages(c.K, c.V, c.table), q, y, off, c.len, 4, max(c.lens),
                               torch.full((2, 1), -1, dtype=torch.int64, device="cuda"))
    ws = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_TREE, p))
    ebd.ebd_attend_tree(p, q, c.K, c.V, y, ws, lse=lse, status=st)
    return q, y, lse, st


@pytest.mark.parametrize("seqs,new,least,context,kv,G,window", [
    (24, 40, 40, 600, 8, 4, 0),     # blocks of 256 query rows, 160 of them taken
    (12, 64, 0, 3000, 8, 4, 0),     # token counts down to none, over 0 to 3000 rows
    (6, 100, 1, 2500, 4, 4, 0),
    (20, 55, 0, 700, 2, 7, 90),
    (40, 70, 1, 300, 4, 2, 0),
    (3, 200, 1, 5000, 1, 4, 2000),
])
def test_tree_batches_of_different_lengths(seqs, new, least, context, kv, G, window):
    rng = random.Random(seqs + new)
    held = [context] + [rng.randrange(context) for _ in range(seqs - 2)] + [0]
    news = [new] + [rng.randint(least, new) for _ in range(seqs - 2)] + [least]
    if least < new:
        news[1:seqs - 1] = [m * m // new for m in news[1:seqs - 1]]  # few tokens for most
    lens = [h + m for h, m in zip(held, news)]
    c = ref.Cache(lens, kv, 16, _gen(seqs), fill=math.nan)
    words = -(-new // 64)
    mask, pos = [], []
    for h, m in zip(held, news):
        a, d = step.masks_of(step.tree(m, rng), words)
        mask += a
        pos += [h + x for x in d]
    q, y, lse, st = _call(c, news, G, mask, pos, window=window, pad=3)
    assert not bool(st.any())
    assert bool((y[sum(news):] == 7).all()) and bool((lse[sum(news):] == 7).all())
    _check(c, news, G, mask, pos, q, y, lse, window, few=3 if seqs * kv > 100 else 6)
