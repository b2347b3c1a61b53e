"""The rows of accepted paths moved together on the GPU, against the definition."""
import random

import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _want(c, news, paths):
    """The pools after the move, by the definition (all rows read before any is written)."""
    K, V = c.K.clone(), c.V.clone()
    P, N = c.table.shape[1], c.K.shape[0]
    for s, (m, path) in enumerate(zip(news, paths)):
        first = c.lens[s] - m

        def place(r):
            pg = int(c.table[s, r // c.page]) if 0 <= r < P * c.page else -1  # noqa: B023
            return (pg, r % c.page) if 0 <= pg < N else None

        for i, a in enumerate(path):
            x, y = place(first + a), place(first + i)
            if a != i and x and y:
                for new, old in ((K, c.K), (V, c.V)):
                    new[y[0], :, y[1]] = old[x[0], :, x[1]]
    return K, V


def _call(c, news, paths, most, out=True, kept=None):
    import paper_2607_21475_amd as ebd

    off = torch.tensor([0] + [sum(news[:i + 1]) for i in range(len(news))], device="cuda")
    path = torch.full((len(news), most), -9, dtype=torch.int32)
    for s, p in enumerate(paths):
        path[s, :len(p)] = torch.tensor(p, dtype=torch.int32)
    kept = torch.tensor([len(p) for p in paths] if kept is None else kept, dtype=torch.int32, device="cuda")
    st = torch.full((len(news),), 64, dtype=torch.int32, device="cuda")
    new_len = torch.full((len(news),), 7, dtype=torch.int32, device="cuda") if out else None
    p = ebd.keep_rows_params(ebd.pages(c.K, c.V, c.table), off, c.len, path.cuda(), kept, len_out=new_len)
    ebd.ebd_keep_rows(p, c.K, c.V, status=st)
    return st, new_len


def _path(n, kept, rng):
    return sorted(rng.sample(range(n), kept))


@pytest.mark.parametrize("held,news,kv,page,order,most", [
    ([0], [1], 1, 16, "heads", 1), ([100], [26], 8, 16, "heads", 6), ([5, 0, 31, 64], [8, 60, 7, 0], 2, 32, "tokens", 16),
    ([3], [700], 1, 16, "heads", 650), ([40, 41, 42], [9, 9, 9], 17, 64, "tokens", 9),
    ([7 + s for s in range(300)], [s % 20 for s in range(300)], 2, 16, "heads", 12), ([12, 1], [5, 4], 300, 16, "heads", 4),
])
def test_keep(held, news, kv, page, order, most):
    print("keep", held[:4], news[:4], kv, page, order, most, flush=True)
    rng = random.Random(sum(held) + most)
    c = ref.Cache([h + m for h, m in zip(held, news)], kv, page, _gen(most), order)
    for full in (False, True):
        paths = [_path(m, min(m, most) if full else rng.randint(0, min(m, most)), rng) for m in news]
        K, V = _want(c, news, paths)
        st, new_len = _call(c, news, paths, most)
        assert bool((st == 64).all())
        assert torch.equal(c.K, K) and torch.equal(c.V, V)
        assert new_len.tolist() == [h + len(p) for h, p in zip(held, paths)]


def test_keep_overlapping_rows():
    """Paths that shift everything by one, or keep a token far behind: rows are read before they are written over."""
    c = ref.Cache([40 + 600, 30 + 40], 2, 16, _gen(1))
    news, paths = [600, 40], [list(range(1, 600)), [0, 1, 2] + list(range(20, 40))]
    K, V = _want(c, news, paths)
    st, _ = _call(c, news, paths, 600, out=False)
    assert bool((st == 64).all()) and torch.equal(c.K, K) and torch.equal(c.V, V)


def test_keep_paths_out_of_place():
    """Nothing moves for a sequence whose path or count is wrong; the others' rows do."""
    import paper_2607_21475_amd as ebd

    news = [6] * 9
    paths = [[1, 3], [3, 1], [2, 2], [0, 6], [-1, 2], [1, 3], [1, 3], [0, 2, 5], [2 ** 31 - 1]]
    kept = [2, 2, 2, 2, 2, -1, 5, 3, 1]  # (5: of four places)
    c = ref.Cache([26] * 9, 2, 16, _gen(2))
    c.len[7] = 3  # fewer rows than new tokens
    right = [p if s == 0 else [] for s, p in enumerate(paths)]
    K, V = _want(c, news, right)
    st, new_len = _call(c, news, [p[:4] for p in paths], 4, kept=kept)
    assert st.tolist() == [64] + [64 | ebd.EBD_ST_BAD_LAYOUT] * 8
    assert torch.equal(c.K, K) and torch.equal(c.V, V)
    assert new_len.tolist() == [22] + [26] * 6 + [3, 26]


def test_keep_rows_without_a_page():
    import paper_2607_21475_amd as ebd

    c = ref.Cache([30 + 20, 30 + 20, 30 + 20, 30 + 20], 2, 16, _gen(3))
    c.table[0, 2] = -1          # rows 32 .. 47
    c.table[1, 3] = 1 << 20     # rows 48, 49
    c.table = c.table[:, :4].contiguous()
    news, paths = [20] * 4, [[3, 5, 18, 19], [0, 18, 19], [1, 4], [0, 1, 2]]
    c.lens = [50, 50, 50, 50]
    K, V = _want(c, news, paths)
    st, new_len = _call(c, news, paths, 4)
    flag = 64 | ebd.EBD_ST_BAD_PAGE
    assert st.tolist() == [flag, flag, 64, 64]
    assert torch.equal(c.K, K) and torch.equal(c.V, V) and new_len.tolist() == [34, 33, 32, 33]


def test_keep_into_the_lengths_and_in_a_graph():
    """len_out is len: each replay keeps a path of what the program appended between."""
    import paper_2607_21475_amd as ebd

    rng = random.Random(4)
    news = [12, 9, 5]
    c = ref.Cache([40 + m + 60 for m in news], 2, 16, _gen(4))
    off = torch.tensor([0, 12, 21, 26], device="cuda")
    path = torch.zeros((3, 5), dtype=torch.int32, device="cuda")
    kept = torch.zeros(3, dtype=torch.int32, device="cuda")
    p = ebd.keep_rows_params(ebd.pages(c.K, c.V, c.table), off, c.len, path, kept, len_out=c.len)
    ebd.ebd_keep_rows(p, c.K, c.V)
    assert c.len.tolist() == [n - m for n, m in zip(c.lens, news)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ebd.ebd_keep_rows(p, c.K, c.V)
    held = [40, 40, 40]
    for _ in range(4):
        c.lens = [h + m for h, m in zip(held, news)]
        c.len.copy_(torch.tensor(c.lens))
        paths = [_path(m, rng.randint(0, 5), rng) for m in news]
        for s, q in enumerate(paths):
            path[s, :len(q)] = torch.tensor(q, dtype=torch.int32, device="cuda")
        kept.copy_(torch.tensor([len(q) for q in paths]))
        torch.cuda.synchronize()
        K, V = _want(c, news, paths)
        graph.replay()
        held = [h + len(q) for h, q in zip(held, paths)]
        assert torch.equal(c.K, K) and torch.equal(c.V, V) and c.len.tolist() == held
