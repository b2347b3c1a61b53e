"""The operators of a speculative serving step together, as a server uses them."""
import math
import random

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


class _View:
    """What step_ref.attend_row reads of a cache."""

    def __init__(self, c):
        self.K, self.V, self.table, self.page = c.K, c.V, c.page_table, c.K.shape[2]


def _accept(parents, rng, most):
    """A path from the root down a tree."""
    path, at = [], -1
    while len(path) < most:
        down = [j for j, up in enumerate(parents) if up == at]
        if not down or rng.random() < 0.2:
            break
        at = rng.choice(down)
        path.append(at)
    return path


def test_a_server_that_drafts():
    """Prompts, drafted trees of which a path is kept, sequences that end and come again: every step's attention against
    the formula over the rows that the cache should hold, and these rows read out and evicted at the end."""
    import paper_2607_21475_amd as ebd
    from paper_2607_21475_amd import cache as ec

    rng, g = random.Random(6), _gen(6)
    S, kv, G, page, most = 5, 2, 3, 16, 6
    c = ebd.PagedCache.pool(S, 60, kv, page, max_pages=20)
    f = step.frequencies(96)
    rot = ebd.rotary(f)
    wk, wq = 1 + 0.2 * torch.randn(kv, 128, generator=g, device="cuda"), 1 + 0.2 * torch.randn(128, generator=g, device="cuda")
    k_norm, q_norm = ebd.head_norm(wk, EPS), ebd.head_norm(wq, EPS)
    view = _View(c)
    held = [[] for _ in range(S)]  # what each sequence's rows are: (K, its tolerance, V) of each
    ws = {"plan": None, "tree": None}
    for turn in range(9):
        prompt = turn == 0 or turn == 5
        count = [rng.randint(30, 90) if prompt and not h else rng.randint(1, 20) for h in held]
        if turn == 4:
            count[1] = count[3] = -1
        trees = [step.chains(m, 1) if prompt and not h else step.tree(max(m, 0), rng) for m, h in zip(count, held)]
        T = sum(max(m, 0) for m in count) + 2
        parent = torch.tensor([x for t in trees for x in t] + [5, 5], dtype=torch.int32, device="cuda")
        st = torch.zeros(S, dtype=torch.int32, device="cuda")
        new = c.plan(torch.tensor(count, dtype=torch.int32, device="cuda"), T, parent=parent, mask_words=2, ws=ws["plan"],
                     status=st)
        ws["plan"] = new["ws"]
        for s, m in enumerate(count):
            if m < 0:
                held[s] = []
        k, v, q = (ref.spaced((T, h, 128), g, True) for h in (kv, kv, kv * G))
        # by slots, and by the sequences' rows: the same
        qr = c.append(k, v, new["new_off"], rot, pos=new["pos"], q=q, k_norm=k_norm, q_norm=q_norm,
                      slots=new["slots"] if turn % 2 else None, status=st)
        out = c.attend_tree(qr, new["new_off"], max(count), 320, new["mask"], qpos=new["pos"], window=70, ws=ws["tree"], status=st)
        ws["tree"] = out["ws"]
        assert not bool(st.any())
        # against the formula
        pos, mask = new["pos"].tolist(), new["mask"].tolist()
        ky, kt = step.norm_rope(k, wk, EPS, new["pos"], f)
        qy, qt = step.norm_rope(q, wq, EPS, new["pos"], f)
        ref.check(qr[:-2], qy[:-2], qt[:-2], "q")
        assert bool((qr[-2:] == 0).all()) and bool((out["y"][-2:] == 0).all()) and bool((out["lse"][-2:] == -math.inf).all())
        t0, paths = 0, []
        for s, m in enumerate(count):
            m = max(m, 0)
            first = len(held[s])
            for j in range(0, m, 1 if m < 10 else 7):
                words, depth = step.masks_of(trees[s], 2)
                assert pos[t0 + j] == first + depth[j] and mask[t0 + j] == words[j]
                rows = step.sees(first, first + m, None, mask[t0 + j], pos[t0 + j], 70)
                for h in range(kv):
                    a = slice(h * G, h * G + G)
                    ry, rl, ty, tl = step.attend_row(view, s, h, qr[t0 + j, a], rows, None, 8)
                    ref.check(out["y"][t0 + j, a], ry, ty, "y")
                    ref.check(out["lse"][t0 + j, a], rl, tl, "lse")
            path = list(range(m)) if prompt and not first else _accept(trees[s], rng, most)
            paths.append(path)
            held[s] += [(ky[t0 + j], kt[t0 + j], v[t0 + j]) for j in path]
            t0 += m
        longest = max(len(p) for p in paths)
        path = torch.zeros((S, max(longest, 1)), dtype=torch.int32)
        for s, p in enumerate(paths):
            path[s, :len(p)] = torch.tensor(p, dtype=torch.int32)
        c.keep(new["new_off"], path.cuda(), torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda"), status=st)
        assert not bool(st.any()) and c.len.tolist() == [len(h) for h in held]
    sizes = [len(h) for h in held]
    K, V, so = c.gather(sizes)
    assert min(sizes) > 20
    for s in range(S):
        for h in range(kv):
            a, b = int(so[s * kv + h]), int(so[s * kv + h + 1])
            ref.check(K[a:b], torch.stack([x[0][h] for x in held[s]]), torch.stack([x[1][h] for x in held[s]]), "K")
            assert torch.equal(V[a:b], torch.stack([x[2][h] for x in held[s]]))
    units = [n for n in sizes for _ in range(kv)]
    qd = ref.spaced((S * kv, G, 128), g, False)
    sc, _ = ec.importance_scores(K, so, qd, max(units))
    kept = ec.evict(K, V, sc, so, units, budget_frac=0.5, n_sink=2, n_recent=8)
    res = ec.attend_certify(kept, qd)
    assert bool(torch.isfinite(res["y"]).all()) and bool((res["r"] >= 0).all())


def test_a_captured_step_and_its_eager_twin():
    """Plan, append, attention and the kept paths as one graph, replayed over steps of other counts, trees and paths; the
    same steps eagerly on a twin cache give the same bits, with the program's own work between."""
    import paper_2607_21475_amd as ebd

    rng, g = random.Random(9), _gen(9)
    S, kv, G, page, T, most = 7, 2, 4, 32, 7 * 12, 4
    f = step.frequencies(128)
    rot = ebd.rotary(f, ebd.EBD_ROPE_PAIRS)
    wk, wq = (1 + 0.2 * torch.randn(128, generator=g, device="cuda") for _ in range(2))
    k_norm, q_norm = ebd.head_norm(wk, EPS), ebd.head_norm(wq, EPS)
    dev = dict(device="cuda")
    count, kept = (torch.zeros(S, dtype=torch.int32, **dev) for _ in range(2))
    parent, path = torch.zeros(T, dtype=torch.int32, **dev), torch.zeros((S, most), dtype=torch.int32, **dev)
    k, v = (torch.zeros((T, kv, 128), dtype=BF, **dev) for _ in range(2))
    q = torch.zeros((T, kv * G, 128), dtype=BF, **dev)

    class Step:
        def __init__(self):
            c = self.c = ebd.PagedCache.pool(S, 90, kv, page, max_pages=16)
            c.K.zero_(), c.V.zero_()
            self.off, self.slots = torch.empty(S + 1, dtype=torch.int64, **dev), torch.empty(T, dtype=torch.int64, **dev)
            self.pos, self.mask = torch.empty(T, dtype=torch.int32, **dev), torch.empty((T, 1), dtype=torch.int64, **dev)
            self.qr, self.y, self.lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((T, kv * G), **dev)
            self.st = torch.zeros(S, dtype=torch.int32, **dev)
            self.plan = ebd.plan_step_params(count, c.len, c.page_table, page, c.free_pages, c.free_state, self.off,
                                             slots=self.slots, pos=self.pos, parent=parent, mask=self.mask)
            self.app = ebd.append_norm_params(c.pages, k, v, k_norm=k_norm, q_norm=q_norm, rot=rot, pos=self.pos, q=q,
                                              q_out=self.qr, slots=self.slots)
            self.att = ebd.attend_tree_params(c.pages, self.qr, self.y, self.off, c.len, 12, 16 * page, self.mask, qpos=self.pos)
            self.kept = ebd.keep_rows_params(c.pages, self.off, c.len, path, kept, len_out=c.len)
            self.w1 = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_PLAN_STEP, self.plan))
            self.w2 = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_TREE, self.att))

        def run(self):
            ebd.ebd_plan_step(self.plan, self.w1, status=self.st)
            ebd.ebd_append_norm(self.app, k, v, self.c.K, self.c.V, q, self.qr)
            ebd.ebd_attend_tree(self.att, self.qr, self.c.K, self.c.V, self.y, self.w2, lse=self.lse, status=self.st)
            ebd.ebd_keep_rows(self.kept, self.c.K, self.c.V, status=self.st)

        def state(self):
            c = self.c
            return [c.K, c.V, c.page_table, c.len, c.free_pages, c.free_state, self.off, self.slots, self.pos, self.mask,
                    self.qr, self.y, self.lse, self.st]

    a, b = Step(), Step()
    a.run(), b.run()  # (no tokens yet)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for i in range(8):
        n = [-1 if i == 5 and s % 3 == 0 else rng.randint(1, 12) for s in range(S)]
        trees = [step.tree(max(m, 0), rng) for m in n]
        count.copy_(torch.tensor(n, dtype=torch.int32))
        flat = [x for t in trees for x in t]
        parent[:len(flat)] = torch.tensor(flat, dtype=torch.int32, device="cuda")
        paths = [_accept(t, rng, most) for t in trees]
        kept.copy_(torch.tensor([len(x) for x in paths], dtype=torch.int32))
        path.zero_()
        for s, x in enumerate(paths):
            path[s, :len(x)] = torch.tensor(x, dtype=torch.int32, device="cuda")
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        for x in (a, b):
            x.y.fill_(7), x.lse.fill_(7), x.w1.fill_(255 - i), x.w2.fill_(i)
        torch.cuda.synchronize()
        graph.replay()
        b.run()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y), i
        assert not bool(a.st.any())
    assert int(a.c.len.sum()) > 20


def test_calls_on_another_device_or_before_their_tensors():
    """A call's tensors must be those its parameters were made for, and on the current device."""
    import paper_2607_21475_amd as ebd

    c = ebd.PagedCache.pool(2, 4, 1, 16)
    off = torch.tensor([0, 1, 2], device="cuda")
    q = torch.zeros((2, 2, 128), dtype=BF, device="cuda")
    mask = torch.ones((2, 1), dtype=torch.int64, device="cuda")
    p = ebd.attend_tree_params(c.pages, q, torch.empty_like(q), off, c.len, 1, 16, mask)
    ws = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_TREE, p))
    with pytest.raises(ValueError, match="shape and strides"):
        ebd.ebd_attend_tree(p, q[:1], c.K, c.V, torch.empty_like(q), ws)
    with pytest.raises(ValueError, match="must be on"):
        ebd.ebd_attend_tree(p, q.cpu(), c.K, c.V, torch.empty_like(q), ws)
    with pytest.raises(TypeError, match="workspace"):
        ebd.ebd_attend_tree(p, q, c.K, c.V, torch.empty_like(q), None)
    with pytest.raises(ValueError, match="mask"):
        ebd.attend_tree_params(c.pages, q, torch.empty_like(q), off, c.len, 1, 16, mask[:1])
    with pytest.raises(ValueError, match="on the GPU"):
        ebd.keep_rows_params(c.pages, off, c.len, torch.zeros((2, 1), dtype=torch.int32), c.len)
    with pytest.raises(ValueError, match="ring"):
        ebd.PagedCache.allocate([3], 1).plan(c.len[:1], 3)
