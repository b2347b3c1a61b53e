"""Plans of a serving step on the GPU, against the definition: every whole number has to be the same."""
import random

import pytest
import torch

import step_ref as step

pytestmark = pytest.mark.gpu
I32 = torch.int32


def _server(rng, held, page, P, spare, holes=0.0):
    """(table, ring, state) of sequences that hold these rows; some entries name no page of the pool."""
    used = [-(-n // page) for n in held]
    N = sum(used) + spare
    ids = list(range(N))
    rng.shuffle(ids)
    table, at = [], 0
    for u in used:
        row = ids[at:at + u] + [rng.choice([-1, -1, N, N + 7, -2 ** 31, 2 ** 31 - 1]) for _ in range(P - u)]
        table.append([-1 if rng.random() < holes else x for x in row])
        at += u
    head = rng.randrange(N)
    ring = [-5] * N
    for i, x in enumerate(ids[at:]):
        ring[(head + i) % N] = x
    return table, ring, [head, N - at]


def _run(count, lens, table, page, ring, state, room, parent=None, words=0, want_slots=True, want_pos=True):
    import paper_2607_21475_amd as ebd

    dev = dict(device="cuda")
    t = {"count": torch.tensor(count, dtype=I32, **dev), "len": torch.tensor(lens, dtype=I32, **dev),
         "table": torch.tensor(table, dtype=I32, **dev).view(len(lens), -1 if lens else 4), "ring": torch.tensor(ring, dtype=I32, **dev),
         "state": torch.tensor(state, dtype=I32, **dev), "new_off": torch.full((len(lens) + 1,), 7, **dev)}
    t["slots"] = torch.full((room,), 7, **dev) if want_slots else None
    t["pos"] = torch.full((room,), 7, dtype=I32, **dev) if want_pos else None
    t["parent"] = t["mask"] = None
    if parent is not None:
        t["parent"] = torch.tensor(parent + [9] * (room - len(parent)), dtype=I32, **dev)
        t["mask"] = torch.full((room, words), 7, **dev)
    t["status"] = torch.full((len(lens),), 64, dtype=I32, **dev)
    p = ebd.plan_step_params(t["count"], t["len"], t["table"], page, t["ring"], t["state"], t["new_off"], slots=t["slots"],
                             pos=t["pos"], parent=t["parent"], mask=t["mask"])
    ws = ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_PLAN_STEP, p))
    ws.fill_(255)
    ebd.ebd_plan_step(p, ws, status=t["status"])
    return t, p, ws


def _check(t, want):
    for name in ("len", "table", "ring", "state", "new_off", "slots", "pos"):
        if t[name] is not None:
            assert t[name].tolist() == want[name], name
    if t["mask"] is not None:
        assert t["mask"].tolist() == want["mask"]
    assert t["status"].tolist() == [64 | x for x in want["status"]]


CASES = [
    # sequences, most rows held, most new tokens, page, spare pages, tree, mask words, ended, holes
    (1, 0, 1, 16, 3, False, 0, 0, 0), (1, 100, 64, 16, 9, True, 1, 0, 0), (1, 5, 4096, 16, 300, False, 0, 0, 0),
    (1, 3, 4096, 32, 140, True, 64, 0, 0), (5, 40, 7, 16, 20, True, 2, 1, 0.2), (64, 4000, 1, 16, 70, False, 0, 0, 0),
    (63, 900, 66, 64, 200, True, 2, 9, 0.1), (300, 200, 3, 16, 400, False, 0, 40, 0), (257, 70, 61, 16, 1500, True, 1, 17, 0),
    (1000, 64, 5, 16, 900, True, 1, 100, 0), (700, 300, 1, 128, 800, False, 0, 0, 0.05), (40, 9000, 700, 16, 2100, False, 0, 5, 0),
    (4100, 20, 2, 16, 5000, False, 0, 50, 0), (65536, 3, 1, 16, 9000, False, 0, 300, 0), (33, 2, 300, 16, 900, True, 5, 0, 0),
]


@pytest.mark.parametrize("seqs,held,new,page,spare,tree,words,ended,holes", CASES)
def test_plan(seqs, held, new, page, spare, tree, words, ended, holes):
    print("plan", seqs, held, new, page, spare, tree, words, ended, holes, flush=True)
    rng = random.Random(seqs * 31 + new)
    lens = [rng.randint(0, held) for _ in range(seqs)]
    count = [rng.randint(0 if seqs > 1 else new, new) for _ in range(seqs)]
    for s in rng.sample(range(seqs), ended):
        count[s] = rng.choice([-1, -7, -2 ** 31])
    P = (held + new) // page + 2
    table, ring, state = _server(rng, lens, page, P, spare, holes)
    parent = [x for n in count for x in step.tree(max(n, 0), rng)] if tree else None
    room = sum(max(n, 0) for n in count) + rng.randint(0, 5)
    want = step.plan(count, lens, table, page, ring, state, room, parent, words)
    t, p, ws = _run(count, lens, table, page, ring, state, room, parent, words)
    _check(t, want)


def test_plan_steps_one_after_another():
    """A server's life on one set of buffers: sequences come, decode, draft, fall back, end and come again; the pages held
    and free are a partition of the pool after every step."""
    import paper_2607_21475_amd as ebd

    rng = random.Random(3)
    S, page, P, N = 20, 16, 12, 40
    lens, table, ring, state = [0] * S, [[-1] * P for _ in range(S)], list(range(N)), [0, N]
    count = [rng.randint(0, 40) for _ in range(S)]
    t, p, ws = _run(count, lens, table, page, ring, state, 900)
    full = 0
    for i in range(60):
        want = step.plan(count, lens, table, page, ring, state, 900)
        _check(t, want)
        lens, table, ring, state = want["len"], want["table"], want["ring"], want["state"]
        full += any(want["status"])
        held = [x for r in table for x in r if x >= 0]
        free = [ring[(state[0] + k) % N] for k in range(state[1])]
        assert sorted(held + free) == list(range(N))
        lens = [max(n - rng.randint(0, 3), 0) for n in lens]  # drafted tokens that were not kept
        count = [rng.choice([-1, 0, 1, 1, rng.randint(0, 30)]) if n < 100 else -1 for n in lens]
        t["len"].copy_(torch.tensor(lens, dtype=I32))
        t["count"].copy_(torch.tensor(count, dtype=I32))
        t["status"].fill_(64)
        ebd.ebd_plan_step(p, ws, status=t["status"])
    assert full > 0  # the pool was too small now and then


@pytest.mark.parametrize("seqs", [3, 600])
def test_plan_where_something_is_missing(seqs):
    """Too few pages, tables too short, too little room, parents out of place, masks too short, rows past 2^30, lengths
    below zero, a ring that cannot be."""
    rng = random.Random(seqs)
    pad = [1] * (seqs - 3)
    lens, page = [30, -4, 7] + [17] * (seqs - 3), 16
    table, ring, state = _server(rng, [max(n, 0) for n in lens], page, 6, 4)
    count, room = [40, 70, 20] + pad, 130 + seqs
    parent = [x for n in count for x in step.tree(n, rng)]
    parent[3], parent[41], parent[45], parent[110] = 3, 2 ** 31 - 1, -2, -2 ** 31
    for kw in (dict(), dict(parent=parent, words=1)):
        _check(_run(count, lens, table, page, ring, state, room, **kw)[0],
               step.plan(count, lens, table, page, ring, state, room, **kw))
    cut = dict(room=50)
    _check(_run(count, lens, table, page, ring, state, **cut)[0], step.plan(count, lens, table, page, ring, state, **cut))
    cut = dict(room=90, parent=parent[:90], words=2)
    _check(_run(count, lens, table, page, ring, state, **cut)[0], step.plan(count, lens, table, page, ring, state, **cut))
    for bad in ([-1, 2], [len(ring), 1], [0, -1], [0, len(ring) + 1]):
        _check(_run(count, lens, table, page, ring, bad, room)[0], step.plan(count, lens, table, page, ring, bad, room))
    lens[0], count[0], count[1] = 2 ** 30 - 1, 2, 2 ** 31 - 1
    _check(_run(count, lens, table, page, ring, state, room)[0], step.plan(count, lens, table, page, ring, state, room))


def test_plan_without_some_outputs():
    rng = random.Random(8)
    lens, count = [20, 3], [5, 30]
    table, ring, state = _server(rng, lens, 16, 5, 4)
    parent = step.tree(5, rng) + step.chains(30, 3)
    want = step.plan(count, lens, table, 16, ring, state, 35)
    trees = step.plan(count, lens, table, 16, ring, state, 35, parent, 1)
    for kw in (dict(want_slots=False), dict(want_pos=False)):
        _check(_run(count, lens, table, 16, ring, state, 35, **kw)[0], want)
        _check(_run(count, lens, table, 16, ring, state, 35, parent, 1, **kw)[0], trees)
    t = _run(count, lens, table, 16, ring, state, 0, want_slots=False, want_pos=False)[0]
    _check(t, want)


@pytest.mark.parametrize("seqs,new,tree", [(9, 40, True), (900, 6, False)])
def test_plan_in_a_graph(seqs, new, tree):
    """A captured step replayed, with other counts and the program's own work between."""
    import paper_2607_21475_amd as ebd

    rng = random.Random(seqs)
    lens = [rng.randint(0, 90) for _ in range(seqs)]
    table, ring, state = _server(rng, lens, 16, 40, 30 * seqs)
    room = seqs * new
    make = lambda: [rng.choice([rng.randint(0, new), rng.randint(0, new), -1]) for _ in range(seqs)]  # noqa: E731
    count = make()
    parents = lambda: [x for n in count for x in step.tree(max(n, 0), rng)] if tree else None  # noqa: E731
    parent = parents()
    t, p, ws = _run(count, lens, table, 16, ring, state, room, parent, 1)
    want = step.plan(count, lens, table, 16, ring, state, room, parent, 1)
    _check(t, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ebd.ebd_plan_step(p, ws, status=t["status"])
    for _ in range(4):
        count = make()
        parent = parents()
        t["count"].copy_(torch.tensor(count, dtype=I32))
        if tree:
            t["parent"].fill_(9)
            t["parent"][:len(parent)] = torch.tensor(parent, dtype=I32, device="cuda")
        t["status"].fill_(64)
        ws.fill_(255)
        torch.cuda.synchronize()
        before = [want[k] for k in ("len", "table", "ring", "state")]
        graph.replay()
        want = step.plan(count, before[0], before[1], 16, before[2], before[3], room, parent, 1)
        _check(t, want)


@pytest.mark.parametrize("seqs", [4, 300])
def test_plan_from_a_ring_of_bad_pages(seqs):
    """Numbers outside the pool among the free pages: taken in their turn, and flagged."""
    rng = random.Random(seqs)
    lens, count = [rng.randint(0, 40) for _ in range(seqs)], [rng.randint(0, 50) for _ in range(seqs)]
    table, ring, state = _server(rng, lens, 16, 7, 4 * seqs)
    for i in range(0, state[1], 3):
        ring[(state[0] + i) % len(ring)] = rng.choice([-1, len(ring), 2 ** 31 - 1])
    want = step.plan(count, lens, table, 16, ring, state, 50 * seqs)
    assert 0 < sum(x > 0 for x in want["status"])
    _check(_run(count, lens, table, 16, ring, state, 50 * seqs)[0], want)


@pytest.mark.parametrize("room", [3, 5000])
def test_plan_without_sequences(room):
    """Every token is padding then: nothing may be left of what slots, positions and masks held."""
    for parent, words in ((None, 0), ([], 2)):
        t = _run([], [], torch.zeros((0, 4), dtype=I32).tolist(), 16, [3, 4, 5], [1, 2], room, parent, words)[0]
        assert t["new_off"].tolist() == [0] and t["state"].tolist() == [1, 2] and t["ring"].tolist() == [3, 4, 5]
        assert bool((t["slots"] == -1).all()) and bool((t["pos"] == -1).all())
        assert words == 0 or bool((t["mask"] == 0).all())
