"""Plans of deep trees on the GPU: prompts and drafts that are chains, alone and beside small trees."""
import random

import pytest

import step_ref as step
from test_gpu_plan import _check, _run, _server

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("chains,width,trees,words", [
    ([4096], 1, 0, 64), ([4096], 3, 0, 64), ([700, 65, 1000], 1, 40, 16), ([1500, 64, 900], 1, 150, 24), ([4096, 4100], 1, 200, 64),
])
def test_plan_of_chains(chains, width, trees, words):
    """One launch for up to 128 sequences and 4096 tokens, three otherwise; tokens past the masks' words among them."""
    print("plan of chains", chains, width, trees, words, flush=True)
    rng = random.Random(sum(chains) + trees)
    count = chains + [rng.randint(0, 9) for _ in range(trees)]
    if trees and sum(count) > 4096 and trees < 100:
        raise ValueError("for one launch")
    parents = [step.chains(m, width) for m in chains] + [step.tree(m, rng) for m in count[len(chains):]]
    order = list(range(len(count)))
    rng.shuffle(order)
    count, parents = [count[i] for i in order], [parents[i] for i in order]
    lens = [rng.randint(0, 60) for _ in count]
    page = 32
    P = (60 + max(count)) // page + 2
    table, ring, state = _server(rng, lens, page, P, sum(-(-m // page) + 1 for m in count))
    parent = [x for p in parents for x in p]
    room = len(parent) + (0 if len(count) == 1 else 3)
    want = step.plan(count, lens, table, page, ring, state, room, parent, words)
    t, _, _ = _run(count, lens, table, page, ring, state, room, parent, words)
    _check(t, want)
