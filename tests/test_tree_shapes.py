"""CPU check of the attention of drafted trees: the batches that its GPU tests run for each kernel shape are planned for it."""
import os

import pytest

import tree_shapes
from paper_2607_21475_amd import build


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not installed")
    return tree_shapes.planner(str(tmp_path_factory.mktemp("plan")))


@pytest.mark.parametrize("name", tree_shapes.BATCHES)
def test_batches_have_their_shapes(planner, name):
    news, held, kv, G, window, shape, split = tree_shapes.BATCHES[name]
    for pad in (0, 2):
        (rows, pairs, nsplit), *others = planner(tree_shapes.params(news, held, kv, G, window, pad=pad))
        assert not others and (rows, pairs) == shape and (nsplit > 1) == split, (rows, pairs, nsplit)
    new, rows = tree_shapes.bounds(name)
    for kw in (dict(max_new=new), dict(max_rows=rows)):
        (rows, pairs, nsplit), *others = planner(tree_shapes.params(news, held, kv, G, window, **kw))
        assert not others and (rows, pairs) == shape and (nsplit > 1) == split, (kw, rows, pairs, nsplit)
