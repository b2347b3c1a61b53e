"""Attention of drafted trees on the GPU by every shape of its kernels: values that are all alike."""
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
