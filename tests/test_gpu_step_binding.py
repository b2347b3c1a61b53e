"""Calls of a step through the binding on the GPU that the other tests do not make."""
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


def test_one_row_of_weights_expanded_over_the_heads():
    """The forward call takes it; its gradient is that of the row, which the gradients' call asks for."""
    import paper_2607_21475_amd as ebd

    g = _gen(3)
    x, dy = ref.spaced((19, 5, 128), g, False), ref.spaced((19, 5, 128), g, False)
    row = 1 + 0.3 * torch.randn(128, generator=g, device="cuda")
    wide = ebd.head_norm(row.expand(5, 128), EPS)
    y = torch.empty_like(x)
    ebd.ebd_norm_rope(ebd.norm_rope_params(x, y, wide), x, y)
    ref.check(y, *step.norm_rope(x, row, EPS, None, None), "y")
    dx = torch.empty_like(x)
    with pytest.raises(ValueError, match="expanded"):
        ebd.norm_rope_backward_params(x, dy, dx, wide)
    p = ebd.norm_rope_backward_params(x, dy, dx, ebd.head_norm(row, EPS))
    dw = torch.full((128,), 7.0, device="cuda")
    ebd.ebd_norm_rope_backward(p, x, dy, dx, dw, ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_NORM_ROPE_BACKWARD, p)))
    (rx, tx), (rw, tw) = step.norm_rope_gradients(x, row, EPS, dy, None, None)
    ref.check(dx, rx, tx, "dx")
    ref.check(dw, rw, tw, "dw")


def test_layers_that_share_a_plan():
    """Three layers of pools of their own and one table and len: a step planned once, appended, attended to and kept in each;
    every layer's rows are then those of the accepted paths."""
    import random

    import paper_2607_21475_amd as ebd

    g, rng = _gen(8), random.Random(8)
    S, kv, G, page = 3, 2, 2, 16
    layers = [ebd.PagedCache.pool(S, 30, kv, page, max_pages=8)]
    for _ in range(2):
        a = layers[0]
        layers.append(ebd.PagedCache(torch.empty_like(a.K), torch.empty_like(a.V), a.page_table, a.len))
    held = [[[] for _ in range(S)] for _ in layers]  # (K, V) of each row
    for count in ([20, 33, 5], [9, 12, 7], [4, 1, 17]):
        trees = [step.tree(m, rng) for m in count]
        parent = torch.tensor([x for t in trees for x in t], dtype=torch.int32, device="cuda")
        st = torch.zeros(S, dtype=torch.int32, device="cuda")
        new = layers[0].plan(torch.tensor(count, dtype=torch.int32, device="cuda"), sum(count), parent=parent, status=st)
        paths = [sorted(rng.sample(range(m), rng.randint(1, m))) for m in count]
        path = torch.zeros((S, max(len(x) for x in paths)), dtype=torch.int32)
        for s, x in enumerate(paths):
            path[s, :len(x)] = torch.tensor(x, dtype=torch.int32)
        kept = torch.tensor([len(x) for x in paths], dtype=torch.int32, device="cuda")
        for i, c in enumerate(layers):
            k, v, q = (ref.spaced((sum(count), h, 128), g, False) for h in (kv, kv, kv * G))
            c.append(k, v, new["new_off"], q=q, slots=new["slots"], status=st)
            c.attend_tree(q, new["new_off"], max(count), 8 * page, new["mask"], qpos=new["pos"], status=st)
            c.keep(new["new_off"], path.cuda(), kept, status=st, update_len=i == len(layers) - 1)
            t0 = 0
            for s, m in enumerate(count):
                held[i][s] += [(k[t0 + j], v[t0 + j]) for j in paths[s]]
                t0 += m
        assert not bool(st.any()) and layers[0].len.tolist() == [len(h) for h in held[0]]
        for c, rows in zip(layers, held):
            K, V, so = c.gather([len(h) for h in rows])
            for s in range(S):
                for h in range(kv):
                    a, b = int(so[s * kv + h]), int(so[s * kv + h + 1])
                    assert torch.equal(K[a:b], torch.stack([x[0][h] for x in rows[s]]))
                    assert torch.equal(V[a:b], torch.stack([x[1][h] for x in rows[s]]))
