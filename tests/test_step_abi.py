"""CPU checks of the entry points of a serving step: bad arguments are refused before any device work."""
import ctypes

import pytest
import torch

import paper_2607_21475_amd as ebd
from paper_2607_21475_amd import paged

from test_paged_abi import BAD_PAGES, FAKE, _pages, _rot

LIB = ebd._lib
BAD, UNSUPPORTED, NO_WS, OK = ebd.EBD_ERR_INVALID_ARG, ebd.EBD_ERR_UNSUPPORTED, ebd.EBD_ERR_WORKSPACE, ebd.EBD_OK
ROWS = paged.ebd_rows(1024, 128)


def _norm(**kw):
    n = paged.ebd_norm()
    n.weight, n.head_stride, n.eps = FAKE, 128, 1e-6
    for k, v in kw.items():
        setattr(n, k, v)
    return n


BAD_NORMS = [dict(weight=FAKE + 8), dict(head_stride=64), dict(head_stride=130), dict(head_stride=-128),
             dict(head_stride=1 << 40), dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
             dict(eps=1e-40), dict(reserved=1)]


def _with(p, **kw):
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _norm_rope(x=FAKE, y=FAKE, **kw):
    p = paged.ebd_norm_rope_params()
    _with(p, num_tokens=4, num_heads=2, head_dim=128, pos=FAKE, rot=_rot(), norm=_norm(), x=ROWS, y=ROWS)
    return LIB.ebd_norm_rope(ctypes.byref(_with(p, **kw)), x, y, None)


def test_norm_rope_refusals():
    assert LIB.ebd_norm_rope(None, FAKE, FAKE, None) == BAD
    for kw in BAD_NORMS + [dict(weight=None)]:
        assert _norm_rope(norm=_norm(**kw)) == BAD, kw
    for kw in (dict(rot_dim=7), dict(layout=2), dict(flags=2), dict(amplitude=float("nan"))):
        assert _norm_rope(rot=_rot(**kw)) == BAD, kw
    for kw in (dict(num_tokens=-1), dict(num_heads=-1), dict(reserved=1), dict(pos=None)):
        assert _norm_rope(**kw) == BAD, kw
    for args in ((None, FAKE), (FAKE, None), (FAKE + 2, FAKE), (FAKE, FAKE + 8)):
        assert _norm_rope(*args) == BAD, args
    p = paged.ebd_norm_rope_params()
    _with(p, num_tokens=4, num_heads=2, head_dim=128, pos=FAKE, rot=_rot(), norm=_norm(), x=ROWS, y=paged.ebd_rows(-8, 128))
    assert LIB.ebd_norm_rope(ctypes.byref(p), FAKE, FAKE, None) == BAD
    assert _norm_rope(head_dim=64) == UNSUPPORTED and _norm_rope(num_tokens=1 << 24) == UNSUPPORTED
    assert _norm_rope(num_heads=1 << 17) == UNSUPPORTED
    assert _norm_rope(num_tokens=0) == OK and _norm_rope(num_heads=0) == OK


def _backward(args=None, ws=FAKE, ws_bytes=1 << 40, **kw):
    p = paged.ebd_norm_rope_backward_params()
    _with(p, num_tokens=4, num_heads=2, head_dim=128, pos=FAKE, rot=_rot(), norm=_norm(), x=ROWS, dy=ROWS, dx=ROWS)
    _with(p, **kw)
    a = [FAKE] * 4
    for i, v in (args or {}).items():
        a[i] = v
    size = LIB.ebd_workspace_size(ebd.EBD_WS_NORM_ROPE_BACKWARD, ctypes.byref(p))
    return LIB.ebd_norm_rope_backward(ctypes.byref(p), *a, ws, ws_bytes, None), size


def test_norm_rope_backward_refusals():
    for kw in BAD_NORMS + [dict(weight=None)]:
        assert _backward(norm=_norm(**kw)) == (BAD, 0), kw
    for kw in (dict(num_tokens=-1), dict(num_heads=-1), dict(reserved=1), dict(rot=_rot(rot_dim=130)),
               dict(x=paged.ebd_rows(4, 128)), dict(dy=paged.ebd_rows(1 << 40, 128)), dict(dx=paged.ebd_rows(8, -8))):
        assert _backward(**kw) == (BAD, 0), kw
    assert _backward(pos=None)[0] == BAD
    for i in range(4):
        assert _backward({i: None})[0] == BAD and _backward({i: FAKE + 2})[0] == BAD, i
    for kw in (dict(head_dim=64), dict(num_tokens=1 << 24), dict(num_heads=1 << 17)):
        assert _backward(**kw) == (UNSUPPORTED, 0), kw
    need = _backward()[1]
    assert need >= 256
    assert _backward(ws=None)[0] == NO_WS and _backward(ws=FAKE + 64)[0] == NO_WS and _backward(ws_bytes=need - 1)[0] == NO_WS


def _append(args=None, slots=None, k_norm=None, q_norm=None, **kw):
    p = paged.ebd_append_norm_params()
    a = p.append
    _with(a, pages=_pages(), rot=_rot(), num_tokens=5, new_off=FAKE, len=FAKE, q_heads=8, k_rows=ROWS, v_rows=ROWS,
          q_rows=ROWS, q_out_rows=ROWS)
    _with(a, **kw)
    p.k_norm, p.q_norm, p.slots = k_norm or _norm(), q_norm or _norm(), slots
    t = [FAKE] * 6 + [None]
    for i, v in (args or {}).items():
        t[i] = v
    return LIB.ebd_append_norm(ctypes.byref(p), *t, None)


def test_append_norm_refusals():
    assert LIB.ebd_append_norm(None, *[FAKE] * 6, None, None) == BAD
    for kw, code in BAD_PAGES:
        assert _append(pages=_pages(**kw)) == code, kw
        if "num_seqs" not in kw and "page_table" not in kw:
            assert _append(slots=FAKE, pos=FAKE, pages=_pages(**kw)) == code, kw
    for kw in BAD_NORMS:
        assert _append(k_norm=_norm(**kw)) == BAD and _append(q_norm=_norm(**kw)) == BAD, kw
    assert _append(rot=_rot(rot_dim=3)) == BAD and _append(num_tokens=-1) == BAD and _append(reserved=3) == BAD
    assert _append(new_off=None) == BAD and _append(len=None) == BAD
    for i in range(6):
        assert _append({i: None}) == BAD and _append({i: FAKE + 8}) == BAD, i
        assert _append({i: None}, slots=FAKE, pos=FAKE) == BAD, i
    assert _append(q_heads=0) == BAD and _append({4: None, 5: None}) == BAD
    for rows in ("k_rows", "v_rows", "q_rows", "q_out_rows"):
        assert _append(**{rows: paged.ebd_rows(512, 12)}) == BAD, rows
    assert _append(num_tokens=1 << 24) == UNSUPPORTED and _append(q_heads=1 << 17) == UNSUPPORTED
    assert _append(slots=FAKE) == BAD  # a rotation without positions
    assert _append(slots=FAKE + 4, pos=FAKE) == BAD
    assert _append(num_tokens=0) == OK and _append(pages=_pages(num_seqs=0)) == OK


def test_norms_of_the_binding():
    x = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="weight"):
        ebd.head_norm(torch.zeros(128, dtype=torch.bfloat16))
    with pytest.raises(TypeError, match="weight"):
        ebd.head_norm(None)
    with pytest.raises(ValueError, match="GPU"):
        ebd.head_norm(torch.zeros(128))
    with pytest.raises(TypeError, match="head_norm"):
        ebd.norm_rope_params(x, x, None)


def _plan(ws=FAKE, ws_bytes=1 << 40, **kw):
    p = paged.ebd_plan_step_params()
    _with(p, num_seqs=3, page_size=16, num_pages=40, max_pages=8, num_tokens=20, count=FAKE, len=FAKE, page_table=FAKE,
          free_pages=FAKE, free_state=FAKE, new_off=FAKE, slots=FAKE, pos=FAKE, parent=FAKE, mask=FAKE, mask_words=1)
    _with(p, **kw)
    size = LIB.ebd_workspace_size(ebd.EBD_WS_PLAN_STEP, ctypes.byref(p))
    return LIB.ebd_plan_step(ctypes.byref(p), None, ws, ws_bytes, None), size


def test_plan_refusals():
    assert LIB.ebd_plan_step(None, None, FAKE, 1 << 40, None) == BAD
    for kw in (dict(num_seqs=-1), dict(num_pages=0), dict(max_pages=0), dict(page_size=0), dict(num_tokens=-1),
               dict(reserved=1), dict(parent=None), dict(mask=None), dict(mask_words=0), dict(mask_words=65),
               dict(new_off=FAKE + 4), dict(slots=FAKE + 4), dict(mask=FAKE + 4)):
        assert _plan(**kw) == (BAD, 0), kw
    for kw in (dict(count=None), dict(len=None), dict(page_table=None), dict(free_pages=None), dict(free_state=None),
               dict(new_off=None)):
        assert _plan(**kw)[0] == BAD, kw
    for kw in (dict(page_size=8), dict(page_size=48), dict(page_size=1 << 17), dict(num_seqs=65537),
               dict(num_tokens=1 << 24), dict(num_pages=(1 << 30) + 1), dict(max_pages=(1 << 30) + 1)):
        assert _plan(**kw) == (UNSUPPORTED, 0), kw
    need = _plan()[1]
    assert _plan(ws=None)[0] == NO_WS and _plan(ws=FAKE + 8)[0] == NO_WS and _plan(ws_bytes=need - 1)[0] == NO_WS
    assert _plan(num_seqs=0, new_off=None)[0] == BAD  # (its one entry is written, and every token is padding)


def test_plans_of_the_binding():
    i32 = torch.int32
    z = lambda *shape, dtype=i32: torch.zeros(shape, dtype=dtype)  # noqa: E731
    args = dict(count=z(2), len=z(2), page_table=z(2, 4), page_size=16, free_pages=z(9), free_state=z(2),
                new_off=z(3, dtype=torch.int64))
    for kw, what in ((dict(page_table=z(8)), "page_table"), (dict(free_pages=z(0)), "free_pages"),
                     (dict(parent=z(5)), "go together"), (dict(mask=z(5, 1, dtype=torch.int64)), "go together"),
                     (dict(slots=z(4, dtype=torch.int64), pos=z(5)), "same number"),
                     (dict(), "CUDA|GPU|cuda|device")):
        with pytest.raises((ValueError, TypeError), match=what):
            ebd.plan_step_params(**{**args, **kw})


def _tree_params(mask=FAKE, words=1, reserved=0, **kw):
    from test_paged_abi import _attend_params

    p = paged.ebd_attend_tree_params()
    p.attend, p.mask, p.mask_words, p.reserved = _attend_params(**kw), mask, words, reserved
    return p


def _tree(args=None, ws=FAKE, ws_bytes=1 << 40, **kw):
    a = [FAKE] * 4 + [None, None]
    for i, v in (args or {}).items():
        a[i] = v
    p = _tree_params(**kw)
    size = LIB.ebd_workspace_size(ebd.EBD_WS_ATTEND_TREE, ctypes.byref(p))
    return LIB.ebd_attend_tree(ctypes.byref(p), *a, ws, ws_bytes, None), size


def test_tree_refusals():
    assert LIB.ebd_attend_tree(None, *[FAKE] * 4, None, None, FAKE, 1 << 40, None) == BAD
    assert LIB.ebd_workspace_size(ebd.EBD_WS_ATTEND_TREE, None) == 0
    for kw, code in BAD_PAGES:
        assert _tree(pages=_pages(**kw)) == (code, 0), kw
    for kw in (dict(words=0), dict(words=65), dict(reserved=1), dict(group=0), dict(max_new=-1), dict(num_tokens=-1),
               dict(max_rows=-1), dict(window=-1), dict(scale=-1.0), dict(q_rows=paged.ebd_rows(-8, 128))):
        assert _tree(**kw) == (BAD, 0), kw
    for kw in (dict(mask=None), dict(mask=FAKE + 4), dict(max_new=0), dict(new_off=None), dict(len=None)):
        assert _tree(**kw)[0] == BAD, kw
    for i in range(4):
        assert _tree({i: None})[0] == BAD and _tree({i: FAKE + 8})[0] == BAD, i
    for kw in (dict(max_rows=(1 << 30) + 1), dict(num_tokens=1 << 24), dict(max_new=1 << 29)):
        assert _tree(**kw) == (UNSUPPORTED, 0), kw
    need = _tree(max_rows=1 << 20)[1]
    assert need > 256 and _tree(max_rows=1 << 20, ws_bytes=need - 1)[0] == NO_WS
    assert _tree(ws=None)[0] == NO_WS and _tree(ws=FAKE + 64)[0] == NO_WS
    assert _tree(num_tokens=0, mask=None)[0] == OK and _tree(pages=_pages(num_seqs=0))[0] == OK


def _keep(K=FAKE, V=FAKE, **kw):
    p = paged.ebd_keep_rows_params()
    _with(p, pages=_pages(), new_off=FAKE, len=FAKE, path=FAKE, kept=FAKE, len_out=None, max_kept=4)
    return LIB.ebd_keep_rows(ctypes.byref(_with(p, **kw)), K, V, None, None)


def test_keep_refusals():
    assert LIB.ebd_keep_rows(None, FAKE, FAKE, None, None) == BAD
    for kw, code in BAD_PAGES:
        assert _keep(pages=_pages(**kw)) == code, kw
    for kw in (dict(max_kept=-1), dict(reserved=1), dict(new_off=None), dict(len=None), dict(path=None), dict(kept=None),
               dict(K=None), dict(V=None), dict(K=FAKE + 8), dict(V=FAKE + 2)):
        assert _keep(**kw) == BAD, kw
    assert _keep(pages=_pages(num_seqs=1 << 24)) == UNSUPPORTED and _keep(max_kept=1 << 24) == UNSUPPORTED
    assert _keep(pages=_pages(num_seqs=0)) == OK


def test_sizes_of_calls_without_tokens_heads_or_sequences():
    """Workspace sizes are numbers whatever is zero (a division by any of these would end the process)."""
    for heads in (0, 1, 200):
        for tokens in (0, 1, 100000):
            for stride in (0, 128):
                code, size = _backward(num_heads=heads, num_tokens=tokens, norm=_norm(head_stride=stride), ws=None)
                assert size >= 256 and code in ((OK,) if not heads and stride else (NO_WS,))
    for seqs in (0, 1, 5, 3000):
        for tokens in (0, 1, 100, 40000):
            for new in (0, 1, 8, 64, 500):
                for window in (0, 7):
                    kw = dict(pages=_pages(num_seqs=seqs), num_tokens=tokens, max_new=new, window=window, max_rows=5000)
                    p = _tree_params(words=8, **kw)
                    assert LIB.ebd_workspace_size(ebd.EBD_WS_ATTEND_TREE, ctypes.byref(p)) >= 256, (seqs, tokens, new)
                    assert LIB.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, ctypes.byref(p.attend)) >= 256
