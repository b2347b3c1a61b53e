"""CPU checks of the paged-cache entry points: bad arguments are refused before any device work."""
import ctypes

import pytest
import torch

import paper_2607_21475_amd as ebd
from paper_2607_21475_amd import paged

FAKE = 0x100000  # aligned, never dereferenced: validation fails before any device access
LIB = ebd._lib
BAD, UNSUPPORTED, NO_WS = ebd.EBD_ERR_INVALID_ARG, ebd.EBD_ERR_UNSUPPORTED, ebd.EBD_ERR_WORKSPACE


def _rot(**kw):
    r = paged.ebd_rotary()
    r.freq, r.rot_dim, r.layout, r.amplitude, r.flags = FAKE, 128, 0, 1.0, 0
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _pages(**kw):
    P = paged.ebd_pages()
    P.num_seqs, P.kv_heads, P.head_dim, P.page_size, P.num_pages, P.max_pages = 2, 4, 128, 16, 100, 8
    P.page_table = FAKE
    P.page_stride, P.head_stride, P.row_stride = 4 * 16 * 128, 16 * 128, 128
    for k, v in kw.items():
        setattr(P, k, v)
    return P


BAD_PAGES = [(dict(num_seqs=-1), BAD), (dict(kv_heads=0), BAD), (dict(num_pages=0), BAD), (dict(max_pages=0), BAD),
             (dict(page_table=None), BAD), (dict(row_stride=4), BAD), (dict(head_stride=0), BAD),
             (dict(page_stride=-8), BAD), (dict(page_stride=1001), BAD), (dict(head_dim=64), UNSUPPORTED),
             (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=1 << 17), UNSUPPORTED),
             (dict(kv_heads=1 << 17), UNSUPPORTED), (dict(row_stride=1 << 26), UNSUPPORTED),
             (dict(page_stride=1 << 40), UNSUPPORTED)]


def _rope(x=FAKE, y=FAKE, p=None, **kw):
    p = p or paged.ebd_rope_params()
    p.num_tokens, p.num_heads, p.head_dim, p.pos, p.rot = 4, 2, 128, FAKE, kw.pop("rot", _rot())
    p.x = p.y = paged.ebd_rows(256, 128)
    for k, v in kw.items():
        setattr(p, k, v)
    return LIB.ebd_rope(ctypes.byref(p), x, y, None)


def test_rope_refusals():
    assert LIB.ebd_rope(None, FAKE, FAKE, None) == BAD
    for kw in (dict(rot_dim=0), dict(rot_dim=130), dict(rot_dim=7), dict(layout=2), dict(flags=2),
               dict(amplitude=float("nan")), dict(freq=None), dict(freq=FAKE + 4)):
        assert _rope(rot=_rot(**kw)) == BAD, kw
    assert _rope(num_tokens=-1) == BAD and _rope(num_heads=-1) == BAD and _rope(reserved=1) == BAD
    assert _rope(pos=None) == BAD and _rope(x=None) == BAD and _rope(y=None) == BAD
    assert _rope(x=FAKE + 2) == BAD and _rope(y=FAKE + 8) == BAD
    for r in ((-8, 128), (256, 4), (1 << 40, 128)):
        p = paged.ebd_rope_params()
        p.num_tokens, p.num_heads, p.head_dim, p.pos, p.rot = 4, 2, 128, FAKE, _rot()
        p.x, p.y = paged.ebd_rows(256, 128), paged.ebd_rows(*r)
        assert LIB.ebd_rope(ctypes.byref(p), FAKE, FAKE, None) == BAD, r
    assert _rope(head_dim=64) == UNSUPPORTED and _rope(num_tokens=1 << 24) == UNSUPPORTED
    assert _rope(num_heads=1 << 17) == UNSUPPORTED
    assert _rope(num_tokens=0) == ebd.EBD_OK and _rope(num_heads=0) == ebd.EBD_OK


def _append(args=None, **kw):
    p = paged.ebd_append_paged_params()
    p.pages, p.rot = kw.pop("pages", _pages()), kw.pop("rot", _rot())
    p.num_tokens, p.new_off, p.len, p.q_heads = 5, FAKE, FAKE, 8
    p.k_rows = p.v_rows = paged.ebd_rows(512, 128)
    p.q_rows = p.q_out_rows = paged.ebd_rows(1024, 128)
    for k, v in kw.items():
        setattr(p, k, v)
    a = [FAKE] * 6 + [None]
    for i, v in (args or {}).items():
        a[i] = v
    return LIB.ebd_append_paged(ctypes.byref(p), *a, None)


def test_append_refusals():
    for kw, code in BAD_PAGES:
        assert _append(pages=_pages(**kw)) == code, kw
    assert _append(rot=_rot(rot_dim=3)) == BAD and _append(rot=_rot(layout=-1)) == BAD
    assert _append(num_tokens=-1) == BAD and _append(q_heads=-1) == BAD and _append(reserved=3) == BAD
    assert _append(new_off=None) == BAD and _append(len=None) == BAD
    for i in range(6):
        assert _append({i: None}) == BAD, i
        assert _append({i: FAKE + 8}) == BAD, i
    assert _append(q_heads=0) == BAD  # queries without heads
    assert _append({4: None, 5: None}) == BAD  # heads without queries
    for rows in ("k_rows", "v_rows", "q_rows", "q_out_rows"):
        assert _append(**{rows: paged.ebd_rows(512, 12)}) == BAD, rows
    assert _append(num_tokens=1 << 24) == UNSUPPORTED and _append(q_heads=1 << 17) == UNSUPPORTED
    assert _append(num_tokens=0) == ebd.EBD_OK and _append(pages=_pages(num_seqs=0)) == ebd.EBD_OK


def _attend_params(**kw):
    p = paged.ebd_attend_paged_params()
    p.pages = kw.pop("pages", _pages())
    p.group, p.max_new, p.num_tokens, p.max_rows = 4, 3, 5, 128
    p.new_off = p.len = FAKE
    p.q_rows = p.y_rows = paged.ebd_rows(16 * 128, 128)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _attend(args=None, ws=FAKE, ws_bytes=1 << 40, **kw):
    a = [FAKE] * 4 + [None, None]
    for i, v in (args or {}).items():
        a[i] = v
    return LIB.ebd_attend_paged(ctypes.byref(_attend_params(**kw)), *a, ws, ws_bytes, None)


def test_attend_refusals():
    for kw, code in BAD_PAGES:
        assert _attend(pages=_pages(**kw)) == code, kw
        n = LIB.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, ctypes.byref(_attend_params(pages=_pages(**kw))))
        assert n == 0, kw
    for kw in (dict(group=0), dict(max_new=-1), dict(max_new=0), dict(num_tokens=-1), dict(max_rows=-1), dict(window=-1),
               dict(scale=-1.0), dict(scale=float("inf")), dict(new_off=None), dict(len=None),
               dict(q_rows=paged.ebd_rows(-8, 128)), dict(y_rows=paged.ebd_rows(128, 4))):
        assert _attend(**kw) == BAD, kw
    for i in range(4):
        assert _attend({i: None}) == BAD and _attend({i: FAKE + 8}) == BAD, i
    assert _attend({4: FAKE + 2}) == BAD  # lse
    for kw in (dict(max_rows=(1 << 30) + 1), dict(num_tokens=1 << 24), dict(group=1 << 15),
               dict(max_new=1 << 29), dict(pages=_pages(num_seqs=1 << 24))):
        assert _attend(**kw) == UNSUPPORTED, kw
    assert _attend(ws=None) == NO_WS and _attend(ws=FAKE + 64) == NO_WS and _attend(ws_bytes=255) == NO_WS
    need = LIB.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, ctypes.byref(_attend_params(max_rows=1 << 20)))
    assert need > 256 and _attend(max_rows=1 << 20, ws_bytes=need - 1) == NO_WS
    assert _attend(num_tokens=0) == ebd.EBD_OK and _attend(pages=_pages(num_seqs=0)) == ebd.EBD_OK
    assert LIB.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, None) == 0


def test_gather_refusals():
    def call(args=None, **kw):
        p = paged.ebd_gather_paged_params()
        p.pages, p.max_rows, p.seq_off = kw.pop("pages", _pages()), 100, FAKE
        for k, v in kw.items():
            setattr(p, k, v)
        a = [FAKE] * 4 + [None]
        for i, v in (args or {}).items():
            a[i] = v
        return LIB.ebd_gather_paged(ctypes.byref(p), *a, None)

    for kw, code in BAD_PAGES:
        assert call(pages=_pages(**kw)) == code, kw
    assert call(max_rows=-1) == BAD and call(seq_off=None) == BAD
    for i in range(4):
        assert call({i: None}) == BAD and call({i: FAKE + 4}) == BAD, i
    assert call(max_rows=(1 << 30) + 1) == UNSUPPORTED
    assert call(max_rows=1 << 30, pages=_pages(num_seqs=64)) == UNSUPPORTED  # work-groups
    assert call(max_rows=0) == ebd.EBD_OK and call(pages=_pages(num_seqs=0)) == ebd.EBD_OK


def test_workspace_grows_with_the_splits_only():
    size = lambda **kw: ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, _attend_params(**kw))  # noqa: E731
    assert size(max_rows=0) >= 256
    many = _pages(num_seqs=4096, kv_heads=8)
    assert size(pages=many, max_new=1, max_rows=4096) == 256  # enough units: nothing is split


def test_binding_refuses_wrong_tensors():
    bf = torch.bfloat16
    cpu = torch.zeros((4, 2, 128), dtype=bf)
    pos = torch.zeros(4, dtype=torch.int32)
    freq = torch.zeros(64, dtype=torch.float64)
    with pytest.raises(ValueError):
        ebd.rotary(freq)  # not on the GPU
    with pytest.raises(ValueError):
        ebd.rotary(torch.zeros(65, dtype=torch.float64))
    with pytest.raises(ValueError):
        ebd.rope_params(cpu, cpu, pos, ebd.rotary(None))
    with pytest.raises(TypeError):
        ebd.rope_params(cpu.float(), cpu, pos, ebd.rotary(None))
    with pytest.raises(ValueError):
        ebd.rope_params(cpu, cpu[:3], pos, ebd.rotary(None))
    with pytest.raises(ValueError):  # rows that share memory
        ebd.rope_params(cpu, cpu[:1].expand(4, 2, 128), pos, ebd.rotary(None))
    with pytest.raises(ValueError):  # ... though no stride is below a row's length
        ebd.rope_params(cpu, torch.as_strided(cpu, (4, 2, 128), (128, 128, 1)), pos, ebd.rotary(None))
    K = torch.zeros((3, 2, 16, 128), dtype=bf)
    table = torch.zeros((1, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        ebd.pages(K, K[:2], table)
    with pytest.raises(ValueError):
        ebd.pages(K[..., :64], K[..., :64], table)
    with pytest.raises(TypeError):
        ebd.pages(K.half(), K.half(), table)
    with pytest.raises(ValueError):
        ebd.pages(K, K.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3), table)
    with pytest.raises(ValueError):
        ebd.pages(K[:1].expand(3, 2, 16, 128), K[:1].expand(3, 2, 16, 128), table)


def test_binding_names_what_is_not_a_tensor():
    K = torch.zeros(2, 1, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="page_table"):
        ebd.pages(K, K, [[0, 1]])
    with pytest.raises(ValueError, match="page_table"):
        ebd.pages(K, K, None)
    with pytest.raises(TypeError, match="freq"):
        ebd.rotary([1.0, 0.1])
    with pytest.raises(TypeError, match="workspace"):
        ebd.ebd_attend_paged(_attend_params(), K, K, K, K, None)


def test_rope_frequencies():
    f, a = ebd.rope_frequencies(8, 10000.0, device="cpu")
    assert a == 1.0 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14)
    assert torch.equal(ebd.rope_frequencies(8, 1e4, "linear", 4.0, device="cpu")[0], f / 4)
    n, _ = ebd.rope_frequencies(8, 1e4, "ntk", 4.0, device="cpu")
    assert n[0] == 1 and abs(float(n[-1] / f[-1]) - 0.25) < 1e-12 and bool((n[1:-1] < f[1:-1]).all())
    # turns over 6284 positions: about 1000, 100, 10, 1
    b, a = ebd.rope_frequencies(8, 1e4, "bands", 8.0, original=6284, low=2.0, high=18.0, device="cpu")
    t = 6284 * 0.01 / (2 * 3.141592653589793)
    g = (t - 2) / 16
    assert a == 1.0 and torch.equal(b[:2], f[:2]) and float(b[3]) == float(f[3]) / 8
    assert abs(float(b[2]) - (g * 0.01 + (1 - g) * 0.01 / 8)) < 1e-15
    y, a = ebd.rope_frequencies(8, 1e4, "yarn", 8.0, original=6284, device="cpu")
    assert abs(a - 1.2079441541679836) < 1e-15 and torch.equal(y[:2], f[:2]) and f[2] / 8 < y[2] < f[2]
    for kw in (dict(rot_dim=7), dict(rot_dim=130), dict(base=-1.0), dict(factor=0.0), dict(scaling="other"),
               dict(scaling="bands", factor=2.0), dict(scaling="yarn", factor=2.0, original=10, low=5.0, high=5.0),
               dict(scaling="ntk", rot_dim=2)):
        with pytest.raises(ValueError):
            ebd.rope_frequencies(**{"rot_dim": 8, **kw}, device="cpu")


def test_paged_cache_allocates_room():
    c = ebd.PagedCache.allocate([65, 0, 16], 2, page_size=16, spare=1, device="cpu")
    assert c.K.shape == (7, 2, 16, 128) and c.V.shape == c.K.shape
    assert c.page_table.tolist() == [[0, 1, 2, 3, 4], [-1] * 5, [5, -1, -1, -1, -1]] and c.len.tolist() == [0, 0, 0]
