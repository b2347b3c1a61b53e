"""CPU checks of the paged-cache entry points' limits and of the layouts that the binding takes."""
import ctypes

import pytest
import torch

import paper_2607_21475_amd as ebd
from paper_2607_21475_amd import paged

FAKE = 0x100000  # aligned, never dereferenced: validation fails before any device access
LIB = ebd._lib
BAD, UNSUPPORTED = ebd.EBD_ERR_INVALID_ARG, ebd.EBD_ERR_UNSUPPORTED


def _pages(**kw):
    P = paged.ebd_pages()
    P.num_seqs, P.kv_heads, P.head_dim, P.page_size, P.num_pages, P.max_pages = 2, 4, 128, 16, 100, 8
    P.page_table = FAKE
    P.page_stride, P.head_stride, P.row_stride = 4 * 16 * 128, 16 * 128, 128
    for k, v in kw.items():
        setattr(P, k, v)
    return P


def test_gather_needs_a_row_count_that_is_none_below_zero():
    p = paged.ebd_gather_paged_params()
    p.pages, p.max_rows, p.seq_off, p.num_rows = _pages(), 100, FAKE, -1
    assert LIB.ebd_gather_paged(ctypes.byref(p), FAKE, FAKE, FAKE, FAKE, None, None) == BAD


def _attend_params(seqs, **kw):
    p = paged.ebd_attend_paged_params()
    p.pages = _pages(num_seqs=seqs, kv_heads=8, page_stride=8 * 16 * 128)
    p.group, p.max_new, p.num_tokens, p.max_rows, p.new_off, p.len = 4, 64, 64, 600, FAKE, FAKE
    p.q_rows = p.y_rows = paged.ebd_rows(32 * 128, 128)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_sequences_without_new_tokens_need_no_workspace():
    """One chunk of 256 query rows among many idle sequences: partial sums (a block's 128 query rows take 520 bytes each) for
    its own splits, at most 32 for each of the 17 blocks that 256 rows may lie in, and 8 heads."""
    size = lambda seqs, **kw: ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, _attend_params(seqs, **kw))  # noqa: E731
    most = 512 + 17 * 32 * 8 * 128 * 520
    for rows in (600, 10000):
        n = size(64, max_rows=rows)
        assert n <= most and all(size(seqs, max_rows=rows) == n for seqs in (256, 1000, 70000)), rows
    assert size(64, max_rows=10000) > most // 2
    wide = dict(group=40, max_new=8, num_tokens=8)  # more query heads than the launch of short sequences serves
    assert size(64, max_rows=1 << 20, **wide) == size(10000, max_rows=1 << 20, **wide) <= 512 + (320 // 128 + 8) * 32 * 8 * 128 * 520


def test_attend_refuses_launches_of_too_many_work_groups():
    def call(seqs, **kw):
        return LIB.ebd_attend_paged(ctypes.byref(_attend_params(seqs, **kw)), FAKE, FAKE, FAKE, FAKE, None, None, FAKE, 0, None)

    assert call(1000) == ebd.EBD_ERR_WORKSPACE  # the launches are in bounds, the workspace is not
    assert call((1 << 20) + 1, max_new=1) == UNSUPPORTED
    # five tokens of each sequence, over so many rows that a block's are split: the splits' launch is in bounds, the one
    # that joins them, a work-group for four query rows of every block, is not
    assert call(80000, num_tokens=400000, max_rows=1 << 22) == UNSUPPORTED
    assert call(50000, num_tokens=250000, max_rows=1 << 22) == ebd.EBD_ERR_WORKSPACE  # (57812 blocks of 8 heads: 14.8 million)
    assert call(80000, num_tokens=400000, max_rows=1 << 12) == ebd.EBD_ERR_WORKSPACE


def test_outputs_whose_rows_lie_apart_are_taken():
    """Every second head of an odd number, heads or tokens outermost, gaps of any size: no two rows share an element."""
    x = torch.zeros(40000, dtype=torch.bfloat16)
    for t in (x[:1920].view(5, 3, 128)[:, ::2], x[:1920].view(3, 5, 128)[::2].transpose(0, 1), x[:1920].view(5, 3, 128)[::3],
              torch.as_strided(x, (4, 2, 128), (392, 264, 1)), torch.as_strided(x, (4, 2, 128), (0, 128, 1))[:1],
              x[:3840].view(2, 5, 3, 128)[:, ::2, ::2], x[:0].view(0, 3, 128)):
        seen = (torch.arange(40000)[:, None].new_zeros(40000)).index_add_(
            0, torch.as_strided(torch.arange(40000), t.shape, t.stride()).reshape(-1), torch.ones(t.numel(), dtype=torch.long))
        assert int(seen.max()) <= 1
        paged._distinct(t, "t")
    for shape, stride in (((4, 2, 128), (391, 264, 1)), ((4, 2, 128), (263, 136, 1)), ((2, 2, 128), (0, 128, 1)),
                          ((3, 2, 128), (128, 128, 1)), ((2, 4, 2, 128), (1000, 264, 136, 1))):
        with pytest.raises(ValueError, match="share memory"):
            paged._distinct(torch.as_strided(x, shape, stride), "t")
