"""CPU checks of the paged-cache entry points' limits and of the layouts that the binding takes."""
import ctypes

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
