"""Batches of drafted trees for each shape of ebd_attend_tree's kernels, and what the launch plan makes of a call."""
import ctypes
import os
import subprocess

from paper_2607_21475_amd import build, paged

# The plan's functions are not exported: its source once more, with a window into it.
SOURCE = r"""
#include "paged_api.cpp"

extern "C" int tree_shape(const ebd_attend_tree_params *p, int32_t *out) {
  const AttendPagedPlan plan = attend_paged_plan(&p->attend, true);
  for (int i = 0; i < plan.parts; ++i) {
    out[3 * i] = plan.part[i].rows;
    out[3 * i + 1] = plan.part[i].pairs;
    out[3 * i + 2] = plan.part[i].nsplit;
  }
  return plan.parts;
}
"""


def planner(folder):
    """f(params) -> [(query rows of a block, whether two groups of waves take two tiles at a time, splits) of each launch]."""
    src, obj, lib = (os.path.join(folder, "shape." + end) for end in ("cpp", "o", "so"))
    with open(src, "w") as f:
        f.write(SOURCE)
    for cmd in ([build.HIPCC, *build.FLAGS, "-c", src, "-o", obj],
                [build.HIPCC, "-shared", "-fPIC", "--offload-arch=" + build.ARCH, "-Wl,-Bsymbolic", "-Wl,-rpath," + build.PKG,
                 "-o", lib, obj, build.LIB]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
    call = ctypes.CDLL(lib).tree_shape

    def shapes(p):
        out = (ctypes.c_int32 * 6)()
        n = call(ctypes.byref(p), out)
        return [(out[3 * i], bool(out[3 * i + 1]), out[3 * i + 2]) for i in range(n)]

    return shapes


def params(news, held, kv, G, window=0, page=16, pad=0, max_new=None, max_rows=None):
    """The host fields of a call."""
    p = paged.ebd_attend_tree_params()
    a = p.attend
    lens = [h + m for h, m in zip(held, news)]
    a.pages.num_seqs, a.pages.kv_heads, a.pages.head_dim, a.pages.page_size = len(news), kv, 128, page
    a.pages.num_pages = a.pages.max_pages = 1 << 20
    a.group, a.num_tokens, a.window = G, sum(news) + pad, window
    a.max_new = max(news) if max_new is None else max_new
    a.max_rows = max(lens) if max_rows is None else max_rows
    p.mask_words = max(1, -(-a.max_new // 64))
    return p


# name: new tokens, rows held before, KV heads, query heads of each, window, (query rows of a block, two groups of waves),
# whether the sequences' rows are split.  Up to 64 query rows of a sequence: other kernels, by their blocks of rows.
BATCHES = {
    "rows16": ([3, 2, 4], [700, 37, 2500], 2, 4, 0, (16, False), True),
    "rows32": ([7, 8, 5], [700, 37, 2500], 2, 4, 0, (32, False), True),
    "rows64": ([15, 9, 16], [700, 37, 2500], 2, 4, 0, (64, False), True),
    "four": ([101, 70, 90], [300, 37, 90], 100, 1, 0, (128, False), False),
    "four_window": ([101, 70, 90], [300, 37, 90], 100, 1, 45, (128, False), False),
    "four_blocks": ([300], [40], 128, 1, 0, (128, False), False),
    "four_splits": ([70, 65, 70], [6000, 5900, 6000], 32, 1, 0, (128, False), True),
    "pairs": ([70, 66], [40, 9], 2, 1, 0, (128, True), False),
    "pairs_window": ([150, 100], [900, 700], 2, 2, 45, (128, True), False),
    "pairs_splits": ([150], [3001], 2, 2, 0, (128, True), True),
    "long": ([70, 69, 70], [300, 37, 90], 64, 2, 0, (256, False), False),
    "long_window": ([70, 69, 70], [300, 37, 90], 64, 2, 45, (256, False), False),
    "long_splits": ([130, 128, 130], [3000, 2900, 3000], 16, 1, 0, (256, False), True),
}


def bounds(name):
    """(max_new, max_rows) a little below a batch's truth, by which it keeps its shape."""
    news, held, *_ = BATCHES[name]
    return max(news) - 1, max(h + m for h, m in zip(held, news)) - 3
