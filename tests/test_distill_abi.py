"""Row losses of the distillation written over the teacher's entries, of which other rows are read later: refused on the host."""
import ctypes

import pytest

from paper_2410_15651_b200 import binding, build

STRIDE, WORKSPACE = 4, 5


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_row_losses_over_the_entries(lib):
    buf = (ctypes.c_char * 65536)()
    p = (ctypes.addressof(buf) + 255) // 256 * 256       # never dereferenced

    def call(row, sb, st, K, wsn=100):                   # [2,4,K] entries: ids at p + 4096, log-probs at p + 8192
        return lib.rlhf_distill_loss_fwd_bwd(p, 0, 32, 8, p + 4096, p + 8192, sb, st, K, p, 2, 4, 8, 0, 1.0, 1.0, p, row, p + 1024, 32,
                                             8, p, wsn, None)

    for at in (4096, 8192):
        end = at + 4 * (16 + 3 * 4 + 4)                  # of the entries, strides 16 and 4, K = 4
        for row in (at, at + 4, end - 4, at - 4 * 8 + 4):
            assert call(p + row, 16, 4, 4) == STRIDE, row
        for row in (end, at - 4 * 8):                    # beside them: the next check answers
            assert call(p + row, 16, 4, 4) == WORKSPACE, row
        assert call(p + at + 4 * 40, 16, 4, 4) == WORKSPACE
        assert call(p + at + 4 * 40, 40, 4, 4) == STRIDE
        assert call(p + at, 4, 1, 1) == STRIDE           # one entry per token: the same layout
    assert call(None, 16, 4, 4) == WORKSPACE
