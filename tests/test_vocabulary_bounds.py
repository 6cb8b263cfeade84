"""What bounds linear_cross_entropy's pieces, and what it refuses without rows: on the CPU, with made-up addresses."""
import ctypes as C

import pytest

from paper_2212_08580_b200.binding import load_library
from tests.test_vocabulary_arguments import ce, workspace

MB = 1 << 20


@pytest.mark.parametrize("rows,piece_rows,most", [(250, 100, 64), (250, 65, 64), (300, 127, 64), (1000, 191, 128), (700, 255, 192), (90, 1, 64)])
def test_pieces_hold_at_most_piece_rows(rows, piece_rows, most):
    """The buffer of row numbers (4 bytes a row, in 256 bytes) of a partition in pieces is that of one piece of whole 64s; nothing has less
    than 64 rows."""
    for layout in (0, 1):
        pieces = workspace(ce(rows=rows, each=rows, classes=200, piece_rows=piece_rows, feature_major=layout), 1, 0)
        assert pieces <= workspace(ce(rows=most, each=most, classes=200, feature_major=layout), 1, 0)


def test_no_rows_refuse_shared_memory():
    """The weights would be lost: their gradient is set to 0 without rows too."""
    lib = load_library()

    def run(W=MB, dW=2 * MB, ld=64, layout=0):
        return lib.ngc_linear_cross_entropy(C.byref(ce(rows=0, feature_major=layout)), None, 64, W, ld, None, None, None, 0, dW, ld, 0, None, None, None,
                                            None, 0, None)

    assert run(dW=MB) == -1 and run(dW=MB, ld=500, layout=1) == -1
    assert run(dW=MB + 2 * 64) == -1
    assert run(dW=MB + 2 * 499 * 64) == -1  # (500 classes: the last row)


def test_no_rows_refuse_a_status_in_other_memory():
    lib = load_library()

    def run(ws, n=256):
        return lib.ngc_linear_cross_entropy(C.byref(ce(rows=0)), None, 64, MB, 64, None, None, None, 0, 2 * MB, 64, 0, None, None, None, ws, n, None)

    assert run(2 * MB + 256) == -1 and run(MB + 4) == -1 and run(3 * MB + 2) == -1
