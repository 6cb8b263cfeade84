"""What bounds linear_cross_entropy's pieces: on the CPU, with made-up addresses."""
import pytest

from tests.test_vocabulary_arguments import ce, workspace


@pytest.mark.parametrize("rows,piece_rows,most", [(250, 100, 64), (250, 65, 64), (300, 127, 64), (1000, 191, 128), (700, 255, 192), (90, 1, 64)])
def test_pieces_hold_at_most_piece_rows(rows, piece_rows, most):
    """The buffer of row numbers (4 bytes a row, in 256 bytes) of a partition in pieces is that of one piece of whole 64s; nothing has less
    than 64 rows."""
    for layout in (0, 1):
        pieces = workspace(ce(rows=rows, each=rows, classes=200, piece_rows=piece_rows, feature_major=layout), 1, 0)
        assert pieces <= workspace(ce(rows=most, each=most, classes=200, feature_major=layout), 1, 0)
