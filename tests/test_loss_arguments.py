"""What the loss functions hand to the library, without one: sizes that its integers cannot hold."""
import pytest
import torch

import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200 import training


class Fake:
    """As much of a tensor as the checks ask for."""

    def __init__(self, shape, dtype=torch.float32):
        self.shape, self.dtype = shape, dtype

    def get_device(self):
        return torch.cuda.current_device() if torch.cuda.is_initialized() else -2

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def stride(self):
        return (self.shape[1], 1)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def element_size(self):
        return 1


class Library:
    """Keeps what it is called with."""

    def __init__(self):
        self.calls = []

    def ngc_policy_loss(self, cfg, *rest):
        self.calls.append((cfg._obj, rest))
        return 0

    def ngc_preference_loss(self, cfg, *rest):
        self.calls.append((cfg._obj, rest))
        return 0


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(training, "load_library", lambda: lib)
    return lib


def policy(rows, classes, each, parts):
    v = Fake((rows,))
    x = Fake((rows, classes))
    ngc.policy_loss(x, Fake((rows,), torch.int32), v, v, x, v, v, Fake((parts,)), rows_per_partition=each)


def preference(rows, classes, pairs):
    x = Fake((rows, classes))
    ngc.preference_loss(x, Fake((rows,), torch.int32), Fake((2 * pairs + 1,), torch.int64), Fake((2 * pairs,)), x,
                        Fake((2 * pairs,)), Fake((pairs,)), Fake((1 << 40,), torch.uint8))


@pytest.mark.parametrize("each", [7, 8, 1 << 31, (1 << 63) - 1, 1 << 63, (1 << 64) + 1, 1 << 100])
def test_partitions_of_more_rows_than_there_are(library, each):
    policy(7, 10, each, 1)
    (cfg, _), = library.calls
    assert cfg.rows == 7 and cfg.rows_per_partition >= 7


def test_ordinary_partitions(library):
    policy(7, 10, 3, 3)
    assert library.calls[0][0].rows_per_partition == 3
    policy(0, 10, 1 << 70, 0)
    assert library.calls[1][0].rows_per_partition >= 1


@pytest.mark.parametrize("classes", [1 << 31, (1 << 32) + 16, 1 << 40])
def test_classes_beyond_the_librarys_count_are_refused(library, classes):
    with pytest.raises(ngc.NgcError):
        policy(2, classes, 1, 2)
    with pytest.raises(ngc.NgcError):
        preference(2, classes, 1)
    assert not library.calls


@pytest.mark.parametrize("pairs", [1 << 31, (1 << 32) + 3])
def test_pairs_beyond_the_librarys_count_are_refused(library, pairs):
    with pytest.raises(ngc.NgcError):
        preference(2, 10, pairs)
    assert not library.calls


def test_the_most_classes_and_pairs(library):
    policy(1, (1 << 31) - 1, 1, 1)
    preference(1, (1 << 31) - 1, 0x3ffffffe)
    assert library.calls[0][0].n_classes == (1 << 31) - 1 and library.calls[1][0].pairs == 0x3ffffffe
