"""What the loss functions hand to the library, and what it refuses of it: sizes that its integers cannot hold, memory that
arguments share."""
import ctypes as C

import pytest
import torch

import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200 import training
from paper_2212_08580_b200.binding import PolicyLossConfig, PreferenceLossConfig


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


# ---- memory that arguments share: 64 rows of 16 fp32 classes, addresses that nothing is read from

ROWS = 64
PLACES = dict(logits=0x100000, grad=0x200000, actions=0x300000, old=0x310000, ref=0x320000, adv=0x330000, weight=0x340000,
              logp=0x350000, row_loss=0x360000, loss=0x370000)


def policy_memory(each=8, **kw):
    a = {**PLACES, **kw}
    cfg = PolicyLossConfig(rows=ROWS, rows_per_partition=each, n_classes=16, dtype=ngc.NGC_F32, scale=1.0, clip_low=0.2,
                           clip_high=0.2, kl_coef=0.1)
    return ngc.load_library().ngc_policy_loss(C.byref(cfg), a["logits"], 16, a["actions"], a["old"], a["ref"], a["adv"],
                                              a["weight"], a["grad"], 16, a["logp"], a["row_loss"], a["loss"], None)


VECTOR, MATRIX = 4 * ROWS, 4 * ROWS * 16
REFUSED = [(out, PLACES[other] + off, 8)
           for out, others in (("logp", ("row_loss", "loss", "actions", "logits", "grad")), ("row_loss", ("loss", "actions", "logits", "grad")),
                               ("loss", ("logits", "grad")))
           for other in others for off in (0, 4)]
REFUSED += [(out, PLACES["logits"] + MATRIX - 4, 8) for out in ("logp", "row_loss", "loss")]
REFUSED += [(out, PLACES[x] + off, 8) for out in ("logp", "row_loss") for x in ("old", "ref", "adv", "weight") for off in (4, VECTOR - 4, 4 - VECTOR)]
REFUSED += [("grad", PLACES[x] + off, 8) for x in ("actions", "old", "ref", "adv", "weight") for off in (0, 4 - MATRIX, VECTOR - 4)]
REFUSED += [("loss", PLACES["old"] + 4, 1), ("loss", PLACES["actions"], 1), ("loss", PLACES["row_loss"] + 4, 1), ("loss", PLACES["row_loss"], 8)]


@pytest.mark.parametrize("name,at,each", REFUSED)
def test_policy_outputs_in_other_arguments_memory_are_refused(name, at, each):
    assert policy_memory(each, **{name: at}) == -1


PAIRS = 9
PAIR_PLACES = dict(logits=0x100000, grad=0x200000, labels=0x300000, begin=0x310000, ref=0x320000, weight=0x330000,
                   seq=0x340000, loss=0x350000, ws=0x400000)


def preference_memory(**kw):
    a = {**PAIR_PLACES, **kw}
    cfg = PreferenceLossConfig(rows=ROWS, pairs=PAIRS, n_classes=16, dtype=ngc.NGC_F32, length_mean=0, scale=1.0, beta=0.1,
                               label_smoothing=0.0)
    return ngc.load_library().ngc_preference_loss(C.byref(cfg), a["logits"], 16, a["labels"], a["begin"], a["ref"],
                                                  a["weight"], a["grad"], 16, a["seq"], a["loss"], a["ws"], 1 << 16, None)


SIZE = dict(logits=MATRIX, grad=MATRIX, labels=VECTOR, begin=8 * (2 * PAIRS + 1), ref=8 * PAIRS, weight=4 * PAIRS, seq=8 * PAIRS,
            loss=4 * PAIRS)
PAIR_REFUSED = [("ws", (PAIR_PLACES[x] + SIZE[x] - 4) // 16 * 16) for x in SIZE]
PAIR_REFUSED += [("seq", PAIR_PLACES[x] + off) for x in ("logits", "grad", "labels", "begin", "weight", "loss") for off in (0, 4 - SIZE["seq"])]
PAIR_REFUSED += [("loss", PAIR_PLACES[x] + off) for x in ("logits", "grad", "labels", "begin", "ref") for off in (0, SIZE[x] - 4)]
PAIR_REFUSED += [("grad", PAIR_PLACES[x]) for x in ("labels", "begin", "ref", "weight")]
PAIR_REFUSED += [("seq", PAIR_PLACES["ref"] + 4), ("seq", PAIR_PLACES["ref"] - 8), ("loss", PAIR_PLACES["weight"] + 4)]


@pytest.mark.parametrize("name,at", PAIR_REFUSED)
def test_preference_outputs_in_other_arguments_memory_are_refused(name, at):
    assert preference_memory(**{name: at}) == -1
