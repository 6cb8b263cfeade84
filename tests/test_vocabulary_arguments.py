"""What linear_cross_entropy and dropout hand to the library, and what they refuse before it: sizes that its integers cannot hold, layouts,
memory that arguments share.  The library's own checks, which come before anything is launched, are asked with made-up addresses."""
import ctypes as C

import pytest
import torch

import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200 import training
from paper_2212_08580_b200.binding import NGC_BF16, NGC_F32, DropoutConfig, LinearCrossEntropyConfig, load_library

BF16, F32 = torch.bfloat16, torch.float32


class Fake:
    """As much of a tensor as the checks ask for."""

    def __init__(self, shape, dtype=BF16, stride=None, at=1 << 20, device=-2):
        self.shape, self.dtype, self.at, self.device = tuple(shape), dtype, at, device
        if stride is None:
            stride, n = [], 1
            for s in reversed(shape):
                stride.insert(0, n)
                n *= s
        self.strides = tuple(stride)

    def get_device(self):
        return self.device if not torch.cuda.is_initialized() else torch.cuda.current_device() if self.device == -2 else -1

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at

    def element_size(self):
        return 1

    def unsqueeze(self, i):
        return Fake((1, *self.shape), self.dtype, (self.shape[0] * self.strides[0], *self.strides), self.at)

    def __getitem__(self, i):
        return Fake(self.shape[1:], self.dtype, self.strides[1:], self.at)


class Library:
    """Keeps what it is called with."""

    def __init__(self):
        self.calls = []

    def ngc_dropout(self, cfg, *rest):
        self.calls.append((cfg._obj, rest))
        return 0

    def ngc_linear_cross_entropy(self, cfg, *rest):
        self.calls.append((cfg._obj, rest))
        return 0

    def ngc_linear_cross_entropy_workspace_bytes(self, cfg, *rest):
        self.calls.append((cfg._obj, rest))
        return 4096


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(training, "load_library", lambda: lib)
    return lib


def call(rows=8, d=16, classes=20, x=None, weight=None, **more):
    parts = -(-rows // more["rows_per_partition"]) if more.get("rows_per_partition") else 1
    f32 = {"dtype": F32}
    args = [x or Fake((rows, d)), weight or Fake((classes, d)), Fake((rows,), torch.int32), Fake((rows,), **f32), Fake((rows,), **f32),
            Fake((parts,), **f32), Fake((1 << 20,), torch.uint8)]
    ngc.linear_cross_entropy(*args, **more)


def test_layouts_and_numbers_reach_the_library(library):
    call(x=Fake((8, 16), stride=(24, 1)), weight=Fake((20, 16), stride=(1, 32)), dweight=Fake((2, 20, 16), stride=(640, 1, 40)),
         dx=Fake((8, 16), stride=(18, 1)), rows_per_partition=5, scale=0.5, dropout=0.25, seed=(1 << 64) - 1, step=(1 << 32) - 1,
         first_row=(1 << 63) - 1, piece_rows=1 << 40)
    cfg, rest = library.calls[-1]
    assert (cfg.rows, cfg.rows_per_partition, cfg.d, cfg.n_classes, cfg.feature_major, cfg.keep_rows) == (8, 5, 16, 20, 1, 0)
    assert (cfg.scale, cfg.dropout, cfg.seed, cfg.step, cfg.first_row, cfg.piece_rows) == (0.5, 0.25, (1 << 64) - 1, (1 << 32) - 1, (1 << 63) - 1, 1 << 31)
    assert rest[1] == 24 and rest[3] == 32 and rest[7] == 18 and rest[9] == 40 and rest[10] == 640
    call(keep_rows=True, rows_per_partition=1 << 60)
    cfg, rest = library.calls[-1]
    assert (cfg.feature_major, cfg.keep_rows, cfg.rows_per_partition) == (0, 1, 8) and rest[6] is None and rest[8] is None


def test_single_rows_and_columns_have_any_stride(library):
    call(rows=1, d=1, classes=7, x=Fake((1, 1), stride=(99, 5)), weight=Fake((7, 1), stride=(1, 77)))
    assert library.calls[-1][0].feature_major == 0
    call(rows=3, d=5, classes=1, weight=Fake((1, 5), stride=(77, 1)), dweight=Fake((1, 5), stride=(3, 1)))
    assert library.calls[-1][0].feature_major == 0
    # one class, one feature: the weights may be read either way, and are read as their gradient is
    call(rows=3, d=5, classes=1, weight=Fake((1, 5), stride=(1, 1)), dweight=Fake((1, 5), stride=(1, 4)))
    assert library.calls[-1][0].feature_major == 1 and library.calls[-1][1][3] == 1 and library.calls[-1][1][9] == 4
    call(rows=3, d=1, classes=6, weight=Fake((6, 1), stride=(1, 1)), dweight=Fake((6, 1), stride=(3, 1)))
    assert library.calls[-1][0].feature_major == 0 and library.calls[-1][1][9] == 3
    with pytest.raises(ngc.NgcError):
        call(rows=3, d=1, classes=6, weight=Fake((6, 1), stride=(2, 9)), dweight=Fake((6, 1), stride=(0, 7)))


@pytest.mark.parametrize("more", [
    dict(x=Fake((1 << 31, 16)), rows=1 << 31), dict(d=(1 << 20) + 1), dict(classes=(1 << 24) + 1), dict(x=Fake((8, 16), F32)),
    dict(x=Fake((8, 17))), dict(x=Fake((8,))), dict(x=Fake((8, 16), stride=(15, 1))), dict(x=Fake((8, 16), stride=(32, 2))),
    dict(weight=Fake((20, 16), stride=(32, 2))), dict(weight=Fake((20, 16), stride=(15, 1))), dict(weight=Fake((20, 16), F32)),
    dict(weight=Fake((0, 16))), dict(weight=Fake((20, 16), device=0)), dict(dweight=Fake((20, 16), stride=(1, 20))),
    dict(dweight=Fake((2, 20, 16))), dict(dweight=Fake((20, 16)), rows_per_partition=4), dict(dweight=Fake((20,))),
    dict(dx=Fake((8, 15))), dict(rows_per_partition=0), dict(piece_rows=-1), dict(seed=1 << 64), dict(step=-1), dict(first_row=1 << 63),
    dict(row_weight=Fake((7,), F32)), dict(row_weight=Fake((8,), BF16))])
def test_refused_before_the_library(library, more):
    with pytest.raises(ngc.NgcError):
        call(**more)
    assert not library.calls


def test_dropout_arguments(library):
    ngc.dropout(Fake((4, 9), F32, (12, 1)), Fake((4, 9), F32, (11, 1)), 0.5, seed=3, step=7, first_row=9, residual=Fake((4, 9), F32, (10, 1)))
    cfg, rest = library.calls[-1]
    assert (cfg.rows, cfg.columns, cfg.dtype, cfg.p, cfg.seed, cfg.step, cfg.first_row) == (4, 9, NGC_F32, 0.5, 3, 7, 9)
    assert (rest[1], rest[3], rest[5]) == (12, 10, 11)
    n = len(library.calls)
    for x, out in ((Fake((4, 9)), Fake((4, 9), F32)), (Fake((4, 0)), Fake((4, 0))), (Fake((4, 1 << 31)), Fake((4, 1 << 31))),
                   (Fake((4, 9)), Fake((4, 9), stride=(8, 1))), (Fake((4, 9), torch.float16), Fake((4, 9), torch.float16)), (Fake((4,)), Fake((4,)))):
        with pytest.raises(ngc.NgcError):
            ngc.dropout(x, out, 0.5, seed=1)
    assert len(library.calls) == n


def ce(rows=100, each=100, d=64, classes=500, **more):
    return LinearCrossEntropyConfig(**{**dict(rows=rows, rows_per_partition=each, piece_rows=0, d=d, n_classes=classes, feature_major=0, keep_rows=0,
                                             scale=1.0, dropout=0.0, seed=0, first_row=0, step=0), **more})


def workspace(cfg, dx=1, dw=1, at=1 << 20, ld=None):
    return load_library().ngc_linear_cross_entropy_workspace_bytes(C.byref(cfg), at, ld or (cfg.n_classes if cfg.feature_major else cfg.d), dx, dw)


def test_workspace_sizes():
    some, more = workspace(ce(), 0, 0), workspace(ce(), 1, 1)
    assert 0 < some < more
    assert workspace(ce(rows=1 << 20, each=1 << 20, classes=100_000)) < 5 << 30  # pieces
    assert workspace(ce(rows=4096, each=4096, classes=100_000, piece_rows=256)) < workspace(ce(rows=4096, each=4096, classes=100_000))
    assert workspace(ce(), ld=65) > workspace(ce(), ld=64)  # weights that are copied
    assert workspace(ce(), at=(1 << 20) + 2) > workspace(ce())
    assert workspace(ce(keep_rows=1)) < workspace(ce())
    assert workspace(ce(rows=0)) >= 0
    for bad in (ce(rows=-1), ce(each=0), ce(piece_rows=-1), ce(d=0), ce(classes=0), ce(d=(1 << 20) + 1), ce(classes=(1 << 24) + 1), ce(scale=0.0),
                ce(scale=float("nan")), ce(scale=1e39), ce(dropout=-0.1), ce(dropout=1.1), ce(dropout=float("nan"))):
        assert workspace(bad) == 0
    assert workspace(ce(), ld=63) == 0 and workspace(ce(), at=(1 << 20) + 1) == 0 and workspace(ce(), at=0) == 0


def test_library_refuses_before_anything_is_launched():
    lib = load_library()
    cfg = ce()
    MB = 1 << 20

    def run(cfg=cfg, **more):
        a = dict(X=1 * MB, ldx=64, W=2 * MB, ldw=64, labels=3 * MB, weight=0, dX=0, ld_dx=0, dW=0, ld_dw=0, part=0, logp=4 * MB, row=5 * MB, loss=6 * MB,
                 ws=16 * MB, n=1 << 30)
        a.update(more)
        return lib.ngc_linear_cross_entropy(C.byref(cfg), a["X"], a["ldx"], a["W"], a["ldw"], a["labels"], a["weight"] or None, a["dX"] or None,
                                            a["ld_dx"], a["dW"] or None, a["ld_dw"], a["part"], a["logp"], a["row"], a["loss"] or None, a["ws"], a["n"], None)

    for more in (dict(ldx=63), dict(ldw=63), dict(X=MB + 1), dict(labels=3 * MB + 2), dict(weight=7 * MB + 1), dict(dX=8 * MB, ld_dx=63),
                 dict(dX=8 * MB + 1, ld_dx=64), dict(dW=8 * MB, ld_dw=63), dict(X=0), dict(labels=0), dict(logp=0), dict(row=0), dict(ws=0),
                 dict(ldx=1 << 40), dict(dW=8 * MB, ld_dw=1 << 40)):
        assert run(**more) == -1, more
    assert lib.ngc_linear_cross_entropy(None, MB, 64, MB, 64, MB, None, None, 0, None, 0, 0, MB, MB, None, MB, 1, None) == -1
    drop = DropoutConfig(rows=4, columns=8, dtype=NGC_BF16, p=0.5, seed=1, first_row=0, step=0)

    def out(cfg=drop, x=MB, ldx=8, res=0, ldr=0, to=2 * MB, ldo=8):
        return lib.ngc_dropout(C.byref(cfg), x, ldx, res or None, ldr, to, ldo, None)

    for more in (dict(x=0), dict(to=0), dict(ldx=7), dict(ldo=7), dict(x=MB + 1), dict(res=3 * MB, ldr=7), dict(res=3 * MB + 1, ldr=8), dict(to=MB + 2),
                 dict(to=MB, ldo=9), dict(res=2 * MB + 16, ldr=8), dict(ldx=1 << 44)):
        assert out(**more) == -1, more
    for bad in (dict(rows=-1), dict(columns=0), dict(dtype=2), dict(p=-0.5), dict(p=1.5), dict(p=float("nan"))):
        assert out(DropoutConfig(**{**dict(rows=4, columns=8, dtype=NGC_BF16, p=0.5, seed=1, first_row=0, step=0), **bad})) == -1
    assert out(DropoutConfig(rows=0, columns=8, dtype=NGC_BF16, p=0.5, seed=1, first_row=0, step=0)) == 0
