"""linear_cross_entropy at logits far from zero: classes ruled out by a constant feature and weights
of -1e4 and less, as a padded vocabulary or a restricted set of tokens has them.

A ruled-out class has e^z = 0 in every precision, so what is left is the problem without these classes, at that problem's tolerances
(tests/test_gpu_vocabulary.py)."""
import copy

import pytest
import torch

from tests.test_gpu_vocabulary import BF16, Problem

gpu = pytest.mark.gpu
MASKS = [-1e4, -2.3e7, -1e9, -1.7e9, -1e30]
# rows, d, classes: the few-rows form (scored where they are, and packed), the logits' form, a row in one tile of 256 and of 128 classes
SHAPES = [(100, 64, 700), (300, 64, 700), (300, 64, 250), (200, 64, 120), (90, 1024, 1000)]


def ruled_out(p, out, value, rows=None):
    """The classes `out` (a truth value each) get the logit `value` in all rows (or some), whatever else there is."""
    flat = p.weight if p.layout == "classes" else p.weight.t()
    flat = flat.contiguous()
    w = flat if p.layout == "classes" else flat.t()
    p.weight = w
    w[:, 0] = torch.where(out, torch.tensor(value, dtype=BF16, device="cuda"), torch.zeros_like(w[:, 0]))
    p.x[:, 0] = 1.0 if rows is None else rows.to(BF16)
    p.out = out
    inside = (~out).nonzero().squeeze(1)
    live = (p.labels >= 0) & (p.labels < p.classes)
    p.labels = torch.where(live, inside[p.labels.long() % inside.numel()].to(torch.int32), p.labels)
    return p


def check_without(p):
    """As the problem of the other classes."""
    q, inside = copy.copy(p), (~p.out).nonzero().squeeze(1)
    number = torch.full((p.classes,), -1, dtype=torch.int64, device="cuda")
    number[inside] = torch.arange(inside.numel(), device="cuda")
    live = (p.labels >= 0) & (p.labels < p.classes)
    q.labels = torch.where(live, number[p.labels.long().clamp(0, p.classes - 1)], -1).to(torch.int32)
    q.weight, q.classes = p.weight[inside], inside.numel()
    if p.dw is not None:
        assert (p.dw[:, p.out] == 0).all()
        q.dw = p.dw[:, inside]
    assert (p.logp <= 0).all()
    q.check()


def masks_of(classes):
    c = torch.arange(classes, device="cuda")
    yield "first half", c < classes // 2
    yield "second half", c >= classes // 2
    yield "a group", (c >= 32) & (c < min(160, classes - 32))
    yield "all but three", (c % (classes // 3)) != 5
    yield "every other", c % 2 == 0


@gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,d,classes", SHAPES)
@pytest.mark.parametrize("value", MASKS)
@pytest.mark.parametrize("grads", [True, False])
def test_classes_ruled_out(layout, rows, d, classes, value, grads):
    for which, out in masks_of(classes):
        p = ruled_out(Problem(rows, d, classes, seed=rows + d, layout=layout), out, value)
        p.run(dx=grads, dw=grads)
        assert torch.isfinite(p.logp).all() and torch.isfinite(p.loss).all(), which
        check_without(p)


@gpu
@pytest.mark.parametrize("value", [-2.3e7, -1e9])
@pytest.mark.parametrize("options", [dict(each=100), dict(piece_rows=128), dict(each=128, keep_rows=True), dict(scale=0.6), dict(dropout=0.0, scale=1.7)])
def test_ruled_out_in_every_way_of_calling(value, options):
    for which, out in masks_of(900):
        p = ruled_out(Problem(450, 72, 900, seed=8, masked=0.0 if options.get("keep_rows") else 0.2), out, value)
        check_without(p.run(**options))
