"""linear_cross_entropy at logits far from zero and at rows that are nearly certain: classes ruled out by a constant feature and weights
of -1e4 ... the type's lowest value, as a padded vocabulary or a restricted set of tokens has them; labels far above the rest.

A ruled-out class has e^z = 0 in every precision, so what is left is the problem without these classes, at that problem's tolerances
(tests/test_gpu_vocabulary.py)."""
import copy
import math

import pytest
import torch

from tests.test_gpu_vocabulary import BF16, Problem, U

gpu = pytest.mark.gpu
LOWEST = torch.finfo(torch.bfloat16).min
MASKS = [-1e4, -2.3e7, -1e9, -1.7e9, -1e30, -3e38, LOWEST]
# rows, d, classes: the few-rows form (scored where they are, and packed), the logits' form, a row in one tile of 256 and of 128 classes
SHAPES = [(100, 64, 700), (300, 64, 700), (300, 64, 250), (200, 64, 120), (90, 1024, 1000), (260, 1300, 600)]


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
@pytest.mark.parametrize("value", MASKS)
@pytest.mark.parametrize("rows,d,classes", SHAPES)
def test_one_class_left(rows, d, classes, value):
    """log p = 0 and no gradient."""
    out = torch.ones(classes, dtype=torch.bool, device="cuda")
    out[classes // 2] = False
    p = ruled_out(Problem(rows, d, classes), out, value).run()
    assert (p.logp == 0).all() and (p.row_loss == 0).all() and (p.dx == 0).all() and (p.dw == 0).all()


@gpu
@pytest.mark.parametrize("value", MASKS + [1e9, 3e38])
@pytest.mark.parametrize("rows,d,classes", SHAPES)
@pytest.mark.parametrize("grads", [True, False])
def test_all_classes_alike(rows, d, classes, value, grads):
    """Every class at one logit, however far: log p = -log(classes), to what a logarithm in fp32 gives."""
    p = ruled_out(Problem(rows, d, classes, weighted=False, masked=0.0), torch.zeros(classes, dtype=torch.bool, device="cuda"), value)
    p.x[:, 1:] = 0.0
    p.weight[:, 0] = value
    p.run(dx=grads, dw=grads)
    want = -math.log(classes)
    # (sums of ones are exact; a logarithm to base 2, its product with ln 2, two roundings of a number below 16)
    assert ((p.logp.double() - want).abs() <= 8 * U * abs(want)).all()
    if grads:
        G = torch.full((rows, classes), 1.0 / classes, dtype=torch.float64, device="cuda")
        G[torch.arange(rows, device="cuda"), p.labels.long()] -= 1.0
        e_G = G.abs() * (2.0 ** -8 + 2.0 ** -11 + 32 * U)
        x = p.x.double()
        want, slack = G.t() @ x, e_G.t() @ x.abs() + (rows + 8) * U * (G.abs().t() @ x.abs())
        assert ((p.dw[0].double() - want).abs() <= slack + 2.0 ** -8 * want.abs()).all()


@gpu
@pytest.mark.parametrize("value", [-1e4, -1e9, LOWEST])
@pytest.mark.parametrize("rows,d,classes", SHAPES)
def test_label_ruled_out(rows, d, classes, value):
    """A label among the ruled-out classes: log p is as far as its logit, and G is that of the others but -1 at the label."""
    out = torch.arange(classes, device="cuda") >= classes // 2
    p = ruled_out(Problem(rows, d, classes, weighted=False, masked=0.0), out, value)
    p.labels.fill_(classes - 1)
    p.run()
    z = p.x.double() @ p.weight.double().t()
    want = torch.log_softmax(z, 1)[:, -1]
    assert torch.isfinite(p.logp).all()
    assert ((p.logp.double() - want).abs() <= 2 * (d + 8) * U * want.abs()).all()
    G = z.softmax(1)
    e_G = G * (2 * (d + 8) * U * (p.x.double().abs() @ p.weight[~out].double().abs().t()).amax(1, keepdim=True) + 160 * U) + 2.0 ** -38
    G[:, -1] -= 1.0
    e_G = e_G + G.abs() * (2.0 ** -8 + 2.0 ** -11)
    x = p.x.double()
    want, slack = G.t() @ x, e_G.t() @ x.abs() + (rows + 8) * U * (G.abs().t() @ x.abs())
    assert ((p.dw[0].double() - want).abs() <= slack + 2.0 ** -8 * want.abs()).all()


@gpu
@pytest.mark.parametrize("value", [-1e9, LOWEST])
@pytest.mark.parametrize("options", [dict(each=100), dict(piece_rows=128), dict(each=128, keep_rows=True), dict(scale=0.6), dict(dropout=0.0, scale=1.7)])
def test_ruled_out_in_every_way_of_calling(value, options):
    if value == LOWEST and options.get("scale", 0.0) > 1.0:
        value = -1e38  # (finite after scaling too)
    for which, out in masks_of(900):
        p = ruled_out(Problem(450, 72, 900, seed=8, masked=0.0 if options.get("keep_rows") else 0.2), out, value)
        check_without(p.run(**options))


@gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,d,classes", SHAPES)
def test_minus_infinity_among_the_logits(layout, rows, d, classes):
    """Finite operands whose product leaves fp32 (-2 times the lowest value): a class of e^-inf = 0, in whole groups as well."""
    for which, out in masks_of(classes):
        p = ruled_out(Problem(rows, d, classes, layout=layout), out, LOWEST)
        p.x[:, 0] = 2.0
        p.run(dx=False, dw=False)
        assert torch.isfinite(p.logp).all(), which
        check_without(p)


@gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,d,classes", SHAPES)
@pytest.mark.parametrize("top", [8.0, 20.0, 35.0, 100.0, 300.0])
def test_rows_that_are_nearly_certain(layout, rows, d, classes, top):
    """Features along the label's weights.  log p is at most 0, and as exact as 1 - p is small: with e_z the error of a logit,
    |error of log p| <= (1 - p) 2 e_z (and the second order) + what fp32 holds of 1 + (1 - p)."""
    p = Problem(rows, d, classes, layout=layout, masked=0.0, weighted=False)
    w = p.weight.float()[p.labels.long()]
    p.x.copy_((w * (top / w.square().sum(1, keepdim=True))).to(BF16))
    p.run(dx=True, dw=True)
    x, w = p.x.double(), p.weight.double()
    z = x @ w.t()
    y = p.labels.long().unsqueeze(1)
    logp = torch.log_softmax(z, 1).gather(1, y).squeeze(1)
    rest = -torch.expm1(logp)
    e_z = (d + 8) * U * (x.abs() @ w.abs().t()).amax(1)
    assert (p.logp <= 0).all() and (p.row_loss >= 0).all()
    off = (p.logp.double() - logp).abs()
    # (sums of powers near 1: a rounding each for up to 64 of a thread's, a tree of 8, two joins; the powers' own 2^-22)
    slack = rest * (2 * e_z + 4 * e_z ** 2) + 4 * U + rest * 128 * U + 4 * U * logp.abs()
    assert (off <= slack).all(), float((off / slack).max())
    p.each, p.scale, p.options = rows, 1.0, {}
    p.check()


@gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,d,classes", SHAPES + [(1, 256, 500), (400, 64, 90), (500, 96, 3000)])
@pytest.mark.parametrize("top", [4.0, 9.0, 14.0, 20.0, 40.0, 60.0])
def test_small_log_p_has_its_digits(layout, rows, d, classes, top):
    """log p = -log1p(sum of the others' powers): relative to itself, an error of 2 e_z for the logits, 2^-22 for each power, and for sums
    of at most 64 in a chain, however near to 1 p is.  Down to where a power leaves fp32."""
    p = Problem(rows, d, classes, seed=3, layout=layout, masked=0.0, weighted=False, spread=0.5)
    w = p.weight.float()[p.labels.long()]
    p.x.copy_((w * (top / w.square().sum(1, keepdim=True))).to(BF16))
    x, w = p.x.double(), p.weight.double()
    z = x @ w.t()
    y = p.labels.long().unsqueeze(1)
    others = (z - z.gather(1, y)).scatter(1, y, -math.inf)
    want = -torch.log1p(others.exp().sum(1))
    e_z = (d + 8) * U * (x.abs() @ w.abs().t()).amax(1)
    certain = want > -0.5
    assert int(certain.sum()) >= rows // 2 or top < 10.0
    for grads in (True, False):
        p.run(dx=grads, dw=grads)
        off = (p.logp.double() - want).abs()[certain]
        slack = (want.abs() * (torch.expm1(2 * e_z) + 70 * U))[certain]
        assert (p.logp < 0).all() and (off <= slack).all(), float((off / slack).max())
