"""ngc_policy_loss and ngc_preference_loss under finite masks: classes that are ruled out by a large negative logit."""
import math

import pytest
import torch

import tests.test_gpu_losses as losses
from tests.test_gpu_losses import Policy, preference

gpu = pytest.mark.gpu
MASKS = [-1e4, -1e9, -1e10, -1e12, -1e20, -1e30]
SCALES = [0.7, 1.0, 1.3, 1 / 0.3]
# teams of lanes, a warp per row, blocks of several sizes, rows of several rounds
CLASSES = [13, 300, 1500, 5000, 20000, 70001]


def legal(rows, classes, labels):
    """Which classes each row may choose; the label always may, but in the row of nothing but masks."""
    keep = torch.zeros((rows, classes), dtype=torch.bool, device="cuda")
    at = torch.arange(classes, device="cuda")
    keep[1, :: max(1, classes // 16)] = True
    keep[2, : (classes + 1) // 2] = True
    keep[3, classes // 2:] = True
    keep[4, (at * 7) % 5 == 0] = True
    keep[5] = True
    keep[6, int(labels[6]) ^ 1 if (int(labels[6]) ^ 1) < classes else 0] = True
    for r in range(7):
        keep[r, int(labels[r])] = True
    return keep             # row 0: the label alone; row 7: nothing


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", CLASSES)
def test_policy_under_finite_masks(classes, dtype):
    for scale in SCALES:
        p = Policy(8, classes, dtype, scale=scale, each=3, seed=classes)
        logits = p.logits.clone()
        keep = legal(8, classes, p.labels)
        for mask in MASKS:
            p.logits.copy_(torch.where(keep, logits, torch.tensor(mask, dtype=p.dtype, device="cuda")))
            p.anchor()
            p.run()
            p.check()
            assert abs(p.logp[7].item() + math.log(classes)) <= 1e-6 * (1 + math.log(classes)), (scale, mask)
            want = p.grad.clone()
            p.run(grad=p.logits)                      # in place
            torch.cuda.synchronize()
            assert torch.equal(p.logits, want), (scale, mask)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", CLASSES)
def test_preference_under_finite_masks(classes, dtype):
    for scale in SCALES:
        p = preference([3, 2, 1, 2], classes, dtype, scale=scale, seed=classes)
        p.labels.clamp_(min=0)
        logits = p.logits.clone()
        keep = legal(8, classes, p.labels)
        for mask in MASKS:
            p.logits.copy_(torch.where(keep, logits, torch.tensor(mask, dtype=p.dtype, device="cuda")))
            p.anchor()
            p.run()
            p.check()
            want = p.grad.clone()
            p.run(grad=p.logits)
            torch.cuda.synchronize()
            assert torch.equal(p.logits, want), (scale, mask)


@gpu
@pytest.mark.parametrize("classes", CLASSES)
def test_rows_of_large_logits(classes):
    """A row that lies far from zero as a whole has the probabilities of the same row around zero (whole numbers beside
    2^e, which fp32 holds exactly up to e = 24)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(classes)
    for e in (10, 16, 19, 20, 21, 23):
        for sign in (1.0, -1.0):
            x = torch.randint(-6, 1, (6, classes), generator=g, device="cuda").float() + sign * 2.0 ** e
            p = Policy(6, classes, "f32", seed=e)
            p.logits.copy_(x)
            p.anchor()
            p.run()
            p.check()
            q = preference([2, 1, 2, 1], classes, "f32", seed=e)
            q.logits.copy_(x)
            q.anchor()
            q.run()
            q.check()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", CLASSES)
def test_masks_of_every_magnitude(classes, dtype):
    """From where an fp32 shift no longer holds every whole number to where its product with the scale is infinite."""
    g = torch.Generator(device="cuda")
    g.manual_seed(classes)
    for e in range(24, 128, 4):
        p = Policy(3, classes, dtype, seed=e)
        mask = -(2.0 ** e) * (1.0 + torch.rand(1, generator=g, device="cuda").item())
        p.logits[0, : classes - 1] = mask        # one class is left
        p.labels[0] = classes - 1
        p.logits[1] = mask                       # none is
        p.logits[2, ::2] = mask
        p.labels[2] = 1
        p.anchor()
        p.run()
        p.check()


class ExactRest(losses.Reference):
    """1 - p of the label from the other classes: 64 bits of p itself end at 1.1e-16, below which 1 - p of well separated logits
    lies.  What that moves is then compared within the half step of bf16 (2^-8), with as much again for fp32 errors."""

    def gradient(self, k, dk, dtype):
        want, tol = super().gradient(k, dk, dtype)
        rest = self.p.scatter(1, self.at, 0.0).sum(1, keepdim=True)
        lost = (1.0 - self.p.gather(1, self.at)) - rest
        move = torch.zeros_like(want).scatter_(1, self.at, (k.unsqueeze(1) * lost).where(self.live.unsqueeze(1), rest * 0.0))
        return want - move, torch.where(self.live.unsqueeze(1), tol + 2.0 ** -7 * move.abs(), 0.0)


@gpu
@pytest.mark.parametrize("classes", CLASSES)
def test_bf16_gradients_of_logits_far_from_zero(classes, monkeypatch):
    """The powers of a gradient belong to the sum they are divided by, wherever the row lies: the coefficient in one part,
    times logits of 2^e, is off by 2^(e - 23)."""
    monkeypatch.setattr(losses, "Reference", ExactRest)
    g = torch.Generator(device="cuda")
    g.manual_seed(classes)
    for e in (10, 13, 15, 16, 17):
        for sign in (1.0, -1.0):
            x = torch.randint(-6, 1, (6, classes), generator=g, device="cuda").float() * 2.0 ** (e - 7) + sign * 2.0 ** e
            p = Policy(6, classes, "bf16", seed=e)
            p.logits.copy_(x)
            p.logits[5] = sign * 2.0 ** e
            p.anchor()
            p.run()
            p.check()
            q = preference([2, 1, 2, 1], classes, "bf16", seed=e)
            q.logits.copy_(p.logits)
            q.anchor()
            q.run()
            q.check()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [13, 300, 5000, 70001])
@pytest.mark.parametrize("scale", [0.7, 1.0])
def test_a_label_at_the_types_lowest_value(classes, dtype, scale):
    """log p is scale times that value (what the other classes add is far below its rounding), not -infinity.  Beside ordinary
    logits (rows 0, 1), and beside logits of a magnitude that leaves the difference in the range or not (2, 3)."""
    low = torch.finfo(losses.DTYPES[dtype]).min
    p = Policy(4, classes, dtype, scale=scale, ref=False)
    p.old, p.ref = torch.full((4,), -3.0, device="cuda"), None
    p.logits[2:] = -2.0 ** 100
    p.logits[3] = 2.0 ** 125
    for r in range(4):
        p.logits[r, int(p.labels[r])] = low
    p.run()
    torch.cuda.synchronize()
    top = torch.tensor([0.0, 0.0, -2.0 ** 100, 2.0 ** 125], dtype=torch.float64, device="cuda")
    want = scale * (low - top)
    want[:2] = scale * low
    fits = want.abs() <= torch.finfo(torch.float32).max
    got = p.logp.double()
    assert ((got - want).abs() <= 4 * losses.U * want.abs())[fits].all() and (got[~fits] == -math.inf).all(), got.tolist()
    q = preference([1, 1, 1, 1], classes, dtype, scale=scale)
    q.labels.copy_(p.labels)
    q.logits.copy_(p.logits)
    q.run()
    torch.cuda.synchronize()
    assert ((q.seq_logp.double() - want).abs() <= 4 * losses.U * want.abs())[fits].all()
    assert p.grad.isfinite().all()
