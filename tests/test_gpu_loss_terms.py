"""The policy loss's terms where its rows' numbers are small, large or equal: one class, whose log p is exactly 0."""
import math

import pytest
import torch

import paper_2212_08580_b200 as ngc

gpu = pytest.mark.gpu
U = 2.0 ** -24


def one_class(old, ref, advantage, weight=None, kl=1.0, classes=1, clip=0.2):
    """Losses and gradients of rows whose action is certain (classes = 1) or one of equally likely ones."""
    n = advantage.numel()
    x = torch.zeros((n, classes), device="cuda")
    grad = torch.empty_like(x)
    logp, loss = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    actions = torch.zeros(n, dtype=torch.int32, device="cuda")
    ngc.policy_loss(x, actions, old, advantage, grad, logp, loss, ref_logp=ref, weight=weight, kl_coef=kl,
                    clip_low=clip, clip_high=clip)
    torch.cuda.synchronize()
    return loss, grad, logp


@gpu
def test_kl_term_of_a_policy_next_to_its_reference():
    """With advantage 0 the loss is the KL term alone.  Up to 1/4 a series with at most seven roundings and coefficients
    rounded once, cut off at 1e-8; above, expm1 within one unit of its last place and two roundings."""
    d = torch.cat([s * 10.0 ** torch.linspace(-18, 0.7, 400, dtype=torch.float64) for s in (1.0, -1.0)])
    d = torch.cat([d, torch.tensor([0.0, 0.25, -0.25, 0.24999999, -0.24999999])]).float().cuda()
    zero = torch.zeros_like(d)
    loss, _, logp = one_class(zero, d, zero)
    assert (logp == 0).all() and (loss >= 0).all()
    x = d.double().cpu()
    # (64 bits lose the small ones in the same way: the series there too)
    want = torch.where(x.abs() < 1e-2, x * x / 2 * (1 + x / 3 * (1 + x / 4 * (1 + x / 5 * (1 + x / 6)))), torch.expm1(x) - x)
    tol = 16 * U * want + 1e-8 * want + torch.where(x.abs() >= 0.25, 2 * U * torch.expm1(x).abs(), 0.0) + 2.0 ** -149
    assert ((loss.double().cpu() - want).abs() <= tol).all()


def definition(lp, old, ref, adv, w, kl, clip=0.2):
    ratio = (lp - old).exp()
    free, held = ratio * adv, ratio.clamp(1 - clip, 1 + clip) * adv
    value, slope = -torch.minimum(free, held), torch.where(free <= held, -free, 0.0)
    if ref is not None:
        d = ref - lp
        value, slope = value + kl * (d.exp() - 1 - d), slope + kl * (1 - d.exp())
    return w * value, w * slope


@gpu
@pytest.mark.parametrize("classes", [2, 1024, 1 << 14])
@pytest.mark.parametrize("use_ref", [False, True])
def test_ratios_and_kl_terms_beyond_fp32(classes, use_ref):
    """Ratios and e^d up to e^200: what the advantage, the weight and kl_coef bring back into the range of fp32 is finite,
    and a row of advantage 0 has no share of its ratio."""
    lp = torch.full((12,), -math.log(classes), dtype=torch.float64, device="cuda")
    delta = torch.tensor([100.0, 100.0, 100.0, 87.9, 88.1, 88.8, 120.0, 0.1, 150.0, -150.0, 200.0, 3.0], dtype=torch.float64)
    adv = torch.tensor([0.0, 1.0, -1e-20, -1e-5, -1e-5, -1e-5, -1e-30, 0.5, 2.0, 1.0, 0.0, -1.0], device="cuda")
    d = torch.tensor([0.0, -0.1, 0.2, 88.5, 89.0, 95.0, 100.0, 110.0, -100.0, 0.1, 1.0, 0.5], dtype=torch.float64)
    old, ref = (lp - delta.cuda()).float(), (lp + d.cuda()).float()
    w = torch.full((12,), 1e-9, device="cuda")
    loss, grad, _ = one_class(old, ref if use_ref else None, adv, w, kl=0.05, classes=classes)
    want, slope = definition(lp, old.double(), ref.double() if use_ref else None, adv.double(), w.double(), 0.05)
    # log p within 4e-8 (and 2 U of itself), which the exponentials carry over; exp and expm1 two units in the last place,
    # products and the sum
    tol = (2 * 4e-8 + 4 * U * math.log(classes) + 16 * U) * (want.abs() + slope.abs() + 0.05 * 1e-9 * 10)
    assert want.abs().max() < 3e38 and loss.isfinite().all()
    assert ((loss.double() - want).abs() <= tol).all()
    k = slope.unsqueeze(1) * (torch.nn.functional.one_hot(torch.zeros(12, dtype=torch.int64), classes).cuda().double() - 1 / classes)
    assert grad.isfinite().all()
    assert ((grad.double() - k).abs() <= 2 * tol.unsqueeze(1) * (k.abs() / slope.abs().clamp(min=1e-300).unsqueeze(1)) + 1e-38).all()
    assert loss[0] == 0 or use_ref


@gpu
@pytest.mark.parametrize("classes", [40, 5000])
@pytest.mark.parametrize("scale", [1e-32, 3e-39, 2e-44])
def test_scales_below_the_range_of_normal_numbers(classes, scale):
    """Every class alike: p = 1 / classes, whatever is left of the coefficient's digits.  The weight brings the gradient back."""
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn((6, classes), device="cuda").to(dtype)
        grad = torch.empty_like(x)
        logp, loss = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
        w = torch.full((6,), 1e38, device="cuda")
        old = torch.full((6,), -math.log(classes), device="cuda")
        ngc.policy_loss(x, torch.zeros(6, dtype=torch.int32, device="cuda"), old, -w / w, grad, logp, loss, weight=w, scale=scale)
        torch.cuda.synchronize()
        assert ((logp.double() + math.log(classes)).abs() <= 4e-7).all()
        s = float(torch.tensor(scale, dtype=torch.float32))
        want = -s * 1e38 / classes * torch.ones(classes, dtype=torch.float64, device="cuda")
        want[0] += s * 1e38
        half = 0.0 if dtype == torch.float32 else 2.0 ** -8
        assert ((grad.double() - want).abs() <= (half + 2e-6) * want.abs()).all()
