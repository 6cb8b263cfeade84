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
