"""Outputs of the losses that take the place of inputs: the same results as apart from them."""
import pytest
import torch

import paper_2212_08580_b200 as ngc
from tests.test_gpu_losses import Policy, preference

gpu = pytest.mark.gpu


def spoil(p):
    """Rows of every kind: left out, of nothing but masks, far from zero."""
    p.weight[2] = 0.0
    p.labels[3] = -1
    p.logits[4] = torch.finfo(p.dtype).min
    p.logits[5] = 1e6
    p.logits[6, ::2] = -1e10


@gpu
@pytest.mark.parametrize("classes", [20, 1500, 9000, 40000])
@pytest.mark.parametrize("logp_at,loss_at", [("old", "advantage"), ("advantage", "ref"), ("ref", "weight"), ("weight", "old")])
def test_policy_rows_in_place_of_inputs(classes, logp_at, loss_at):
    p = Policy(40, classes, "bf16", each=7)
    spoil(p)
    p.anchor()
    p.run()
    torch.cuda.synchronize()
    want = [x.clone() for x in (p.grad, p.logp, p.row_loss, p.loss)]
    outs = (getattr(p, logp_at), getattr(p, loss_at), p.loss)
    p.run(outs=outs)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, (p.grad,) + outs))


@gpu
@pytest.mark.parametrize("classes", [20, 9000])
def test_policy_sums_in_place_of_rows_and_inputs(classes):
    p = Policy(40, classes, "f32", each=1)
    spoil(p)
    p.anchor()
    p.run()
    torch.cuda.synchronize()
    want = p.row_loss.clone()
    assert torch.equal(p.loss, want)
    for at in ("row_loss", "old", "advantage"):
        q = Policy(40, classes, "f32", each=1)
        spoil(q)
        q.anchor()
        row_loss = torch.zeros(40, device="cuda")
        loss = row_loss if at == "row_loss" else getattr(q, at)
        q.run(outs=(torch.zeros(40, device="cuda"), row_loss, loss))
        torch.cuda.synchronize()
        assert torch.equal(row_loss, want) and torch.equal(loss, want)
    q = Policy(40, classes, "f32", each=8)
    spoil(q)
    q.anchor()
    q.run()
    torch.cuda.synchronize()
    want = q.loss.clone()
    q.run(outs=(torch.zeros(40, device="cuda"), torch.zeros(40, device="cuda"), q.advantage[:5]))
    torch.cuda.synchronize()
    assert torch.equal(q.advantage[:5], want)


@gpu
@pytest.mark.parametrize("classes", [20, 9000])
def test_preference_pairs_in_place_of_inputs(classes):
    p = preference([5, 3, 0, 4, 9, 2], classes, "f32")
    p.run()
    torch.cuda.synchronize()
    want = [x.clone() for x in (p.grad, p.seq_logp, p.pair_loss)]
    outs = (p.ref, p.weight)
    p.run(outs=outs)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, (p.grad,) + outs))


@gpu
def test_outputs_that_share_memory_are_refused():
    p = Policy(40, 20, "f32", each=7)
    p.anchor()
    buf = torch.zeros(100, device="cuda")
    with pytest.raises(ngc.NgcError):
        p.run(outs=(buf[:40], buf[:40], p.outputs()[2]))
    with pytest.raises(ngc.NgcError):
        p.run(outs=(buf[:40], buf[39:79], p.outputs()[2]))
    with pytest.raises(ngc.NgcError):
        p.run(outs=(buf[:40], buf[40:80], buf[38:44]))
    p.run(outs=(buf[:40], buf[40:80], buf[80:86]))          # side by side
    p.check()
