"""Training the softmax model on cross-entropy over many classes under a gradient code: features, dropout, loss, partial
gradients, encode, decode, update."""
import subprocess
import sys

import numpy as np
import pytest
import torch

import ngc_inputs
import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200 import gd_loop
from tests._philox import kept, threshold
from tests._util import model_of, rel_l2

gpu = pytest.mark.gpu


def problem(n=6, rows=96, d=40, C=1000, levels=(0, 1, 2), seed=900, out=0.1):
    w = ngc_inputs.Workload("vocabulary_case", seed, n, levels, "softmax", rows, d, "bf16", n_classes=C)
    g = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn((n, rows, d), generator=g, device="cuda").bfloat16()
    theta = torch.randn(d * C, generator=g, device="cuda") * 0.3
    labels = torch.randint(0, C, (n * rows,), generator=g, device="cuda", dtype=torch.int32)
    labels[torch.rand(n * rows, generator=g, device="cuda") < out] = -1
    return w, X, theta, labels, ngc.Plan(n, levels, seed=3)


def expected(w, X, theta, labels, p=0.0, seed=0, step=0):
    """Gradient of theta and loss of every task, in 64 bits, at weights rounded to bf16."""
    rows = w.n * w.rows
    x = X.reshape(rows, w.d).double()
    if p:
        keep = torch.from_numpy(kept(rows, w.d, p, seed, step)).cuda()
        x = torch.where(keep, x * (65536.0 / (65536 - threshold(p))), 0.0)
    live = labels >= 0
    th = theta.bfloat16().double().requires_grad_()
    lp = torch.log_softmax(x @ th.view(w.d, w.n_classes), 1).gather(1, labels.clamp(min=0).long().unsqueeze(1)).squeeze(1)
    loss = torch.where(live, -lp, 0.0)
    return torch.autograd.grad(loss.sum(), th)[0], loss.detach().view(w.n, w.rows).sum(1)


@gpu
@pytest.mark.parametrize("C,d", [(1000, 40), (257, 72), (33, 33), (5003, 16)])
@pytest.mark.parametrize("p", [0.0, 0.25])
@pytest.mark.parametrize("side", [False, True])
def test_one_coded_iteration(C, d, p, side):
    """theta moves by the decoded gradient, which is the gradient of the whole data: G and the partial gradients are rounded to bf16
    (2^-8 of an element at most, each), and the decode adds up to sum |a_i| |b_ij| rounded partial gradients: of one norm each here, with
    weights below 20, so 20 2^-7 is far above what happens and far below what a wrong row, mask or task would do (0.2 and more)."""
    w, X, theta, labels, plan = problem(C=C, d=d)
    loss = gd_loop.VocabularyLoss(labels, w.n, dropout=p, seed=77)
    want, sums = expected(w, X, theta, labels, p, 77, 0)
    was = theta.clone()
    stream = torch.cuda.Stream() if side else None
    h = gd_loop.run(plan, model_of(w), theta, X, None, 1, 0.5, 11, loss=loss, stream=stream.cuda_stream if side else 0)
    torch.cuda.synchronize()
    assert len(h.latency) == 1 and not loss.gave_up()
    moved = (was.double() - theta.double()) / 0.5
    assert rel_l2(moved.cpu().numpy(), want.cpu().numpy()) < 0.02
    assert rel_l2(loss.loss.double().cpu().numpy(), sums.cpu().numpy()) < 1e-4


@gpu
def test_every_component_code_decodes_the_same_gradient():
    """Whichever workers answer, the masks of a partition agree between them: the decoded gradient does not depend on the code."""
    w, X, theta, labels, _ = problem(out=0.3)
    got = []
    for levels in ((0,), (1,), (2,)):
        th = theta.clone()
        loss = gd_loop.VocabularyLoss(labels, w.n, dropout=0.5, seed=5)
        gd_loop.run(ngc.Plan(w.n, levels, seed=3), model_of(w), th, X, None, 1, 1.0, 4, loss=loss)
        got.append((theta.double() - th.double()).cpu().numpy())
    for other in got[1:]:
        assert rel_l2(other, got[0]) < 1e-4


@gpu
@pytest.mark.parametrize("optimizer", ["gd", "adamw8"])
def test_iterations_draw_new_masks_and_repeat(optimizer):
    w, X, theta, labels, plan = problem()
    runs = []
    for seed in (1, 1, 2):
        th = theta.clone()
        loss = gd_loop.VocabularyLoss(labels, w.n, dropout=0.5, seed=seed)
        gd_loop.run(plan, model_of(w), th, X, None, 3, 1e-3, 4, loss=loss, optimizer=optimizer)
        runs.append(th)
    assert torch.equal(runs[0], runs[1]) and not torch.equal(runs[0], runs[2])
    a, _ = expected(w, X, theta, labels, 0.5, 1, 0)
    b, _ = expected(w, X, theta, labels, 0.5, 1, 1)
    assert rel_l2(a.cpu().numpy(), b.cpu().numpy()) > 0.1


@gpu
def test_two_codes_with_several_partitions_per_task():
    """k = 2 n partitions: a task is two of them."""
    n, rows, d, C = 4, 32, 24, 300
    w = ngc_inputs.Workload("vocabulary_case", 901, n, (0, 1), "softmax", rows, d, "bf16", n_classes=C)
    g = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randn((2 * n, rows, d), generator=g, device="cuda").bfloat16()
    theta = torch.randn(d * C, generator=g, device="cuda") * 0.3
    labels = torch.randint(0, C, (2 * n * rows,), generator=g, device="cuda", dtype=torch.int32)
    loss = gd_loop.VocabularyLoss(labels, n)
    double = ngc_inputs.Workload("vocabulary_case", 901, n, (0, 1), "softmax", 2 * rows, d, "bf16", n_classes=C)
    want, _ = expected(double, X, theta, labels)
    was = theta.clone()
    gd_loop.run(ngc.Plan(n, (0, 1), n_partitions=2 * n, seed=3), model_of(w), theta, X, None, 1, 1.0, 3, loss=loss)
    assert rel_l2((was.double() - theta.double()).cpu().numpy(), want.cpu().numpy()) < 0.02


@gpu
def test_refusals():
    w, X, theta, labels, plan = problem()
    with pytest.raises(ValueError):
        gd_loop.VocabularyLoss(labels, 7)
    with pytest.raises(ValueError):
        gd_loop.VocabularyLoss(labels, 0)
    with pytest.raises(ValueError):
        gd_loop.run(plan, model_of(w), theta, X, None, 1, 1.0, 3, loss=gd_loop.VocabularyLoss(labels, 3))
    f32 = ngc.Model.make("softmax", "f32", w.rows, w.d, w.n_classes)
    with pytest.raises(ValueError):
        gd_loop.run(plan, f32, theta, X, None, 1, 1.0, 3, loss=gd_loop.VocabularyLoss(labels, w.n))
    with pytest.raises(ngc.NgcError):
        gd_loop.run(plan, model_of(w), theta, X, None, 1, 1.0, 3, loss=gd_loop.VocabularyLoss(labels, w.n, dropout=2.0))


@gpu
@pytest.mark.parametrize("extra", [["--dropout", "0.1"], ["--optimizer", "adamw", "--classes", "777"]])
def test_command(extra):
    out = subprocess.run([sys.executable, "-m", "paper_2212_08580_b200.gd_loop", "--loss", "vocabulary", "--iters", "3", *extra],
                         capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    lines = out.stdout.strip().splitlines()
    assert len(lines) == 6 and "nan" not in out.stdout
    # every scheme decodes the same gradients
    final = [float(line.split()[-1]) for line in lines[1:]]
    assert np.ptp(final) <= 1e-2 * abs(final[0])
