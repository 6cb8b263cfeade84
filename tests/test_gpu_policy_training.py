"""The softmax model's two halves around a loss of the caller's, and training on such a loss under a gradient code."""
import numpy as np
import pytest
import torch

import ngc_inputs
import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200 import gd_loop
from tests._util import model_of, rel_l2

U = 2.0 ** -24
gpu = pytest.mark.gpu


def problem(n=6, rows=100, d=72, C=48, q=1, seed=900, levels=(0, 1, 2)):
    w = ngc_inputs.Workload("half_case", seed, n, levels, "softmax", rows, d, "bf16", n_classes=C)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    X = torch.randn((n * q, rows, d), generator=g, device="cuda").mul_(d ** -0.5).bfloat16()
    theta = torch.randn(d * C, generator=g, device="cuda")
    return w, X, theta, ngc.Plan(n, levels, n_partitions=n * q, seed=3), g


def test_halves_refuse_other_models_and_bad_arguments():
    p = ngc.Plan(4, [0, 1], seed=1)
    good = ngc.Model.make("softmax", "bf16", 8, 64, 16)
    at = type("A", (), {"data_ptr": lambda self: 0x1000})()
    off = type("A", (), {"data_ptr": lambda self: 0x1004})()
    for m in (ngc.Model.make("lsq", "f32", 8, 64), ngc.Model.make("softmax", "f32", 8, 64, 16),
              ngc.Model.make("softmax", "bf16", 8, 64, 20), ngc.Model.make("softmax", "bf16", 8, 63, 16),
              ngc.Model.make("softmax", "bf16", 8, 64, 272)):
        with pytest.raises(ngc.NgcError):
            p.shard_logits(m, at, at, 4, at)
        with pytest.raises(ngc.NgcError):
            p.shard_weight_gradients(m, at, at, 4, at, 1 << 20)
    for bad in ((off, at, 4, at), (at, off, 4, at), (at, at, 5, at), (at, at, 0, at), (at, at, 4, off)):
        with pytest.raises(ngc.NgcError):
            p.shard_logits(good, *bad)
    for bad in ((off, at, 4, at, 1024), (at, off, 4, at, 1024), (at, at, 4, off, 1024), (at, at, 4, at, 1020),
                (at, at, 4, at, 1026), (at, at, 9, at, 1024)):
        with pytest.raises(ngc.NgcError):
            p.shard_weight_gradients(good, *bad)


@gpu
@pytest.mark.parametrize("n,rows,d,C,q", [(6, 100, 72, 48, 1), (3, 1, 8, 16, 1), (4, 257, 200, 256, 2), (2, 300, 520, 256, 1),
                                          (5, 64, 64, 240, 3)])
def test_logits_and_weight_gradients(n, rows, d, C, q):
    w, X, theta, p, g = problem(n, rows, d, C, q, levels=(0,))
    m = model_of(w)
    logits = torch.empty((n * q * rows, C), dtype=torch.bfloat16, device="cuda")
    p.shard_logits(m, theta, X, n, logits)
    W = theta.view(d, C).bfloat16().double()     # the kernels' operand
    x = X.reshape(-1, d).double()
    z, size = x @ W, x.abs() @ W.abs()
    # fp32 sums of d exact products, one rounding to bf16 (half a step: 2^-8)
    assert ((logits.double() - z).abs() <= 2.0 ** -8 * z.abs() + 1.01 * d * U * size + 1e-38).all()
    delta = torch.randn((n * q * rows, C), generator=g, device="cuda").bfloat16()
    ld = d * C + 4
    G = torch.full((n, ld), 7.0, device="cuda")
    p.shard_weight_gradients(m, X, delta, n, G, ld)
    torch.cuda.synchronize()
    xs, ds = X.double().view(n, q * rows, d), delta.double().view(n, q * rows, C)
    want, size = torch.bmm(xs.transpose(1, 2), ds), torch.bmm(xs.abs().transpose(1, 2), ds.abs())
    got = G[:, :d * C].view(n, d, C).double()
    assert ((got - want).abs() <= 1.01 * (q * rows + 2) * U * size + 1e-38).all()
    assert (G[:, d * C:] == 7.0).all()
    assert p.device_status() < 1e-6


def expected_gradient(kind, w, X, theta, loss):
    """Sum over all rows of the loss's gradient with respect to theta, in 64 bits throughout."""
    th = theta.double().clone().requires_grad_()
    z = X.reshape(-1, w.d).double() @ th.view(w.d, w.n_classes)
    labels = loss.fixed[0].long()
    lp = torch.log_softmax(z, 1).gather(1, labels.unsqueeze(1)).squeeze(1)
    o = loss.options
    if kind == "policy":
        _, old, adv = (x.double() for x in loss.fixed)
        r, d = (lp - old).exp(), o["ref_logp"].double() - lp
        value = -torch.minimum(r * adv, r.clamp(1 - o["clip_low"], 1 + o["clip_high"]) * adv) + o["kl_coef"] * (d.exp() - d - 1)
    else:
        begin, ref = loss.fixed[1], loss.fixed[2].double()
        total = torch.cat([lp.new_zeros(1), lp.cumsum(0)])
        seq = total[begin[1:]] - total[begin[:-1]] - ref
        value = -torch.nn.functional.logsigmoid(o["beta"] * (seq[0::2] - seq[1::2]))
    return torch.autograd.grad(value.sum(), th)[0]


def make_loss(kind, w, X, theta, g):
    rows, C = w.n * w.rows, w.n_classes
    labels = torch.randint(0, C, (rows,), generator=g, device="cuda", dtype=torch.int32)
    z = X.reshape(rows, w.d).double() @ theta.double().view(w.d, C)
    lp = torch.log_softmax(z, 1).gather(1, labels.long().unsqueeze(1)).squeeze(1)
    if kind == "policy":
        # ratios that stay clear of the clip's borders, so that bf16 logits cannot push a row across one
        shift = torch.tensor([-0.6, -0.05, 0.08, 0.7], device="cuda")[torch.randint(0, 4, (rows,), generator=g, device="cuda")]
        return gd_loop.PolicyLoss(labels, (lp + shift).float(), torch.randn(rows, generator=g, device="cuda"), w.rows,
                                  ref_logp=(lp + 0.2).float(), kl_coef=0.1, clip_low=0.3, clip_high=0.3)
    begin = torch.arange(0, rows + 1, 5, device="cuda")   # sequences of five rows, pairs of ten within a partition
    ref = lp.view(-1, 5).sum(1) + torch.randn(rows // 5, generator=g, device="cuda")
    return gd_loop.PreferenceLoss(labels, begin, ref.float(), beta=0.7)


@gpu
@pytest.mark.parametrize("kind", ["policy", "preference"])
@pytest.mark.parametrize("C", [48, 256])
@pytest.mark.parametrize("side", [False, True])
def test_one_coded_iteration(kind, C, side):
    """Logits, loss, partial gradients, code, stragglers, decode, plain step: theta moves by the full gradient.  The
    logits (and the gradient of each row) are rounded to bf16, 2^-8 of values of a few units: one percent in the norm."""
    w, X, theta, p, g = problem(C=C)
    loss = make_loss(kind, w, X, theta, g)
    want = expected_gradient(kind, w, X, theta, loss)
    th = theta.clone()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream().cuda_stream if side else 0
    h = gd_loop.run(p, model_of(w), th, X, None, 1, 1.0, 11, p_fail=0.2, stream=stream, loss=loss)
    torch.cuda.synchronize()
    moved = (theta.double() - th.double()).cpu().numpy()
    assert len(h.level) == 1 and rel_l2(moved, want.cpu().numpy()) < 1e-2
    assert loss.loss.isfinite().all() and p.device_status() < 1e-6


@gpu
@pytest.mark.parametrize("kind", ["policy", "preference"])
@pytest.mark.parametrize("optimizer", ["adamw", "adamw8"])
def test_iterations_with_adamw(kind, optimizer):
    """Several iterations run, under different responsive sets, and do what their parts do one by one."""
    w, X, theta, p, g = problem()
    m = model_of(w)
    loss = make_loss(kind, w, X, theta, g)
    a, b = theta.clone(), theta.clone()
    gd_loop.run(p, m, a, X, None, 4, 0.02, 21, optimizer=optimizer, loss=loss)
    l = theta.numel()
    grad = torch.empty(l, device="cuda")
    opt = gd_loop.make_optimizer(optimizer, m, b, grad, 0.02)
    logits = torch.empty((w.n * w.rows, w.n_classes), dtype=torch.bfloat16, device="cuda")
    G, coded = torch.empty((w.n + 2, l), device="cuda"), torch.empty((w.n + 2, l), device="cuda")
    for it in range(4):
        info = p.select(np.ascontiguousarray(ngc.sample_times(21 + it, w.n, 3, 0.5, 0.5, 0.0)))
        p.shard_logits(m, b, X, w.n, logits)
        loss(logits, 0)
        p.shard_weight_gradients(m, X, logits, w.n, G, l)
        G[w.n:].copy_(G[:2])
        p.shard_encode_decode(m, info.layer, 0, w.n, G, l, info.responsive(), coded, grad)
        opt.update(grad_scale=1.0 / (w.n * w.rows))
    torch.cuda.synchronize()
    assert torch.equal(a, b) and not torch.equal(a, theta)


@gpu
def test_a_loss_needs_the_softmax_model():
    w = ngc_inputs.Workload("lsq_case", 7, 4, (0, 1), "lsq", 16, 64, "f32")
    X, y, theta = ngc_inputs.make_data(w, "cuda")
    with pytest.raises(ValueError):
        gd_loop.run(ngc.Plan(4, [0, 1], seed=1), model_of(w), theta, X, y, 1, 0.1, 1, loss=lambda z, s: None)


@gpu
def test_a_pair_that_no_worker_sees_whole_is_refused():
    """100 rows a partition, one or two partitions a task."""
    for q, begin, bad in ((1, [0, 40, 100, 130, 200], False), (1, [0, 40, 101, 130, 200], True), (1, [90, 100, 110], True),
                          (1, [60, 60, 100, 100, 200], False), (1, [30, 30, 30, 100, 100], False), (2, [0, 90, 200, 300, 400], False),
                          (2, [0, 90, 200, 300, 401], True), (1, [100, 100, 300], True)):
        w, X, theta, p, g = problem(q=q)
        labels = torch.randint(0, w.n_classes, (w.n * q * w.rows,), generator=g, device="cuda", dtype=torch.int32)
        before = theta.clone()
        loss = gd_loop.PreferenceLoss(labels, torch.tensor(begin, device="cuda"), torch.zeros(len(begin) - 1, device="cuda"))
        call = lambda: gd_loop.run(p, model_of(w), theta, X, None, 1, 1.0, 11, loss=loss)
        if bad:
            with pytest.raises(ValueError):
                call()
        else:
            call()
        torch.cuda.synchronize()
        assert torch.equal(theta, before) or not bad


@gpu
@pytest.mark.parametrize("side", [False, True])
def test_rows_that_no_sequence_holds_do_not_train(side):
    """Rows before the first and behind the last sequence: no loss, so no gradient."""
    w, X, theta, p, g = problem(C=48)
    loss = make_loss("preference", w, X, theta, g)
    labels, begin, ref = loss.fixed
    for first, last in ((0, 100), (4, 120), (6, 60)):
        part = gd_loop.PreferenceLoss(labels, begin[first:last + 1].contiguous(), ref[first:last].contiguous(), beta=0.7)
        want = expected_gradient("preference", w, X, theta, part)
        th = theta.clone()
        torch.cuda.synchronize()
        stream = torch.cuda.Stream().cuda_stream if side else 0
        gd_loop.run(p, model_of(w), th, X, None, 1, 1.0, 11, stream=stream, loss=part)
        torch.cuda.synchronize()
        moved = (theta.double() - th.double()).cpu().numpy()
        assert rel_l2(moved, want.cpu().numpy()) < 1e-2, (first, last)   # (bf16 logits, as above)
