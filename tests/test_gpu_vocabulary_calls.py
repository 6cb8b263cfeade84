"""Calls of linear_cross_entropy and dropout that their documentation allows: no rows, streams, workspaces of other types, column
blocks of one buffer; what the coded loop keeps and tells."""
import pytest
import torch

import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200 import gd_loop
from tests._util import model_of, rel_l2
from tests.test_gpu_vocabulary import BF16, F32, Problem
from tests.test_gpu_vocabulary_training import expected, problem

gpu = pytest.mark.gpu


def no_rows(p, **more):
    p.x, p.labels, p.row_weight, p.rows = p.x[:0], p.labels[:0], None, 0
    p.outputs(1, True, True)
    ws = torch.full((256,), 255, dtype=torch.uint8, device="cuda")
    args = {"dx": p.dx, "dweight": p.dw[0], **more}
    ngc.linear_cross_entropy(p.x, p.weight, p.labels, p.logp, p.row_loss, p.loss[:0], ws, **args)
    return ws


@gpu
def test_no_rows_clear_the_status():
    p = Problem(8, 40, 30)
    assert not ngc.linear_cross_entropy_gave_up(no_rows(p))
    assert (p.dw == 0).all()
    assert not ngc.linear_cross_entropy_gave_up(no_rows(p, dweight=None))


@gpu
def test_no_rows_leave_the_weights():
    p = Problem(8, 40, 30)
    was = p.weight.clone()
    with pytest.raises(ngc.NgcError):
        no_rows(p, dweight=p.weight)
    assert torch.equal(p.weight, was)


@gpu
def test_gave_up_waits_for_every_stream():
    ws = torch.zeros(1024, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
        ws[:4].view(torch.int32).fill_(1)
    assert ngc.linear_cross_entropy_gave_up(ws)


@gpu
@pytest.mark.parametrize("dtype", [torch.uint8, torch.int8, BF16, F32, torch.float64])
def test_workspaces_of_any_type(dtype):
    p = Problem(40, 32, 300)
    p.run()
    p.workspace = p.workspace[: p.workspace.numel() // 8 * 8].view(dtype)
    p.run(outputs=False)
    assert not ngc.linear_cross_entropy_gave_up(p.workspace)
    p.workspace.view(torch.uint8)[:4].view(torch.int32).fill_(1)
    assert ngc.linear_cross_entropy_gave_up(p.workspace)


@gpu
def test_a_loop_goes_on_with_its_masks():
    """A loss that is run again draws the masks of the iterations after the last one's."""
    w, X, theta, labels, plan = problem()
    loss = gd_loop.VocabularyLoss(labels, w.n, dropout=0.5, seed=9)
    for step, iters in ((0, 1), (1, 1), (4, 3)):
        gd_loop.run(plan, model_of(w), theta, X, None, iters, 0.0, 4, loss=loss)
        _, sums = expected(w, X, theta, labels, 0.5, 9, step)
        assert rel_l2(loss.loss.double().cpu().numpy(), sums.cpu().numpy()) < 1e-4
    loss.iteration = 1  # (a run that is taken up again)
    gd_loop.run(plan, model_of(w), theta, X, None, 1, 0.0, 4, loss=loss)
    _, sums = expected(w, X, theta, labels, 0.5, 9, 1)
    assert rel_l2(loss.loss.double().cpu().numpy(), sums.cpu().numpy()) < 1e-4


@gpu
def test_features_that_are_not_contiguous_on_a_side_stream(monkeypatch):
    """The copy of such features is work of the loop's stream too."""
    w, X, theta, labels, plan = problem()
    want, _ = expected(w, X, theta, labels)
    wide = torch.zeros((w.n, w.rows + 5, w.d), dtype=BF16, device="cuda")
    wide[:, : w.rows] = X
    was = theta.clone()
    loss = gd_loop.VocabularyLoss(labels, w.n)
    gd_loop.run(plan, model_of(w), theta.clone(), X, None, 1, 0.5, 11, loss=loss)  # (kernels are loaded)
    torch.cuda.synchronize()
    real = plan.select

    def late(times):
        torch.cuda._sleep(400_000_000)  # (the current stream falls behind)
        return real(times)

    monkeypatch.setattr(plan, "select", late)
    s = torch.cuda.Stream()
    gd_loop.run(plan, model_of(w), theta, wide[:, : w.rows], None, 1, 0.5, 11, loss=loss, stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert rel_l2(((was.double() - theta.double()) / 0.5).cpu().numpy(), want.cpu().numpy()) < 0.02


@gpu
@pytest.mark.parametrize("side", [False, True])
@pytest.mark.parametrize("when", [0, 2])
def test_a_loop_tells_that_a_wait_gave_up(monkeypatch, side, when):
    """The status word set from the host's side behind one iteration's call: the run ends with an error, once."""
    w, X, theta, labels, plan = problem()
    loss = gd_loop.VocabularyLoss(labels, w.n)
    calls = []
    real = gd_loop.linear_cross_entropy

    def spoiled(*args, stream=0, **more):
        real(*args, stream=stream, **more)
        if len(calls) == when:
            with gd_loop._on(stream):
                args[6][:4].view(torch.int32).fill_(1)
        calls.append(stream)

    monkeypatch.setattr(gd_loop, "linear_cross_entropy", spoiled)
    s = torch.cuda.Stream() if side else None
    stream = s.cuda_stream if side else 0
    with pytest.raises(ngc.NgcError) as e:
        gd_loop.run(plan, model_of(w), theta, X, None, 3, 0.1, 4, loss=loss, stream=stream)
    assert e.value.status == -5 and len(calls) == 3
    h = gd_loop.run(plan, model_of(w), theta, X, None, 2, 0.1, 4, loss=loss, stream=stream)
    assert len(h.latency) == 2 and not loss.gave_up()


@gpu
@pytest.mark.parametrize("columns", [64, 40, 37])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_dropout_between_column_blocks(columns, dtype):
    buf = torch.randn((50, 3 * columns + 1), device="cuda").to(dtype)
    was = buf.clone()
    x, residual, out = (buf[:, i * columns:(i + 1) * columns] for i in range(3))
    want = torch.empty((50, columns), dtype=dtype, device="cuda")
    ngc.dropout(x.contiguous(), want, 0.3, seed=4, residual=residual.contiguous())
    ngc.dropout(x, out, 0.3, seed=4, residual=residual)
    assert torch.equal(out, want)
    assert torch.equal(buf[:, : 2 * columns], was[:, : 2 * columns]) and torch.equal(buf[:, 3 * columns:], was[:, 3 * columns:])
    for shared in (buf[:, 1: columns + 1], buf[:, columns - 1: 2 * columns - 1]):  # a column of x, of the residual, of both
        with pytest.raises(ngc.NgcError):
            ngc.dropout(x, shared, 0.3, seed=4, residual=residual)
    # blocks that touch around a row's end
    flat = torch.randn(51 * 3 * columns, device="cuda").to(dtype)
    a, b = flat[: 50 * 3 * columns].view(50, 3 * columns), flat[2 * columns: 2 * columns + 50 * 3 * columns].view(50, 3 * columns)
    with pytest.raises(ngc.NgcError):
        ngc.dropout(a[:, : columns], b[:, 1: columns + 1], 0.3, seed=4)  # (columns 2 c + 1 .. 3 c: the last one is the next row's first)
    ngc.dropout(a[:, : columns], b[:, : columns], 0.3, seed=4)


@gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("d,classes", [(64, 320), (72, 130), (33, 301)])
@pytest.mark.parametrize("keep", [False, True])
def test_gradients_beside_their_operands(layout, d, classes, keep):
    """Features and their gradient, weights and theirs, as column blocks of one buffer each; none writes the other's."""
    if keep and d % 8:
        d += 7
    want = Problem(200, d, classes, layout=layout, masked=0.0 if keep else 0.3).run()
    p = Problem(200, d, classes, layout=layout, masked=0.0 if keep else 0.3)
    p.outputs(1)
    rows = torch.zeros((200, 2 * d), dtype=BF16, device="cuda")
    rows[:, :d] = p.x
    a, b = (classes, d) if layout == "classes" else (d, classes)
    both = torch.zeros((a, 2 * b), dtype=BF16, device="cuda")
    both[:, :b] = p.weight if layout == "classes" else p.weight.t()
    was = rows[:, :d].clone(), both[:, :b].clone()
    p.x, p.dx, p.dx_full = rows[:, :d], rows[:, d:], p.dx_full
    w, dw = both[:, :b], both[:, b:]
    p.weight, p.dw = (w, dw.unsqueeze(0)) if layout == "classes" else (w.t(), dw.t().unsqueeze(0))
    n = ngc.linear_cross_entropy_workspace_bytes(p.x, p.weight, dx=p.dx, dweight=p.dw, keep_rows=keep)
    p.workspace = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    p.run(outputs=False, keep_rows=keep).check()
    assert torch.equal(rows[:, :d], was[0]) and torch.equal(both[:, :b], was[1])
    if not keep:
        assert torch.equal(p.logp, want.logp)
    for wrong in (rows[:, d - 1:2 * d - 1], rows[:, 1:d + 1]):
        with pytest.raises(ngc.NgcError):
            ngc.linear_cross_entropy(p.x, p.weight, p.labels, p.logp, p.row_loss, p.loss, p.workspace, dx=wrong, dweight=p.dw)
