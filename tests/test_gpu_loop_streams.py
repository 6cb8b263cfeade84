"""gd_loop.run on a stream that is not torch's current one: its memory belongs to that stream."""
import pytest
import torch

import ngc_inputs
import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200 import gd_loop
from tests._util import model_of

gpu = pytest.mark.gpu


def lsq(plan_levels=(0, 1, 2)):
    w = ngc_inputs.Workload("loop_case", 78, 6, plan_levels, "lsq", 64, 4096, "f32", unit_x=True)
    X, y, theta = ngc_inputs.make_data(w, "cuda")
    return w, X, y, theta, ngc.Plan(w.n, w.levels, seed=2)


def torch_calls(monkeypatch):
    """Records which stream is torch's current one when memory is asked for."""
    seen = []
    empty = torch.empty

    def record(*args, **kw):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", record)
    return seen


@gpu
@pytest.mark.parametrize("optimizer", ["gd", "adamw"])
def test_memory_of_the_loop_comes_from_its_stream(optimizer, monkeypatch):
    """What the loop frees when it returns may still be in use on its stream, and only there."""
    w, X, y, theta, plan = lsq()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    seen = torch_calls(monkeypatch)
    gd_loop.run(plan, model_of(w), theta, X, y, 2, 1e-3, 5, stream=side.cuda_stream, optimizer=optimizer)
    torch.cuda.synchronize()
    assert seen and set(seen) == {side.cuda_stream}


@gpu
@pytest.mark.parametrize("optimizer", ["gd", "adamw"])
def test_work_behind_the_loop_on_the_current_stream_leaves_it_alone(optimizer):
    w, X, y, theta, plan = lsq()
    want = theta.clone()
    gd_loop.run(plan, model_of(w), want, X, y, 3, 1e-3, 5, optimizer=optimizer)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    gd_loop.run(plan, model_of(w), theta, X, y, 3, 1e-3, 5, stream=side.cuda_stream, optimizer=optimizer)
    junk = [torch.full((n,), 1e9, device="cuda") for n in (w.n_params, w.n * w.n_params, 2 * w.n * w.n_params) for _ in range(8)]
    torch.cuda.synchronize()
    assert torch.equal(theta, want) and all((x == 1e9).all() for x in junk)


def policy_problem():
    w = ngc_inputs.Workload("loop_loss", 79, 6, (0, 1, 2), "softmax", 100, 72, "bf16", n_classes=48)
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    X = torch.randn((w.n, w.rows, w.d), generator=g, device="cuda").mul_(w.d ** -0.5).bfloat16()
    theta = torch.randn(w.d * w.n_classes, generator=g, device="cuda")
    rows = w.n * w.rows
    labels = torch.randint(0, w.n_classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    both = torch.randn((2, w.rows, w.n), generator=g, device="cuda")
    return w, X, theta, ngc.Plan(w.n, w.levels, seed=3), labels, both


def make(kind, w, labels, both):
    """A loss whose inputs its making copies (matrices that lie transposed)."""
    if kind == "policy":
        return gd_loop.PolicyLoss(labels, both[0].t(), both[1].t(), w.rows)
    begin = torch.arange(0, labels.numel() + 1, 5, device="cuda")
    return gd_loop.PreferenceLoss(labels.view(w.rows, w.n).t(), begin, both.view(-1)[: begin.numel() - 1], beta=0.7)


@gpu
@pytest.mark.parametrize("kind", ["policy", "preference"])
@pytest.mark.parametrize("own_stream", [False, True])
def test_a_loss_made_on_one_stream_and_used_on_another(kind, own_stream):
    """The inputs are copied, and the buffers may still be written, behind a long wait on the stream that the loss is made
    on; the loss is dropped while the loop's stream still works on it, and its memory is asked for again at once."""
    w, X, theta, plan, labels, both = policy_problem()
    m = model_of(w)
    want = theta.clone()
    gd_loop.run(plan, m, want, X, None, 2, 1e-3, 9, loss=make(kind, w, labels, both))
    torch.cuda.synchronize()
    side, maker = torch.cuda.Stream(), torch.cuda.Stream() if own_stream else torch.cuda.current_stream()
    late = torch.zeros_like(both)
    torch.cuda.synchronize()
    with torch.cuda.stream(maker):
        torch.cuda._sleep(100_000_000)
        late.copy_(both)
        loss = make(kind, w, labels, late)
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    gd_loop.run(plan, m, theta, X, None, 2, 1e-3, 9, stream=side.cuda_stream, loss=loss)
    sizes = [x.numel() for x in (loss.loss,) + ((loss.logp, loss.row_loss) if kind == "policy" else (loss.seq_logp,))]
    del loss
    with torch.cuda.stream(maker):
        junk = [torch.full((n,), 1e9, device="cuda") for n in sizes * 4]
    torch.cuda.synchronize()
    assert torch.equal(theta, want) and not torch.equal(theta, policy_problem()[2])
    assert all((x == 1e9).all() for x in junk)
