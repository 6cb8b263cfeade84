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
