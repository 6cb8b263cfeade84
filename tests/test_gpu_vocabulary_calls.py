"""Calls of linear_cross_entropy that its documentation allows: no rows, streams, workspaces of other types."""
import pytest
import torch

import paper_2212_08580_b200 as ngc
from tests.test_gpu_vocabulary import BF16, F32, Problem

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
