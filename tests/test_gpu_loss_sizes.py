"""The losses at sizes where 32-bit arithmetic ends."""
import math

import pytest
import torch

import paper_2212_08580_b200 as ngc
from tests.test_gpu_losses import Policy, preference

gpu = pytest.mark.gpu
U = 2.0 ** -24


@gpu
@pytest.mark.parametrize("rows", [(1 << 31) - 33, (1 << 31) - 1])
def test_preference_sequences_that_end_at_the_largest_rows(rows):
    """Rows of two classes: the last sequences end at, and start at, the last row."""
    pairs = 64
    need = rows * (4 + 4) + ngc.preference_workspace_bytes(rows, pairs)
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip(f"needs {need >> 30} GB of device memory")
    logits = torch.zeros((rows, 2), dtype=torch.bfloat16, device="cuda")
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    ws = torch.empty(ngc.preference_workspace_bytes(rows, pairs), dtype=torch.uint8, device="cuda")
    # 62 pairs of equal lengths, one that ends at the last row, one of two empty sequences there
    at = [i * (rows // 125) for i in range(125)] + [rows - 7, rows, rows, rows]
    begin = torch.tensor(at, dtype=torch.int64, device="cuda")
    assert begin.numel() == 2 * pairs + 1
    n = (begin[1:] - begin[:-1]).double()
    ref = (-math.log(2) * n).float()
    seq, loss = torch.full((2 * pairs,), 5.0, device="cuda"), torch.full((pairs,), 5.0, device="cuda")
    weight = torch.ones(pairs, device="cuda")
    ngc.preference_loss(logits, labels, begin, ref, logits, seq, loss, ws, pair_weight=weight, beta=0.5)
    torch.cuda.synchronize()
    want = -math.log(2) * n
    # each row is off by 4e-8 at most, the sums of up to 2^24.04 rows are in 64 bits
    assert ((seq.double() - want).abs() <= 4e-8 * n + 2 * U * want.abs()).all()
    lp = seq.double()                                   # what the losses were made of, up to its rounding to fp32
    off = 0.5 * 2 * 2 * U * (want[0::2].abs() + want[1::2].abs()) + 0.5 * 4e-8 * 2 * n[0::2]
    h = 0.5 * ((lp - ref.double())[0::2] - (lp - ref.double())[1::2])
    assert ((loss.double() - torch.nn.functional.softplus(-h)).abs() <= 1.01 * off + 2 * U * (1 + loss.double())).all()
    slope = 0.5 * torch.sigmoid(-h)                     # gradient of a chosen row: -slope (onehot - p), p = 1/2
    for q, r in ((0, 0), (61, at[124] - 1), (62, rows - 8), (62, at[124])):
        chosen = r < at[2 * q + 1]
        x = -slope[q] / 2 * (1 if chosen else -1)
        assert abs(logits[r, 0].item() - x.item()) <= (2.0 ** -8 + 0.51 * off[q].item()) * abs(x.item()) + 1e-30, (q, r)
        assert logits[r, 1].item() == -logits[r, 0].item()
    r = rows - 3                                        # the rejected sequence of pair 62
    assert abs(logits[r, 0].item() - slope[62].item() / 2) <= (2.0 ** -8 + 0.51 * off[62].item()) * slope[62].item()
    del logits, labels, ws
    torch.cuda.empty_cache()


@gpu
def test_policy_of_the_most_rows():
    rows, each = (1 << 31) - 1, 1 << 20
    need = rows * 20
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip(f"needs {need >> 30} GB of device memory")
    logits = torch.zeros((rows, 2), dtype=torch.bfloat16, device="cuda")
    actions = torch.zeros(rows, dtype=torch.int32, device="cuda")
    old = torch.full((rows,), -math.log(2), device="cuda")
    parts = -(-rows // each)
    row_loss, loss = torch.full((rows,), 5.0, device="cuda"), torch.full((parts,), 5.0, device="cuda")
    old[-1] = math.inf                                   # a ratio of 0: the last row's loss is 0
    adv = torch.ones(1, device="cuda").expand(rows).contiguous()
    ngc.policy_loss(logits, actions, old, adv, logits, None, row_loss, loss, rows_per_partition=each)
    torch.cuda.synchronize()
    n = torch.full((parts,), float(each), dtype=torch.float64, device="cuda")
    n[-1] = rows - (parts - 1) * each - 1
    # a row's ratio is one within its log p (4e-8) and old's rounding and the exponential's (2^-23 each)
    assert ((loss.double() + n).abs() <= (4e-8 + 2.0 ** -22) * n + 2 * U * n).all()
    assert row_loss[-1] == 0 and (logits[-1] == 0).all()
    for r in (0, (1 << 30) + 7, rows - 2):
        assert logits[r, 0].item() == -0.5 and logits[r, 1].item() == 0.5
    del logits, actions, old, adv, row_loss
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("dtype,classes", [("bf16", 40), ("bf16", 5000), ("f32", 20000)])
def test_rows_whose_offsets_pass_32_bits(dtype, classes):
    """Five rows 2^30 elements apart."""
    pad = (1 << 30) - classes
    if torch.cuda.mem_get_info()[0] < (56 << 30):
        pytest.skip("needs 56 GB of device memory")
    p = Policy(5, classes, dtype, pad=pad, each=2)
    p.anchor()
    p.run()
    p.check()
    want = p.grad.clone()
    p.run(grad=p.logits)
    torch.cuda.synchronize()
    assert torch.equal(p.logits, want)
    del p, want
    torch.cuda.empty_cache()
    p = preference([2, 1], classes, dtype, pad=pad, before=1, behind=1)
    p.run()
    p.check()
    del p
    torch.cuda.empty_cache()
