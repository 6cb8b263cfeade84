"""How exact log p is, over many rows: a systematic error of a row, however small, adds up over a sequence.

A pair whose rejected sequence is empty has the loss log(1 + e^-h), h = beta (lp - ref): with ref next to lp and a large beta
the loss, a number near ln 2 in fp32, tells lp to 2^-25 / (beta / 2), far better than lp itself rounded to fp32."""
import math

import pytest
import torch

import paper_2212_08580_b200 as ngc

gpu = pytest.mark.gpu
U = 2.0 ** -24
# teams of lanes of every width, a warp or a block per row, rows of one and of several rounds
CLASSES = [13, 300, 631, 1500, 5000, 20000, 32000, 70001]
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows_for(classes, long=False):
    return min(65536, (1 << 28) // classes) if long else max(2048, min(16384, (1 << 26) // classes))


def problem(rows, classes, dtype, seed, offset=0.0, raise_label=6.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, classes), generator=g, device="cuda").mul_(2.0)
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    at = labels.long().unsqueeze(1)
    x.scatter_add_(1, at, raise_label * torch.rand((rows, 1), generator=g, device="cuda"))
    if offset:
        x = (x * 8).round_() / 8 + offset         # exact in fp32 up to an offset of 2^20
    return x.to(KINDS[dtype]), labels


def exact_logp(x, labels, scale):
    out = torch.empty(labels.numel(), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // x.shape[1])
    for a in range(0, labels.numel(), step):
        z = x[a:a + step].double() * scale
        out[a:a + step] = torch.log_softmax(z, 1).gather(1, labels[a:a + step].long().unsqueeze(1)).squeeze(1)
    return out


def kernel_logp(x, labels, begin, lp, scale, beta):
    """log p of the sequences in `begin`, each the chosen one of a pair with an empty one, from the losses."""
    pairs = begin.numel() - 1
    both = torch.stack([begin[:-1], begin[1:]], 1).view(-1)
    both = torch.cat([both, begin[-1:]])
    ref = torch.zeros((pairs, 2), device="cuda")
    ref[:, 0] = lp.float()
    seq, loss = torch.empty(2 * pairs, device="cuda"), torch.empty(pairs, device="cuda")
    ws = torch.empty(ngc.preference_workspace_bytes(labels.numel(), pairs), dtype=torch.uint8, device="cuda")
    ngc.preference_loss(x, labels, both, ref.view(-1), None, seq, loss, ws, scale=scale, beta=beta)
    torch.cuda.synchronize()
    h = -torch.log(torch.expm1(loss.double()))
    return ref[:, 0].double() + h / beta


# Errors of a row: the logarithm's fraction (log1p within a unit of the last place of a number below 0.41: 2^-26 rms) and the
# sum's roundings, each 2^-24 / sqrt(3) of what a step of the tree adds, some 10 of them: 1.1e-7 at most, half of it where
# the steps' sizes differ; the powers' errors (2^-22 at most) average out over the classes that count.  Of systematic ones
# only what is left of the powers' mean: 1e-9 between octaves, and up to 5e-9 where bf16 logits take few of the fractions
# over which that mean is one; four deviations of a mean of 2048 rows are 4e-9.
MEAN, RMS = 1e-8, 1e-7
# Steep rows: a running sum drops terms below half its last place and rounds up those above, which of terms spread evenly
# over the orders of magnitude costs 0.31 * 2^-24 for each that lies within a factor e.  At scale 1 / 0.3 some 64 terms of
# a lane lie around that place with a deviation of 6.7 nats, 3.8 to a factor e; half of them come behind the largest one,
# and the last place is 0.72 * 2^-23 of a sum on average: 2.5e-8.
STEEP = MEAN + 2.5e-8


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", CLASSES)
@pytest.mark.parametrize("scale", [1.0, 0.9, 1 / 0.3])
def test_log_p_has_no_systematic_error(classes, dtype, scale):
    rows = rows_for(classes)
    x, labels = problem(rows, classes, dtype, classes, raise_label=6.0 / scale)
    lp = exact_logp(x, labels, scale)
    begin = torch.arange(rows + 1, device="cuda")
    off = kernel_logp(x, labels, begin, lp, scale, 1000.0) - lp
    mean, rms = off.mean().item(), off.square().mean().sqrt().item()
    assert abs(mean) <= (STEEP if scale > 1 else MEAN) and rms <= RMS, (mean, rms)


@gpu
@pytest.mark.parametrize("classes", [13, 300, 5000, 32000])
def test_log_p_of_rows_far_from_zero(classes):
    """Just below and above the shift from which rows subtract their largest logit first."""
    rows = rows_for(classes)
    for offset in (150_000.0, 2.0 ** 20, -2.0 ** 20):
        x, labels = problem(rows, classes, "f32", classes, offset)
        lp = exact_logp(x, labels, 1.0)
        off = kernel_logp(x, labels, torch.arange(rows + 1, device="cuda"), lp, 1.0, 1000.0) - lp
        mean, rms = off.mean().item(), off.square().mean().sqrt().item()
        # Below, a term's exponent loses up to 2^-22 of its own: 1.7e-7 in e, 1e-7 rms, averaged over the classes.  Above, all
        # logits of all rows are multiples of 1/8 below the largest, so that every row takes its powers at the same places,
        # some 2 sqrt(pi) 16 = 57 that count, and the error of a power (7e-8 rms) averages over those alone: four
        # deviations of such a mean.
        assert abs(mean) <= MEAN + 4 * 7e-8 / math.sqrt(57) and rms <= 2 * RMS, (offset, mean, rms)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [64, 256, 300, 5000, 32000])
def test_long_sequences(classes, dtype):
    """The error of a sequence grows with the root of its length and with the small mean, not with a row's largest error."""
    rows = rows_for(classes, long=True)
    x, labels = problem(rows, classes, dtype, 3 + classes)
    lp = exact_logp(x, labels, 1.0)
    begin = torch.tensor([0, rows // 4, rows], device="cuda")
    want = torch.stack([lp[: rows // 4].sum(), lp[rows // 4:].sum()])
    got = kernel_logp(x, labels, begin, want, 1.0, 10.0)
    n = (begin[1:] - begin[:-1]).double()
    # (the loss tells lp to 2^-25 / 5, and lp - ref, up to half a step of fp32, stays within h = 1)
    assert ((got - want).abs() <= MEAN * n + 5 * RMS * n.sqrt() + 2e-8).all(), ((got - want).tolist(), n.tolist())


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [13, 64, 256, 300, 631, 1500, 5000, 32000, 70001])
def test_policy_ratios_have_no_systematic_error(classes, dtype):
    """With the clip out of the way and advantage 1 the loss is minus the ratio, which next to 1 tells lp - old to 2^-24."""
    rows = rows_for(classes)
    x, labels = problem(rows, classes, dtype, 7 * classes)
    lp = exact_logp(x, labels, 1.0)
    old = lp.float()
    ones = torch.ones(rows, device="cuda")
    logp, loss = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ngc.policy_loss(x, labels, old, ones, None, logp, loss, clip_low=1.0, clip_high=1e30)
    torch.cuda.synchronize()
    off = torch.log(-loss.double()) - (lp - old.double())
    mean, rms = off.mean().item(), off.square().mean().sqrt().item()
    # The exponential and the ratio's last rounding, U each at most.  Numbers between 1 - U and 1 + U, an eighth of the rows,
    # round to 1 from further above than from below, which is U / 4 on average, twice.
    assert abs(mean) <= MEAN + 2 * U / 32 and rms <= RMS + U, (mean, rms)
    assert ((logp.double() - lp).abs() <= U * lp.abs() + 8 * RMS).all()
