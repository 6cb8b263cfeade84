"""How exact log p of linear_cross_entropy is at long contractions, against 64 bits.

The tensor cores add 16 products at a time to an accumulator and cut what does not fit.  Half a step of the accumulator each time, 2^-24
of what it holds, is the allowance here; accumulators go on for at most 256 features, after which they are added in fp32 with
rounding.  What is cut depends on the data: sums that grow evenly lose the most, features with few or one non-zero
element next to nothing.  So a row's allowance is taken from its own partial sums."""
import pytest
import torch

import paper_2212_08580_b200 as ngc
from tests.test_gpu_vocabulary import BF16, F32

gpu = pytest.mark.gpu
U = 2.0 ** -24
KINDS = ["dense", "positive", "cancelling", "few", "one-hot", "leading"]


def problem(kind, rows, d, classes, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((rows, d), device="cuda").normal_(generator=g)
    w = torch.empty((classes, d), device="cuda").normal_(0.0, 2.0 * d ** -0.5, generator=g)
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    at = torch.arange(d, device="cuda")
    if kind == "positive":            # logits of 30 and what sets classes apart
        x, w = x.abs(), w.abs() + 28.0 / d
    elif kind == "cancelling":        # grows to some 100 and comes back
        x = torch.where(at < d // 2, 1.0, -1.0) + 0.02 * x
        w = 200.0 / d * (1.0 + 0.5 * w * d ** 0.5 * 0.05) + 0 * w
    elif kind == "few":               # eight non-zero features, classes told apart by them; whole numbers, so logits are exact
        x = torch.where((at * 8) % d < 8, (3.0 * x).round(), 0.0)
        w = (w * d ** 0.5 * 2.0).round()
    elif kind == "one-hot":
        x = torch.zeros_like(x)
        x[torch.arange(rows, device="cuda"), torch.randint(0, d, (rows,), generator=g, device="cuda")] = 1.0
        w = (w * d ** 0.5 * 8.0).round()
    elif kind == "leading":           # one feature dominates
        x[:, 0] = 1.0
        w[:, 0] = 40.0 + w[:, 0]
    return x.to(BF16), w.to(BF16), labels


def logp_of(x, w, labels, layout, grads):
    weight = w if layout == "classes" else w.t().contiguous().t()
    rows = x.shape[0]
    out = [torch.empty(rows, dtype=F32, device="cuda") for _ in range(2)]
    dx = torch.empty_like(x) if grads else None
    ws = torch.empty(ngc.linear_cross_entropy_workspace_bytes(x, weight, dx=dx), dtype=torch.uint8, device="cuda")
    ngc.linear_cross_entropy(x, weight, labels, *out, None, ws, dx=dx)
    assert not ngc.linear_cross_entropy_gave_up(ws)
    return out[0].double()


def allowance(x, w, labels, each=256):
    """Exact logits, and for each the sum over steps of 16 products of 2^-24 of the accumulator, which begins anew every 256 features,
    and of the additions of these in fp32."""
    rows, d = x.shape
    x, w = x.double(), w.double()
    z = torch.zeros((rows, w.shape[0]), dtype=torch.float64, device="cuda")
    cut = torch.zeros_like(z)
    for a in range(0, d, each):
        s = torch.zeros_like(z)
        for b in range(a, min(d, a + each), 16):
            s += x[:, b:b + 16] @ w[:, b:b + 16].t()
            cut += U * s.abs()
        z += s
        cut += U * z.abs()
    y = labels.long().unsqueeze(1)
    lp = torch.log_softmax(z, 1)
    want = lp.gather(1, y).squeeze(1)
    p = lp.exp()
    # the label's own cut, the others' as they count; powers (2^-22 each), the logarithm and the last product: a rounding or two of numbers below 16
    slack = (1.0 - p.gather(1, y)).squeeze(1) * (cut.gather(1, y).squeeze(1) + (p * cut).sum(1)) + 4 * U * (1.0 + want.abs())
    return want, slack


@gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [256, 1024, 1032, 2048, 4096, 8192])
@pytest.mark.parametrize("rows,classes,grads", [(96, 700, False), (512, 700, False), (512, 700, True), (512, 240, True), (512, 100, False)])
def test_log_p_over_long_features(layout, kind, d, rows, classes, grads):
    x, w, labels = problem(kind, rows, d, classes, d + rows)
    want, slack = allowance(x, w, labels)
    off = logp_of(x, w, labels, layout, grads) - want
    rms = float(off.square().mean().sqrt()), float(slack.square().mean().sqrt())
    assert rms[0] <= rms[1], rms
    # the systematic part, which adds up over a sequence
    assert abs(float(off.mean())) <= float(slack.mean()), (float(off.mean()), float(slack.mean()))


@gpu
@pytest.mark.parametrize("kind", ["few", "one-hot"])
@pytest.mark.parametrize("d", [16384, 131072])
@pytest.mark.parametrize("rows", [64, 200])
def test_exact_logits_stay_exact(kind, d, rows):
    """Logits that are whole numbers and partial sums that fp32 holds: nothing is cut at any length."""
    x, w, labels = problem(kind, rows, d, 300, 5)
    z = x.double() @ w.double().t()
    assert (z == z.round()).all() and float(z.abs().max()) < 2 ** 20
    want = torch.log_softmax(z, 1).gather(1, labels.long().unsqueeze(1)).squeeze(1)
    off = (logp_of(x, w, labels, "classes", False) - want).abs()
    # powers 2^-22 (their arguments: a rounding of (z - max) log2(e) that matters below 20), sums, logarithm, product
    assert (off <= 64 * U + 4 * U * want.abs()).all(), float((off / U).max())
