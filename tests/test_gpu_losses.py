"""ngc_policy_loss and ngc_preference_loss against their definitions in 64 bits."""
import ctypes as C
import math

import pytest
import torch

import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200.binding import PolicyLossConfig, PreferenceLossConfig

gpu = pytest.mark.gpu
U = 2.0 ** -24  # half a step of fp32, relative
LOW, HIGH, KL = 0.2, 0.3, 0.05
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
AT = 0x100000  # an address that nothing is read from


def policy_call(cfg=None, **kw):
    c = dict(rows=4, rows_per_partition=2, n_classes=10, dtype=ngc.NGC_F32, scale=1.0, clip_low=0.2, clip_high=0.2, kl_coef=0.1)
    a = dict(logits=AT, ld=10, actions=AT, old=AT, ref=AT, adv=AT, weight=AT, grad=AT + 4096, ldg=10, logp=AT, row_loss=AT,
             loss=AT)
    c.update({k: v for k, v in kw.items() if k in c})
    a.update({k: v for k, v in kw.items() if k in a})
    return ngc.load_library().ngc_policy_loss(C.byref(PolicyLossConfig(**c)), a["logits"], a["ld"], a["actions"], a["old"],
                                              a["ref"], a["adv"], a["weight"], a["grad"], a["ldg"], a["logp"],
                                              a["row_loss"], a["loss"], None)


@pytest.mark.parametrize("kw", [
    {"rows": -1}, {"rows": 1 << 31}, {"rows_per_partition": 0}, {"n_classes": 0}, {"dtype": ngc.NGC_F64}, {"dtype": 9},
    {"scale": 0.0}, {"scale": -1.0}, {"scale": math.nan}, {"scale": math.inf}, {"scale": 1e-60}, {"scale": 3e38},
    {"clip_low": -0.1}, {"clip_low": 1.5}, {"clip_high": -0.1}, {"clip_high": math.inf}, {"kl_coef": -1.0},
    {"kl_coef": math.nan}, {"ld": 9}, {"ldg": 9}, {"ldg": 12, "grad": AT}, {"logits": None}, {"logits": AT + 2},
    {"grad": AT + 1}, {"actions": None}, {"old": None}, {"adv": None}, {"row_loss": None}, {"actions": AT + 1},
    {"ref": AT + 2}, {"loss": AT + 3}])
def test_policy_refusals(kw):
    assert policy_call(**kw) == -1


def test_policy_without_rows_does_nothing():
    assert policy_call(rows=0, logits=None, actions=None, row_loss=None) == 0


def preference_call(**kw):
    c = dict(rows=4, pairs=2, n_classes=10, dtype=ngc.NGC_BF16, length_mean=0, scale=1.0, beta=0.1, label_smoothing=0.0)
    a = dict(logits=AT, ld=10, labels=AT, begin=AT, ref=AT, weight=AT, grad=AT + 4096, ldg=10, seq=AT, loss=AT, ws=AT,
             ws_bytes=1 << 20)
    c.update({k: v for k, v in kw.items() if k in c})
    a.update({k: v for k, v in kw.items() if k in a})
    return ngc.load_library().ngc_preference_loss(C.byref(PreferenceLossConfig(**c)), a["logits"], a["ld"], a["labels"],
                                                  a["begin"], a["ref"], a["weight"], a["grad"], a["ldg"], a["seq"],
                                                  a["loss"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw", [
    {"rows": -1}, {"rows": 1 << 31}, {"pairs": -1}, {"pairs": 0x3fffffff}, {"n_classes": 0}, {"dtype": ngc.NGC_E4M3},
    {"scale": 0.0}, {"scale": math.inf}, {"beta": math.nan}, {"label_smoothing": -0.1}, {"label_smoothing": 1.1},
    {"ld": 9}, {"ldg": 9}, {"ldg": 11, "grad": AT}, {"logits": None}, {"labels": None}, {"begin": None},
    {"begin": AT + 4}, {"ref": None}, {"seq": None}, {"loss": None}, {"ws": None}, {"ws": AT + 8}, {"ws_bytes": 16},
    {"logits": AT + 1}, {"grad": AT + 1}, {"labels": AT + 2}, {"weight": AT + 1}])
def test_preference_refusals(kw):
    assert preference_call(**kw) == -1


def test_workspace_grows_with_the_rows():
    sizes = [ngc.preference_workspace_bytes(r, 3) for r in (0, 1, 1000, 100000)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and sizes[-1] < 100000 * 64
    assert ngc.preference_workspace_bytes(-1, 3) == 0


def test_tensors_that_are_not_on_the_device_are_refused():
    x, i = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ngc.NgcError):
        ngc.policy_loss(x, i, x[:, 0], x[:, 0], x, x[:, 0], x[:, 0])
    with pytest.raises(ngc.NgcError):
        ngc.preference_loss(x, i, i, x[:, 0], x, x[:, 0], x[:, 0], x)


# ---- on the device


def matrix(g, rows, classes, dtype, pad=0, offset=0, std=2.0):
    """[rows, classes] inside a larger buffer: `pad` more columns, the first element `offset` elements in."""
    flat = torch.full((offset + rows * (classes + pad) + 8,), 99.0, dtype=dtype, device="cuda")
    m = flat[offset:offset + rows * (classes + pad)].view(rows, classes + pad)
    m[:, :classes] = (std * torch.randn((rows, classes), generator=g, device="cuda")).to(dtype)
    return flat, m[:, :classes]


def row_errors(x, scale, top, live_rows):
    """A bound on the relative error of a row's fp32 sums.  A term's exponent: at most three roundings (c, which is kept in two
    parts, a product and a sum), and terms further than 40 below the maximum no longer count; 2^-22 for each 2^x, of
    which a term sees one of its own, and one for every join of partial sums in which the maximum moved if the powers
    between whole-number shifts are not exact: a thread joins its up to V / 1024 rounds, then 5 steps in the warp and
    at most 16 warps, with 8 to spare; one rounding for every addition on that way."""
    joins = x.shape[1] / 1024 + 5 + 16 + 8 + 2
    reach = (scale * (top - x.masked_fill(x == -math.inf, math.inf).amin(1))).clamp(max=40.0)
    return U * (3 * reach + 4 * (joins + 1) + 8 + joins)


class Reference:
    """log p of the labels and p itself in 64 bits, rows that count, and the error of the kernel's log p."""

    def __init__(self, logits, labels, scale, counted):
        self.x = logits.double()
        n = logits.shape[1]
        self.live = counted & (labels >= 0) & (labels < n) & ~(self.x == -math.inf).all(1)
        self.x = torch.where(self.live.unsqueeze(1), self.x, torch.zeros_like(self.x))
        self.at = torch.where(self.live, labels, 0).long().unsqueeze(1)
        self.scale = scale
        lsm = torch.log_softmax(scale * self.x, 1)
        self.p = lsm.exp()
        self.logp = lsm.gather(1, self.at).squeeze(1)
        top = self.x.amax(1)
        self.rel = row_errors(self.x, scale, top, self.live)
        self.dlogp = self.rel + U * (scale * (top - self.x.gather(1, self.at).squeeze(1))).abs() + 2 * U

    def gradient(self, k, dk, dtype):
        """k (onehot - p), and how far the kernel's may be off: the factor, the probability, three roundings, the output."""
        one = torch.zeros_like(self.p).scatter_(1, self.at, 1.0)
        rest = 1.0 - self.p.gather(1, self.at)
        share = torch.where(one > 0, rest, self.p)
        want = k.unsqueeze(1) * (one - self.p)
        reach = (self.scale * (self.x.amax(1, keepdim=True) - self.x)).clamp(max=90.0)
        tol = (dk.unsqueeze(1) + k.abs().unsqueeze(1) * (2 * self.rel.unsqueeze(1) + U * (3 * reach + 8))) * share
        tol = tol + 4 * U * want.abs() + (torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0.0) * want.abs()
        want = torch.where(self.live.unsqueeze(1), want, 0.0)
        return want, torch.where(self.live.unsqueeze(1), 1.01 * tol + 1e-36, 0.0)


class Policy:
    def __init__(self, rows, classes, dtype="f32", seed=0, pad=0, offset=0, grad_offset=None, scale=1.0, ref=True,
                 weight=True, each=None, std=2.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed * 7919 + rows * 31 + classes)
        self.dtype = DTYPES[dtype]
        self.flat, self.logits = matrix(g, rows, classes, self.dtype, pad, offset, std)
        self.grad_flat, self.grad = matrix(g, rows, classes, self.dtype, pad, offset if grad_offset is None else grad_offset)
        self.labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
        self.scale, self.each = scale, each or rows
        self.advantage = torch.randn(rows, generator=g, device="cuda")
        self.weight = torch.rand(rows, generator=g, device="cuda") + 0.5 if weight else None
        self.noise = torch.randn((2, rows), generator=g, device="cuda")
        self.use_ref = ref

    def anchor(self):
        """Old and reference log-probabilities around the present ones, ratios not next to a border of the clip."""
        lp = Reference(self.logits, self.labels, self.scale, self.counted()).logp
        delta = 0.25 * self.noise[0].double()
        for b in (1 - LOW, 1 + HIGH):
            near = ((-delta).exp() - b).abs() < 1e-2
            delta = torch.where(near, delta + 0.05, delta)
        self.old = (lp + delta).float()
        self.ref = (lp + 0.3 * self.noise[1]).float() if self.use_ref else None

    def counted(self):
        return torch.ones_like(self.labels, dtype=torch.bool) if self.weight is None else self.weight != 0

    def outputs(self):
        rows = self.labels.numel()
        return (torch.full((rows,), 55.0, device="cuda"), torch.full((rows,), 55.0, device="cuda"),
                torch.full((-(-rows // self.each),), 55.0, device="cuda"))

    def run(self, grad="own", stream=0, outs=None):
        self.logp, self.row_loss, self.loss = outs or self.outputs()
        ngc.policy_loss(self.logits, self.labels, self.old, self.advantage, self.grad if grad == "own" else grad, self.logp,
                        self.row_loss, self.loss, ref_logp=self.ref, weight=self.weight, rows_per_partition=self.each,
                        scale=self.scale, clip_low=LOW, clip_high=HIGH, kl_coef=KL, stream=stream)

    def expected(self):
        r = Reference(self.logits, self.labels, self.scale, self.counted())
        adv = self.advantage.double()
        w = torch.ones_like(adv) if self.weight is None else self.weight.double()
        ratio = (r.logp - self.old.double()).exp()
        free, held = ratio * adv, ratio.clamp(1 - LOW, 1 + HIGH) * adv
        value = -torch.minimum(free, held)
        slope = torch.where(free <= held, -free, 0.0)
        dvalue = dslope = free.abs() * 1.1 * r.dlogp
        if self.ref is not None:
            d = self.ref.double() - r.logp
            value = value + KL * (d.exp() - 1 - d)
            slope = slope + KL * (1 - d.exp())
            dvalue = dvalue + KL * (d.exp() - 1).abs() * 1.1 * r.dlogp
            dslope = dslope + KL * d.exp() * 1.1 * r.dlogp
        live, zero = r.live, torch.zeros_like(adv)
        loss = torch.where(live, w * value, zero)
        dloss = torch.where(live, 1.01 * (w * dvalue).abs() + 2 * U * loss.abs() + 1e-36, zero)
        k = self.scale * w * slope
        grad, dgrad = r.gradient(k, (self.scale * w * dslope).abs() + 2 * U * k.abs(), self.dtype)
        part = torch.arange(adv.numel(), device="cuda") // self.each
        total = [zero.new_zeros(self.loss.numel()).index_add_(0, part, x) for x in (loss, dloss)]
        return {"logp": (torch.where(live, r.logp, zero), torch.where(live, r.dlogp + U * r.logp.abs(), zero)),
                "row_loss": (loss, dloss), "loss": (total[0], total[1] + 2 * U * total[0].abs()), "grad": (grad, dgrad)}

    def check(self, names=("logp", "row_loss", "loss", "grad")):
        torch.cuda.synchronize()
        want = self.expected()
        for name in names:
            got, (x, tol) = getattr(self, name).double(), want[name]
            bad = ~((got - x).abs() <= tol)
            assert not bad.any(), (name, bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), x[bad][:4].tolist(),
                                   tol.expand_as(x)[bad][:4].tolist())


CLASSES = [1, 2, 3, 7, 8, 9, 10, 33, 255, 256, 257, 1000, 1025, 2047, 2049, 4097, 8200, 16500, 33000, 50021]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", CLASSES)
def test_policy_over_classes(classes, dtype):
    p = Policy(7, classes, dtype, each=3)
    p.anchor()
    p.run()
    p.check()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [70001, 131072, 140000, 262144, 300007])
def test_policy_over_many_classes(classes, dtype):
    p = Policy(3, classes, dtype, scale=1.3)
    p.anchor()
    p.run()
    p.check()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [10, 200, 2000, 9000])
@pytest.mark.parametrize("pad,offset,grad_offset", [(0, 1, 1), (3, 2, 2), (8, 0, 3), (5, 7, 0), (0, 0, 1), (1, 3, 5)])
def test_policy_strides_and_alignments(classes, dtype, pad, offset, grad_offset):
    p = Policy(9, classes, dtype, seed=3, pad=pad, offset=offset, grad_offset=grad_offset, scale=0.7, each=4)
    p.anchor()
    p.run()
    p.check()
    for flat, m in ((p.flat, p.logits), (p.grad_flat, p.grad)):   # nothing outside the rows is written
        inside = torch.zeros_like(flat, dtype=torch.bool)
        torch.as_strided(inside, m.shape, m.stride(), m.storage_offset()).fill_(True)
        assert (flat[~inside] == 99.0).all()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vectors", [0, 1, 2, 3, 4, 7, 8, 9, 16, 17, 24, 25, 32, 40, 48, 60, 64, 96, 97, 128, 160, 192, 193,
                                     256, 257, 320, 321, 383, 385, 513, 770, 1030, 1537])
def test_policy_teams_of_every_length(vectors, dtype):
    """Rows around the lengths at which other threads take them, whole vectors and loose elements, aligned and not, rows left
    out among them."""
    n = 4 if dtype == "f32" else 8
    for classes, pad, offset in ((vectors * n, 0, 0), (vectors * n + 1, n - 1, 0), (vectors * n + n - 1, 0, 3)):
        if classes < 1:
            continue
        p = Policy(37, classes, dtype, seed=vectors, pad=pad, offset=offset, each=10)
        p.labels[::5] = -1
        p.weight[7] = 0.0
        p.logits[35] = torch.finfo(p.dtype).min
        p.labels[36] = classes - 1
        p.anchor()
        p.run()
        p.check()
        want = p.grad.clone()
        p.run(grad=p.logits)
        torch.cuda.synchronize()
        assert torch.equal(p.logits, want)


@gpu
@pytest.mark.parametrize("rows,each", [(8192, 8192), (8193, 8193), (20000, 9000), (70001, 70001), (204800, 1 << 40),
                                       (204800, 8191), (100, 1 << 62)])
def test_policy_sums_over_partitions_of_many_rows(rows, each):
    p = Policy(rows, 4, "f32", each=rows)
    p.each = each
    p.anchor()
    p.run()
    p.check()
    first = p.loss.clone()
    p.run()
    torch.cuda.synchronize()
    assert torch.equal(p.loss, first)


@gpu
@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 1000, 5001])
@pytest.mark.parametrize("classes", [10, 300])
def test_policy_over_rows(rows, classes):
    p = Policy(rows, classes, "bf16", ref=rows % 2 == 0, weight=rows % 3 != 0, each=max(1, rows // 3))
    p.anchor()
    p.run()
    p.check()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [12, 700, 5000, 40000])
def test_policy_rows_that_are_left_out(classes, dtype):
    p = Policy(12, classes, dtype, seed=5, each=4)
    p.weight[1] = 0.0
    p.labels[2], p.labels[3], p.labels[4] = -1, classes, 2 ** 31 - 1
    p.logits[1:4] = math.nan            # what a left-out row holds does not matter
    p.logits[5] = -math.inf             # nothing can be chosen
    p.logits[6, : classes // 2] = -math.inf
    p.labels[6] = classes - 1
    p.logits[7] = torch.finfo(p.dtype).min     # the type's lowest value everywhere: all classes alike
    p.logits[8, 1:] = torch.finfo(p.dtype).min
    p.labels[8] = 0
    p.weight[8:12] = 0.0                # (8 comes back below) the last partition has one row
    p.weight[8] = 1.0
    p.anchor()
    p.run()
    p.check()
    assert (p.grad[1:6] == 0).all() and (p.row_loss[1:6] == 0).all()
    assert (p.grad[6, : classes // 2] == 0).all()
    assert abs(p.logp[7].item() + math.log(classes)) <= 4 * U * math.log(classes) + 1e-6


@gpu
def test_policy_spoilt_rows_stay_alone():
    for classes in (20, 3000, 30000):
        p = Policy(6, classes, "f32", each=2)
        p.anchor()
        p.logits[2, 5] = math.nan
        p.logits[3, 1] = math.inf
        p.run()
        torch.cuda.synchronize()
        assert p.grad[2].isnan().any() and p.grad[3].isnan().any() and p.row_loss[2:4].isnan().all()
        for r in (0, 1, 4, 5):
            assert p.grad[r].isfinite().all() and p.row_loss[r].isfinite()
        assert p.loss[1].isnan() and p.loss[0].isfinite() and p.loss[2].isfinite()


@gpu
@pytest.mark.parametrize("scale", [1 / 1.4426950408889634, 0.5 / 1.4426950408889634, 1.25 / 1.4426950408889634, 1e-3, 40.0])
@pytest.mark.parametrize("classes", [13, 1500, 30001])
def test_scales_with_few_digits(classes, scale):
    """Scales whose product with log2(e) is a short number, and small and large ones, with classes that cannot be chosen."""
    for dtype in DTYPES:
        p = Policy(5, classes, dtype, scale=scale, std=2.0 / scale)
        p.logits[:, 1::3] = -math.inf
        p.labels[:] = 2
        p.anchor()
        p.run()
        p.check()
        q = preference([2, 3], classes, dtype, scale=scale)
        q.run()
        q.check()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [20, 1500, 30000])
def test_policy_infinite_log_probabilities(classes, dtype):
    """An action of probability 0 now (rows 0, 1), before (2, 3) or under the reference (4): what the formulas give."""
    p = Policy(6, classes, dtype, ref=False, weight=False, each=6)
    p.logits[0, 3] = p.logits[1, 3] = -math.inf
    p.labels[:2] = 3
    p.anchor()
    p.old[:2] = -1.0
    p.old[2:4] = -math.inf
    p.advantage[:4] = torch.tensor([2.0, -2.0, 2.0, -2.0], device="cuda")
    p.run()
    torch.cuda.synchronize()
    assert (p.logp[:2] == -math.inf).all() and p.logp[2:].isfinite().all()
    # ratios 0 and infinity: the clipped term counts, but where the free one is lower
    want = torch.tensor([0.0, 2 * (1 - LOW), -2 * (1 + HIGH), math.inf], dtype=torch.float64, device="cuda")
    got = p.row_loss[:4].double()
    assert ((got == want) | ((got - want).abs() <= 3 * U * want.abs())).all(), got.tolist()
    assert (p.grad[:3] == 0).all() and p.grad[4:].isfinite().all() and p.row_loss[4:].isfinite().all()
    p.ref = p.old.clone()
    p.ref[2:4] = -1.0
    p.ref[4] = -math.inf
    p.run()
    torch.cuda.synchronize()
    assert (p.row_loss[[0, 1, 3, 4]] == math.inf).all() and p.row_loss[[2, 5]].isfinite().all()
    assert p.grad[[2, 4, 5]].isfinite().all()


@gpu
@pytest.mark.parametrize("classes", [50, 1500, 40001])
def test_policy_in_place_and_without_gradient(classes):
    p = Policy(5, classes, "bf16", pad=2)
    p.anchor()
    p.run(grad=None)
    p.check(("logp", "row_loss", "loss"))
    p.run()
    torch.cuda.synchronize()
    want = p.grad.clone()
    p.run(grad=p.logits)
    torch.cuda.synchronize()
    assert torch.equal(p.logits, want)


@gpu
@pytest.mark.parametrize("classes", [64, 3000, 20000])
def test_policy_gradient_against_differences(classes):
    """The kernel's gradient against central differences of the loss in 64 bits: their own error is of the order h^2
    (third derivatives of the loss are below 10 here), far below the tolerance."""
    p = Policy(4, classes, "f32", scale=0.9)
    p.anchor()
    p.run()
    torch.cuda.synchronize()
    h = 1e-4

    def loss(x):
        lp = torch.log_softmax(p.scale * x, 1).gather(1, p.labels.long().unsqueeze(1)).squeeze(1)
        ratio, adv = (lp - p.old.double()).exp(), p.advantage.double()
        d = p.ref.double() - lp
        return (p.weight.double() * (-torch.minimum(ratio * adv, ratio.clamp(1 - LOW, 1 + HIGH) * adv)
                                     + KL * (d.exp() - d - 1))).sum()

    for r in range(4):
        for v in {0, int(p.labels[r]), int(p.logits[r].argmax()), classes - 1}:
            e = torch.zeros_like(p.logits, dtype=torch.float64)
            e[r, v] = h
            x = p.logits.double()
            slope = (loss(x + e) - loss(x - e)).item() / (2 * h)
            assert abs(p.grad[r, v].item() - slope) <= 1e-4 * abs(slope) + 1e-6, (r, v)


@gpu
def test_policy_on_another_stream_and_in_a_graph():
    p = Policy(40, 3000, "bf16", each=16)
    p.anchor()
    p.run()
    p.check()
    outs = p.outputs()
    grad = p.grad.clone()
    logits = p.logits.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        p.run(stream=torch.cuda.current_stream().cuda_stream, outs=outs)
    for k in range(2):
        p.logits.copy_(logits if k else -logits)
        p.grad.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p.grad, grad)
    p.check()


@gpu
def test_policy_calls_beside_each_other_and_long_partitions_in_graphs():
    a, b = Policy(20000, 40, "bf16", seed=1), Policy(9000, 300, "f32", seed=2, each=8500)
    graphs, streams = [], []
    for p in (a, b):
        p.anchor()
        p.run()
        p.check()
        p.keep = [x.clone() for x in (p.grad, p.logp, p.row_loss, p.loss)]
        outs = p.outputs()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            p.run(stream=torch.cuda.current_stream().cuda_stream, outs=outs)
        p.grad.zero_()
        graphs.append(g)
        streams.append(side)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for p in (a, b):
        assert all(torch.equal(x, y) for x, y in zip(p.keep, (p.grad, p.logp, p.row_loss, p.loss)))


@gpu
def test_policy_bad_tensors_are_refused():
    p = Policy(4, 16, "f32")
    p.anchor()
    good = dict(logits=p.logits, actions=p.labels, old_logp=p.old, advantage=p.advantage, dlogits=p.grad,
                logp=torch.zeros(4, device="cuda"), row_loss=torch.zeros(4, device="cuda"))
    ngc.policy_loss(**good)
    for bad in ({"logits": p.logits.double()}, {"logits": p.logits.t()}, {"dlogits": p.grad[:3]}, {"logits": p.logits[0]},
                {"dlogits": p.grad.bfloat16()}, {"actions": p.labels.long()}, {"old_logp": p.old[:3]},
                {"advantage": p.advantage.cpu()}, {"row_loss": None}, {"loss": torch.zeros(2, device="cuda")},
                {"rows_per_partition": 0}, {"weight": p.advantage.double()}, {"dlogits": p.grad[:, :8]},
                {"logits": p.logits[:, ::2], "dlogits": p.grad[:, ::2]}):
        with pytest.raises(ngc.NgcError):
            ngc.policy_loss(**{**good, **bad})


class Preference:
    def __init__(self, lengths, classes, dtype="f32", seed=0, pad=0, offset=0, grad_offset=None, scale=1.0, beta=0.3,
                 smooth=0.1, mean=False, weight=True, before=0, behind=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + classes)
        self.dtype = DTYPES[dtype]
        rows = before + sum(lengths) + behind
        self.flat, self.logits = matrix(g, rows, classes, self.dtype, pad, offset)
        self.grad_flat, self.grad = matrix(g, rows, classes, self.dtype, pad, offset if grad_offset is None else grad_offset)
        self.labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
        self.labels[torch.rand(rows, generator=g, device="cuda") < 0.25] = -1
        self.begin = before + torch.tensor([0] + list(lengths)).cumsum(0).to("cuda")
        self.pairs = len(lengths) // 2
        self.scale, self.beta, self.smooth, self.mean = scale, beta, smooth, mean
        self.weight = torch.rand(self.pairs, generator=g, device="cuda") + 0.5 if weight else None
        self.noise = torch.randn(2 * self.pairs, generator=g, device="cuda")
        self.before, self.behind = before, behind

    def reference(self):
        r = Reference(self.logits, self.labels, self.scale, torch.ones_like(self.labels, dtype=torch.bool))
        inside = torch.arange(self.labels.numel(), device="cuda")
        self.owner = (torch.searchsorted(self.begin, inside, right=True) - 1).clamp(0, 2 * self.pairs - 1)
        self.covered = (inside >= self.begin[0]) & (inside < self.begin[-1])
        r.live = r.live & self.covered
        return r

    def sums(self, r):
        z = torch.zeros(2 * self.pairs, dtype=torch.float64, device="cuda")
        add = lambda x: z.index_add(0, self.owner, torch.where(r.live, x, 0.0))
        total, off, count = add(r.logp), add(r.dlogp + 4e-16 * r.logp.abs() * r.logp.numel()), add(torch.ones_like(r.logp))
        count = count.clamp(min=1) if self.mean else torch.ones_like(count)
        return total / count, off / count, count

    def anchor(self):
        self.ref = (self.sums(self.reference())[0] + self.noise / self.beta).float()

    def run(self, grad="own", stream=0, outs=None, ws=None):
        self.seq_logp, self.pair_loss = outs or (torch.full((2 * self.pairs,), 55.0, device="cuda"),
                                                 torch.full((self.pairs,), 55.0, device="cuda"))
        if ws is None:
            ws = torch.full((ngc.preference_workspace_bytes(self.labels.numel(), self.pairs),), 0xAB, dtype=torch.uint8,
                            device="cuda")
        ngc.preference_loss(self.logits, self.labels, self.begin, self.ref, self.grad if grad == "own" else grad,
                            self.seq_logp, self.pair_loss, ws, pair_weight=self.weight, scale=self.scale, beta=self.beta,
                            label_smoothing=self.smooth, length_mean=self.mean, stream=stream)

    def check(self, grad=True):
        torch.cuda.synchronize()
        r = self.reference()
        lp, off, count = self.sums(r)
        ratio = lp - self.ref.double()
        h = self.beta * (ratio[0::2] - ratio[1::2])
        dh = self.beta * (off[0::2] + off[1::2]) + 4e-16 * h.abs()
        w = torch.ones_like(h) if self.weight is None else self.weight.double()
        e = self.smooth
        loss = -w * ((1 - e) * torch.nn.functional.logsigmoid(h) + e * torch.nn.functional.logsigmoid(-h))
        slope = self.beta * w * (torch.sigmoid(h) - (1 - e))
        want = {"seq_logp": (lp, 1.01 * off + 2 * U * lp.abs()),
                "pair_loss": (loss, 1.01 * (w * dh) + 2 * U * loss.abs() + 1e-36)}
        for name, (x, tol) in want.items():
            assert ((getattr(self, name).double() - x).abs() <= tol).all(), name
        if not grad:
            return
        # sigmoid has a slope of at most 1/4, and of at most itself
        dslope = self.beta * w * 1.1 * dh * (torch.sigmoid(h) * torch.sigmoid(-h)) + 1e-15 * slope.abs()
        k, dk = (torch.stack([x, y], 1).view(-1) / count for x, y in ((slope, -slope), (dslope, dslope)))
        k, dk = self.scale * k[self.owner], self.scale * dk[self.owner]
        x, tol = r.gradient(k, dk + 2 * U * k.abs(), self.dtype)
        c = self.covered
        assert ((self.grad.double() - x).abs() <= tol)[c].all()
        assert (self.grad[~c].float() == self.untouched[~c].float()).all()


@pytest.mark.parametrize("call", [policy_call, preference_call])
def test_row_strides_beyond_any_buffer_are_refused(call):
    assert call(ld=1 << 43) == -1 and call(ldg=1 << 62) == -1
    assert call(rows=(1 << 31) - 1, ld=1 << 20, ldg=1 << 20, ws_bytes=1 << 40) == -1


@pytest.mark.parametrize("call", [policy_call, preference_call])
@pytest.mark.parametrize("kw", [
    {"grad": AT + 4}, {"grad": AT + 16, "ld": 16, "ldg": 16}, {"grad": AT + 80, "ld": 40, "ldg": 10},
    {"grad": AT - 40, "ld": 12, "ldg": 12}, {"grad": AT + 4 * 36, "ld": 40, "ldg": 40, "dtype": ngc.NGC_F32}])
def test_gradients_that_share_elements_with_other_logits_are_refused(call, kw):
    assert call(**kw) == -1


@gpu
def test_halves_of_a_wider_matrix():
    """Logits and gradient side by side in one buffer."""
    p = Policy(9, 300, "f32", each=9)
    p.anchor()
    p.run()
    torch.cuda.synchronize()
    want = p.grad.clone()
    both = torch.zeros((9, 600), device="cuda")
    for a, b in ((both[:, :300], both[:, 300:]), (both[:, 300:], both[:, :300])):
        a.copy_(p.logits)
        b.fill_(7.0)
        p.logits, p.grad = a, b
        p.run()
        torch.cuda.synchronize()
        assert torch.equal(b, want)


@gpu
@pytest.mark.parametrize("classes", [50, 5000])
def test_preference_infinite_ratios_and_pairs_without_weight(classes):
    p = preference([3, 2, 3, 2, 3, 2], classes, "f32", smooth=0.0)
    p.labels[[1, 6, 8, 11]] = 2
    p.logits[8, 2] = -math.inf         # pair 1: the rejected sequence cannot have been drawn
    p.logits[11, 2] = -math.inf        # pair 2: the chosen one
    p.run()
    torch.cuda.synchronize()
    assert p.pair_loss[0].isfinite() and p.pair_loss[1] == 0 and p.pair_loss[2] == math.inf
    assert (p.grad[5:10] == 0).all() and p.grad[10:].isfinite().all() and (p.grad[11, 2] < 0)
    p.smooth = 1.0                      # the other way round
    p.run()
    torch.cuda.synchronize()
    assert p.pair_loss[1] == math.inf and p.pair_loss[2] == 0 and (p.grad[10:] == 0).all()
    p.weight = torch.tensor([0.0, 0.0, 1.0], device="cuda")
    p.labels[0] = 3
    p.logits[0] = math.nan
    p.run()
    torch.cuda.synchronize()
    assert (p.pair_loss == 0).all() and (p.grad == 0).all()


LENGTHS = [[1, 1], [0, 3], [4, 0], [0, 0, 2, 5], [3, 1, 0, 7, 12, 2], [40, 25]]


def preference(*args, **kw):
    p = Preference(*args, **kw)
    p.untouched = p.grad.clone()
    p.anchor()
    return p


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("mean", [False, True])
def test_preference_over_lengths(lengths, dtype, mean):
    p = preference(lengths, 301, dtype, mean=mean, before=len(lengths) % 3, behind=2)
    p.run()
    p.check()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [1, 2, 9, 256, 1025, 8200, 33000, 70001, 140000, 300007])
def test_preference_over_classes(classes, dtype):
    p = preference([3, 2, 4, 1], classes, dtype, scale=0.8, behind=1)
    p.run()
    p.check()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vectors", [0, 1, 7, 8, 9, 16, 17, 32, 33, 64, 65, 128, 129, 256, 257, 640, 641, 1280, 1281, 1920, 1921,
                                     2560, 2561, 3840, 3841, 5120, 5121])
def test_preference_teams_of_every_length(vectors, dtype):
    """Rows around the lengths at which other threads take them, whole vectors and loose elements, aligned and not, rows left
    out among them, and rows before, between and behind what the teams of a warp or a block hold."""
    n = 4 if dtype == "f32" else 8
    for classes, pad, offset in ((vectors * n, 0, 0), (vectors * n + 1, n - 1, 0), (vectors * n + n - 1, 0, 3)):
        if classes < 1:
            continue
        p = preference([9, 4, 0, 11], classes, dtype, seed=vectors, pad=pad, offset=offset, before=5, behind=7)
        p.labels[6] = classes - 1
        p.labels[12] = 0
        p.logits[12] = torch.finfo(p.dtype).min
        p.labels[13] = 0
        p.logits[13] = -math.inf
        p.labels[14] = -1
        p.logits[14] = math.nan
        p.anchor()
        p.run()
        p.check()
        want = p.grad.clone()
        p.run(grad=p.logits)
        torch.cuda.synchronize()
        assert torch.equal(p.logits[5:-7], want[5:-7])


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset,grad_offset", [(0, 1, 1), (3, 2, 2), (8, 0, 3), (5, 7, 0)])
def test_preference_strides_and_alignments(dtype, pad, offset, grad_offset):
    for classes in (60, 2000, 9000):
        p = preference([5, 6, 2, 8], classes, dtype, pad=pad, offset=offset, grad_offset=grad_offset, before=1, behind=1)
        p.run()
        p.check()
        for flat, m in ((p.flat, p.logits), (p.grad_flat, p.grad)):
            inside = torch.zeros_like(flat, dtype=torch.bool)
            torch.as_strided(inside, m.shape, m.stride(), m.storage_offset()).fill_(True)
            assert (flat[~inside] == 99.0).all()


@gpu
@pytest.mark.parametrize("classes", [100, 12000])
def test_preference_rows_that_are_left_out(classes):
    p = preference([6, 6, 3, 3], classes, "f32", mean=True, weight=False)
    p.labels[6:12] = torch.tensor([-1, classes, -5, 2 ** 31 - 1, -1, -1], device="cuda", dtype=torch.int32)  # a whole sequence
    p.logits[6:12] = math.nan
    p.logits[0] = -math.inf
    p.logits[1, 1:] = -math.inf
    p.labels[1] = 0
    p.logits[2] = torch.finfo(torch.float32).min
    p.labels[2] = classes - 1
    p.anchor()
    p.run()
    p.check()
    assert p.seq_logp[1] == 0 and (p.grad[6:12] == 0).all() and (p.grad[0] == 0).all()


@gpu
def test_preference_many_pairs_long_sequences_and_bad_offsets():
    g = torch.Generator().manual_seed(3)
    lengths = torch.randint(0, 40, (600,), generator=g).tolist()
    p = preference(lengths, 70, "bf16", smooth=0.0)
    p.run()
    p.check()
    p = preference([3000, 2500], 130, "f32", beta=0.01)
    p.run()
    p.check()
    # offsets outside the rows, or descending: every access stays inside the buffers
    p = preference([5, 5, 5, 5], 64, "f32")
    for begin in ([-9, 5, 100, 7, 1 << 40], [20, 10, 5, 2, 0], [3, 3, 3, 3, 3]):
        p.begin = torch.tensor(begin, device="cuda")
        p.run()
    torch.cuda.synchronize()
    assert (p.flat[-8:] == 99.0).all() and (p.grad_flat[-8:] == 99.0).all()


@gpu
@pytest.mark.parametrize("classes", [50, 5000])
def test_preference_in_place_without_gradient_and_extreme_ratios(classes):
    p = preference([5, 8], classes, "f32")
    p.run(grad=None)
    p.check(grad=False)
    p.run()
    torch.cuda.synchronize()
    want = p.grad.clone()
    logits = p.logits.clone()
    p.run(grad=p.logits)
    torch.cuda.synchronize()
    assert torch.equal(p.logits, want)
    p.logits.copy_(logits)
    for far in (3000.0, -3000.0):       # a ratio whose sigmoid leaves the range of exp
        p.ref[0] += far
        p.run()
        p.check()


@gpu
def test_preference_gradient_against_differences():
    p = preference([4, 3, 2, 5], 200, "f32", scale=1.1, mean=True)
    p.run()
    torch.cuda.synchronize()
    h = 1e-4

    def loss(x):
        lp = torch.log_softmax(p.scale * x, 1).gather(1, p.labels.clamp(min=0).long().unsqueeze(1)).squeeze(1)
        total, _, count = p.sums(type("R", (), {"live": p.labels >= 0, "logp": lp, "dlogp": lp})())
        ratio = total - p.ref.double()
        z = p.beta * (ratio[0::2] - ratio[1::2])
        ls = torch.nn.functional.logsigmoid
        return (-p.weight.double() * ((1 - p.smooth) * ls(z) + p.smooth * ls(-z))).sum()

    for r in range(14):
        for v in (0, max(0, int(p.labels[r])), 199):
            e = torch.zeros_like(p.logits, dtype=torch.float64)
            e[r, v] = h
            x = p.logits.double()
            slope = (loss(x + e) - loss(x - e)).item() / (2 * h)
            assert abs(p.grad[r, v].item() - slope) <= 1e-4 * abs(slope) + 1e-6, (r, v)


@gpu
def test_preference_two_graphs_with_workspaces_of_their_own():
    a, b = preference([30, 20, 25, 30], 3000, "bf16", seed=1), preference([10, 41], 3000, "bf16", seed=2)
    graphs, streams = [], []
    for p in (a, b):
        p.run()
        torch.cuda.synchronize()
        p.keep = p.grad.clone()
        p.grad.zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        ws = torch.empty(ngc.preference_workspace_bytes(p.labels.numel(), p.pairs), dtype=torch.uint8, device="cuda")
        outs = (torch.zeros(2 * p.pairs, device="cuda"), torch.zeros(p.pairs, device="cuda"))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            p.run(stream=torch.cuda.current_stream().cuda_stream, outs=outs, ws=ws)
        graphs.append(g)
        streams.append(side)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for p in (a, b):
        assert torch.equal(p.grad, p.keep)
        p.check()


@gpu
def test_preference_bad_tensors_are_refused():
    p = preference([3, 2], 16, "f32")
    ws = torch.empty(ngc.preference_workspace_bytes(5, 1), dtype=torch.uint8, device="cuda")
    good = dict(logits=p.logits, labels=p.labels, seq_begin=p.begin, ref_logp=p.ref, dlogits=p.grad,
                seq_logp=torch.zeros(2, device="cuda"), pair_loss=torch.zeros(1, device="cuda"), workspace=ws)
    ngc.preference_loss(**good)
    for bad in ({"workspace": ws[:16]}, {"workspace": ws[8:]}, {"seq_begin": p.begin.int()}, {"seq_begin": p.begin[:2]},
                {"ref_logp": p.ref[:1]}, {"labels": p.labels.long()}, {"pair_loss": torch.zeros(2, device="cuda")},
                {"dlogits": p.grad.bfloat16()}, {"logits": p.logits.half(), "dlogits": p.grad.half()},
                {"label_smoothing": 2.0}, {"scale": 0.0}, {"pair_weight": p.ref}):
        with pytest.raises(ngc.NgcError):
            ngc.preference_loss(**{**good, **bad})


@gpu
def test_results_do_not_vary_from_run_to_run():
    p = Policy(300, 777, "bf16", each=100)
    p.anchor()
    q = preference([120, 90, 60, 100], 3001, "f32")
    first = None
    for _ in range(3):
        p.run()
        q.run()
        torch.cuda.synchronize()
        now = [x.clone() for x in (p.grad, p.row_loss, p.loss, p.logp, q.grad, q.seq_logp, q.pair_loss)]
        assert first is None or all(torch.equal(x, y) for x, y in zip(first, now))
        first = now


# Logits that do not stay in L2 between the two reads.
LARGE = {"many short pairs": ([11, 8, 0, 0, 9, 14, 1, 0, 0, 7] * 34, 36000, "bf16"),
         "a pair longer than a group": ([5, 6, 700, 350, 3, 0, 0, 2, 40, 41], 33001, "bf16"),
         "few classes": ([60, 50, 70, 64] * 24, 4500, "f32"),
         "fp32": ([200, 100, 90, 60], 50021, "f32"),
         "very long rows": ([30, 20, 25, 10], 300007, "f32")}


@gpu
@pytest.mark.parametrize("name", LARGE)
@pytest.mark.parametrize("mean", [False, True])
def test_preference_large(name, mean):
    lengths, classes, dtype = LARGE[name]
    p = preference(lengths, classes, dtype, mean=mean, before=3, behind=5, beta=0.05)
    p.labels[10:14] = -1
    p.logits[20] = torch.finfo(p.dtype).min
    p.logits[21] = -math.inf
    p.anchor()
    assert p.logits.numel() * p.logits.element_size() > 64 << 20
    p.run()
    p.check()
    first = [x.clone() for x in (p.grad, p.seq_logp, p.pair_loss)]
    p.run()                                      # the same again, bit for bit
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, (p.grad, p.seq_logp, p.pair_loss)))
    p.run(grad=p.logits)                         # in place
    torch.cuda.synchronize()
    assert torch.equal(p.logits[3:-5], first[0][3:-5])


@gpu
def test_preference_large_in_graphs_and_beside_each_other():
    a = preference([300, 280, 4, 9], 60000, "bf16", seed=5)
    b = preference([90, 100] * 4, 50000, "bf16", seed=6)
    graphs, streams = [], []
    for p in (a, b):
        p.run()
        torch.cuda.synchronize()
        p.keep = p.grad.clone()
        p.grad.zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        ws = torch.empty(ngc.preference_workspace_bytes(p.labels.numel(), p.pairs), dtype=torch.uint8, device="cuda")
        outs = (torch.zeros(2 * p.pairs, device="cuda"), torch.zeros(p.pairs, device="cuda"))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            p.run(stream=torch.cuda.current_stream().cuda_stream, outs=outs, ws=ws)
        graphs.append(g)
        streams.append(side)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for p in (a, b):
        assert torch.equal(p.grad, p.keep)
        p.check()


@gpu
@pytest.mark.parametrize("classes", [64, 70000])
def test_preference_offsets_that_do_not_ascend(classes):
    """Nothing outside the buffers is touched, and the losses say that something is wrong."""
    p = preference([150, 150, 150, 150], classes, "f32", behind=4)
    for begin, bad in (([0, 200, 100, 300, 600], [0]), ([600, 300, 200, 100, 0], [0, 1]), ([-5, 100, 300, 500, 1 << 40], []),
                       ([5, 5, 5, 5, 5], []), ([700, 700, 800, 800, 900], [])):
        p.begin = torch.tensor(begin, device="cuda")
        p.run()
        torch.cuda.synchronize()
        for q in range(2):
            assert p.pair_loss[q].isnan() or q not in bad, begin
            assert p.pair_loss[q].isfinite() or bad, begin
    assert (p.flat[-8:] == 99.0).all() and (p.grad_flat[-8:] == 99.0).all()


@gpu
@pytest.mark.parametrize("fill", [0, 0xAB])
def test_preference_offsets_outside_the_first_and_the_last_one(fill):
    """Rows there have no statistics: a pair that ascends among them says so, whatever the workspace holds."""
    p = preference([50, 50, 50, 50, 50, 50], 40, "f32")
    ws = torch.full((ngc.preference_workspace_bytes(300, 3),), fill, dtype=torch.uint8, device="cuda")
    for begin, bad in (([50, 60, 70, 5, 6, 10, 20], [0, 1, 2]), ([50, 60, 250, 5, 30, 40, 100], [0, 1, 2]),
                       ([0, 60, 120, 100, 130, 140, 300], [1])):
        p.begin = torch.tensor(begin, device="cuda")
        p.run(ws=ws)
        torch.cuda.synchronize()
        assert p.pair_loss.isnan().nonzero().view(-1).tolist() == bad, begin
