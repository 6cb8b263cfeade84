"""Softmax cross entropy straight from features and weights, against its definition in 64 bits.

Tolerances, element by element (u = 2^-23 is a step of fp32 next to 1; the tensor cores' sums of exact products may cut instead of round):
  logits       e_z  = scale stretch (d + 8) u max_v sum |x W_v|,
  logp         e_lp = 2 e_z + 4 u (max |z| + |lse| + 1) + 128 u         (the powers, their sums of at most 64 in a chain, the logarithm),
  G            e_G  = |g| p e_lp + |G| (2^-8 + 2^-11) + |g| 2^-38       (bf16; powers in fp16 and where that ends),
  dX           e_G |W| + (classes + 8) u |G| |W| + 2^-8 |dX|,  dW likewise with rows in the place of classes.
"""
import math
import random
import subprocess
import sys

import pytest
import torch

import paper_2212_08580_b200 as ngc
from tests._philox import kept, threshold

BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -23


class Problem:
    def __init__(self, rows, d, classes, seed=1, layout="classes", masked=0.2, weighted=True, spread=1.0, pad=0, shift=0, w_pad=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.rows, self.d, self.classes = rows, d, classes
        flat = torch.empty(rows * (d + pad) + shift, dtype=BF16, device="cuda").normal_(generator=g)
        self.x = flat[shift:].view(rows, d + pad)[:, :d]
        a, b = (classes, d) if layout == "classes" else (d, classes)
        flat = torch.empty(a * (b + w_pad) + shift, dtype=BF16, device="cuda").normal_(0.0, 2.0 * spread / math.sqrt(d), generator=g)
        w = flat[shift:].view(a, b + w_pad)[:, :b]
        self.weight = w if layout == "classes" else w.t()
        self.layout = layout
        self.labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
        if masked:
            out = torch.rand(rows, generator=g, device="cuda") < masked
            self.labels[out] = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.5, -1, classes).to(torch.int32)[out]
        self.row_weight = None
        if weighted:
            self.row_weight = torch.rand(rows, generator=g, device="cuda") + 0.1
            self.row_weight[torch.rand(rows, generator=g, device="cuda") < masked / 2] = 0.0

    def live(self):
        keep = (self.labels >= 0) & (self.labels < self.classes)
        return keep if self.row_weight is None else keep & (self.row_weight != 0)

    def outputs(self, parts, dx=True, dw=True, extra=3):
        f32 = {"dtype": F32, "device": "cuda"}
        self.logp, self.row_loss, self.loss = (torch.full((n,), 7.0, **f32) for n in (self.rows, self.rows, parts))
        self.dx_full = torch.full((self.rows, self.d + extra), 7.0, dtype=BF16, device="cuda")
        self.dx = self.dx_full[:, : self.d] if dx else None
        a, b = (self.classes, self.d) if self.layout == "classes" else (self.d, self.classes)
        self.dw_full = torch.full((parts, a, b + extra), 7.0, dtype=BF16, device="cuda")
        dwm = self.dw_full[:, :, :b]
        self.dw = (dwm if self.layout == "classes" else dwm.transpose(1, 2)) if dw else None
        self.extra = extra

    def run(self, each=None, dx=True, dw=True, stream=0, outputs=True, scale=1.0, **options):
        each = self.each = self.rows if each is None else each
        self.scale, self.options = scale, options
        if outputs:
            self.outputs(-(-self.rows // each), dx, dw)
        sizes = {k: options[k] for k in ("keep_rows", "piece_rows") if k in options}
        n = ngc.linear_cross_entropy_workspace_bytes(self.x, self.weight, dx=self.dx, dweight=self.dw, rows_per_partition=each, **sizes)
        if outputs:
            self.workspace = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # (NaN wherever nothing is written)
        ngc.linear_cross_entropy(self.x, self.weight, self.labels, self.logp, self.row_loss, self.loss, self.workspace, dx=self.dx,
                                 dweight=self.dw, row_weight=self.row_weight, rows_per_partition=each, scale=scale, stream=stream,
                                 **options)
        return self

    def check_some(self, rows):
        """log p and gradients of some rows, each of them a partition."""
        live = self.live()
        for i in rows.tolist():
            if not live[i]:
                assert self.logp[i] == 0 and (self.dx[i] == 0).all() and (self.dw[i] == 0).all()
                continue
            x, w, y = self.x[i].double(), self.weight.double(), int(self.labels[i])
            z = w @ x
            logp = torch.log_softmax(z, 0)
            e_lp = 2 * (self.d + 8) * U * float((w.abs() @ x.abs()).max()) + 4 * U * (float(z.abs().max()) + abs(float(z.logsumexp(0))) + 1) + 128 * U
            assert abs(float(self.logp[i]) - float(logp[y])) <= e_lp
            k = 1.0 if self.row_weight is None else float(self.row_weight[i])
            G = k * logp.exp()
            e_G = G * e_lp + k * 2.0 ** -38
            G[y] -= k
            e_G += G.abs() * (2.0 ** -8 + 2.0 ** -11)
            want = G @ w
            assert ((self.dx[i].double() - want).abs() <= e_G @ w.abs() + 16 * U * (G.abs() @ w.abs()) + 2.0 ** -8 * want.abs()).all()
            want = G.unsqueeze(1) * x
            assert ((self.dw[i].double() - want).abs() <= e_G.unsqueeze(1) * x.abs() + (2.0 ** -8 + 16 * U) * want.abs()).all()

    def check(self):
        opt, scale, p = self.options, self.scale, self.options.get("dropout", 0.0)
        live = self.live()
        r = live.nonzero().squeeze(1)
        x, w = self.x[r].double(), self.weight.double()
        mask, stretch = None, 1.0
        if p:
            mask = torch.from_numpy(kept(self.rows, self.d, p, opt["seed"], opt.get("step", 0), opt.get("first_row", 0))).cuda()[r]
            stretch = 65536.0 / (65536 - threshold(p)) if threshold(p) < 65536 else 0.0
            x = torch.where(mask, x * stretch, 0.0)
        z = scale * (x @ w.t())
        lse = torch.logsumexp(z, 1, keepdim=True)
        y = self.labels[r].long().unsqueeze(1)
        logp = (z - lse).gather(1, y)
        weight = torch.ones_like(logp) if self.row_weight is None else self.row_weight[r].double().unsqueeze(1)
        size = scale * (x.abs() @ w.abs().t()).amax(1, keepdim=True) if r.numel() else logp
        e_lp = 2 * (self.d + 8) * U * size + 4 * U * (z.abs().amax(1, keepdim=True) + lse.abs() + 1) + 128 * U
        assert not ngc.linear_cross_entropy_gave_up(self.workspace)
        assert (self.logp[~live] == 0).all() and (self.row_loss[~live] == 0).all()
        off = (self.logp[r].double().unsqueeze(1) - logp).abs()
        assert (off <= e_lp).all(), ("logp", float((off / e_lp).max()))
        off = (self.row_loss[r].double().unsqueeze(1) + weight * logp).abs()
        assert (off <= weight * e_lp + U * (weight * logp).abs()).all(), "row_loss"
        parts = -(-self.rows // self.each)
        at = torch.arange(self.rows, device="cuda") // self.each
        total = torch.zeros(parts, dtype=torch.float64, device="cuda").index_add_(0, at, self.row_loss.double())
        assert ((self.loss.double() - total).abs() <= U * total.abs()).all(), "loss"
        g = scale * weight
        prob = (z - lse).exp()
        G = prob.clone()
        G.scatter_add_(1, y, -torch.ones_like(logp))
        G *= g
        e_G = g * prob * e_lp + G.abs() * (2.0 ** -8 + 2.0 ** -11) + g * 2.0 ** -38
        if self.dx is not None:
            want, slack = G @ w, e_G @ w.abs() + (self.classes + 8) * U * (G.abs() @ w.abs())
            if mask is not None:
                want, slack = torch.where(mask, want * stretch, 0.0), torch.where(mask, slack * stretch, 0.0)
            off = (self.dx[r].double() - want).abs()
            assert (off <= slack + 2.0 ** -8 * want.abs() + 1e-38).all(), ("dx", float((off / (slack + 1e-38)).max()))
            assert (self.dx[~live] == 0).all()
            assert (self.dx_full[:, self.d:] == 7.0).all()
        if self.dw is not None:
            assert (self.dw_full[:, :, self.dw_full.shape[2] - self.extra:] == 7.0).all()
            for j in range(parts):
                s = (r // self.each) == j
                want = G[s].t() @ x[s]
                slack = e_G[s].t() @ x[s].abs() + (int(s.sum()) + 8) * U * (G[s].abs().t() @ x[s].abs())
                off = (self.dw[j].double() - want).abs()
                assert (off <= slack + 2.0 ** -8 * want.abs() + 1e-38).all(), ("dw", j, float((off / (slack + 1e-38)).max()))
        return self


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,d,classes", [(1, 1, 1), (1, 1, 2), (1, 64, 300), (2, 8, 3), (3, 33, 130), (63, 64, 64), (64, 72, 257),
                                            (65, 127, 1000), (130, 520, 63), (257, 200, 513), (1025, 64, 1024), (1500, 129, 3001),
                                            (300, 1300, 777), (40, 64, 20000), (2100, 16, 17)])
def test_against_the_definition(layout, rows, d, classes):
    Problem(rows, d, classes, seed=rows + d + classes, layout=layout).run(scale=0.7).check()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,each,masked", [(1000, 1000, 0.0), (1000, 333, 0.3), (900, 64, 0.5), (3000, 1100, 0.9), (70, 7, 0.5),
                                              (5000, 2500, 0.2), (129, 128, 0.2), (200, 1, 0.4)])
def test_partitions(layout, rows, each, masked):
    Problem(rows, 80, 210, seed=each, layout=layout, masked=masked).run(each=each).check()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("piece_rows,each", [(1, None), (64, None), (200, None), (300, 250), (300, 700), (1000, 100), (5000, None)])
def test_pieces_of_rows(layout, piece_rows, each):
    rows = 90 if piece_rows == 1 else 1000
    whole = Problem(rows, 72, 333, layout=layout).run(each=each).check()
    parts = Problem(rows, 72, 333, layout=layout).run(each=each, piece_rows=piece_rows).check()
    assert (whole.logp == parts.logp).all() and (whole.row_loss == parts.row_loss).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dx,dw", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("rows,each", [(1, None), (300, None), (1300, 400)])
def test_outputs_that_are_wanted(dx, dw, rows, each):
    both = Problem(rows, 200, 1111, seed=4).run(each=each).check()
    some = Problem(rows, 200, 1111, seed=4).run(each=each, dx=dx, dw=dw).check()
    assert (some.logp == both.logp).all() and (some.loss == both.loss).all()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows", [1, 32, 33, 200, 256, 257, 350, 512, 513, 700, 1024, 1025, 4000])
@pytest.mark.parametrize("d,classes", [(64, 257), (72, 3001), (1300, 1000), (33, 20011), (520, 40000)])
def test_scoring(layout, rows, d, classes):
    Problem(rows, d, classes, seed=rows + classes, layout=layout, masked=0.3).run(dx=False, dw=False, scale=1.3).check()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,each,piece_rows", [(1, 1, 0), (5, 1, 0), (100, 1, 0), (100, 7, 0), (128, 128, 0), (100, 1, 30), (90, 20, 64)])
@pytest.mark.parametrize("pad,classes", [(0, 2000), (8, 4097), (3, 2000)])
def test_scoring_few_rows(layout, rows, each, piece_rows, pad, classes):
    """With and without a copy of the features, labels on either side of the classes, losses per row and per partition."""
    p = Problem(rows, 64, classes, seed=rows + pad, layout=layout, masked=0.4 if rows > 1 else 0.0, pad=pad)
    p.run(each=each, dx=False, dw=False, piece_rows=piece_rows).check()
    p.labels.fill_(classes)
    p.run(each=each, dx=False, dw=False, piece_rows=piece_rows)
    assert (p.logp == 0).all() and (p.row_loss == 0).all() and (p.loss == 0).all()


@pytest.mark.gpu
def test_scoring_spoiled_and_left_out_rows():
    p = Problem(300, 64, 5000, masked=0.3, weighted=False)
    live = p.live().nonzero().squeeze(1)
    p.x[~p.live()] = float("nan")
    p.x[live[3], 5] = float("nan")
    p.x[live[-1], 0] = float("inf")
    p.run(dx=False, dw=False)
    bad = torch.zeros(300, dtype=torch.bool, device="cuda")
    bad[live[[3, -1]]] = True
    assert (p.logp.isnan() == bad).all()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("pad,shift,w_pad", [(1, 0, 0), (0, 1, 0), (8, 8, 8), (3, 5, 7), (0, 0, 1), (0, 4, 0)])
def test_strides_and_alignments(layout, pad, shift, w_pad):
    Problem(150, 104, 330, seed=pad + shift, layout=layout, pad=pad, shift=shift, w_pad=w_pad).run(each=100).check()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,each", [(1000, None), (1001, None), (1000, 128), (64, 64), (1, None), (1000, 320)])
@pytest.mark.parametrize("piece_rows", [0, 256])
def test_rows_that_stay_where_they_are(layout, rows, each, piece_rows):
    Problem(rows, 136, 270, layout=layout).run(each=each, keep_rows=True, piece_rows=piece_rows).check()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("p", [0.1, 0.5, 1.0])
@pytest.mark.parametrize("rows,d", [(300, 200), (33, 129), (1500, 72)])
def test_dropout_on_the_features(layout, p, rows, d):
    Problem(rows, d, 500, layout=layout).run(each=100 if rows < 1000 else None, dropout=p, seed=(5 << 40) + 3, step=9,
                                             first_row=12345).check()


@pytest.mark.gpu
def test_dropout_agrees_with_the_operator_and_between_shards():
    """Workers that hold some of the rows drop what the whole drops: both are the definition's by the mask of rows 256 ..  (Not bit
    for bit: few rows take another kernel, whose sums have another order.)"""
    whole = Problem(512, 64, 300, masked=0.0).run(each=128, dropout=0.3, seed=7, step=2).check()
    part = Problem(512, 64, 300, masked=0.0)
    part.x, part.labels, part.row_weight, part.rows = part.x[256:384], part.labels[256:384], part.row_weight[256:384], 128
    part.run(each=128, dropout=0.3, seed=7, step=2, first_row=256).check()
    assert ((part.dx == 0) == (whole.dx[256:384] == 0)).all()
    # rows dropped beforehand (powers of two round nothing): p = 0.5 stretches by 2
    inside = Problem(100, 64, 300, seed=9).run(dropout=0.5, seed=3)
    before = Problem(100, 64, 300, seed=9)
    ngc.dropout(before.x, before.x, 0.5, seed=3)
    before.run()
    back = torch.empty_like(before.dx)
    ngc.dropout(before.dx, back, 0.5, seed=3)
    for a, b in ((inside.logp, before.logp), (inside.dw, before.dw), (inside.dx, back)):
        assert (a.double() - b.double()).norm() <= 2.0 ** -8 * b.double().norm()


@pytest.mark.gpu
def test_left_out_rows_may_hold_anything():
    p = Problem(400, 96, 520, masked=0.4)
    clean = Problem(400, 96, 520, masked=0.4).run(each=130)
    out = ~p.live()
    p.x[out] = float("nan")
    p.x[out.nonzero()[0]] = float("inf")
    p.run(each=130)
    for a, b in ((p.logp, clean.logp), (p.dx, clean.dx), (p.dw, clean.dw), (p.loss, clean.loss)):
        assert torch.equal(a, b)
    clean.check()


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
def test_no_row_counts(keep):
    p = Problem(700, 64, 300)
    p.labels.fill_(-100)
    p.run(each=192, keep_rows=keep)
    assert (p.logp == 0).all() and (p.loss == 0).all() and (p.dx == 0).all() and (p.dw == 0).all()
    assert not ngc.linear_cross_entropy_gave_up(p.workspace)
    # one partition of several, and in pieces
    p = Problem(700, 64, 300, masked=0.0, weighted=False)
    p.labels[192:384] = -1
    p.run(each=192, keep_rows=keep).check()
    p = Problem(700, 64, 300, masked=0.0, weighted=False)
    p.labels[:600] = -1
    p.run(piece_rows=128, keep_rows=keep).check()


@pytest.mark.gpu
def test_no_rows():
    p = Problem(8, 40, 30)
    p.x, p.labels, p.row_weight, p.rows = p.x[:0], p.labels[:0], None, 0
    p.outputs(1, True, True)
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    ngc.linear_cross_entropy(p.x, p.weight, p.labels, p.logp, p.row_loss, p.loss[:0], ws, dx=p.dx, dweight=p.dw[0])
    assert (p.dw == 0).all() and (p.dw_full[:, :, 40:] == 7.0).all()


@pytest.mark.gpu
def test_a_spoiled_row_spoils_its_own_outputs():
    p = Problem(300, 64, 400, masked=0.0, weighted=False)
    p.x[7, 3] = float("nan")
    p.x[250, 1] = float("inf")
    p.run(each=100)
    bad = torch.zeros(300, dtype=torch.bool, device="cuda")
    bad[[7, 250]] = True
    assert (p.logp.isnan() == bad).all() and (p.dx.isnan().any(1) == bad).all()
    assert p.dw.isnan().flatten(1).any(1).tolist() == [True, False, True]
    assert p.loss.isnan().tolist() == [True, False, True]


@pytest.mark.gpu
@pytest.mark.parametrize("spread,scale", [(20.0, 1.0), (200.0, 1.0), (1.0, 1e-3), (1.0, 300.0), (0.0, 1.0)])
def test_far_and_flat_logits(spread, scale):
    Problem(200, 128, 700, spread=spread).run(scale=scale).check()


@pytest.mark.gpu
def test_weights_of_any_size_and_sign():
    p = Problem(200, 64, 300, masked=0.0)
    p.row_weight.copy_(torch.linspace(-3.0, 3.0, 200))
    p.row_weight[::7] *= 1e-20
    p.row_weight[1::7] *= 1e20
    want = Problem(200, 64, 300, masked=0.0, weighted=False).run()
    p.run(each=1, dw=False)
    assert (p.logp == want.logp).all()
    off = (p.row_loss.double() + p.row_weight.double() * want.logp.double()).abs()
    assert (off <= U * (p.row_weight.double() * want.logp.double()).abs()).all()
    off = (p.dx.double() - p.row_weight.double().unsqueeze(1) * want.dx.double()).norm(dim=1)
    assert (off <= 2.0 ** -6 * (p.row_weight.double().unsqueeze(1) * want.dx.double()).norm(dim=1)).all()


@pytest.mark.gpu
def test_gradients_against_differences():
    """Central differences of the losses in x and W: h^2 / 6 of the third derivative and the losses' own rounding."""
    p = Problem(40, 32, 90, masked=0.1).run()
    p.check()
    g = torch.Generator(device="cuda").manual_seed(3)

    def total(x, w):
        q = Problem(40, 32, 90, masked=0.1)
        q.x, q.weight = x, w
        q.run(dx=False, dw=False)
        return float(q.row_loss.double().sum()), q

    for which in ("x", "w"):
        base = (p.x if which == "x" else p.weight).contiguous()
        grad = (p.dx if which == "x" else p.dw[0]).double()
        h = torch.where(torch.rand(base.shape, generator=g, device="cuda") < 0.5, 1.0, -1.0) * 0.03
        up, down = (base.float() + h).to(BF16), (base.float() - h).to(BF16)
        step = (up.double() - down.double()) / 2
        args = ((up, p.weight), (down, p.weight)) if which == "x" else ((p.x, up), (p.x, down))
        (a, _), (b, _) = total(*args[0]), total(*args[1])
        want = float((grad * step).sum())
        # logits move by at most about 32 * 0.03 * (their operand) < 1.5: third-order terms stay below 1.5^3 / 6 per unit weight,
        # far above rounding; signs are random, so they are typically a hundredth of that
        assert abs((a - b) / 2 - want) <= 0.05 * abs(want) + 0.02 * float((grad.abs() * step.abs()).sum())


@pytest.mark.gpu
def test_results_do_not_vary_and_workspaces_keep_nothing():
    a = Problem(700, 200, 3000).run(each=300)
    b = Problem(700, 200, 3000).run(each=300)
    other = Problem(700, 200, 3000, seed=2)
    other.outputs(3)
    other.workspace = b.workspace
    other.run(each=300, outputs=False)
    b.run(each=300, outputs=False)
    for name in ("logp", "row_loss", "loss", "dx", "dw"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


@pytest.mark.gpu
def test_graphs_and_streams():
    p = Problem(900, 128, 2000)
    p.run(each=450)  # (kernels are loaded)
    p.outputs(2)
    p.workspace.fill_(255)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        p.run(each=450, stream=s.cuda_stream, outputs=False)
    for seed in (11, 12):
        q = Problem(900, 128, 2000, seed=seed, masked=0.1 * (seed - 10))
        p.x.copy_(q.x)
        p.labels.copy_(q.labels)
        p.row_weight.copy_(q.row_weight)
        graph.replay()
        torch.cuda.synchronize()
        p.check()
    # two calls beside each other, each with its workspace
    a, b = Problem(600, 64, 1500, seed=3), Problem(600, 64, 1500, seed=4)
    t = torch.cuda.Stream()
    for q in (a, b):
        q.run()
    torch.cuda.synchronize()
    for _ in range(3):
        a.run(stream=s.cuda_stream, outputs=False)
        b.run(stream=t.cuda_stream, outputs=False)
    torch.cuda.synchronize()
    a.check()
    b.check()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("rows,d,classes,each,options", [
    (6400, 2100, 4200, None, {}), (6400, 2100, 4200, None, dict(dropout=0.2, seed=3)), (7000, 1100, 2600, 6200, dict(keep_rows=False)),
    (19000, 600, 520, None, {}), (6272, 2056, 4160, None, dict(keep_rows=True)), (12800, 1040, 2100, 6400, dict(keep_rows=True))])
def test_units_of_two_tiles(layout, rows, d, classes, each, options):
    """Contractions long enough, and tiles enough, for two tiles that share an operand; odd numbers of them at the edges."""
    Problem(rows, d, classes, layout=layout, masked=0.1).run(each=each, **options).check()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["classes", "features"])
@pytest.mark.parametrize("piece_rows", [192, 512])
def test_pieces_with_dropout_and_odd_rows(layout, piece_rows):
    """Every piece goes on where the last one's masks, partitions and sums ended."""
    Problem(1500, 129, 700, layout=layout, pad=3, shift=1, w_pad=1).run(each=700, piece_rows=piece_rows, dropout=0.3, seed=1 << 63, step=5,
                                                                       first_row=1 << 33).check()


@pytest.mark.gpu
def test_a_wait_that_gave_up_shows():
    p = Problem(10, 16, 300).run()
    assert not ngc.linear_cross_entropy_gave_up(p.workspace)
    p.workspace[:4].view(torch.int32).fill_(1)
    assert ngc.linear_cross_entropy_gave_up(p.workspace)
    p.run(outputs=False).check()  # (a call begins anew)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(40))
def test_drawn_shapes_and_options(seed):
    """Any combination, over a workspace of random bytes."""
    rng = random.Random(seed)
    rows, d, classes = (int(math.exp(rng.uniform(0.0, math.log(n)))) for n in (3000, 1500, 6000))
    p = Problem(rows, d, classes, seed=seed, layout=rng.choice(["classes", "features"]), masked=rng.choice([0.0, 0.0, 0.3, 0.9]),
                weighted=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 8]), shift=rng.choice([0, 0, 1, 8]), w_pad=rng.choice([0, 0, 3, 8]))
    each = rng.choice([None, rng.randint(1, rows), rng.randint(1, max(1, rows // 3))])
    if each and -(-rows // each) * d * classes > 40_000_000:
        each = None
    options = {"scale": rng.choice([1.0, 0.3])}
    if rng.random() < 0.4:
        options.update(dropout=rng.choice([0.1, 0.7]), seed=rng.getrandbits(64), step=rng.getrandbits(32), first_row=rng.getrandbits(40))
    elif d % 8 == 0 and p.x.data_ptr() % 16 == 0 and p.x.stride(0) % 8 == 0 and (not each or each >= rows or each % 64 == 0):
        options["keep_rows"] = rng.random() < 0.7
    if rng.random() < 0.3:
        options["piece_rows"] = rng.randint(max(1, rows // 8), rows)
    dx, dw = rng.choice([(True, True), (True, True), (False, True), (True, False), (False, False)])
    p.outputs(-(-rows // (each or rows)), dx, dw)
    sizes = {k: v for k, v in options.items() if k in ("keep_rows", "piece_rows")}
    n = ngc.linear_cross_entropy_workspace_bytes(p.x, p.weight, dx=p.dx, dweight=p.dw, rows_per_partition=each, **sizes)
    p.workspace = torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
    p.run(each=each, outputs=False, **options).check()


@pytest.mark.gpu
def test_many_small_partitions():
    """More partitions than a piece takes."""
    p = Problem(9001, 8, 5, masked=0.3).run(each=1)
    assert (p.loss == p.row_loss).all()
    p.check_some(torch.tensor([0, 1, 4095, 4096, 8191, 8192, 9000], device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("grads", [False, True])
def test_long_features_and_large_vocabularies(grads):
    Problem(3, 70001, 300, masked=0.0).run(dx=grads, dw=grads).check()
    Problem(200, 33000, 40, masked=0.2).run(dx=grads, dw=grads).check()
    Problem(2, 8, 3_000_001, masked=0.0, layout="features").run(dx=grads, dw=grads).check()


@pytest.mark.gpu
def test_first_call_of_a_process_may_be_captured():
    code = """
import torch, paper_2212_08580_b200 as ngc
x, w = torch.randn(700, 128, device="cuda").bfloat16(), torch.randn(3000, 128, device="cuda").bfloat16()
y = torch.randint(0, 3000, (700,), device="cuda", dtype=torch.int32)
logp, row = torch.zeros(700, device="cuda"), torch.zeros(700, device="cuda")
dx, dw, out = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(x)
ws = torch.empty(ngc.linear_cross_entropy_workspace_bytes(x, w, dx=dx, dweight=dw), dtype=torch.uint8, device="cuda")
s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(g, stream=s):
    ngc.dropout(x, out, 0.5, seed=1, stream=s.cuda_stream)
    ngc.linear_cross_entropy(out, w, y, logp, row, None, ws, dx=dx, dweight=dw, dropout=0.1, stream=s.cuda_stream)
g.replay()
torch.cuda.synchronize()
z = torch.randn(1, device="cuda")
assert float(dx.float().norm()) > 0 and float(dw.float().norm()) > 0 and float(logp.max()) < 0 and not ngc.linear_cross_entropy_gave_up(ws)
print("done")
"""
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert got.stdout.strip() == "done", got.stderr


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """70001 rows x 40000 classes: 2.8e9 powers in one piece; some rows against the definition."""
    p = Problem(70001, 16, 40000, masked=0.0, weighted=False)
    p.run(piece_rows=80000)
    at = torch.tensor([0, 1, 33333, 53687, 53688, 69999, 70000], device="cuda")
    z = p.x[at].double() @ p.weight.double().t()
    lse = torch.logsumexp(z, 1, keepdim=True)
    y = p.labels[at].long().unsqueeze(1)
    e_lp = 2 * 24 * U * (p.x[at].double().abs() @ p.weight.double().abs().t()).amax(1, keepdim=True) + 4 * U * (z.abs().amax(1, keepdim=True) + lse.abs() + 1) + 128 * U
    assert ((p.logp[at].double().unsqueeze(1) - (z - lse).gather(1, y)).abs() <= e_lp).all()
    G = (z - lse).exp()
    prob = G.clone()
    G.scatter_add_(1, y, -torch.ones_like(e_lp))
    e_G = prob * e_lp + G.abs() * (2.0 ** -8 + 2.0 ** -11) + 2.0 ** -38
    w = p.weight.double()
    want = G @ w
    off = (p.dx[at].double() - want).abs()
    assert (off <= e_G @ w.abs() + 40008 * U * (G.abs() @ w.abs()) + 2.0 ** -8 * want.abs()).all()
    assert not ngc.linear_cross_entropy_gave_up(p.workspace)


@pytest.mark.gpu
def test_refusals():
    p = Problem(64, 40, 50, masked=0.0)
    p.run(each=32)
    x, w, ws = p.x, p.weight, p.workspace

    def call(x=x, weight=w, labels=p.labels, logp=p.logp, row_loss=p.row_loss, loss=p.loss, workspace=ws, **more):
        options = {"dx": p.dx, "dweight": p.dw, "row_weight": p.row_weight, "rows_per_partition": 32, **more}
        ngc.linear_cross_entropy(x, weight, labels, logp, row_loss, loss, workspace, **options)

    call()
    nan = float("nan")
    bad = [dict(x=x.float()), dict(weight=w.float()), dict(x=x[:, :39]), dict(labels=p.labels.long()), dict(labels=p.labels[:63]),
           dict(logp=p.logp[:63]), dict(loss=p.loss[:1]), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=1e39),
           dict(scale=1e-50), dict(dropout=-0.1), dict(dropout=1.1), dict(dropout=nan), dict(seed=-1), dict(step=1 << 32),
           dict(first_row=-1), dict(rows_per_partition=0), dict(piece_rows=-1), dict(rows_per_partition=31), dict(workspace=ws[:-1]),
           dict(workspace=ws[16:]), dict(workspace=ws.cpu()), dict(dx=p.dx[:63]), dict(dx=p.dx.float()), dict(dx=x), dict(dweight=p.dw[:1]),
           dict(dweight=p.dw.float()), dict(dweight=p.dw.transpose(1, 2).contiguous().transpose(1, 2)), dict(logp=p.row_loss),
           dict(row_weight=p.row_weight[:60]), dict(row_weight=p.logp), dict(loss=p.logp[:2]), dict(x=x.cpu()), dict(weight=None),
           dict(x=x[:, ::2], weight=w[:, ::2]), dict(dweight=p.dw[:1].expand(2, -1, -1)), dict(keep_rows=True, dropout=0.5),
           dict(keep_rows=True, rows_per_partition=16, dweight=torch.empty((4, 50, 40), dtype=BF16, device="cuda"),
                loss=torch.empty(4, device="cuda")),
           dict(keep_rows=True, x=torch.empty((64, 41), dtype=BF16, device="cuda")[:, :40], dweight=None)]
    for change in bad:
        with pytest.raises(ngc.NgcError):
            call(**change)
    shared = torch.zeros(64 * 40 + 64 * 40, dtype=BF16, device="cuda")
    with pytest.raises(ngc.NgcError):
        call(x=shared[: 64 * 40].view(64, 40), dx=shared[40: 40 + 64 * 40].view(64, 40))
    call(x=shared[: 64 * 40].view(64, 40), dx=shared[64 * 40:].view(64, 40))
    call()
    p.check()
