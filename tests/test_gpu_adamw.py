"""ngc_adamw_update against the update written out in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import ngc_inputs
import paper_2212_08580_b200 as ngc
from paper_2212_08580_b200 import gd_loop
from paper_2212_08580_b200.binding import AdamWConfig, AdamWTensor
from tests._util import model_of

LR, B1, B2, EPS = 2e-3, 0.9, 0.999, 1e-8
U = 2.0 ** -24  # half a step of fp32, relative
BLOCK = 256
gpu = pytest.mark.gpu


def cfg(**kw):
    base = dict(lr=LR, beta1=B1, beta2=B2, eps=EPS, grad_scale=1.0, step=1, step_dev=None, theta_dtype=ngc.NGC_F32,
                grad_dtype=ngc.NGC_F32, state_dtype=ngc.NGC_F32)
    return AdamWConfig(**{**base, **kw})


def entry(at=0x1000, numel=64, **kw):
    base = dict(theta=at, grad=at + 0x100000, m=at + 0x200000, v=at + 0x300000, m_scale=at + 0x400000,
                v_scale=at + 0x500000, numel=numel, weight_decay=0.0)
    return AdamWTensor(**{**base, **kw})


def call(c, *entries):
    table = (AdamWTensor * max(1, len(entries)))(*entries)
    return ngc.load_library().ngc_adamw_update(C.byref(c), table, len(entries), None)


@pytest.mark.parametrize("kw", [
    {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": 1.0}, {"beta2": math.nan}, {"eps": 0.0}, {"eps": 1e-60}, {"eps": 1e-38}, {"eps": -1e-8}, {"eps": math.inf}, {"lr": math.inf},
    {"grad_scale": math.nan}, {"step": 0}, {"step": -3}, {"step_dev": 0x1004}, {"theta_dtype": ngc.NGC_F64},
    {"grad_dtype": ngc.NGC_E4M3}, {"state_dtype": ngc.NGC_BF16}, {"theta_dtype": 17}])
def test_bad_settings_are_refused(kw):
    assert call(cfg(**kw), entry()) == -1


@pytest.mark.parametrize("kw", [
    {"theta": None}, {"grad": None}, {"m": None}, {"v": None}, {"theta": 0x1002}, {"grad": 0x2001}, {"m": 0x3002},
    {"numel": -1}, {"numel": 1 << 50}, {"weight_decay": math.nan}])
def test_bad_tensors_are_refused(kw):
    assert call(cfg(), entry(**kw)) == -1


def test_missing_scales_overlaps_and_null_arguments_are_refused():
    small = cfg(state_dtype=ngc.NGC_E4M3)
    assert call(small, entry(m_scale=None)) == -1
    assert call(small, entry(v_scale=None)) == -1
    a = entry()
    assert call(cfg(), a, a) == -1                                             # the same tensor twice
    assert call(cfg(), entry(0x9000), entry(0x1000), entry(0x1000 + 4 * 63)) == -1   # one element shared, unordered list
    assert call(cfg(), entry(0x1000), entry(0x9000, m=0x201000 + 4)) == -1     # only the states overlap
    lib = ngc.load_library()
    assert lib.ngc_adamw_update(None, None, 0, None) == -1
    c = cfg()
    assert lib.ngc_adamw_update(C.byref(c), None, 1, None) == -1
    assert lib.ngc_adamw_update(C.byref(c), None, -1, None) == -1
    assert lib.ngc_adamw_update(C.byref(c), None, 0, None) == 0                # nothing to do
    assert call(c, entry(numel=0, theta=None)) == 0


def test_ranges_of_different_kinds_that_overlap_are_refused():
    small = cfg(state_dtype=ngc.NGC_E4M3)
    a = entry()
    assert call(cfg(), entry(m=a.v)) == -1
    assert call(cfg(), entry(v=a.theta + 4 * 63)) == -1
    assert call(cfg(), entry(0x9000), entry(m=0x9000)) == -1                   # another tensor's theta
    assert call(small, entry(m_scale=a.v_scale)) == -1
    assert call(small, entry(v_scale=a.m)) == -1
    assert call(small, entry(0x9000, numel=600), entry(m_scale=0x409000 + 8)) == -1  # the last of three scales


@pytest.mark.parametrize("kw", [{"lr": 1e300}, {"grad_scale": -1e300}])
def test_settings_beyond_fp32_are_refused(kw):
    assert call(cfg(**kw), entry()) == -1
    assert call(cfg(), entry(weight_decay=1e300)) == -1


def test_tensors_that_are_not_on_the_device_are_refused():
    x = torch.zeros(8)
    with pytest.raises(ngc.NgcError):
        ngc.AdamW([x], [x.clone()], lr=1e-3)


# ---- on the device


def e4m3_state(x):
    """Codes and scales of some state to start from (any valid pair will do)."""
    n = x.numel()
    pad = torch.zeros(-(-max(n, 1) // BLOCK) * BLOCK, device=x.device)
    pad[:n] = x
    top = pad.view(-1, BLOCK).abs().amax(1).clamp(min=1e-30)
    codes = (pad.view(-1, BLOCK) * (448.0 / top).unsqueeze(1)).clamp(-448, 448).to(torch.float8_e4m3fn).view(-1)[:n]
    return codes.contiguous(), (top / 448.0)[:-(-n // BLOCK)].contiguous()


def per_element(scale, n):
    return scale.double().repeat_interleave(BLOCK)[:n]


class Problem:
    def __init__(self, sizes, state="f32", theta=torch.float32, grad=torch.float32, offset=0, seed=0, zero=False):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def rand(n, std, dtype):   # `offset` elements into a larger buffer: any alignment
            return (torch.randn(n + offset, generator=g, device="cuda") * std).to(dtype)[offset:]

        self.state = state
        self.theta = [rand(n, 0.5, theta) for n in sizes]
        self.grad = [rand(n, 0.1, grad) for n in sizes]
        m, v = [rand(n, 0.05, torch.float32) for n in sizes], [rand(n, 0.1, torch.float32).square() for n in sizes]
        if zero:
            m, v = [x.zero_() for x in m], [x.zero_() for x in v]
        if offset and state == "f32":
            v = [torch.cat([torch.zeros(offset, device="cuda"), x])[offset:] for x in v]
        self.m_scale = self.v_scale = None
        if state == "e4m3":
            a, b = [e4m3_state(x) for x in m], [e4m3_state(x.sqrt()) for x in v]
            self.m, self.m_scale = [x for x, _ in a], [x for _, x in a]
            self.v, self.v_scale = [x for x, _ in b], [x for _, x in b]
            if offset:
                self.m, self.v = ([torch.cat([torch.zeros(offset, dtype=torch.uint8, device="cuda"), x.view(torch.uint8)])
                                   [offset:].view(torch.float8_e4m3fn) for x in y] for y in (self.m, self.v))
        else:
            self.m, self.v = m, v
        self.decay = [0.1 * (i % 2) for i in range(len(sizes))]

    def optimizer(self, **kw):
        return ngc.AdamW(self.theta, self.grad, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=self.decay, m=self.m, v=self.v,
                         m_scale=self.m_scale, v_scale=self.v_scale, **kw)

    def moments(self):
        if self.state == "f32":
            return [x.double() for x in self.m], [x.double() for x in self.v]
        return ([x.double() * per_element(s, x.numel()) for x, s in zip(self.m, self.m_scale)],
                [(x.double() * per_element(s, x.numel())) ** 2 for x, s in zip(self.v, self.v_scale)])

    def expected(self, t, grad_scale=1.0, lr=LR):
        """In 64 bits: theta, m, v after the step, and how far fp32 arithmetic may be off each."""
        out = []
        for th, g, m, v, wd in zip([x.double() for x in self.theta], [x.double() * grad_scale for x in self.grad],
                                   *self.moments(), self.decay):
            a, b = B1 * m, (1 - B1) * g
            c, d = B2 * v, (1 - B2) * g * g
            m1, v1 = a + b, c + d
            bc1, bc2 = 1 - B1 ** t, 1 - B2 ** t
            den = (v1 / bc2).sqrt() + EPS
            step = m1 / bc1 / den
            new = th - lr * (step + wd * th)
            # roundings: the constant, the scaled gradient, the state read from 8 bits (two for v), each product, the sum
            dm = U * (5 * a.abs() + 5 * b.abs())
            dv = U * (7 * c + 7 * d)
            # v enters by its root (half of its relative error); root, correction, product, eps and quotient: one each
            dstep = dm / bc1 / den + step.abs() * (dv / v1.clamp(min=1e-300) / 2 + 7 * U)
            dnew = U * new.abs() + lr * (dstep + 4 * U * (step.abs() + (wd * th).abs()))
            out.append((new, dnew, m1, dm, v1, dv))
        return out

    def check(self, want):
        for i, (new, dnew, m1, dm, v1, dv) in enumerate(want):
            half = torch.finfo(self.theta[i].dtype).eps / 2
            tol = 1.01 * dnew + (1.01 * half * new.abs() if half > U else 0.0)
            assert ((self.theta[i].double() - new).abs() <= tol + 1e-38).all(), ("theta", i)
            if self.state == "f32":
                assert ((self.m[i].double() - m1).abs() <= 1.01 * dm + 1e-38).all(), ("m", i)
                assert ((self.v[i].double() - v1).abs() <= 1.01 * dv + 1e-38).all(), ("v", i)
                continue
            n = m1.numel()
            for name, codes, scale, x, dx in (("m", self.m[i], self.m_scale[i], m1, dm),
                                              ("v", self.v[i], self.v_scale[i], v1.sqrt(), dv / v1.sqrt().clamp(min=1e-300))):
                pad = torch.zeros(scale.numel() * BLOCK, dtype=torch.float64, device="cuda")
                pad[:n] = x.abs()
                top = pad.view(-1, BLOCK).amax(1) / 448
                pad[:n] = dx
                off = pad.view(-1, BLOCK).amax(1) / 448
                assert ((scale.double() - top).abs() <= 1.01 * off + 2 * U * top).all(), (name, i)
                s = per_element(scale, n)
                # half a step of the format: 2^-4 of the value, or 2^-10 of the scale among the subnormals; the smallest
                # positive root is lifted to a whole step of them, 2^-9
                low = 2.0 ** -9 if name == "v" else 2.0 ** -10
                tol = torch.maximum(2.0 ** -4 * x.abs(), low * s) * (1 + 1e-5) + 1.01 * dx
                got = codes.double() * s
                assert ((got - x).abs() <= tol).all(), (name, i)
                if name == "v":
                    assert (got[x > 0] > 0).all()


SIZES = [[1], [3], [255], [256], [257], [2047, 2048, 2049], [0, 5, 1000, 0, 70001]]


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_one_step(sizes, state):
    p = Problem(sizes, state, seed=len(sizes))
    want = p.expected(5)
    p.optimizer().update(step=5)
    torch.cuda.synchronize()
    p.check(want)


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("theta,grad", [("float32", "bfloat16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("offset", [0, 1, 2, 3])
def test_types_and_alignments(state, theta, grad, offset):
    p = Problem([4096, 777], state, getattr(torch, theta), getattr(torch, grad), offset, seed=offset)
    if offset == 1:
        p.grad = [torch.cat([x, x])[3:3 + x.numel()] for x in p.grad]   # the gradient aligned in another way
    want = p.expected(12, grad_scale=0.25)
    p.optimizer().update(step=12, grad_scale=0.25)
    torch.cuda.synchronize()
    p.check(want)


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("count", [48, 49, 440, 441, 1000])
def test_many_tensors(count, state):
    p = Problem([(i * 37) % 700 for i in range(count)], state, seed=count)
    want = p.expected(3)
    p.optimizer().update(step=3)
    torch.cuda.synchronize()
    p.check(want)


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_first_steps_from_zero_and_without_gradient(state):
    p = Problem([600, 300], state, zero=True, seed=4)
    p.grad[1].zero_()
    start = p.theta[1].clone()
    opt = p.optimizer()
    for t in (1, 2, 3):
        want = p.expected(t)
        opt.update()
        torch.cuda.synchronize()
        p.check(want)
    assert opt.step == 3
    # no gradient, no moments: only the decay moves theta, by lr * 0.1 a step (two roundings each)
    assert ((p.theta[1].double() - start.double() * (1 - LR * 0.1) ** 3).abs() <= 3 * 3 * U * start.double().abs()).all()
    assert (p.m[1].double() == 0).all() and (p.v[1].double() == 0).all()


@gpu
def test_states_made_by_the_object_start_at_zero():
    for state in ("f32", "e4m3"):
        th, g = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
        opt = ngc.AdamW([th], [g], lr=LR, state_dtype=state)
        opt.update()
        torch.cuda.synchronize()
        # after one step from zero m / (1 - b1) = g and v / (1 - b2) = g^2: every element moves by lr
        assert (th.double() - (1 - LR)).abs().max() <= 2 * U + LR * 20 * U


@gpu
def test_small_second_moments_are_not_lost_in_eight_bits():
    # one element a million times larger than the rest of its block: the others' roots fall below the format's range
    th, g = torch.zeros(256, device="cuda"), torch.full((256,), 1e-6, device="cuda")
    g[7] = 1.0
    opt = ngc.AdamW([th], [g], lr=LR, state_dtype="e4m3")
    for _ in range(20):
        opt.update()
    torch.cuda.synchronize()
    assert (opt.v[0].view(torch.uint8) > 0).all()
    assert th.abs().max().item() <= 20 * LR * 1.2     # no element takes more than a step of about lr


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_a_nan_stays_in_its_element_or_block(state):
    p = Problem([1024, 512], state, seed=9)
    p.grad[0][300] = math.nan
    want = p.expected(2)
    p.optimizer().update(step=2)
    torch.cuda.synchronize()
    assert torch.isnan(p.theta[0][300]) and torch.isnan(p.theta[0]).sum() == 1
    keep = torch.ones(1024, dtype=torch.bool, device="cuda")
    keep[256:512] = False
    new, dnew = want[0][0], want[0][1]
    assert ((p.theta[0].double() - new).abs() <= 1.01 * dnew)[keep].all()
    m, v = p.moments()
    assert torch.isfinite(m[0][keep]).all() and torch.isfinite(v[0][keep]).all()
    assert torch.isfinite(m[1]).all() and torch.isfinite(v[1]).all()


@gpu
def test_step_number_on_the_device_in_a_replayed_graph():
    a, b = Problem([5000, 33], "e4m3", seed=1), Problem([5000, 33], "e4m3", seed=1)
    count = torch.ones(1, dtype=torch.int64, device="cuda")
    opt = a.optimizer()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        opt.update(step_dev=count, stream=torch.cuda.current_stream().cuda_stream)
        count.add_(1)
    ref = b.optimizer()
    for t in range(1, 5):
        graph.replay()
        ref.update(step=t)
    torch.cuda.synchronize()
    assert count.item() == 5
    for x, y in zip(a.theta + a.m_scale + a.v_scale, b.theta + b.m_scale + b.v_scale):
        assert torch.equal(x, y)
    for x, y in zip(a.m + a.v, b.m + b.v):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@gpu
def test_neighbouring_memory_is_left_alone():
    buf = torch.full((3, 1000), 7.0, device="cuda")
    codes = torch.full((2, 1000), 17, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, 10), 5.0, device="cuda")
    opt = ngc.AdamW([buf[0][100:401]], [buf[1][100:401]], lr=LR, m=[codes[0][100:401].view(torch.float8_e4m3fn)],
                    v=[codes[1][100:401].view(torch.float8_e4m3fn)], m_scale=[scales[0][4:6]], v_scale=[scales[1][4:6]])
    opt.update()
    torch.cuda.synchronize()
    for x, old in ((buf[0], 7.0), (codes[0], 17), (codes[1], 17)):
        assert (x[:100] == old).all() and (x[401:] == old).all()
    assert (scales[:, :4] == 5.0).all() and (scales[:, 6:] == 5.0).all() and (buf[1:] == 7.0).all()


@gpu
def test_bad_lists_are_refused():
    x = torch.zeros(300, device="cuda")
    g, m, v = x.clone(), x.clone(), x.clone()
    for bad in (lambda: ngc.AdamW([x], [g[:299]], lr=LR), lambda: ngc.AdamW([x], [], lr=LR),
                lambda: ngc.AdamW([x.double()], [g], lr=LR), lambda: ngc.AdamW([x[::2]], [g[:150]], lr=LR),
                lambda: ngc.AdamW([x], [g], lr=LR, m=[m]), lambda: ngc.AdamW([x], [g], lr=LR, m=[m], v=[v[:10]]),
                lambda: ngc.AdamW([x], [g], lr=LR, weight_decay=[0.1, 0.2]),
                lambda: ngc.AdamW([x], [g], lr=LR, m=[m.to(torch.float8_e4m3fn)], v=[v.to(torch.float8_e4m3fn)]),
                lambda: ngc.AdamW([x], [g], lr=LR, state_dtype="int8"),
                lambda: ngc.AdamW([x, x], [g, g], lr=LR).update(),
                lambda: ngc.AdamW([x], [g], lr=LR).update(step=0)):
        with pytest.raises(ngc.NgcError):
            bad()


@gpu
@pytest.mark.parametrize("optimizer", ["adamw", "adamw8"])
def test_gradient_descent_loop_with_adamw(optimizer):
    """The loop's iterates are those of the update applied to the gradients that the plan decodes."""
    w = ngc_inputs.shrink(ngc_inputs.WORKLOADS["mlp30"], rows=60)
    X, y, theta = ngc_inputs.make_data(w, "cuda")
    a, b = theta.clone(), theta.clone()
    plan = ngc.Plan(w.n, w.levels, seed=w.seed)
    gd_loop.run(plan, model_of(w), a, X, y, 3, 1e-2, 55, optimizer=optimizer, weight_decay=0.1)
    coded = torch.empty((w.n, w.n_params), device="cuda")
    grad = torch.empty(w.n_params, device="cuda")
    opt = gd_loop.make_optimizer(optimizer, model_of(w), b, grad, 1e-2, 0.1)
    assert [p.numel() for p in opt.params] == [784 * 512, 512, 5120, 10]
    tasks = w.levels[-1] + 1
    for it in range(3):
        t = np.ascontiguousarray(ngc.sample_times(55 + it, w.n, tasks, 0.5, 0.5, 0.0))
        plan.step(model_of(w), b, X, y, t, coded, grad)
        opt.update(grad_scale=1.0 / (w.n * w.rows))
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.isfinite(a).all() and not torch.equal(a, theta)


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_an_object_made_on_one_stream_and_used_on_another(state):
    th, g = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(20_000_000)            # the zeros of the states come behind this
        opt = ngc.AdamW([th], [g], lr=LR, state_dtype=state)
    other = torch.cuda.Stream()
    opt.update(stream=other.cuda_stream)
    torch.cuda.synchronize()
    assert (opt.m[0].float() != 0).all() and (th.double() - (1 - LR)).abs().max() <= 2 * U + LR * 20 * U


@gpu
def test_a_refused_update_leaves_the_settings():
    th, g = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
    opt = ngc.AdamW([th], [g], lr=LR)
    with pytest.raises(ngc.NgcError):
        opt.update(lr=math.nan)
    assert opt.step == 0
    opt.update()
    torch.cuda.synchronize()
    assert opt.step == 1 and (th.double() - (1 - LR)).abs().max() <= 2 * U + LR * 20 * U


@gpu
def test_a_device_counter_that_has_not_started_counts_as_the_first_step():
    th, g = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
    opt = ngc.AdamW([th], [g], lr=LR)
    opt.update(step_dev=torch.zeros(1, dtype=torch.int64, device="cuda"))
    torch.cuda.synchronize()
    assert (th.double() - (1 - LR)).abs().max() <= 2 * U + LR * 20 * U


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_two_updates_beside_each_other_and_interleaved_tensors(state):
    """Two objects on two streams; the second one's tensors lie in one buffer, kinds mixed."""
    a = Problem([70001, 300], state, seed=21)
    th, g = torch.ones(2, 256, device="cuda"), torch.full((256,), 0.5, device="cuda")
    flat = torch.zeros(2, 256 * 8 + 16, dtype=torch.uint8, device="cuda")
    kind = torch.float8_e4m3fn if state == "e4m3" else torch.float32
    size = 256 * (1 if state == "e4m3" else 4)
    b = ngc.AdamW([th[0], th[1]], [g, g], lr=LR, m=[x[:size].view(kind) for x in flat],
                  v=[x[size:2 * size].view(kind) for x in flat], m_scale=[x[-16:-12].view(torch.float32) for x in flat],
                  v_scale=[x[-8:-4].view(torch.float32) for x in flat])
    want = a.expected(5)
    opt = a.optimizer()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    opt.update(step=5, stream=one.cuda_stream)
    b.update(stream=two.cuda_stream)
    torch.cuda.synchronize()
    a.check(want)
    assert (th.double() - (1 - LR)).abs().max() <= 2 * U + LR * 20 * U


@gpu
def test_step_numbers_beyond_64_bits_are_refused():
    th, g = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
    opt = ngc.AdamW([th], [g], lr=LR)
    for step in (1 << 63, (1 << 64) + 1, -(1 << 64) + 1):
        with pytest.raises(ngc.NgcError):
            opt.update(step=step)
    torch.cuda.synchronize()
    assert (th == 1.0).all() and opt.step == 0


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_states_are_not_made_during_a_capture(state):
    """A replay would zero them again: every step a first one."""
    th, g = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
    p = Problem([300], state)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        with pytest.raises(ngc.NgcError):
            ngc.AdamW([th], [g], lr=LR, state_dtype=state)
        p.optimizer().update(step=1, stream=torch.cuda.current_stream().cuda_stream)   # states of the caller's: as before
    want = p.expected(1)
    graph.replay()
    torch.cuda.synchronize()
    p.check(want)
    ngc.AdamW([th], [g], lr=LR, state_dtype=state).update()
    torch.cuda.synchronize()
    assert (th.double() - (1 - LR)).abs().max() <= 2 * U + LR * 20 * U


@pytest.mark.parametrize("settings,entries", [
    ({}, [{"grad": 0x1000 + 4}]),                                               # theta, one element off
    ({}, [{"grad": 0x201000 - 4 * 63}]),                                        # the first element of m
    ({}, [{}, {"at": 0x9000, "grad": 0x1000}]),                                 # another tensor's theta
    ({}, [{"at": 0x9000, "grad": 0x301000}, {}]),                               # another tensor's v
    ({"grad_dtype": ngc.NGC_BF16}, [{"grad": 0x1000}]),                         # half of its own theta's bytes
    ({"theta_dtype": ngc.NGC_BF16}, [{"grad": 0x1000}]),                        # its own theta and what lies behind it
    ({"state_dtype": ngc.NGC_E4M3}, [{"grad": 0x201000}]),                      # codes
    ({"state_dtype": ngc.NGC_E4M3}, [{"grad": 0x401000 - 4 * 60}]),             # a scale
    ({"step_dev": 0x1008}, [{}]), ({"step_dev": 0x301000}, [{}, {"at": 0x9000}]),
    ({}, [{"at": 0x1000 * (9 - i), "grad": 0x700000} for i in range(7)] + [{"at": 0x600000, "grad": 0x203000 + 8}])])
def test_gradients_in_memory_that_is_written_are_refused(settings, entries):
    assert call(cfg(**settings), *(entry(**{"at": 0x1000, **e}) for e in entries)) == -1


@gpu
@pytest.mark.parametrize("kind", ["theta", "m", "v", "each other"])
@pytest.mark.parametrize("order", [1, -1])
def test_gradients_in_their_own_tensors_memory(kind, order):
    """A gradient that is its tensor's theta, m or v (a weight of its own, say), element for element, or another's gradient."""
    p = Problem([5000, 300, 4099], seed=12)
    for x in (p.theta, p.grad, p.m, p.v, p.decay):
        x[:] = x[::order]
    if kind == "each other":
        p.grad = [p.grad[0 if order == 1 else 2][:n] for n in (x.numel() for x in p.theta)]
    else:
        p.grad = list(getattr(p, kind))
    want = p.expected(4)
    p.optimizer().update(step=4)
    torch.cuda.synchronize()
    p.check(want)
