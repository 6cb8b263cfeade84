"""Gradient descent (Eq. 1) driven by a gradient code, with the latency of every iteration taken from the
straggler model of Section II-D: per-task times rho + Exp(lambda), a worker failing with probability p_e,
constants gamma and eps added once per iteration.

    python -m paper_2212_08580_b200.gd_loop --iters 50        # nested code vs fixed codes vs uncoded, least squares
    python -m paper_2212_08580_b200.gd_loop --optimizer adamw8        # AdamW with 8-bit states instead of the plain step
    python -m paper_2212_08580_b200.gd_loop --loss policy             # a softmax policy, or --loss preference

Every scheme sees the same per-task times in the same iteration, so the latencies are directly comparable:
a nested code with levels 0..s_bar stops as early as the best fixed code of the iteration (Section III).
An iteration whose pattern no component code can decode (more hard stragglers than the largest tolerance) is
repeated with fresh times and its waiting time is not counted: the model's latency is infinite there.

Only argument marshalling happens here; gradients, encode, decode and update run in the CUDA library.
"""
from __future__ import annotations

import argparse
from contextlib import contextmanager
from dataclasses import dataclass, field

import numpy as np

from . import AdamW, NgcError, Plan, gd_update, policy_loss, preference_loss, preference_workspace_bytes, sample_times
from .binding import NGC_F64, NGC_MLP, NGC_SOFTMAX


@dataclass
class History:
    latency: list = field(default_factory=list)        # model time of every completed iteration
    level: list = field(default_factory=list)          # component code that decoded it
    tasks_done: list = field(default_factory=list)     # partial gradients computed by all workers together
    undecodable: int = 0                               # patterns that had to be redrawn

    @property
    def total_latency(self) -> float:
        return float(np.sum(self.latency))


OPTIMIZERS = ("gd", "adamw", "adamw8")


def parameter_tensors(model, theta):
    """The weight matrices and bias vectors that a model's flat theta consists of, as (view, is a bias)."""
    if model.kind != NGC_MLP:
        return [(theta, False)]
    sizes = (model.d * model.hidden, model.hidden, model.hidden * model.n_classes, model.n_classes)
    return [(part, i % 2 == 1) for i, part in enumerate(theta.split(sizes))]


def make_optimizer(name: str, model, theta, grad, lr: float, weight_decay: float = 0.0) -> AdamW:
    """AdamW over a model's tensors, states in fp32 ("adamw") or in 8 bits ("adamw8"); biases are not decayed."""
    parts = parameter_tensors(model, theta)
    return AdamW([p for p, _ in parts], [g for g, _ in parameter_tensors(model, grad)], lr=lr,
                 weight_decay=[0.0 if bias else weight_decay for _, bias in parts],
                 state_dtype="e4m3" if name == "adamw8" else "f32")


class PolicyLoss:
    """policy_loss over the rows of all partitions, for `run`: called with the logits, it replaces them by their
    gradient.  `loss` holds the sum over each partition after every iteration."""

    def __init__(self, actions, old_logp, advantage, rows_per_partition: int, **options):
        import torch
        self.made_on = torch.cuda.current_stream()
        rows = actions.numel()
        self.fixed = (actions.reshape(-1), old_logp.reshape(-1), advantage.reshape(-1))
        self.logp, self.row_loss = (torch.empty(rows, dtype=torch.float32, device=actions.device) for _ in range(2))
        self.loss = torch.empty(rows // rows_per_partition, dtype=torch.float32, device=actions.device)
        self.options = dict(options, rows_per_partition=rows_per_partition)

    def __call__(self, logits, stream: int):
        policy_loss(logits, *self.fixed, logits, self.logp, self.row_loss, self.loss, stream=stream, **self.options)


class PreferenceLoss:
    """preference_loss over pairs of consecutive rows' sequences, for `run`.  A pair lies within one task of a worker (a
    partition, or the consecutive ones that make up a task), which is all that a worker sees; `run` refuses others.
    Rows that no sequence holds do not train (called on its own, the loss leaves them as they are).  `loss` holds the loss of
    every pair after every iteration."""

    def __init__(self, labels, seq_begin, ref_logp, **options):
        import torch
        self.made_on = torch.cuda.current_stream()
        pairs = ref_logp.numel() // 2
        device = labels.device
        self.fixed = (labels.reshape(-1), seq_begin, ref_logp)
        self.seq_logp = torch.empty(2 * pairs, dtype=torch.float32, device=device)
        self.loss = torch.empty(pairs, dtype=torch.float32, device=device)
        self.workspace = torch.empty(preference_workspace_bytes(labels.numel(), pairs), dtype=torch.uint8, device=device)
        self.options = options

    def held_rows(self, rows_per_task: int):
        """First row of the first sequence and end of the last one; raises where a pair's rows belong to more than one task."""
        import torch
        with torch.cuda.stream(self.made_on):
            begin = self.fixed[1].cpu()
        first, last = begin[:-1:2], begin[2::2]
        split = (last > first) & (first // rows_per_task != (last - 1) // rows_per_task)
        if split.any():
            raise ValueError(f"pair {int(split.nonzero()[0])} lies in more than one task of {rows_per_task} rows")
        first, last = (min(max(int(r), 0), self.fixed[0].numel()) for r in (begin[0], begin[-1]))
        return first, max(first, last)

    def __call__(self, logits, stream: int):
        preference_loss(logits, *self.fixed, logits, self.seq_logp, self.loss, self.workspace, stream=stream,
                        **self.options)


def _torch_stream(stream: int):
    import torch
    return torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()


def _on(stream: int):
    """torch's work and memory on the stream that the library is given."""
    import torch
    return torch.cuda.stream(_torch_stream(stream))


@contextmanager
def _between(stream: int, loss):
    """Work on `stream` behind what torch's current stream, and the one that the loss was made on, have been given, and the
    later work of those two behind it: they own buffers that it uses."""
    import torch
    here, others = _torch_stream(stream), {torch.cuda.current_stream()}
    if getattr(loss, "made_on", None) is not None:
        others.add(loss.made_on)
    others.discard(here)
    for s in others:
        here.wait_stream(s)
    try:
        yield
    finally:
        for s in others:
            s.wait_stream(here)


class _LossStep:
    """What plan.step does for the softmax model, with a loss of the logits in place of cross-entropy."""

    def __init__(self, plan: Plan, model, theta, loss):
        import torch
        if model.kind != NGC_SOFTMAX:
            raise ValueError("a loss of the logits goes with the softmax model")
        rows = plan.k * model.rows_per_partition
        self.held = (0, rows)
        if isinstance(loss, PreferenceLoss):
            self.held = loss.held_rows(rows // plan.n)
        self.plan, self.model, self.loss = plan, model, loss
        l = int(theta.numel())
        self.logits = torch.empty((rows, model.n_classes), dtype=torch.bfloat16, device=theta.device)
        self.window = torch.empty((plan.n + plan.levels[-1], l), dtype=torch.float32, device=theta.device)
        f64 = plan.coded_dtype(model) == NGC_F64
        self.coded = torch.empty_like(self.window, dtype=torch.float64 if f64 else torch.float32)
        self.partial = torch.empty(l, dtype=self.coded.dtype, device=theta.device)

    def __call__(self, theta, X, times, grad, stream: int):
        plan, model, n = self.plan, self.model, self.plan.n
        info = plan.select(times)
        plan.shard_logits(model, theta, X, n, self.logits, stream)
        self.loss(self.logits, stream)
        first, last = self.held
        with _on(stream):  # the other rows still hold their logits
            if first > 0:
                self.logits[:first].zero_()
            if last < self.logits.shape[0]:
                self.logits[last:].zero_()
        plan.shard_weight_gradients(model, X, self.logits, n, self.window, self.window.stride(0), stream)
        with _on(stream):
            if info.sigma:  # the windows of the last workers go on with the first groups
                self.window[n:n + info.sigma].copy_(self.window[:info.sigma])
            plan.shard_encode_decode(model, info.layer, 0, n, self.window, self.window.stride(0), info.responsive(),
                                     self.coded, self.partial, stream)
            grad.copy_(self.partial)
        return info


def run(plan: Plan, model, theta, X, y, iters: int, step: float, seed: int, rho: float = 0.5, lam: float = 0.5,
        p_fail: float = 0.0, times_width: int | None = None, stream: int = 0, optimizer: str = "gd",
        weight_decay: float = 0.0, loss=None) -> History:
    """`iters` iterations of theta <- theta - step * g on the device, g decoded by `plan` under a fresh seeded
    straggler pattern per iteration.  theta is updated in place; returns the latency record.

    `times_width` = tasks per worker that are drawn (default: what this plan needs).  Schemes that are to see the
    same times must be given the same width (the largest any of them needs); each reads the first columns.

    `optimizer` "adamw" or "adamw8" replaces the plain step by AdamW (states in fp32 or in 8 bits) with learning rate
    `step`, `weight_decay` on the weight matrices, and the mean of the gradient over all rows.

    `loss` (softmax model, y unused): a PolicyLoss or PreferenceLoss that is trained on instead of cross-entropy;
    workers and the largest tolerance together are then at most 128.

    `stream` (a cudaStream_t as an integer): the iterations wait for what torch's current stream, and the one that the loss was
    made on, have been given so far, and their later work waits for the iterations."""
    if optimizer not in OPTIMIZERS:
        raise ValueError(f"optimizer is one of {OPTIMIZERS}")
    with _between(stream, loss):
        return _run(plan, model, theta, X, y, iters, step, seed, rho, lam, p_fail, times_width, stream, optimizer,
                    weight_decay, loss)


def _run(plan, model, theta, X, y, iters, step, seed, rho, lam, p_fail, times_width, stream, optimizer, weight_decay,
         loss) -> History:
    import torch
    l = int(theta.numel())
    cdt = plan.coded_dtype(model)
    tasks = plan.levels[-1] + 1
    width = max(tasks, times_width or 0)
    mean = 1.0 / (plan.k * model.rows_per_partition)
    coded = opt = loss_step = None
    with _on(stream):
        if loss is None:
            coded = torch.empty((plan.n, l), dtype=torch.float64 if cdt == NGC_F64 else torch.float32, device=theta.device)
        grad = torch.empty(l, dtype=torch.float32, device=theta.device)
        if optimizer != "gd":
            opt = make_optimizer(optimizer, model, theta, grad, step, weight_decay)
        if loss is not None:
            loss_step = _LossStep(plan, model, theta, loss)
    hist = History()
    draw = 0
    for _ in range(iters):
        while True:
            t = sample_times(seed + draw, plan.n, width, rho, lam, p_fail)[:, :tasks]
            draw += 1
            try:
                if loss_step is None:
                    info = plan.step(model, theta, X, y, np.ascontiguousarray(t), coded, grad, stream)
                else:
                    info = loss_step(theta, X, np.ascontiguousarray(t), grad, stream)
                break
            except NgcError as e:
                if e.status != -2:      # NGC_ERR_UNDECODABLE
                    raise
                hist.undecodable += 1
        if opt is None:
            gd_update(theta, grad, step, stream)
        else:
            opt.update(grad_scale=mean, stream=stream)
        hist.latency.append(info.latency)
        hist.level.append(info.layer)
        hist.tasks_done.append(int(sum(info.tasks_done[: plan.n])))
    return hist


def _demo_loss(kind: str, w, X):
    """A policy or preference problem on data X: a hidden linear score says how good each class is for a row."""
    import torch
    rows, C = w.n * w.rows, w.n_classes
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    score = X.reshape(rows, w.d).float() @ torch.randn((w.d, C), generator=g, device="cuda")
    even = torch.full((rows,), -float(np.log(C)), device="cuda")  # log-probabilities under theta = 0
    if kind == "policy":
        actions = torch.randint(0, C, (rows,), generator=g, device="cuda", dtype=torch.int32)
        reward = score.gather(1, actions.long().unsqueeze(1)).squeeze(1)
        return PolicyLoss(actions, even, (reward - reward.mean()) / reward.std(), w.rows, ref_logp=even, kl_coef=0.01)
    # rows 2 p and 2 p + 1 hold the same data; the better of two drawn classes was chosen
    two = torch.randint(0, C, (rows // 2, 2), generator=g, device="cuda")
    better = score[0::2].gather(1, two)
    swap = better[:, :1] < better[:, 1:]
    labels = torch.where(swap, two.flip(1), two).to(torch.int32)
    return PreferenceLoss(labels.reshape(-1).contiguous(), torch.arange(rows + 1, device="cuda"), even, beta=1.0)


def _main():
    import torch

    import ngc_inputs
    from . import Model

    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--iters", type=int, default=50)
    ap.add_argument("--n", type=int, default=8)
    ap.add_argument("--s-bar", type=int, default=3)
    ap.add_argument("--p-fail", type=float, default=0.0,
                    help="probability that a worker never responds; a redrawn iteration (column 'redrawn') had "
                         "infinite latency under that scheme and shifts its later draws")
    ap.add_argument("--seed", type=int, default=2212)
    ap.add_argument("--optimizer", choices=OPTIMIZERS, default="gd")
    ap.add_argument("--loss", choices=("lsq", "policy", "preference"), default="lsq")
    args = ap.parse_args()
    w = ngc_inputs.Workload("gd_demo", 77, args.n, (0,), "lsq", 512, 256, "f32", unit_x=True)
    if args.loss != "lsq":
        w = ngc_inputs.Workload("gd_demo", 77, args.n, (0,), "softmax", 512, 64, "bf16", n_classes=16)
    X, y, theta0 = ngc_inputs.make_data(w, "cuda")
    model = Model.make(w.kind, w.x_dtype, w.rows, w.d, w.n_classes)
    step = 0.5 / (w.n * w.rows) if args.optimizer == "gd" else 0.05
    loss = None
    if args.loss != "lsq":
        if args.loss == "preference":
            X[:, 1::2] = X[:, 0::2]
        theta0.zero_()
        loss = _demo_loss(args.loss, w, X)
        step = 20.0 / (w.n * w.rows) if args.optimizer == "gd" else step
    schemes = [("nested 0..%d" % args.s_bar, list(range(args.s_bar + 1)))]
    schemes += [("fixed sigma=%d" % s, [s]) for s in range(args.s_bar + 1)]
    print(f"{'scheme':16s} {'total latency':>14s} {'mean':>8s} {'tasks/iter':>11s} {'redrawn':>8s} {'final loss':>12s}")
    for name, levels in schemes:
        plan = Plan(args.n, levels, seed=1, gamma=0.0, eps=0.1)
        theta = theta0.clone()
        h = run(plan, model, theta, X, y, args.iters, step, args.seed, p_fail=args.p_fail, times_width=args.s_bar + 1,
                optimizer=args.optimizer, loss=loss)
        torch.cuda.synchronize()
        if loss is None:
            r = (X.reshape(-1, w.d) @ theta - y.reshape(-1)).double()
            final = 0.5 * float(r @ r)
        else:
            final = float(loss.loss.double().sum())  # at the last iteration's theta
        print(f"{name:16s} {h.total_latency:14.2f} {np.mean(h.latency):8.3f} {np.mean(h.tasks_done):11.1f} "
              f"{h.undecodable:8d} {final:12.4e}")


if __name__ == "__main__":
    _main()
