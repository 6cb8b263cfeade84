"""Cases, plain forms and 64-bit values of the training operators: the AdamW update over many tensors
(states in fp32, or in e4m3 with one fp32 scale per 256 elements), the clipped policy loss with its KL term,
and the preference loss over pairs of packed sequences, each loss with the gradient of its logits.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU from a seed, `run` is one pass
(`own` false: elementary torch operations; true: the library's kernels), `exact` the same outputs from the
definitions in 64 bits.
"""
import math
import random

import torch

own = False

BLOCK = 256           # elements that share one scale of an e4m3 state
E4M3_MAX = 448.0      # largest value of the format
E4M3_TINY = 2.0 ** -9  # its smallest positive value
NOTHING = 2.0 ** -110  # a block whose largest magnitude is below this counts as zero
LR, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MOST_LOGITS = 268_435_456   # logits of a drawn case
MOST_PARAMS = 300_000_000   # parameters of a drawn case


def listed():
    return [
        # the parameters of the least-squares workload with 100 workers: one short vector, where the call itself counts
        {"name": "adamw_lsq100", "op": "adamw", "layout": "one", "size": 16384, "theta": "f32", "grad": "f32",
         "state": "f32", "t": 7},
        # the 784-512-10 network: two matrices, and two biases that are not decayed
        {"name": "adamw_mlp30", "op": "adamw", "layout": "mlp", "theta": "f32", "grad": "f32", "state": "e4m3", "t": 40},
        # a stack of 24 attention and feed-forward blocks, fp32 throughout: the memory traffic is all that counts
        {"name": "adamw_stack_f32", "op": "adamw", "layout": "stack", "layers": 24, "width": 1024, "theta": "f32",
         "grad": "f32", "state": "f32", "t": 1000},
        # the same stack with odd widths and its states in 8 bits
        {"name": "adamw_stack_e4m3", "op": "adamw", "layout": "stack", "layers": 24, "width": 1021, "theta": "f32",
         "grad": "f32", "state": "e4m3", "t": 1000},
        # one sampled token of one episode
        {"name": "policy_token", "op": "policy", "rows": 1, "classes": 32000, "dtype": "bf16", "parts": 1, "kl": True,
         "masked": 0.0, "forbidden": False, "scale": 1.0, "pad": 0},
        # the softmax workload's rows and classes as a policy: 50 partitions of 4096 rows, 256 actions
        {"name": "policy_softmax50", "op": "policy", "rows": 204800, "classes": 256, "dtype": "bf16", "parts": 50,
         "kl": True, "masked": 0.0, "forbidden": False, "scale": 1.0, "pad": 0},
        # a training batch of a token model: 8192 tokens, a quarter of them prompt or padding
        {"name": "policy_tokens", "op": "policy", "rows": 8192, "classes": 32000, "dtype": "bf16", "parts": 8, "kl": True,
         "masked": 0.25, "forbidden": False, "scale": 1.0, "pad": 0},
        # fp32 logits over an odd vocabulary, with a temperature, forbidden tokens and no reference model
        {"name": "policy_odd_f32", "op": "policy", "rows": 1999, "classes": 50021, "dtype": "f32", "parts": 3, "kl": False,
         "masked": 0.1, "forbidden": True, "scale": 0.8, "pad": 0},
        # a handful of short answers
        {"name": "preference_short", "op": "preference", "pairs": 4, "length": 24, "classes": 4096, "dtype": "bf16",
         "smooth": 0.0, "mean": False, "scale": 1.0, "pad": 0},
        # a training batch: 16 pairs of answers of about 256 tokens
        {"name": "preference_batch", "op": "preference", "pairs": 16, "length": 256, "classes": 32000, "dtype": "bf16",
         "smooth": 0.0, "mean": False, "scale": 1.0, "pad": 0},
        # two pairs of long answers over a large vocabulary
        {"name": "preference_long", "op": "preference", "pairs": 2, "length": 512, "classes": 131072, "dtype": "bf16",
         "smooth": 0.1, "mean": True, "scale": 1.0, "pad": 0},
        # fp32 logits over an odd vocabulary, rows of a wider buffer
        {"name": "preference_odd_f32", "op": "preference", "pairs": 7, "length": 100, "classes": 10007, "dtype": "f32",
         "smooth": 0.05, "mean": False, "scale": 0.9, "pad": 5},
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["adamw", "policy", "preference"])
    if op == "adamw":
        total = _log_uniform(rng, 1000, MOST_PARAMS)
        return {"op": op, "layout": "mixed", "size": total, "tensors": min(_log_uniform(rng, 1, 400), total),
                "mix": rng.randrange(1 << 30), "theta": rng.choice(["f32", "f32", "bf16"]),
                "grad": rng.choice(["f32", "bf16"]), "state": rng.choice(["f32", "e4m3"]), "t": _log_uniform(rng, 1, 100000)}
    dtype = rng.choice(["f32", "bf16"])
    most = MOST_LOGITS // 2 if dtype == "f32" else MOST_LOGITS
    common = {"dtype": dtype, "scale": rng.choice([1.0, round(rng.uniform(0.5, 1.5), 2)]), "pad": rng.choice([0, 0, 5, 8])}
    if op == "policy":
        classes = _log_uniform(rng, 10, 200_000)
        rows = _log_uniform(rng, 1, min(262_144, most // classes))
        return {"op": op, "rows": rows, "classes": classes, "parts": rng.randint(1, min(rows, 60)), "kl": rng.random() < 0.6,
                "masked": rng.choice([0.0, round(rng.uniform(0.0, 0.5), 2)]), "forbidden": rng.random() < 0.4, **common}
    classes = _log_uniform(rng, 200, 160_000)
    pairs = _log_uniform(rng, 1, 32)
    length = _log_uniform(rng, 1, max(1, min(4096, most // (classes * pairs * 4))))
    return {"op": op, "pairs": pairs, "length": length, "classes": classes, "smooth": rng.choice([0.0, 0.1]),
            "mean": rng.random() < 0.4, **common}


# ---- what the cases consist of


def _sizes(case):
    """Elements and weight decay of every tensor of an AdamW case."""
    if case["layout"] == "one":
        return [(case["size"], 0.01)]
    if case["layout"] == "mlp":
        return [(784 * 512, 0.01), (512, 0.0), (512 * 10, 0.01), (10, 0.0)]
    if case["layout"] == "stack":
        w = case["width"]
        block = [(w, 0.0), (w * w, 0.1), (w * w, 0.1), (w * w, 0.1), (w * w, 0.1), (w, 0.0), (4 * w * w, 0.1), (4 * w, 0.0),
                 (4 * w * w, 0.1), (w, 0.0)]
        return block * case["layers"]
    rng = random.Random(case["mix"])
    parts = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(case["tensors"])]
    unit = case["size"] / sum(parts)
    return [(max(1, int(p * unit)), rng.choice([0.0, 0.1])) for p in parts]


def _lengths(case):
    """Tokens of every sequence of a preference case: chosen and rejected answer in turn, some of them empty."""
    rng = random.Random(case["pairs"] * 1_000_003 + case["length"])
    return [0 if rng.random() < 0.02 else rng.randint(max(1, case["length"] // 2), case["length"] + case["length"] // 2)
            for _ in range(2 * case["pairs"])]


def _counted(case):
    """Which tokens of a preference case have a label: the last two thirds of every sequence."""
    return [n - n // 3 for n in _lengths(case)]


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "adamw":
        n = sum(s for s, _ in _sizes(case))
        state = 16 if case["state"] == "f32" else 4
        scales = 0 if case["state"] == "f32" else 16 * sum(-(-s // BLOCK) for s, _ in _sizes(case))
        return {"bytes": n * (2 * size[case["theta"]] + size[case["grad"]] + state) + scales, "flops": 15 * n}
    e = size[case["dtype"]]
    if case["op"] == "policy":
        rows, classes = case["rows"], case["classes"]
        live = rows * (1.0 - case["masked"])
        return {"bytes": int((live + rows) * classes * e) + rows * (4 * (4 + (1 if case["kl"] else 0)) + 8) + 4 * case["parts"],
                "flops": int(live * classes * 8)}
    tokens, live, classes = sum(_lengths(case)), sum(_counted(case)), case["classes"]
    return {"bytes": (live + tokens) * classes * e + tokens * 4 + case["pairs"] * (16 + 16 + 8 + 4), "flops": live * classes * 8}


# ---- inputs


def _logits(g, rows, classes, dtype, pad):
    """Rows of logits as a model's last layer gives them, `pad` unused columns behind each."""
    full = torch.empty((rows, classes + pad), dtype=dtype, device="cuda")
    full.normal_(0.0, 2.0, generator=g)
    return full[:, :classes]


def _like(logits):
    """A buffer for the gradient with the same row stride."""
    return torch.zeros((logits.shape[0], logits.stride(0)), dtype=logits.dtype, device="cuda")[:, : logits.shape[1]]


def _raise_labels(g, logits, labels):
    """The tokens that were sampled are likelier than the rest."""
    up = 12.0 * torch.rand((labels.numel(), 1), generator=g, device="cuda")
    at = labels.clamp(min=0).long().unsqueeze(1)
    logits.scatter_(1, at, (logits.gather(1, at).float() + up).to(logits.dtype))


def _label_logp(logits, labels, scale):
    """log softmax(scale * logits) at the labels, for inputs only."""
    out = torch.empty(labels.numel(), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 26) // logits.shape[1])
    for a in range(0, labels.numel(), step):
        z = logits[a:a + step].float() * scale
        y = labels[a:a + step].clamp(min=0).long().unsqueeze(1)
        out[a:a + step] = z.gather(1, y).squeeze(1) - torch.logsumexp(z, 1)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    f32 = {"dtype": torch.float32, "device": "cuda"}
    if case["op"] == "adamw":
        # every tensor starts on a multiple of 256 elements of one buffer, as an allocator would place it
        sizes, at, total = _sizes(case), [], 0
        for n, _ in sizes:
            at.append(total)
            total += -(-n // BLOCK) * BLOCK
        inside = torch.zeros(total, dtype=torch.bool, device="cuda")
        for (n, _), a in zip(sizes, at):
            inside[a:a + n] = True

        def filled(std):
            return torch.randn(total, generator=g, **f32).mul_(std).mul_(inside)

        # gradients of very different size from tensor to tensor, moments of the size that such gradients leave
        level = torch.exp(2.0 * torch.randn(len(sizes), generator=g, **f32))
        index = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"),
                                        torch.tensor([-(-n // BLOCK) for n, _ in sizes], device="cuda"))
        per_block = level[index].mul_(1e-3).unsqueeze(1)
        s = {"case": case, "sizes": sizes, "at": at, "step": case["t"],
             "decay": torch.tensor([d for _, d in sizes], **f32)[index].unsqueeze(1),
             "theta": filled(0.05).to(DTYPES[case["theta"]]),
             "grad": (filled(1.0).view(-1, BLOCK) * per_block).view(-1).to(DTYPES[case["grad"]])}
        m = (filled(0.3).view(-1, BLOCK) * per_block).view(-1)
        v = (filled(1.0).view(-1, BLOCK) * per_block).view(-1).square_()
        if case["state"] == "f32":
            s["m"], s["v"] = m, v
        else:
            s["m"], s["m_scale"] = _to_e4m3(m, False)
            s["v"], s["v_scale"] = _to_e4m3(v.sqrt_(), True)
        return s
    dtype, classes = DTYPES[case["dtype"]], case["classes"]
    if case["op"] == "policy":
        rows = case["rows"]
        logits = _logits(g, rows, classes, dtype, case["pad"])
        if case["forbidden"]:
            logits[:, : max(1, classes // 8)] = -math.inf
        low = max(1, classes // 8) if case["forbidden"] else 0
        actions = torch.randint(low, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
        _raise_labels(g, logits, actions)
        logp = _label_logp(logits, actions, case["scale"])
        weight = (torch.rand(rows, generator=g, **f32) >= case["masked"]).float() / rows
        weight[0] = 1.0 / rows  # a batch without any counted token is not trained on
        s = {"case": case, "logits": logits, "actions": actions, "advantage": torch.randn(rows, generator=g, **f32),
             "old_logp": logp - 0.2 * torch.randn(rows, generator=g, **f32),
             "ref_logp": logp - 0.3 * torch.randn(rows, generator=g, **f32) if case["kl"] else None, "weight": weight,
             "rows_per_partition": -(-rows // case["parts"])}
        s["out"] = {"dlogits": _like(logits), "logp": torch.zeros(rows, **f32),
                    "row_loss": torch.zeros(rows, **f32),
                    "loss": torch.zeros(-(-rows // s["rows_per_partition"]), **f32)}
        return s
    lengths, counted, pairs = _lengths(case), _counted(case), case["pairs"]
    rows = sum(lengths)
    begin = torch.tensor([0] + lengths).cumsum(0).to(device="cuda", dtype=torch.int64)
    logits = _logits(g, rows, classes, dtype, case["pad"])
    targets = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    _raise_labels(g, logits, targets)
    place = torch.arange(rows, device="cuda")
    sequence = torch.bucketize(place, begin[1:], right=True)
    prompt = torch.tensor([n - c for n, c in zip(lengths, counted)], device="cuda")
    targets[place - begin[sequence] < prompt[sequence]] = -1
    logp = torch.where(targets >= 0, _label_logp(logits, targets, case["scale"]), 0.0).double()
    total = torch.zeros(2 * pairs, dtype=torch.float64, device="cuda").index_add_(0, sequence, logp)
    if case["mean"]:
        total /= torch.tensor(counted, dtype=torch.float64, device="cuda").clamp(min=1)
    beta = 2.0 if case["mean"] else 0.1
    s = {"case": case, "logits": logits, "targets": targets, "begin": begin, "beta": beta,
         "ref_logp": total.float() + torch.randn(2 * pairs, generator=g, **f32) / beta,
         "pair_weight": torch.rand(pairs, generator=g, **f32) + 0.5}
    s["out"] = {"dlogits": _like(logits), "seq_logp": torch.zeros(2 * pairs, **f32),
                "pair_loss": torch.zeros(pairs, **f32)}
    return s


# ---- plain forms


def _to_e4m3(x, positive):
    """Codes and scales of the 8-bit form of `x`; where `positive`, nothing above zero becomes zero."""
    b = x.view(-1, BLOCK)
    top = b.abs().amax(1, keepdim=True)
    some = top >= NOTHING
    q = torch.where(some, b * torch.where(some, E4M3_MAX / top, 0.0), 0.0)
    if positive:
        q = torch.where((b > 0) & some, q.clamp(min=E4M3_TINY), q)
    return q.to(torch.float8_e4m3fn).view(-1), torch.where(some, top / E4M3_MAX, 0.0).view(-1)


def _plain_adamw(s):
    t, small = s["step"], s["case"]["state"] == "e4m3"
    m, v = s["m"], s["v"]
    if small:
        m = (m.float().view(-1, BLOCK) * s["m_scale"].unsqueeze(1)).view(-1)
        v = (v.float().view(-1, BLOCK) * s["v_scale"].unsqueeze(1)).view(-1).square_()
    g = s["grad"].float()
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    update = (m * (1.0 / (1.0 - BETA1 ** t))) / (torch.sqrt(v) * (1.0 / math.sqrt(1.0 - BETA2 ** t)) + EPS)
    theta = s["theta"].float()
    theta = theta - LR * (update.view(-1, BLOCK) + s["decay"] * theta.view(-1, BLOCK)).view(-1)
    s["theta"].copy_(theta)
    if small:
        for name, x in (("m", m), ("v", v.sqrt_())):
            codes, scales = _to_e4m3(x, name == "v")
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scales)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    s["step"] += 1


def _softmax(logits, labels, scale):
    """Probabilities and the labels' log-probabilities (in 64 bits); labels outside the classes count as class 0."""
    z = logits.float() * scale
    at = torch.where((labels >= 0) & (labels < logits.shape[1]), labels, 0).long().unsqueeze(1)
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    logp = (z.gather(1, at) - top).double() - total.double().log()
    return e / total, logp.squeeze(1), at


def _gradient(p, at, factor, dtype):
    """factor * (onehot - p), row by row."""
    factor = factor.float().unsqueeze(1)
    d = -factor * p
    d.scatter_add_(1, at, factor)
    return torch.where(factor == 0, 0.0, d).to(dtype)


def _plain_policy(s):
    case, rows = s["case"], s["case"]["rows"]
    p, logp, at = _softmax(s["logits"], s["actions"], case["scale"])
    weight, advantage = s["weight"].double(), s["advantage"].double()
    live = (weight != 0) & (s["actions"] >= 0) & (s["actions"] < case["classes"])
    ratio = torch.exp(logp - s["old_logp"].double())
    free, held = ratio * advantage, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * advantage
    loss = -torch.minimum(free, held)
    slope = torch.where(free <= held, -free, 0.0)
    if s["ref_logp"] is not None:
        d = s["ref_logp"].double() - logp
        loss = loss + KL * (torch.expm1(d) - d)
        slope = slope - KL * torch.expm1(d)
    loss = torch.where(live, weight * loss, 0.0)
    slope = torch.where(live, weight * slope, 0.0)
    out = s["out"]
    out["dlogits"].copy_(_gradient(p, at, case["scale"] * slope, out["dlogits"].dtype))
    out["logp"].copy_(torch.where(live, logp, 0.0))
    out["row_loss"].copy_(loss)
    each = s["rows_per_partition"]
    filled = torch.zeros(out["loss"].numel() * each, dtype=torch.float64, device="cuda")
    filled[:rows] = loss
    out["loss"].copy_(filled.view(-1, each).sum(1))
    return out


def _plain_preference(s):
    case, begin, targets = s["case"], s["begin"], s["targets"]
    p, logp, at = _softmax(s["logits"], targets, case["scale"])
    live = (targets >= 0) & (targets < case["classes"])
    sequence = torch.bucketize(torch.arange(targets.numel(), device="cuda"), begin[1:], right=True)
    zero = torch.zeros(1, dtype=torch.float64, device="cuda")
    running = torch.cat([zero, torch.where(live, logp, 0.0).cumsum(0)])
    total = running[begin[1:]] - running[begin[:-1]]
    count = torch.ones_like(total)
    if case["mean"]:
        seen = torch.cat([zero, live.double().cumsum(0)])
        count = (seen[begin[1:]] - seen[begin[:-1]]).clamp(min=1)
        total = total / count
    ratio = total - s["ref_logp"].double()
    h = s["beta"] * (ratio[0::2] - ratio[1::2])
    weight, smooth = s["pair_weight"].double(), case["smooth"]
    softplus = torch.log1p(torch.exp(-h.abs()))  # -log sigmoid(|h|)
    loss = (1.0 - smooth) * (softplus + (-h).clamp(min=0)) + smooth * (softplus + h.clamp(min=0))
    slope = s["beta"] * weight * (smooth / (1.0 + torch.exp(-h)) - (1.0 - smooth) / (1.0 + torch.exp(h)))
    per_sequence = torch.stack([slope, -slope], 1).view(-1) / count
    factor = torch.where(live, case["scale"] * per_sequence[sequence], 0.0)
    out = s["out"]
    out["dlogits"].copy_(_gradient(p, at, factor, out["dlogits"].dtype))
    out["seq_logp"].copy_(total)
    out["pair_loss"].copy_(weight * loss)
    return out


def _own(s):
    import paper_2212_08580_b200 as ngc

    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "adamw":
        if "optimizer" not in s:  # a training program makes it once
            blocks = [-(-n // BLOCK) for n, _ in s["sizes"]]

            def cut(name):
                return [s[name][a:a + n] for (n, _), a in zip(s["sizes"], s["at"])]

            def cut_scales(name):
                return [s[name][a // BLOCK:a // BLOCK + b] for b, a in zip(blocks, s["at"])] if name in s else None

            s["optimizer"] = ngc.AdamW(cut("theta"), cut("grad"), lr=LR, betas=(BETA1, BETA2), eps=EPS,
                                       weight_decay=[d for _, d in s["sizes"]], m=cut("m"), v=cut("v"),
                                       m_scale=cut_scales("m_scale"), v_scale=cut_scales("v_scale"))
        s["optimizer"].update(step=s["step"], stream=stream)
        s["step"] += 1
        return
    out = s["out"]
    if case["op"] == "policy":
        ngc.policy_loss(s["logits"], s["actions"], s["old_logp"], s["advantage"], out["dlogits"], out["logp"],
                        out["row_loss"], out["loss"], ref_logp=s["ref_logp"], weight=s["weight"],
                        rows_per_partition=s["rows_per_partition"], scale=case["scale"], clip_low=CLIP_LOW,
                        clip_high=CLIP_HIGH, kl_coef=KL if case["kl"] else 0.0, stream=stream)
        return
    if "workspace" not in s:
        s["workspace"] = torch.empty(ngc.preference_workspace_bytes(s["targets"].numel(), case["pairs"]),
                                     dtype=torch.uint8, device="cuda")
    ngc.preference_loss(s["logits"], s["targets"], s["begin"], s["ref_logp"], out["dlogits"], out["seq_logp"],
                        out["pair_loss"], s["workspace"], pair_weight=s["pair_weight"], scale=case["scale"],
                        beta=s["beta"], label_smoothing=case["smooth"], length_mean=case["mean"], stream=stream)


def run(s):
    op = s["case"]["op"]
    if own:
        _own(s)
    elif op == "adamw":
        _plain_adamw(s)
    elif op == "policy":
        _plain_policy(s)
    else:
        _plain_preference(s)
    if op == "adamw":
        return {k: s[k] for k in ("theta", "m", "v", "m_scale", "v_scale") if k in s}
    return s["out"]


# ---- the same outputs from the definitions, in 64 bits


def _exact_e4m3(x):
    """Scales and codes of blocks of 256, the codes by their distance to the format's values."""
    b = x.view(-1, BLOCK)
    top = b.abs().max(1, keepdim=True).values
    scale = top / E4M3_MAX
    q = torch.where(top > 0, b / torch.where(top > 0, scale, 1.0), 0.0)
    # the spacing of the format at |q|: 2^(e - 3) for 2^e <= |q| < 2^(e+1), e at least -6
    spacing = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(q / spacing) * spacing, scale


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        t, small = case["t"], case["state"] == "e4m3"
        g = s["grad"].double().view(-1, BLOCK)
        if small:
            m0 = s["m"].to(torch.float64).view(-1, BLOCK) * s["m_scale"].double().unsqueeze(1)
            v0 = (s["v"].to(torch.float64).view(-1, BLOCK) * s["v_scale"].double().unsqueeze(1)) ** 2
        else:
            m0, v0 = s["m"].double().view(-1, BLOCK), s["v"].double().view(-1, BLOCK)
        m = BETA1 * m0 + (1.0 - BETA1) * g
        v = BETA2 * v0 + (1.0 - BETA2) * g ** 2
        del m0, v0, g
        theta = s["theta"].double().view(-1, BLOCK)
        step = (m / (1.0 - BETA1 ** t)) / ((v / (1.0 - BETA2 ** t)).sqrt() + EPS)
        out = {"theta": ((1.0 - LR * s["decay"].double()) * theta - LR * step).view(-1)}
        if not small:
            return {**out, "m": m.view(-1), "v": v.view(-1)}
        out["m"], out["m_scale"] = (x.reshape(-1) for x in _exact_e4m3(m))
        root = v.sqrt()
        codes, out["v_scale"] = (x.reshape(-1) for x in _exact_e4m3(root))
        out["v"] = torch.where((root.view(-1) > 0) & (codes == 0), E4M3_TINY, codes)
        return out
    classes, scale = case["classes"], case["scale"]
    if case["op"] == "policy":
        rows = case["rows"]
        keep = (s["weight"] != 0).nonzero().squeeze(1)
        x = s["logits"][keep].double().requires_grad_()
        logp = torch.log_softmax(scale * x, 1).gather(1, s["actions"][keep].long().unsqueeze(1)).squeeze(1)
        advantage, weight = s["advantage"][keep].double(), s["weight"][keep].double()
        ratio = (logp - s["old_logp"][keep].double()).exp()
        loss = -torch.minimum(ratio * advantage, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * advantage)
        if case["kl"]:
            d = s["ref_logp"][keep].double() - logp
            loss = loss + KL * (d.exp() - d - 1.0)
        loss = loss * weight
        (dx,) = torch.autograd.grad(loss.sum(), x)
        f64 = {"dtype": torch.float64, "device": "cuda"}
        out = {"dlogits": torch.zeros((rows, classes), **f64), "logp": torch.zeros(rows, **f64),
               "row_loss": torch.zeros(rows, **f64), "loss": torch.zeros(s["out"]["loss"].numel(), **f64)}
        out["dlogits"][keep] = dx
        out["logp"][keep] = logp.detach()
        out["row_loss"][keep] = loss.detach()
        out["loss"].index_add_(0, keep // s["rows_per_partition"], loss.detach())
        return out
    rows, pairs = s["targets"].numel(), case["pairs"]
    keep = (s["targets"] >= 0).nonzero().squeeze(1)
    x = s["logits"][keep].double().requires_grad_()
    logp = torch.log_softmax(scale * x, 1).gather(1, s["targets"][keep].long().unsqueeze(1)).squeeze(1)
    owner = torch.searchsorted(s["begin"], keep, right=True) - 1
    total = torch.zeros(2 * pairs, dtype=torch.float64, device="cuda").index_add(0, owner, logp)
    if case["mean"]:
        total = total / torch.bincount(owner, minlength=2 * pairs).clamp(min=1)
    ratio = (total - s["ref_logp"].double()).view(pairs, 2)
    h = s["beta"] * (ratio[:, 0] - ratio[:, 1])
    smooth = case["smooth"]
    logsigmoid = torch.nn.functional.logsigmoid
    loss = s["pair_weight"].double() * -((1.0 - smooth) * logsigmoid(h) + smooth * logsigmoid(-h))
    dlogits = torch.zeros((rows, classes), dtype=torch.float64, device="cuda")
    if keep.numel():
        (dlogits[keep],) = torch.autograd.grad(loss.sum(), x)
    return {"dlogits": dlogits, "seq_logp": total.detach(), "pair_loss": loss.detach()}
