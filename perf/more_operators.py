"""Cases, plain forms and 64-bit values of two operators around a model's last layer: softmax cross entropy over a large
vocabulary straight from features and weights (`linear_cross_entropy`: log-probabilities, losses, gradients of the features
and, for each partition of the rows, of the weights), and dropout whose mask is a function of seed, step, row and column
(`dropout`, also inside the first on the features).

A case is a dict of plain values.  `prepare` makes its inputs on the GPU from a seed, `run` is one pass
(`own` false: elementary torch operations; true: the library's kernels), `exact` the same outputs from the
definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MOST_PRODUCTS = 1_000_000_000_000  # rows * d * classes of a drawn case
MOST_LOGITS = 1 << 30              # rows * classes of a drawn case
MOST_ELEMENTS = 64_000_000         # elements of a drawn dropout
GRADS = ("none", "weight", "both")


def _ce(rows, d, classes, grads, **more):
    return {"op": "ce", "rows": rows, "d": d, "classes": classes, "grads": grads, "layout": "classes", "parts": 1, "masked": 0.0,
            "weighted": False, "scale": 1.0, "dropout": 0.0, "pad": 0, "keep": False, **more}


def _drop(rows, columns, dtype, **more):
    return {"op": "dropout", "rows": rows, "columns": columns, "dtype": dtype, "p": 0.1, "residual": False, "backward": False,
            "pad": 0, **more}


def listed():
    return [
        # how likely one token is, as a server scores it: the weights are read once
        {"name": "ce_token", **_ce(1, 4096, 32000, "none")},
        # a prompt of 700 tokens scored over an odd vocabulary, half of them counted
        {"name": "ce_score", **_ce(700, 2048, 50021, "none", masked=0.5)},
        # the softmax workload: 50 partitions of 4096 rows, weights as this framework's models hold them ([d][classes]); all rows
        # count, so they are read where they are
        {"name": "ce_softmax50", **_ce(204800, 1024, 256, "weight", layout="features", parts=50, keep=True)},
        # one short sequence: weights and their gradient are all that moves
        {"name": "ce_short", **_ce(96, 2048, 32000, "both", weighted=True)},
        # a training batch: 8192 tokens, a quarter of them prompt or padding
        {"name": "ce_batch", **_ce(8192, 4096, 32000, "both", masked=0.25)},
        # a larger vocabulary: the rows go through in pieces
        {"name": "ce_large", **_ce(8192, 1024, 131072, "both", weighted=True)},
        # features dropped, eight tasks of workers, weights [d][classes]
        {"name": "ce_dropout", **_ce(4096, 1024, 16000, "both", layout="features", parts=8, dropout=0.1, masked=0.1)},
        # nothing is a multiple of anything, rows of a wider buffer
        {"name": "ce_odd", **_ce(1999, 1021, 10007, "both", masked=0.1, weighted=True, scale=0.8, parts=3, pad=5)},
        # the features of one short sequence
        {"name": "dropout_short", **_drop(64, 1024, "bf16")},
        # a batch on its way into a residual stream, and back
        {"name": "dropout_batch", **_drop(8192, 4096, "bf16", residual=True, backward=True)},
        # many features of few rows, in 32 bits, dropped by half
        {"name": "dropout_f32", **_drop(512, 32000, "f32", p=0.5, backward=True)},
        # odd rows of a wider buffer
        {"name": "dropout_odd", **_drop(1999, 5003, "bf16", p=0.3, residual=True, pad=6)},
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    if rng.random() < 0.35:
        columns = _log_uniform(rng, 10, 40000)
        rows = _log_uniform(rng, 1, MOST_ELEMENTS // columns)
        return _drop(rows, columns, rng.choice(["f32", "bf16"]), p=rng.choice([0.1, 0.5, round(rng.uniform(0.0, 0.9), 3)]),
                     residual=rng.random() < 0.5, backward=rng.random() < 0.5, pad=rng.choice([0, 0, 3, 8]))
    classes = _log_uniform(rng, 100, 160_000)
    d = _log_uniform(rng, 48, 4200)
    if rng.random() < 0.5:
        d = max(64, d // 64 * 64)
    rows = _log_uniform(rng, 1, max(1, min(16384, MOST_PRODUCTS // (classes * d), MOST_LOGITS // classes)))
    grads = rng.choice(GRADS)
    case = _ce(rows, d, classes, grads, layout=rng.choice(["classes", "features"]),
               parts=rng.randint(1, max(1, min(8, rows, 400_000_000 // (classes * d)))) if grads != "none" else 1,
               masked=rng.choice([0.0, round(rng.uniform(0.0, 0.6), 2)]), weighted=rng.random() < 0.5,
               scale=rng.choice([1.0, round(rng.uniform(0.5, 1.5), 2)]), dropout=rng.choice([0.0, 0.0, 0.1]),
               pad=rng.choice([0, 0, 5, 8]))
    # rows may stay where they are if they are aligned and none of them is changed
    case["keep"] = (d % 8 == 0 and case["pad"] % 8 == 0 and not case["dropout"] and case["masked"] == 0.0
                    and (case["parts"] == 1 or _each(case) % 64 == 0))
    return case


def _live(case):
    """Rows that count: all but the first ones (a prompt) of every run of 64."""
    r = np.arange(case["rows"])
    keep = (r % 64) >= int(round(64 * case["masked"]))
    keep[-1] = True  # a batch without any counted token is not trained on
    return keep


def _each(case):
    return -(-case["rows"] // case["parts"])


def _parts(case):
    return -(-case["rows"] // _each(case))


def work(case):
    if case["op"] == "dropout":
        n = case["rows"] * case["columns"]
        passes = 2 + (1 if case["residual"] else 0) + (2 if case["backward"] else 0)
        return {"bytes": n * passes * (4 if case["dtype"] == "f32" else 2), "flops": n * (2 if case["backward"] else 1)}
    rows, d, classes, grads = case["rows"], case["d"], case["classes"], case["grads"]
    live = int(_live(case).sum())
    size = live * d * 2 + classes * d * 2 + rows * (4 + 4 + 4 + (4 if case["weighted"] else 0)) + 4 * _parts(case)
    if grads != "none":
        size += _parts(case) * classes * d * 2
    if grads == "both":
        size += rows * d * 2
    return {"bytes": size, "flops": 2 * live * d * classes * (1 + GRADS.index(grads))}


# ---- inputs


def _rows_of(g, rows, columns, dtype, pad):
    """Rows of a buffer with `pad` unused columns behind each."""
    full = torch.empty((rows, columns + pad), dtype=dtype, device="cuda")
    full.normal_(0.0, 1.0, generator=g)
    return full[:, :columns]


def _like(x):
    return torch.zeros((x.shape[0], x.stride(0)), dtype=x.dtype, device="cuda")[:, : x.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case, "seed": seed * 2654435761 % (1 << 62), "step": seed % 1000, "first_row": seed % 100 * 1000}
    if case["op"] == "dropout":
        dtype = DTYPES[case["dtype"]]
        s["x"] = _rows_of(g, case["rows"], case["columns"], dtype, case["pad"])
        s["residual"] = _rows_of(g, case["rows"], case["columns"], dtype, case["pad"]) if case["residual"] else None
        s["out"] = {"y": _like(s["x"])}
        if case["backward"]:
            s["dy"] = _rows_of(g, case["rows"], case["columns"], dtype, case["pad"])
            s["out"]["dx"] = _like(s["x"])
        return s
    rows, d, classes, bf16 = case["rows"], case["d"], case["classes"], torch.bfloat16
    shape = (classes, d) if case["layout"] == "classes" else (d, classes)
    weight = torch.empty(shape, dtype=bf16, device="cuda").normal_(0.0, 1.5 / math.sqrt(d), generator=g)
    s["weight"] = weight if case["layout"] == "classes" else weight.t()
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    s["x"] = _rows_of(g, rows, d, bf16, case["pad"])
    # features lean towards the weights of the token that followed, some rows far more than others
    lean = torch.rand((rows, 1), generator=g, device="cuda") * 4.0
    step = max(1, (1 << 26) // d)
    for a in range(0, rows, step):
        s["x"][a:a + step] += (lean[a:a + step] * s["weight"][labels[a:a + step].long()].float()).to(bf16)
    s["labels"] = torch.where(torch.from_numpy(_live(case)).to("cuda"), labels, -1)
    live = int(_live(case).sum())
    s["row_weight"] = (torch.rand(rows, generator=g, device="cuda") + 0.5) / live if case["weighted"] else None
    f32 = {"dtype": torch.float32, "device": "cuda"}
    s["out"] = {"logp": torch.zeros(rows, **f32), "row_loss": torch.zeros(rows, **f32), "loss": torch.zeros(_parts(case), **f32)}
    if case["grads"] != "none":
        dw = torch.zeros((_parts(case), *shape), dtype=bf16, device="cuda")
        s["out"]["dweight"] = dw if case["layout"] == "classes" else dw.transpose(1, 2)
    if case["grads"] == "both":
        s["out"]["dx"] = _like(s["x"])
    return s


# ---- plain forms


def _keep(s, rows, columns, p):
    """Which elements a dropout keeps: Philox4x32-10 under the counter (column / 8, row, step), 16 bits for each element."""
    mask = 0xFFFFFFFF
    row = (s["first_row"] + torch.arange(rows, device="cuda", dtype=torch.int64)).unsqueeze(1)
    block = torch.arange(-(-columns // 8), device="cuda", dtype=torch.int64).unsqueeze(0)
    a, b = block.expand(rows, -1), (row & mask).expand(-1, block.shape[1])
    c, e = (row >> 32 & mask).expand_as(b), torch.full_like(block, s["step"]).expand(rows, -1)
    k, m = s["seed"] & mask, s["seed"] >> 32 & mask

    def one(a, b, c, e, k, m):
        # products of 32-bit numbers wrap in the sign bit only: their halves are right
        u, v = a * 0xD2511F53, c * 0xCD9E8D57
        return (v >> 32 & mask) ^ b ^ k, v & mask, (u >> 32 & mask) ^ e ^ m, u & mask

    a, b, c, e = one(a, b, c, e, k, m)
    a, b, c, e = one(a, b, c, e, k + 0x9E3779B9 & mask, m + 0xBB67AE85 & mask)
    a, b, c, e = one(a, b, c, e, k + 2 * 0x9E3779B9 & mask, m + 2 * 0xBB67AE85 & mask)
    a, b, c, e = one(a, b, c, e, k + 3 * 0x9E3779B9 & mask, m + 3 * 0xBB67AE85 & mask)
    a, b, c, e = one(a, b, c, e, k + 4 * 0x9E3779B9 & mask, m + 4 * 0xBB67AE85 & mask)
    a, b, c, e = one(a, b, c, e, k + 5 * 0x9E3779B9 & mask, m + 5 * 0xBB67AE85 & mask)
    a, b, c, e = one(a, b, c, e, k + 6 * 0x9E3779B9 & mask, m + 6 * 0xBB67AE85 & mask)
    a, b, c, e = one(a, b, c, e, k + 7 * 0x9E3779B9 & mask, m + 7 * 0xBB67AE85 & mask)
    a, b, c, e = one(a, b, c, e, k + 8 * 0x9E3779B9 & mask, m + 8 * 0xBB67AE85 & mask)
    a, b, c, e = one(a, b, c, e, k + 9 * 0x9E3779B9 & mask, m + 9 * 0xBB67AE85 & mask)
    bits = torch.stack([a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16, c & 0xFFFF, c >> 16, e & 0xFFFF, e >> 16], 2)
    return bits.view(rows, -1)[:, :columns] >= _threshold(p)


def _threshold(p):
    """An element is dropped where its 16 bits are below this."""
    return int(math.floor(p * 65536.0 + 0.5))


def _stretch(p):
    t = _threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def _plain_dropout(s):
    case, out = s["case"], s["out"]
    keep = _keep(s, case["rows"], case["columns"], case["p"])
    y = torch.where(keep, s["x"].float() * _stretch(case["p"]), 0.0)
    out["y"].copy_(y if s["residual"] is None else y + s["residual"].float())
    if case["backward"]:
        out["dx"].copy_(torch.where(keep, s["dy"].float() * _stretch(case["p"]), 0.0))
    return out


def _plain_ce(s):
    case, out, labels = s["case"], s["out"], s["labels"]
    rows, d, classes = case["rows"], case["d"], case["classes"]
    live = (labels >= 0) & (labels < classes)
    at = torch.where(live, labels, 0).long().unsqueeze(1)
    x, w = torch.where(live.unsqueeze(1), s["x"], 0.0).float(), s["weight"].float()
    if case["dropout"]:
        keep = _keep(s, rows, d, case["dropout"])
        x = torch.where(keep, x * _stretch(case["dropout"]), 0.0)
    z = (x @ w.t()).mul_(case["scale"])
    label_z = z.gather(1, at)
    top = z.amax(1, keepdim=True)
    e = z.sub_(top).exp_()
    total = e.sum(1, keepdim=True)
    logp = torch.where(live, ((label_z - top).double() - total.double().log()).squeeze(1), 0.0)
    weight = live.double() if s["row_weight"] is None else torch.where(live, s["row_weight"].double(), 0.0)
    row_loss = -weight * logp
    out["logp"].copy_(logp)
    out["row_loss"].copy_(row_loss)
    each, parts = _each(case), _parts(case)
    filled = torch.zeros(parts * each, dtype=torch.float64, device="cuda")
    filled[:rows] = row_loss
    out["loss"].copy_(filled.view(parts, each).sum(1))
    if case["grads"] == "none":
        return out
    factor = (case["scale"] * weight).float().unsqueeze(1)
    g = torch.zeros((parts * each, classes), dtype=torch.float32, device="cuda")
    torch.mul(e, factor / total, out=g[:rows])
    del z, e
    g[:rows].scatter_add_(1, at, -factor)
    if case["grads"] == "both":
        dx = g[:rows] @ w
        if case["dropout"]:
            dx = torch.where(keep, dx * _stretch(case["dropout"]), 0.0)
        out["dx"].copy_(dx)
    filled = torch.zeros((parts * each, d), dtype=torch.float32, device="cuda")
    filled[:rows] = x
    out["dweight"].copy_(torch.bmm(g.view(parts, each, classes).transpose(1, 2), filled.view(parts, each, d)))
    return out


def _own(s):
    import paper_2212_08580_b200 as ngc

    case, out, stream = s["case"], s["out"], torch.cuda.current_stream().cuda_stream
    position = {"seed": s["seed"], "step": s["step"], "first_row": s["first_row"], "stream": stream}
    if case["op"] == "dropout":
        ngc.dropout(s["x"], out["y"], case["p"], residual=s["residual"], **position)
        if case["backward"]:
            ngc.dropout(s["dy"], out["dx"], case["p"], **position)
        return out
    grads = {"dx": out.get("dx"), "dweight": out.get("dweight"), "rows_per_partition": _each(case), "keep_rows": case["keep"]}
    if "workspace" not in s:  # a program makes it once
        s["workspace"] = torch.empty(ngc.linear_cross_entropy_workspace_bytes(s["x"], s["weight"], **grads), dtype=torch.uint8,
                                     device="cuda")
    ngc.linear_cross_entropy(s["x"], s["weight"], s["labels"], out["logp"], out["row_loss"], out["loss"], s["workspace"],
                             row_weight=s["row_weight"], scale=case["scale"], dropout=case["dropout"], **grads, **position)
    return out


def run(s):
    if own:
        return _own(s)
    if s["case"]["op"] == "dropout":
        return _plain_dropout(s)
    return _plain_ce(s)


# ---- the same outputs from the definitions, in 64 bits


def _exact_kept(s, rows, columns, p):
    """The same choice, counter by counter on the host."""
    u32, u64 = np.uint32, np.uint64
    row = np.uint64(s["first_row"]) + np.arange(rows, dtype=u64)[:, None]
    n = -(-columns // 8)
    ctr = np.empty((4, rows, n), dtype=u32)
    ctr[0] = np.arange(n, dtype=u32)[None, :]
    ctr[1] = (row & u64(0xFFFFFFFF)).astype(u32)
    ctr[2] = (row >> u64(32)).astype(u32)
    ctr[3] = u32(s["step"])
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32 % 2 ** 32]
    for _ in range(10):
        p0 = ctr[0].astype(u64) * u64(0xD2511F53)
        p1 = ctr[2].astype(u64) * u64(0xCD9E8D57)
        ctr = np.stack([(p1 >> u64(32)).astype(u32) ^ ctr[1] ^ u32(key[0]), p1.astype(u32),
                        (p0 >> u64(32)).astype(u32) ^ ctr[3] ^ u32(key[1]), p0.astype(u32)])
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    halves = np.ascontiguousarray(ctr.transpose(1, 2, 0)).view(np.uint16).reshape(rows, n * 8)[:, :columns]
    return torch.from_numpy(halves.astype(np.int32) >= round(p * 65536)).to("cuda")


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        keep = _exact_kept(s, case["rows"], case["columns"], case["p"])
        share = 1.0 - round(case["p"] * 65536) / 65536
        y = keep * (s["x"].double() / share)
        out = {"y": y + s["residual"].double() if case["residual"] else y}
        if case["backward"]:
            out["dx"] = keep * (s["dy"].double() / share)
        return out
    rows, d, classes, scale = case["rows"], case["d"], case["classes"], case["scale"]
    f64 = {"dtype": torch.float64, "device": "cuda"}
    w = s["weight"].double()
    out = {"logp": torch.zeros(rows, **f64), "row_loss": torch.zeros(rows, **f64), "loss": torch.zeros(_parts(case), **f64)}
    if case["grads"] != "none":
        out["dweight"] = torch.zeros((_parts(case), classes, d), **f64)
    if case["grads"] == "both":
        out["dx"] = torch.zeros((rows, d), **f64)
    kept = _exact_kept(s, rows, d, case["dropout"]) if case["dropout"] else None
    share = 1.0 - round(case["dropout"] * 65536) / 65536
    each, labels = _each(case), s["labels"].long()
    step = max(1, min(each, (1 << 28) // classes))
    for part in range(_parts(case)):
        end = min(rows, (part + 1) * each)
        for a in range(part * each, end, step):
            r = torch.arange(a, min(end, a + step), device="cuda")
            r = r[labels[r] >= 0]
            x = s["x"][r].double()
            if kept is not None:
                x = x * kept[r] / share
            z = torch.log_softmax(scale * (x @ w.t()), 1)
            y = labels[r]
            weight = torch.ones(r.numel(), **f64) if s["row_weight"] is None else s["row_weight"][r].double()
            n = torch.arange(r.numel(), device="cuda")
            out["logp"][r] = z[n, y]
            out["row_loss"][r] = -weight * z[n, y]
            out["loss"][part] += out["row_loss"][r].sum()
            if case["grads"] == "none":
                continue
            p = z.exp_()
            p[n, y] -= 1.0
            p *= (scale * weight).unsqueeze(1)
            out["dweight"][part] += p.t() @ x
            if case["grads"] == "both":
                dx = p @ w
                out["dx"][r] = dx if kept is None else dx * kept[r] / share
    return out
