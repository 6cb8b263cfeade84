"""Dropout whose mask is a function of seed, step and position: values, masks against the published generator, strides and
alignments, in place, shards of rows, graphs, the gradient, refusals.

Tolerance: the kernel stretches in fp32 (one rounding of the factor, one of the product), adds the residual (one more) and rounds once to the type: 3 2^-24
of the terms and half a step of the result."""
import numpy as np
import pytest
import torch

import paper_2212_08580_b200 as ngc
from tests._philox import kept, philox4x32, threshold

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def test_generator_gives_the_published_numbers():
    """The known answers that accompany the generator's publication."""
    got = [int(w) for w in philox4x32([0, 0, 0, 0], (0, 0))]
    assert got == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert [int(w) for w in philox4x32([ones] * 4, (ones, ones))] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    pi = [0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344]
    assert [int(w) for w in philox4x32(pi, (0xA4093822, 0x299F31D0))] == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def rows_of(g, rows, columns, dtype, pad=0, shift=0):
    """A matrix whose rows lie `pad` elements apart and whose first element is `shift` elements into its memory."""
    flat = torch.empty(rows * (columns + pad) + shift, dtype=dtype, device="cuda").normal_(generator=g)
    return flat[shift:].view(rows, columns + pad)[:, :columns]


def check(x, out, p, residual=None, **position):
    keep = torch.from_numpy(kept(*x.shape, p, **position)).cuda()
    share = 1.0 - threshold(p) / 65536
    want = torch.where(keep, x.double() / share, 0.0) if share else torch.zeros_like(x, dtype=torch.float64)
    size = want.abs()
    if residual is not None:
        want, size = want + residual.double(), size + residual.double().abs()
    off = (out.double() - want).abs()
    assert (off <= HALF[x.dtype] * want.abs() + 3 * 2.0 ** -24 * size).all(), float(off.max())
    if residual is None:
        assert ((out == 0) == (~keep | (x == 0))).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,columns,pad,shift", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 0, 0), (5, 9, 3, 1), (64, 1024, 0, 0),
                                                    (33, 1000, 8, 0), (17, 1021, 0, 0), (300, 77, 6, 3), (2, 70001, 1, 2)])
@pytest.mark.parametrize("residual", [False, True])
def test_values(dtype, rows, columns, pad, shift, residual):
    g = torch.Generator(device="cuda").manual_seed(rows * columns + pad)
    x = rows_of(g, rows, columns, dtype, pad, shift)
    res = rows_of(g, rows, columns, dtype, pad + 1, shift) if residual else None
    full = torch.full((rows, columns + 5), 7.0, dtype=dtype, device="cuda")
    position = {"seed": 0x1234567890ABCDEF, "step": 4000000000, "first_row": (1 << 32) - 2}
    ngc.dropout(x, full[:, :columns], 0.3, residual=res, **position)
    check(x, full[:, :columns], 0.3, res, **position)
    assert (full[:, columns:] == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 2.0 ** -16, 0.5, 0.999, 1.0 - 2.0 ** -16, 1.0])
def test_probabilities(p):
    g = torch.Generator(device="cuda").manual_seed(5)
    x = rows_of(g, 200, 320, F32)
    out = torch.empty_like(x)
    ngc.dropout(x, out, p, seed=9)
    check(x, out, p, seed=9)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_in_the_residuals_place(dtype):
    g = torch.Generator(device="cuda").manual_seed(6)
    x, res = rows_of(g, 50, 123, dtype, 5), rows_of(g, 50, 123, dtype, 5)
    was, old = x.clone(), res.clone()
    ngc.dropout(x, res, 0.25, seed=3, residual=res)
    check(was, res, 0.25, old, seed=3)
    ngc.dropout(x, x, 0.25, seed=3)
    check(was, x, 0.25, seed=3)


@pytest.mark.gpu
def test_a_shard_of_rows_drops_what_the_whole_does():
    """Workers that hold the same rows agree, whatever the type and the launch."""
    x = torch.ones((1000, 40), device="cuda")
    whole, part = torch.empty_like(x), torch.empty((100, 40), dtype=BF16, device="cuda")
    ngc.dropout(x, whole, 0.4, seed=77, step=3)
    ngc.dropout(x[:100].to(BF16), part, 0.4, seed=77, step=3, first_row=600)
    assert ((whole[600:700] != 0) == (part != 0)).all()
    ngc.dropout(x[:100].to(BF16), part, 0.4, seed=77, step=4, first_row=600)
    assert ((whole[600:700] != 0) != (part != 0)).any()


@pytest.mark.gpu
def test_dropped_places_may_hold_anything():
    x = torch.full((64, 256), float("nan"), device="cuda")
    keep = torch.from_numpy(kept(64, 256, 0.5, 11)).cuda()
    x[keep] = 2.0
    x[0][~keep[0]] = float("inf")
    out = torch.empty_like(x)
    ngc.dropout(x, out, 0.5, seed=11)
    assert (out[keep] == 4.0).all() and (out[~keep] == 0.0).all()


@pytest.mark.gpu
def test_gradient_is_the_same_call():
    """y is linear in x, so differences of any size are exact up to rounding."""
    g = torch.Generator(device="cuda").manual_seed(8)
    x, dx, dy = (rows_of(g, 30, 41, F32) for _ in range(3))
    a, b, back = (torch.empty_like(x) for _ in range(3))
    ngc.dropout(x, a, 0.2, seed=5, step=2)
    ngc.dropout(x + dx, b, 0.2, seed=5, step=2)
    ngc.dropout(dy, back, 0.2, seed=5, step=2)
    lhs, rhs = ((b.double() - a.double()) * dy.double()).sum(), (back.double() * dx.double()).sum()
    size = (a.double().abs() + b.double().abs()).mul(dy.double().abs()).sum() + (back.double() * dx.double()).abs().sum()
    assert abs(float(lhs - rhs)) <= 4 * 2.0 ** -24 * float(size)


@pytest.mark.gpu
def test_share_of_dropped_elements():
    """Bernoulli: 1e6 draws are within six standard deviations of p; so are neighbours' joint draws."""
    x = torch.ones((1000, 1000), device="cuda")
    out = torch.empty_like(x)
    ngc.dropout(x, out, 0.1, seed=123)
    dropped = (out == 0).double()
    assert abs(float(dropped.mean()) - 6554 / 65536) < 6 * np.sqrt(0.09 / 1e6)
    for both in (dropped[1:] * dropped[:-1], dropped[:, 1:] * dropped[:, :-1], dropped[:, 8:] * dropped[:, :-8]):
        assert abs(float(both.mean()) - 0.01) < 6 * np.sqrt(0.01 / both.numel())


@pytest.mark.gpu
def test_graph_and_stream():
    g = torch.Generator(device="cuda").manual_seed(9)
    x = rows_of(g, 128, 512, BF16)
    out, s = torch.empty_like(x), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ngc.dropout(x, out, 0.1, seed=1, stream=s.cuda_stream)
    x.normal_(generator=g)
    graph.replay()
    torch.cuda.synchronize()
    check(x, out, 0.1, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(30))
def test_drawn_shapes_and_alignments(seed):
    """Rows of any width and place, in memory of their own or in another's; what lies around the output stays."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = [F32, BF16][rng.integers(2)]
    rows, columns = (int(np.exp(rng.uniform(0.0, np.log(n)))) for n in (500, 3000))
    same = rng.random() < 0.6  # all at one place within 16 bytes
    pads, shifts = ([int(rng.integers(0, 17))] * 3, [int(rng.integers(0, 17))] * 3) if same else (rng.integers(0, 17, 3), rng.integers(0, 17, 3))
    x, res = rows_of(g, rows, columns, dtype, int(pads[0]), int(shifts[0])), rows_of(g, rows, columns, dtype, int(pads[1]), int(shifts[1]))
    full = torch.full((rows * (columns + int(pads[2])) + int(shifts[2]) + 40,), 7.0, dtype=dtype, device="cuda")
    out = full[int(shifts[2]):int(shifts[2]) + rows * (columns + int(pads[2]))].view(rows, columns + int(pads[2]))[:, :columns]
    residual = res if rng.random() < 0.5 else None
    p = float(rng.choice([0.0, 0.1, 0.5, 0.9]))
    position = {"seed": int(rng.integers(1 << 62)), "step": int(rng.integers(1 << 32)), "first_row": int(rng.integers(1 << 40))}
    ngc.dropout(x, out, p, residual=residual, **position)
    check(x, out.contiguous(), p, residual, **position)
    out.fill_(7.0)
    assert (full == 7.0).all()
    was = x.clone()
    ngc.dropout(x, x, p, residual=residual, **position)
    check(was, x, p, residual, **position)


@pytest.mark.gpu
def test_more_than_2_31_elements():
    x = torch.ones((3, 800_000_000), dtype=BF16, device="cuda")
    ngc.dropout(x, x, 0.5, seed=4)
    tail = torch.from_numpy(kept(3, 64, 0.5, 4)).cuda()
    assert ((x[:, :64] != 0) == tail).all()
    torch.cuda.synchronize()
    # the last block of the last row, by its own counter
    block = 800_000_000 // 8 - 1
    words = philox4x32([block, 2, 0, 0], (4, 0))
    bits = [h for w in words for h in (int(w) & 0xFFFF, int(w) >> 16)]
    assert (x[2, -8:] != 0).tolist() == [b >= 32768 for b in bits]


@pytest.mark.gpu
@pytest.mark.parametrize("columns", [2 ** 31 - 1, 2 ** 31 - 257])
@pytest.mark.parametrize("shift", [0, 1])
def test_rows_of_nearly_2_31_columns(columns, shift):
    flat = torch.ones(columns + 40, dtype=BF16, device="cuda")
    x = flat[shift:shift + columns].view(1, columns)
    ngc.dropout(x, x, 0.5, seed=4)
    assert (flat[:shift] == 1).all() and (flat[shift + columns:] == 1).all()
    assert ((x[0, :512] != 0) == torch.from_numpy(kept(1, 512, 0.5, 4)[0]).cuda()).all()
    blocks = np.arange(columns // 8 - 63, columns // 8 + 1, dtype=np.uint64)  # the last, of 7 columns, has its own counter too
    words = philox4x32([blocks, 0 * blocks, 0 * blocks, 0 * blocks], (4, 0))
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).reshape(-1)
    tail = bits[:columns - int(blocks[0]) * 8] >= np.uint64(32768)
    assert ((x[0, int(blocks[0]) * 8:] != 0) == torch.from_numpy(tail).cuda()).all()


@pytest.mark.gpu
def test_refusals():
    x, out = torch.zeros((4, 16), device="cuda"), torch.zeros((4, 16), device="cuda")
    flat = torch.zeros(200, device="cuda")
    bad = [
        lambda: ngc.dropout(x, out, -0.1, seed=1),
        lambda: ngc.dropout(x, out, 1.5, seed=1),
        lambda: ngc.dropout(x, out, float("nan"), seed=1),
        lambda: ngc.dropout(x, out.to(BF16), 0.1, seed=1),
        lambda: ngc.dropout(x, out[:3], 0.1, seed=1),
        lambda: ngc.dropout(x.t(), out.t(), 0.1, seed=1),
        lambda: ngc.dropout(x.double(), out.double(), 0.1, seed=1),
        lambda: ngc.dropout(x.cpu(), out, 0.1, seed=1),
        lambda: ngc.dropout(x, out, 0.1, seed=-1),
        lambda: ngc.dropout(x, out, 0.1, seed=1 << 64),
        lambda: ngc.dropout(x, out, 0.1, seed=1, step=1 << 32),
        lambda: ngc.dropout(x, out, 0.1, seed=1, first_row=-1),
        lambda: ngc.dropout(flat[:64].view(4, 16), flat[1:65].view(4, 16), 0.1, seed=1),
        lambda: ngc.dropout(x, flat[:64].view(4, 16), 0.1, seed=1, residual=flat[8:72].view(4, 16)),
        lambda: ngc.dropout(x, "out", 0.1, seed=1),
        lambda: ngc.dropout(torch.zeros((1, 16), device="cuda").expand(4, 16), out, 0.1, seed=1),
    ]
    for call in bad:
        with pytest.raises(ngc.NgcError):
            call()
    ngc.dropout(x[:0], out[:0], 0.1, seed=1)
