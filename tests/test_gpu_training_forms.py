"""Forms of the training operators that programs use: the softmax model's classes, views of flat buffers."""
import pytest
import torch

from tests.test_gpu_adamw import Problem
from tests.test_gpu_losses import preference

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("classes", [16, 48, 64, 128, 240, 256])
def test_preference_as_the_softmax_model_runs_it(classes):
    """bf16 logits of 16 to 256 classes, many rows, in place: short sequences side by side, some labels left out."""
    lengths = [1, 3, 0, 5, 2, 2, 7, 4, 64, 33] * 120
    p = preference(lengths, classes, "bf16", beta=0.5, smooth=0.0)
    p.run()
    p.check()
    want = p.grad.clone()
    p.run(grad=p.logits)
    torch.cuda.synchronize()
    assert torch.equal(p.logits, want)


@gpu
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_adamw_of_many_odd_tensors_in_one_buffer(state):
    """Views of flat buffers one behind the other, at any element, as a program cuts them: no two aligned alike."""
    sizes = [(i * 7919) % 5003 + 1 for i in range(300)]
    total = sum(sizes)
    p, q = Problem(sizes, state, seed=31), Problem(sizes, state, seed=31)
    for name in ("theta", "grad", "m", "v"):
        parts = getattr(q, name)
        flat = torch.cat([x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x for x in parts])
        assert flat.numel() == total
        setattr(q, name, [x.view(parts[0].dtype) for x in flat.split(sizes)])
    want = p.expected(7)
    p.optimizer().update(step=7)
    q.optimizer().update(step=7)
    torch.cuda.synchronize()
    p.check(want)
    for name in ("theta", "m", "v"):
        for x, y in zip(getattr(p, name), getattr(q, name)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), name
