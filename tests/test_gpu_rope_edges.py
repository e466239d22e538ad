"""kvp_rope_apply: the rounding of the angle, and calls that autograd would have to know of."""
import math

import numpy as np
import pytest

from gpu_helpers import note
from oracle import rotary
from paper_2608_11152_amd import kvpattn as kp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [128, 24])  # whole units of a head, and pairs
def test_angles_are_rounded_to_nearest(rot, interleaved):
    """The angle is held to 2^-32 of a turn, rounded: 2^-33 off at most (7.3e-10 radian), and not one-sided.  Seen where
    the sine itself is that small: slow pairs at near positions, x = (0, 1) gives -sin.  The table's half step times 4096
    positions is 2^-53 of a turn; the sine's own steps are relative."""
    import torch
    note(f"rope small angles {rot} {interleaved}")
    T, base = 4096, 1e12
    x = torch.zeros(T, 1, rot, device="cuda")
    i = np.arange(rot // 2)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    x[:, :, second] = 1.0
    pos = np.arange(T, dtype=np.int32)
    rope = kp.Rope(rot, base=base, interleaved=interleaved)
    y = kp.kvp_rope_apply(rope, x, torch.from_numpy(pos).cuda()).cpu().numpy().astype(np.float64)[:, 0]
    angle = pos[:, None] * rotary.frequencies(rot, base)[None, :]
    slow = angle < 2e-6  # there the sine's own rounding, 2^-23 of it, is under 2^-42
    err = np.where(slow, -y[:, first] - np.sin(angle), 0.0)
    assert slow.sum() > 10000
    assert np.abs(err).max() <= 2 * math.pi * 2.0 ** -33 + 2.0 ** -42
    # one-sided errors would average a quarter of a step of 2^-32 turn or more; at random 10000 of them a 200th
    assert abs(err[slow].mean()) <= 2 * math.pi * 2.0 ** -32 / 16


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_autograd_records_the_call(dt, interleaved):
    """The gradient of a weighted sum is the weights turned back, in either direction, also into strided and broadcast
    leaves; and the gradient's own gradient is the weights' turn."""
    import torch
    note(f"rope autograd {dt} {interleaved}")
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    g = torch.Generator().manual_seed(4)
    T, H, d = 9, 4, 64
    rope = kp.Rope(32, interleaved=interleaved, magnitude=1.25)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 1000
    row = torch.randn(T, H + 2, d, generator=g).to(dtype).cuda().requires_grad_()
    w = torch.randn(T, H, d, generator=g).to(dtype).cuda().requires_grad_()
    for grad in (False, True):
        y = kp.kvp_rope_apply(rope, row[:, 1:H + 1], pos, grad=grad)
        with torch.no_grad():
            assert torch.equal(y, kp.kvp_rope_apply(rope, row[:, 1:H + 1], pos, grad=grad))
            want = kp.kvp_rope_apply(rope, w, pos, grad=not grad)
        got, = torch.autograd.grad(y, row, w, create_graph=True)
        assert torch.equal(got[:, 1:H + 1], want) and not bool(got[:, [0, H + 1]].any())
        u = torch.randn(T, H + 2, d, generator=g).to(dtype).cuda()
        back, = torch.autograd.grad(got, w, u)
        with torch.no_grad():
            assert torch.equal(back, kp.kvp_rope_apply(rope, u[:, 1:H + 1], pos, grad=grad))
    one = torch.randn(T, 1, d, generator=g).to(dtype).cuda().requires_grad_()
    y = kp.kvp_rope_apply(rope, one.expand(T, H, d), pos)
    got, = torch.autograd.grad(y.sum(), one)  # the gradient comes broadcast over the head's elements
    with torch.no_grad():
        turned = kp.kvp_rope_apply(rope, torch.ones(T, 1, d, dtype=dtype, device="cuda"), pos, grad=True)
    assert torch.equal(got, H * turned)  # H is a power of two


def test_outputs_in_place_and_autograd():
    import torch
    note("rope in place and autograd")
    rope = kp.Rope(64)
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    x = torch.randn(3, 2, 64, device="cuda", requires_grad=True)
    keep = x.detach().clone()
    for bad in (dict(x=x, out=torch.empty_like(keep)), dict(x=keep, out=x), dict(x=x * 1.0, out=keep)):
        with pytest.raises(ValueError, match="autograd"):
            kp.kvp_rope_apply(rope, bad["x"], pos, out=bad["out"])
    assert torch.equal(x, keep)
    y = x * 1.0
    z = y * y  # saves y
    with torch.no_grad():
        kp.kvp_rope_apply(rope, y, pos, out=y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.sum().backward()
    with torch.inference_mode():
        a = keep * 1.0
        assert torch.equal(kp.kvp_rope_apply(rope, a, pos, out=a), kp.kvp_rope_apply(rope, keep, pos))
