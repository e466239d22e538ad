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
