"""kvp_rope_apply against the 64-bit oracle: layouts, parts of a head, scaled frequencies, far and negative positions,
strides, in place, the gradient, capture.

Tolerance, per element: half a step of the element type relative to the result, plus fp32 arithmetic relative to the
pair's |a| + |b|.  cos and sin: the angle within a quarter turn is a product of three roundings, at most pi / 4 (1.5 steps
of 2^-24 = 1.2), the series' last two steps round (1), the magnitude once (0.5), the integer angle's truncation 2^-32 of a
turn; the products and their sum add 1.5: 5 steps of 2^-24 in all, 8 are allowed."""
import numpy as np
import pytest

from gpu_helpers import note
from oracle import rotary
from paper_2608_11152_amd import kvpattn as kp

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def half_step(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def make(T, H, d, dtype, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randn(T, H, d, generator=g).to(dtype).cuda()


def check(got, x, pos, rot, interleaved, freq, magnitude=1.0, grad=False):
    want = rotary.rotate(f64(x), pos, freq, interleaved, magnitude, grad)
    a = np.abs(f64(x))
    pair = a.copy()
    if interleaved:
        s = a[..., 0:rot:2] + a[..., 1:rot:2]
        pair[..., 0:rot:2], pair[..., 1:rot:2] = s, s
    else:
        s = a[..., :rot // 2] + a[..., rot // 2:rot]
        pair[..., :rot // 2], pair[..., rot // 2:rot] = s, s
    tol = half_step(got.dtype) * np.abs(want) + 8 * 2.0 ** -24 * magnitude * pair
    tol[..., rot:] = 0.0  # copied
    err = np.abs(f64(got) - want)
    assert np.all(err <= tol), (float((err - tol).max()), np.unravel_index(np.argmax(err - tol), err.shape))


SHAPES = [(1, 1, 64, 64), (4, 8, 64, 64), (17, 36, 128, 128), (1000, 3, 128, 64), (33, 5, 128, 32), (7, 2, 80, 20),
          (5, 3, 256, 256), (3, 1, 2, 2), (6, 2, 17, 10), (9, 4, 96, 48), (2, 70, 64, 16), (65, 1, 72, 72)]


@pytest.mark.parametrize("T,H,d,rot", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_against_oracle(T, H, d, rot, interleaved, dt):
    import torch
    note(f"rope {T} {H} {d} {rot} {interleaved} {dt}")
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    x = make(T, H, d, dtype)
    pos = np.random.default_rng(T).integers(0, 131072, T).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    rope = kp.Rope(rot, interleaved=interleaved)
    before = x.clone()
    freq = rotary.frequencies(rot)
    check(kp.kvp_rope_apply(rope, x, p), x, pos, rot, interleaved, freq)
    check(kp.kvp_rope_apply(rope, x, p, grad=True), x, pos, rot, interleaved, freq, grad=True)
    assert torch.equal(x, before)


@pytest.mark.parametrize("kw", [
    dict(factor=8.0), dict(base=500000.0, factor=16.0, original_len=8192, low_turns=1.0, high_turns=4.0),
    dict(factor=40.0, original_len=4096, low_turns=1.0, high_turns=32.0)])
@pytest.mark.parametrize("magnitude", [1.0, 1.3688879454113936])
def test_scaled_frequencies(kw, magnitude):
    import torch
    note(f"rope scaled {kw} {magnitude}")
    x = make(64, 4, 128, torch.float32)
    pos = (np.arange(64) * 16381).astype(np.int32)
    rope = kp.Rope(128, magnitude=magnitude, **kw)
    freq = rotary.frequencies(128, **kw)
    check(kp.kvp_rope_apply(rope, x, torch.from_numpy(pos).cuda()), x, pos, 128, False, freq, magnitude)


@pytest.mark.parametrize("d", [64, 10])
def test_positions_at_the_ends_of_their_type(d):
    import torch
    note("rope far positions")
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, -123456789, 16777217], np.int32)
    x = make(len(pos), 3, d, torch.float32)
    freq = rotary.frequencies(d)
    # the oracle's own angle at 2^31: f is off by a step of 2^-53 relative, the product by half of one: under 2^-21 radian
    want = rotary.rotate(f64(x), pos, freq)
    got = f64(kp.kvp_rope_apply(kp.Rope(d), x, torch.from_numpy(pos).cuda()))
    a = np.abs(f64(x))
    pair = np.concatenate([a[..., :d // 2] + a[..., d // 2:]] * 2, axis=-1)
    assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + (8 * 2.0 ** -24 + 2.0 ** -21) * pair)
    assert np.array_equal(got[0], f64(x)[0])  # position 0 turns nothing


@pytest.mark.parametrize("d,rot", [(128, 128), (64, 32), (20, 10)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_strides_and_in_place(d, rot, dt):
    """Heads of a fused projection's rows, heads-first memory, rows that start off 16-byte lines, and each in place: the
    dense call's bits, and nothing written between the heads."""
    import torch
    note(f"rope strides {d} {rot} {dt}")
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    T, H = 37, 6
    x = make(T, H, d, dtype)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 3
    rope = kp.Rope(rot)
    want = kp.kvp_rope_apply(rope, x, pos)
    fused = torch.full((T, H + 3, d), 7.0, dtype=dtype, device="cuda")
    first = torch.full((H, T, d), 7.0, dtype=dtype, device="cuda").transpose(0, 1)
    odd = torch.full((T * (H * d + 3) + 1,), 7.0, dtype=dtype, device="cuda")[1:].view(T, H * d + 3)[:, :H * d].unflatten(1, (H, d))
    for name, view in (("fused", fused[:, 1:H + 1]), ("heads first", first), ("odd", odd)):
        view.copy_(x)
        assert torch.equal(kp.kvp_rope_apply(rope, view, pos), want), name
        out = torch.full_like(fused, 9.0)[:, 2:H + 2]
        kp.kvp_rope_apply(rope, view, pos, out=out)
        assert torch.equal(out, want), name
        kp.kvp_rope_apply(rope, view, pos, out=view)
        assert torch.equal(view, want), name
    assert bool((fused[:, 0] == 7.0).all()) and bool((fused[:, H + 1:] == 7.0).all())
    y = x.clone()
    assert kp.kvp_rope_apply(rope, y, pos, out=y) is y and torch.equal(y, want)
    wide = x[:, :1].expand(T, H, d)  # one head read for all
    assert torch.equal(kp.kvp_rope_apply(rope, wide, pos), want[:, :1].expand(T, H, d))
    with pytest.raises(kp.KvpError):
        kp.kvp_rope_apply(rope, x, pos, out=x[:, :1].expand(T, H, d))


def test_gradient_is_the_adjoint_and_differences_agree():
    """<R x, g> = <x, R^T g>, and R^T g from differences of R (linear, so any step does: unit vectors here)."""
    import torch
    note("rope gradient")
    T, H, d, rot = 3, 2, 64, 32
    x, g = make(T, H, d, torch.float32), make(T, H, d, torch.float32, seed=1)
    pos = torch.tensor([5, 70000, -9], dtype=torch.int32, device="cuda")
    for interleaved in (False, True):
        rope = kp.Rope(rot, interleaved=interleaved, magnitude=1.25)
        back = f64(kp.kvp_rope_apply(rope, g, pos, grad=True))
        lhs = float((f64(kp.kvp_rope_apply(rope, x, pos)) * f64(g)).sum())
        rhs = float((f64(x) * back).sum())
        scale = float((np.abs(f64(x)) * np.abs(f64(g))).sum()) * 1.25 * 2
        assert abs(lhs - rhs) <= 18 * 2.0 ** -24 * scale  # each side 9 steps of its terms
        e = torch.zeros(d, 1, d, device="cuda")
        e[torch.arange(d), 0, torch.arange(d)] = 1.0
        for t in range(T):
            cols = f64(kp.kvp_rope_apply(rope, e, pos[t].expand(d).contiguous()))[:, 0]  # row c: R e_c
            want = np.einsum("hd,cd->hc", f64(g)[t], cols)
            room = np.einsum("hd,cd->hc", np.abs(f64(g)[t]), np.abs(cols) + 1.25 * 2.0 ** -20)
            assert np.all(np.abs(back[t] - want) <= 20 * 2.0 ** -24 * room + 2.0 ** -23 * np.abs(want))


def test_values_that_are_not_finite_stay_in_their_pair():
    import torch
    note("rope non-finite")
    x = make(5, 2, 64, torch.bfloat16)
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    rope = kp.Rope(32)
    clean = kp.kvp_rope_apply(rope, x, pos)
    x[2, 1, 3] = float("nan")
    x[3, 0, 40] = float("inf")  # a dim that is not rotated
    got = kp.kvp_rope_apply(rope, x, pos)
    assert torch.isnan(got[2, 1, [3, 19]]).all() and got[3, 0, 40] == float("inf")
    same = torch.ones_like(got, dtype=torch.bool)
    same[2, 1, [3, 19]] = False
    same[3, 0, 40] = False
    assert torch.equal(got[same], clean[same])


def test_many_heads_of_many_tokens_and_none():
    """More elements than 2^31 bytes apart: offsets are 64 bits wide."""
    import torch
    note("rope large")
    x = torch.zeros(40000, 1, 128, dtype=torch.bfloat16, device="cuda")
    base = torch.zeros(2, (1 << 31) + 64, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(base, (2, 3, 64), ((1 << 31) + 64, 128, 1))
    near = make(2, 3, 64, torch.bfloat16)
    far.copy_(near)
    pos = torch.tensor([11, 500], dtype=torch.int32, device="cuda")
    rope = kp.Rope(64)
    want = kp.kvp_rope_apply(rope, near, pos)
    assert torch.equal(kp.kvp_rope_apply(rope, far, pos, out=far), want)
    assert torch.equal(far, want)
    assert kp.kvp_rope_apply(rope, x[:0, :, :64], pos).shape == (0, 1, 64)


def test_capture_and_another_stream():
    import torch
    note("rope capture")
    x = make(33, 4, 128, torch.bfloat16)
    pos = torch.arange(33, dtype=torch.int32, device="cuda")
    rope = kp.Rope(128)
    s = torch.cuda.Stream()
    out = torch.zeros_like(x)
    s.wait_stream(torch.cuda.current_stream())
    kp.kvp_rope_apply(rope, x, pos, out=out, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(out, kp.kvp_rope_apply(rope, x, pos))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        kp.kvp_rope_apply(rope, x, pos, out=out, stream=s)
    del rope  # the graph holds its own copy
    for rep in range(4):
        x.copy_(torch.randn_like(x.float()))
        pos.copy_(torch.randint(0, 1 << 20, (33,), dtype=torch.int32))
        want = kp.kvp_rope_apply(kp.Rope(128), x, pos)
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
