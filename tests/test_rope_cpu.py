"""Rotary positions without a GPU: the frequency table of kvp_rope_init, its refusals, those of the calls that take it
(all made before anything is enqueued), and the properties that pin the oracle."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import rotary
from paper_2608_11152_amd import kvpattn as kp

FAKE = 1 << 20  # an aligned address that a refused call never reads


@pytest.mark.parametrize("kw", [
    dict(r=128), dict(r=2), dict(r=20, base=500000.0), dict(r=256, base=1.0), dict(r=64, factor=8.0),
    dict(r=128, base=500000.0, factor=16.0, original_len=8192, low_turns=1.0, high_turns=4.0),
    dict(r=64, factor=40.0, original_len=4096, low_turns=1.0, high_turns=32.0),
    dict(r=64, factor=4.0, original_len=1, low_turns=0.0, high_turns=0.5),
])
def test_frequencies(kw):
    kw = dict(kw)
    r = kw.pop("r")
    rope = kp.Rope(r, **kw)
    got = np.array([int(t) for t in rope.s.turns[:r // 2]], dtype=np.float64) / 2.0 ** 64 * 2.0 * math.pi
    want = rotary.frequencies(r, **kw)
    # the table's half step is 2^-65 of a turn; the oracle's own arithmetic some steps of 2^-53 relative
    assert np.all(np.abs(got - want) <= 2.0 ** -64 * 2 * math.pi + 2.0 ** -48 * want)
    assert all(int(t) == 0 for t in rope.s.turns[r // 2:])


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=258), dict(rotary_dim=-2), dict(base=0.5), dict(base=math.nan),
    dict(base=math.inf), dict(factor=0.5), dict(factor=math.nan), dict(original_len=-1),
    dict(original_len=10, low_turns=4.0, high_turns=4.0), dict(original_len=10, low_turns=-1.0),
    dict(original_len=10, high_turns=math.inf), dict(magnitude=0.0), dict(magnitude=-1.0), dict(magnitude=math.nan),
    dict(magnitude=1e300),
])
def test_init_refusals(kw):
    with pytest.raises(kp.KvpError) as e:
        kp.Rope(**{"rotary_dim": 64, **kw})
    assert e.value.code == kp.KVP_EINVAL


def _apply(rope, x=FAKE, xt=512, xh=64, y=2 * FAKE, yt=512, yh=64, dtype=kp.KVP_BF16, pos=FAKE, T=4, H=8, d=64):
    return kp.lib().kvp_rope_apply(rope, x, xt, xh, y, yt, yh, dtype, pos, T, H, d, 0, None)


@pytest.mark.parametrize("kw,code", [
    (dict(d=0), kp.KVP_EUNSUPPORTED), (dict(d=257), kp.KVP_EUNSUPPORTED), (dict(d=62), kp.KVP_EINVAL),
    (dict(dtype=kp.KVP_FP8_E4M3), kp.KVP_EUNSUPPORTED), (dict(T=-1), kp.KVP_EINVAL), (dict(H=-1), kp.KVP_EINVAL),
    (dict(x=None), kp.KVP_EINVAL), (dict(y=None), kp.KVP_EINVAL), (dict(pos=None), kp.KVP_EINVAL),
    (dict(x=FAKE + 1), kp.KVP_EINVAL), (dict(y=FAKE + 2, dtype=kp.KVP_F32), kp.KVP_EINVAL), (dict(yt=0), kp.KVP_EINVAL),
    (dict(yh=63), kp.KVP_EINVAL), (dict(yt=511), kp.KVP_EINVAL), (dict(xt=-512), kp.KVP_EINVAL),
    (dict(y=FAKE, yt=1024), kp.KVP_EINVAL), (dict(T=1 << 62), kp.KVP_EINVAL),
])
def test_apply_refusals(kw, code):
    rope = kp.Rope(64)
    assert _apply(rope.ref(), **kw) == code


def test_apply_refuses_an_uninitialised_rotation_and_accepts_nothing_to_do():
    assert _apply(None) == kp.KVP_EINVAL
    assert _apply(C.byref(kp.RopeStruct())) == kp.KVP_EINVAL
    rope = kp.Rope(64)
    assert _apply(rope.ref(), T=0, x=None, y=None, pos=None) == kp.KVP_OK
    assert _apply(rope.ref(), H=0) == kp.KVP_OK


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(4, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU tensor"):
        kp.kvp_rope_apply(kp.Rope(64), x, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="cu_new"):
        kp.kv_append_rope(None, 0, kp.Rope(64), x, x, None, [0, 0], [0, 1])


def test_oracle_closed_form_and_norm():
    x = np.zeros((3, 1, 4))
    x[:, 0, 0] = 1.0
    y = rotary.rotate(x, [0, 1, 2], np.array([0.5, 0.1]), interleaved=False)
    assert np.allclose(y[:, 0], [[1, 0, 0, 0], [math.cos(.5), 0, math.sin(.5), 0], [math.cos(1), 0, math.sin(1), 0]])
    y = rotary.rotate(x, [0, 1, 2], np.array([0.5, 0.1]), interleaved=True)
    assert np.allclose(y[:, 0], [[1, 0, 0, 0], [math.cos(.5), math.sin(.5), 0, 0], [math.cos(1), math.sin(1), 0, 0]])
    x = np.random.default_rng(0).normal(size=(5, 2, 16))
    for il in (False, True):
        y = rotary.rotate(x, np.arange(5) * 1000, rotary.frequencies(12), il, magnitude=1.5)
        assert np.allclose((y[..., :12] ** 2).sum(-1), 2.25 * (x[..., :12] ** 2).sum(-1))
        assert np.array_equal(y[..., 12:], x[..., 12:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_scores_depend_on_distance_only(interleaved):
    rng = np.random.default_rng(1)
    q, k, f = rng.normal(size=(1, 1, 64)), rng.normal(size=(1, 1, 64)), rotary.frequencies(64)

    def score(p, r):
        return float((rotary.rotate(q, [p], f, interleaved) * rotary.rotate(k, [r], f, interleaved)).sum())

    assert abs(score(100, 90) - score(5010, 5000)) < 1e-9
    assert abs(score(7, 7) - float((q * k).sum())) < 1e-9


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_gradient_is_the_derivative(interleaved):
    """d/dx of <rotate(x), g> by central differences of a linear map: exact but for rounding."""
    rng = np.random.default_rng(2)
    f = rotary.frequencies(6, base=100.0)
    x, g, pos = rng.normal(size=(2, 1, 8)), rng.normal(size=(2, 1, 8)), [3, 17]
    want = np.empty_like(x)
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = 1.0
        want[i] = ((rotary.rotate(x + e, pos, f, interleaved, 1.2) - rotary.rotate(x - e, pos, f, interleaved, 1.2)) * g).sum() / 2
    assert np.allclose(rotary.rotate(g, pos, f, interleaved, 1.2, grad=True), want)


def test_binding_refuses_what_is_no_gpu_tensor_whether_it_has_a_gradient_or_not():
    import torch
    pos = torch.zeros(4, dtype=torch.int32)
    for x in (np.zeros((4, 8, 64), np.float32), torch.zeros(4, 8, 64, requires_grad=True)):
        with pytest.raises(ValueError, match="GPU tensor"):
            kp.kvp_rope_apply(kp.Rope(64), x, pos)
