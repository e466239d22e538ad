"""Linear attention without a GPU: the calls' refusals (all made before anything is enqueued) and the properties that
pin the oracle."""
import ctypes as C

import numpy as np
import pytest

from oracle import linear
from paper_2608_11152_amd import kvpattn as kp

FAKE = 1 << 20  # an aligned address that a refused call never reads


def _call(chunk, q=FAKE, qs=512, k=FAKE, ks=128, v=FAKE, vs=128, state=FAKE, slots=4, decay=(0.5, 1.0), src=(0, -1),
          dst=(0, 1), cu=(0, 3, 5), n=2, hq=8, hkv=2, d=64, scale=1.0, out=FAKE, od=kp.KVP_BF16, ws=None, ws_bytes=0):
    dec = np.asarray(decay, np.float32)
    s, t, c = (np.asarray(x, np.int32) for x in (src, dst, cu))
    a = (q, qs, k, ks, v, vs, state, slots, dec.ctypes.data_as(C.POINTER(C.c_float)), kp._ptr(s), kp._ptr(t))
    if chunk:
        return kp.lib().linear_chunk_attn(*a, kp._ptr(c), n, hq, hkv, d, scale, out, od, ws, ws_bytes, None)
    return kp.lib().linear_decode_attn(*a, n, hq, hkv, d, scale, out, od, None)


@pytest.mark.parametrize("chunk", [True, False])
@pytest.mark.parametrize("kw,code", [
    (dict(d=96), kp.KVP_EUNSUPPORTED), (dict(hq=6), kp.KVP_EUNSUPPORTED), (dict(hq=7), kp.KVP_EUNSUPPORTED),
    (dict(hq=64), kp.KVP_EUNSUPPORTED), (dict(hq=0), kp.KVP_EUNSUPPORTED), (dict(hkv=0), kp.KVP_EUNSUPPORTED),
    (dict(hkv=129, hq=129, decay=[0.5] * 129), kp.KVP_EUNSUPPORTED), (dict(od=kp.KVP_FP8_E4M3), kp.KVP_EUNSUPPORTED),
    (dict(scale=float("nan")), kp.KVP_EINVAL), (dict(state=None), kp.KVP_EINVAL), (dict(state=FAKE + 8), kp.KVP_EINVAL),
    (dict(slots=0), kp.KVP_EINVAL), (dict(q=None), kp.KVP_EINVAL), (dict(k=FAKE + 2), kp.KVP_EINVAL),
    (dict(vs=129), kp.KVP_EINVAL), (dict(qs=-512), kp.KVP_EINVAL), (dict(out=None), kp.KVP_EINVAL),
    (dict(decay=(0.5, 0.0)), kp.KVP_EINVAL), (dict(decay=(0.5, 1.5)), kp.KVP_EINVAL),
    (dict(decay=(float("nan"), 1.0)), kp.KVP_EINVAL), (dict(decay=(-0.5, 1.0)), kp.KVP_EINVAL),
    (dict(src=(0, 4)), kp.KVP_ERANGE), (dict(src=(-2, 0)), kp.KVP_ERANGE), (dict(dst=(0, 4)), kp.KVP_ERANGE),
    (dict(dst=(1, 1)), kp.KVP_EINVAL), (dict(src=(0, 0), dst=(0, 1)), kp.KVP_EINVAL),
    (dict(src=(2, 0), dst=(0, 2)), kp.KVP_EINVAL), (dict(n=-1), kp.KVP_EINVAL),
])
def test_refusals(chunk, kw, code):
    assert _call(chunk, **kw) == code
    assert kp.lib().kvp_last_error()


@pytest.mark.parametrize("cu", [(1, 3, 5), (0, 3, 2)])
def test_chunk_refuses_bad_offsets(cu):
    assert _call(True, cu=cu) == kp.KVP_EINVAL
    n = C.c_size_t()
    assert kp.lib().linear_chunk_workspace_size(kp._ptr(np.asarray(cu, np.int32)), 2, 2, 64, C.byref(n)) == kp.KVP_EINVAL


def test_nothing_to_do():
    assert _call(True, n=0) == kp.KVP_OK and _call(False, n=0) == kp.KVP_OK


def test_binding_refuses_host_tensors():
    import torch
    x, st = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 64, 64)
    with pytest.raises(ValueError, match="GPU tensor"):
        kp.linear_decode_attn(x, x, x, st, [0.5, 0.5], [0, 1], [0, 1])
    with pytest.raises(ValueError, match="cu has"):
        kp.linear_chunk_attn(x, x, x, st, [0.5, 0.5], [0, 1], [0, 1], [0, 2])
    with pytest.raises(ValueError, match="one slot per sequence"):
        kp.linear_decode_attn(x, x, x, st, [0.5, 0.5], [0, 1], [0])


def _case(n=37, hq=4, hkv=2, d=8, seed=0):
    r = np.random.default_rng(seed)
    return r.normal(size=(n, hq, d)), r.normal(size=(n, hkv, d)), r.normal(size=(n, hkv, d)), r.normal(size=(hkv, d, d))


def test_oracle_equals_the_double_sum():
    q, k, v, S = _case()
    decay = np.array([0.9, 1.0])
    out, _ = linear.sequence(q, k, v, S, decay, 0.3)
    for i in (0, 1, 20, 36):
        for h in range(4):
            g = h // 2
            o = decay[g] ** (i + 1) * q[i, h] @ S[g]
            for j in range(i + 1):
                o = o + decay[g] ** (i - j) * (q[i, h] @ k[j, g]) * v[j, g]
            assert np.allclose(out[i, h], 0.3 * o)


def test_oracle_splits_anywhere_and_keeps_other_slots():
    q, k, v, S = _case(seed=1)
    decay = np.array([0.8, 0.999])
    whole, end = linear.sequence(q, k, v, S, decay, 1.0)
    states = np.stack([S, S + 1, S + 2])
    a, after = linear.chunks(q[:20], k[:20], v[:20], states, decay, [0], [2], [0, 20], 1.0)
    b, last = linear.chunks(q[20:], k[20:], v[20:], after, decay, [2], [2], [0, 17], 1.0)
    assert np.allclose(np.concatenate([a, b]), whole) and np.allclose(last[2], end)
    assert np.array_equal(last[:2], states[:2])
