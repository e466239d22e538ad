"""Refusals of kvp_rope_apply and linear_chunk_workspace_size at the ends of their arguments; pointers are never followed."""
import ctypes as C

import numpy as np
import pytest

from paper_2608_11152_amd import kvpattn as kp

FAKE = 1 << 20


def apply(rope, T, H, ts, hs, d=64):
    return kp.lib().kvp_rope_apply(rope.ref(), FAKE, ts, hs, 1 << 40, ts, hs, kp.KVP_BF16, FAKE, T, H, d, 0, None)


@pytest.mark.parametrize("T,H,ts,hs,code", [
    (1, (1 << 20) + 1, 64, 64, kp.KVP_EUNSUPPORTED),          # heads beyond the kernels' indices
    (3, 3, 1 << 20, (1 << 62) + 8, kp.KVP_EINVAL),            # two head strides pass 64 bits
    (1 << 40, 2, 1 << 40, 1 << 20, kp.KVP_EINVAL),            # and so many token strides
    (1 << 40, 2, 1 << 40, 32, kp.KVP_EINVAL),
    (5, 4, 255, 64, kp.KVP_EINVAL),                           # heads overlap the next token's
])
def test_rope_apply_refusals(T, H, ts, hs, code):
    assert apply(kp.Rope(64), T, H, ts, hs) == code


def test_workspace_size_is_enough_for_any_heads_and_never_negative():
    lib = kp.lib()
    n = C.c_size_t()
    rng = np.random.default_rng(0)
    for _ in range(200):
        lens = rng.integers(0, 10 ** rng.integers(1, 6), size=rng.integers(1, 40))
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        for Hkv, d in ((1, 64), (4, 128), (16, 64)):
            assert lib.linear_chunk_workspace_size(cu.ctypes.data, len(lens), Hkv, d, C.byref(n)) == kp.KVP_OK
            assert n.value % (Hkv * d * d * 4) == 0
            parts = n.value // (Hkv * d * d * 4)
            assert parts <= sum(-(-int(x) // 64) for x in lens)
