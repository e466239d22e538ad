"""The fp32 outputs of the linear attention calls, which linear_chunk_attn and linear_decode_attn return unless told
otherwise, hold what fp32 arithmetic gives: the relative 2-norm error of the whole output against the 64-bit recurrence.

Bound.  A sum of N terms at random signs, each addition rounded to fp32 (off by at most u = 2^-24 of the partial sum, u /
sqrt(3) at random), is off by u sqrt(N / 6) of its size.
  decode: N = 128 products with the state, and the state's own two roundings: u sqrt(128 / 6 + 2) = 4.8 u; 8 u are allowed.
  chunk:  3 parts of 128 products with the state and of 64 with the weights, weights that are sums of 128 products:
          u sqrt((384 + 192 + 128) / 6) = 10.8 u; a state that comes from earlier chunks is a sum of 3 parts of 64
          products each: sqrt(192 / 6) = 5.7 u; the powers of the decay and the last steps 2 u: 12.4 u together; 16 u are
          allowed.
Both are far under what an operand cut to two bf16 parts leaves, 2^-18.7 = 40 u at random."""
import numpy as np
import pytest

from gpu_helpers import note
from paper_2608_11152_amd import kvpattn as kp
from test_gpu_linear import Case, f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def off(got, want):
    return np.linalg.norm(f64(got) - want) / np.linalg.norm(want) / U


@pytest.mark.parametrize("lens,Hq,Hkv,d", [
    ([1, 2, 64, 65], 2, 2, 128), ([40, 64, 17], 4, 2, 64), ([200], 3, 3, 128), ([200], 2, 2, 64),
    ([128, 90], 16, 1, 128),             # query heads shared out
    ([700, 330], 4, 2, 128), ([1500], 1, 1, 64),  # cut into parts
])
@pytest.mark.parametrize("src", [0, -1])
def test_chunk_outputs(lens, Hq, Hkv, d, src):
    import torch
    note(f"linear fp32 chunk {lens} {Hq}/{Hkv} {d} {src}")
    c = Case(lens, Hq, Hkv, d, fused=True)
    dst = list(range(len(lens)))
    src = dst if src == 0 else [-1] * len(lens)
    want, _ = c.oracle(src, dst, d ** -0.5)
    out = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, src, dst, c.cu)
    assert out.dtype == torch.float32
    assert off(out, want[0]) <= 16
    assert off(c.state, want[1]) <= 16


@pytest.mark.parametrize("B,Hq,Hkv,d", [(1, 4, 4, 64), (7, 8, 2, 128), (100, 16, 1, 64), (33, 3, 3, 128)])
def test_token_outputs(B, Hq, Hkv, d):
    note(f"linear fp32 token {B} {Hq}/{Hkv} {d}")
    c = Case([1] * B, Hq, Hkv, d)
    slots = list(range(B))
    want, _ = c.oracle(slots, slots, d ** -0.5)
    out = kp.linear_decode_attn(c.q, c.k, c.v, c.state, c.decay, slots, slots)
    assert off(out, want[0]) <= 8
    assert off(c.state, want[1]) <= 8


def test_a_token_has_the_same_accuracy_through_either_call():
    note("linear fp32 either call")
    c = Case([1] * 64, 8, 2, 128)
    slots = list(range(64))
    want, _ = c.oracle(slots, [-1] * 64, 128 ** -0.5)
    for out in (kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, slots, [-1] * 64, c.cu),
                kp.linear_decode_attn(c.q, c.k, c.v, c.state, c.decay, slots, [-1] * 64)):
        assert off(out, want[0]) <= 16
