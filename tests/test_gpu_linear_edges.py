"""The linear attention calls where sequences and values are at their ends: sequences without tokens, more sequences than a
launch holds, values that are not finite in sequences cut into parts and in shared-out query heads."""
import numpy as np
import pytest

from gpu_helpers import note
from paper_2608_11152_amd import kvpattn as kp
from test_gpu_linear import Case, check, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,Hq,Hkv,d", [([128], 64, 4, 128), ([70, 300], 8, 2, 64)])
def test_sequences_without_tokens_beside_others(lens, Hq, Hkv, d):
    """Idle sequences of every kind: state in place, not kept, from zeros, handed to another slot.  The others' outputs are
    the bits of the call without them."""
    import torch
    note(f"linear idle sequences {lens} {Hq}/{Hkv} {d}")
    idle = 199
    where = [7, 150][:len(lens)]
    n = np.zeros(idle + len(lens), np.int32)
    n[where] = lens
    B = len(n)
    c = Case(list(n), Hq, Hkv, d, slots=2 * B + 1)
    src = np.arange(B, dtype=np.int32)
    dst = src.copy()
    src[1::4], dst[2::4] = -1, -1
    dst[3::4] = B + np.arange(len(dst[3::4]))
    src[where], dst[where] = where, where
    want, room = c.oracle(src, dst, d ** -0.5)
    alone = c.state.clone()
    some = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    ref = kp.linear_chunk_attn(c.q, c.k, c.v, alone, c.decay, where, where, some)
    out = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, src, dst, c.cu)
    assert torch.equal(out, ref) and torch.equal(c.state[where], alone[where])
    check(out, c.state, want, room, c, dst)
    before = c.state.clone()
    none = np.zeros(B + 1, np.int32)
    src, dst = np.arange(B), np.where(np.arange(B) % 2, np.arange(B), -1)
    got = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, src, dst, none, out=out.clone())
    torch.cuda.synchronize()
    assert torch.equal(got, out) and torch.equal(c.state, before)


def test_more_items_than_one_launch_holds():
    """70000 single tokens of 128 heads: out = scale (q . k) v, where the second launch begins among them."""
    import torch
    note("linear many items")
    B, H, d = 70000, 128, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(B, H, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    state = torch.zeros(1, H, d, d, device="cuda")
    none = np.full(B, -1, np.int32)
    out = kp.linear_chunk_attn(q, k, v, state, np.full(H, 0.5), none, none, np.arange(B + 1), scale=0.25, out_dtype=torch.float32)
    for at in (0, 65535, 65536, 69999):
        a, b, c = (f64(t[at]) for t in (q, k, v))
        want = 0.25 * (a * b).sum(-1, keepdims=True) * c
        room = 0.25 * (np.abs(a) * np.abs(b)).sum(-1, keepdims=True) * np.abs(c)
        assert np.all(np.abs(f64(out[at]) - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -16 * room)
    for lo in range(0, B, 10000):  # all of them, in fp32: 64 products, so 2^-17 of the sum of absolute values
        a, b, c = (t[lo:lo + 10000].float() for t in (q, k, v))
        want = 0.25 * (a * b).sum(-1, keepdim=True) * c
        room = 0.25 * (a.abs() * b.abs()).sum(-1, keepdim=True) * c.abs()
        assert bool(((out[lo:lo + 10000] - want).abs() <= 2.0 ** -16 * room).all())
