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


# Values that are not finite.  Tolerance of what must stay: the docstring of test_gpu_linear.py, against the recurrence
# without the bad value.
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("lens,Hq,Hkv,d,at", [
    ([700, 90], 4, 2, 64, 0), ([700, 90], 4, 2, 64, 337), ([700, 90], 4, 2, 128, 63),   # cut: in and around the parts,
    ([700, 90], 4, 2, 128, 64), ([700, 90], 4, 2, 64, 128), ([700, 90], 4, 2, 128, 699),  # at their ends
    ([100, 90], 16, 1, 128, 40), ([100, 90], 16, 1, 64, 99),                             # query heads shared out, in place
    ([2500], 1, 1, 64, 1300), ([4160], 1, 1, 64, 4000),                                  # the other scans
])
def test_bad_values_in_parts_and_shared_out_heads(lens, Hq, Hkv, d, at, what, value):
    """Nothing but the bad token and, through the state, later tokens of its head and sequence changes beyond rounding;
    whatever is changed is not finite."""
    import torch
    note(f"linear non-finite {lens} {Hq}/{Hkv} {d} {at} {what} {value}")
    c = Case(lens, Hq, Hkv, d)
    i = list(range(len(lens)))
    want, room = c.oracle(i, i, d ** -0.5)
    G, h = Hq // Hkv, Hkv - 1
    head = Hq - 1 if what == "q" else h
    getattr(c, what)[at, head, 5] = value
    hit = np.zeros(want[0].shape, bool)
    heads = slice(head, head + 1) if what == "q" else slice(h * G, (h + 1) * G)
    hit[at:at + 1 if what == "q" else lens[0], heads, 5 if what == "v" else slice(None)] = True
    state_hit = np.zeros(want[1].shape, bool)
    if what == "k":
        state_hit[0, h, 5, :] = True
    elif what == "v":
        state_hit[0, h, :, 5] = True
    for dt in (torch.float32, torch.bfloat16):
        state = c.state.clone()
        got = kp.linear_chunk_attn(c.q, c.k, c.v, state, c.decay, i, i, c.cu, out_dtype=dt)
        assert not np.isfinite(f64(got)[hit]).any() and not np.isfinite(f64(state)[state_hit]).any()
        got[torch.from_numpy(hit).cuda()] = torch.from_numpy(want[0][hit]).to(dt).cuda()
        state[torch.from_numpy(state_hit).cuda()] = torch.from_numpy(want[1][state_hit]).float().cuda()
        check(got, state, want, room, c, i)


def test_an_infinity_in_a_state():
    """Both calls: the row of the state stays not finite, other heads and sequences are as they would be."""
    import torch
    note("linear infinite state")
    for lens in ([100, 70], [700, 1], [1, 1]):
        c = Case(lens, 8, 2, 64)
        i = [0, 1]
        want, room = c.oracle(i, i, 0.125)
        c.state[0, 1, 9, 3] = float("inf")
        calls = [lambda s: kp.linear_chunk_attn(c.q, c.k, c.v, s, c.decay, i, i, c.cu)]
        if lens == [1, 1]:
            calls.append(lambda s: kp.linear_decode_attn(c.q, c.k, c.v, s, c.decay, i, i))
        for call in calls:
            state = c.state.clone()
            got = call(state)
            hit = torch.zeros_like(got, dtype=torch.bool)
            hit[:lens[0], 4:, 3] = True
            assert not bool(torch.isfinite(got[hit]).any()) and not bool(torch.isfinite(state[0, 1, 9, 3]))
            got[hit] = torch.from_numpy(want[0]).float().cuda()[hit]
            state[0, 1, 9, 3] = float(want[1][0, 1, 9, 3])
            check(got, state, want, room, c, i)


def test_infinities_of_single_tokens_stay_infinities():
    """linear_decode_attn computes the formulas as they stand: inf times a positive number is inf, in state and output."""
    import torch
    note("linear infinities")
    q, k, v = (torch.ones(1, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    state = torch.ones(1, 2, 64, 64, device="cuda")
    v[0, 1, 7] = float("inf")
    state[0, 0, 2, 3] = float("-inf")
    out = kp.linear_decode_attn(q, k, v, state, [0.5, 0.5], [0], [0], scale=1.0)
    assert bool((state[0, 1, :, 7] == float("inf")).all()) and float(state[0, 0, 2, 3]) == float("-inf")
    assert float(out[0, 1, 7]) == float("inf") and float(out[0, 0, 3]) == float("-inf")
    out[0, 1, 7] = out[0, 0, 3] = 96.0
    assert bool((out == 96.0).all())  # 64 times 0.5 + 1
