"""linear_chunk_attn and linear_decode_attn against the 64-bit recurrence: lengths around every tile, both head sizes,
shared heads, decays from 1 to almost 0, slots that fork, keep nothing or start from zeros, strides, long sequences cut
into parts, values that are not finite, refusals, capture; and a session's steps through both.

Tolerance, per element, with A the same sum over absolute values (the oracle on |q|, |k|, |v|, |state|):
  outputs: half a step of the output type relative to the result, plus 2^-16 A + n 2^-24 A: an operand of a matrix product
           that is not bf16 already is carried as two bf16 parts, which leaves 2^-18 of it, for the state and for the
           weights of a chunk (2^-17 in all); n fp32 additions and decays of a step each.
  states:  n 2^-24 A + 4 * 2^-24 A, n the sequence's tokens; and over the whole state a relative 2-norm error of
           (n / 2 + 8) 2^-24: rounding decay * S is off by up to half a step of 2^-24, and the same way at every
           token where the decay is a step or two below 1 (x (1 - 2^-24) lies between half a step and a whole one under
           x, and goes to the whole one), the rest is at random."""
import numpy as np
import pytest

from gpu_helpers import note
from oracle import linear
from paper_2608_11152_amd import kvpattn as kp

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Case:
    def __init__(self, lens, Hq, Hkv, d, slots=None, fused=False, decay=None, seed=0):
        import torch
        g = torch.Generator().manual_seed(seed)
        self.lens, self.Hq, self.Hkv, self.d = list(lens), Hq, Hkv, d
        T = sum(lens)
        x = torch.randn(T, Hq + 2 * Hkv, d, generator=g).to(torch.bfloat16).cuda()
        self.q, self.k, self.v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        if not fused:
            self.q, self.k, self.v = (t.contiguous() for t in (self.q, self.k, self.v))
        slots = slots or len(lens) + 2
        self.state = torch.randn(slots, Hkv, d, d, generator=g).cuda()
        self.decay = np.asarray(decay if decay is not None else
                                np.exp(-2.0 ** (-8.0 * (np.arange(Hkv) + 1) / Hkv)), np.float32)
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)

    def oracle(self, src, dst, scale):
        a = [f64(t) for t in (self.q, self.k, self.v, self.state)]
        dec = self.decay.astype(np.float64)
        want = linear.chunks(*a, dec, src, dst, self.cu, scale)
        room = linear.chunks(*(np.abs(t) for t in a), dec, src, dst, self.cu, abs(scale))
        return want, room


def check(got, state, want, room, c, dst):
    import torch
    n = np.repeat(c.lens, c.lens)[:, None, None] if sum(c.lens) else np.zeros((0, 1, 1))
    step = torch.finfo(got.dtype).eps / 2
    err = np.abs(f64(got) - want[0])
    tol = step * np.abs(want[0]) + (2.0 ** -16 + n * 2.0 ** -24) * room[0]
    assert np.all(err <= tol), ("out", float((err - tol).max()), np.unravel_index(np.argmax(err - tol), err.shape))
    s, w = f64(state), want[1]
    n = np.full((s.shape[0], 1, 1, 1), -4.0)
    for i, to in enumerate(dst):
        if to >= 0:
            n[to] = c.lens[i]
    tol = (n + 4) * 2.0 ** -24 * room[1]  # slots that are no destination: exactly as before
    err = np.abs(s - w)
    assert np.all(err <= tol), ("state", float((err - tol).max()), np.unravel_index(np.argmax(err - tol), err.shape))
    assert np.linalg.norm(s - w) <= (max(c.lens) / 2 + 8) * 2.0 ** -24 * np.linalg.norm(w)


def run_chunk(c, src, dst, scale=None, **kw):
    scale = c.d ** -0.5 if scale is None else scale
    want, room = c.oracle(src, dst, scale)
    out = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, src, dst, c.cu, scale=scale, **kw)
    check(out, c.state, want, room, c, dst)
    return out


LENS = [[1], [2], [15, 16, 17], [63], [64], [65], [1, 0, 128, 3], [127, 129], [300, 1, 31, 32, 33], [191, 640]]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("Hq,Hkv,d", [(2, 2, 64), (3, 3, 128), (8, 2, 64), (8, 4, 128), (16, 1, 64), (16, 1, 128)])
def test_chunks(lens, Hq, Hkv, d):
    import torch
    note(f"linear chunk {lens} {Hq}/{Hkv} {d}")
    n = len(lens)
    c = Case(lens, Hq, Hkv, d, slots=2 * n + 1, fused=d == 64)
    src = [i if i % 2 == 0 else -1 for i in range(n)]
    dst = [i if i % 2 == 0 else n + i for i in range(n)]
    run_chunk(c, src, dst, out_dtype=torch.float32)
    run_chunk(c, src, dst, out_dtype=torch.bfloat16)


@pytest.mark.parametrize("decay", [1.0, 1.0 - 2.0 ** -24, 0.999, 0.5, 0.01, 1e-30, 1e-44])
@pytest.mark.parametrize("d", [64, 128])
def test_decays(decay, d):
    import torch
    note(f"linear decay {decay} {d}")
    c = Case([150, 64, 1], 2, 2, d, decay=[decay, 0.9])
    run_chunk(c, [0, 1, 2], [0, 1, 2], out_dtype=torch.float32)


@pytest.mark.parametrize("scale", [1.0, -0.5, 0.0, 3.7])
def test_scales(scale):
    import torch
    note(f"linear scale {scale}")
    run_chunk(Case([70, 5], 4, 2, 64), [0, 1], [2, 3], scale=scale, out_dtype=torch.float32)


def test_slots():
    """Forks of one source, a sequence that keeps nothing, one that only hands its state on, one from zeros."""
    import torch
    note("linear slots")
    c = Case([10, 70, 5, 0, 0, 3], 4, 2, 64, slots=9)
    src, dst = [7, 7, 7, 7, -1, 8], [0, 1, -1, 2, 3, 8]
    run_chunk(c, src, dst, out_dtype=torch.float32)
    assert torch.equal(c.state[2], c.state[7]) and not bool(c.state[3].any())


@pytest.mark.parametrize("lens,Hkv,d", [([20000], 1, 64), ([9001, 33, 12000], 2, 128), ([4097], 4, 128)])
def test_long_sequences(lens, Hkv, d):
    import torch
    note(f"linear long {lens} {Hkv} {d}")
    decay = [0.9999, 1.0 - 2.0 ** -20, 0.99, 1.0][:Hkv]
    c = Case(lens, Hkv, Hkv, d, decay=decay)
    run_chunk(c, list(range(len(lens))), list(range(len(lens))), out_dtype=torch.float32)
    c = Case(lens, Hkv, Hkv, d, decay=decay, seed=1)
    run_chunk(c, [-1] * len(lens), [-1] * len(lens), out_dtype=torch.bfloat16)


def test_many_short_sequences():
    import torch
    note("linear many")
    lens = [(7 * i) % 90 for i in range(500)]
    c = Case(lens, 2, 2, 64)
    order = np.random.default_rng(0).permutation(502)[:500]
    run_chunk(c, [-1] * 500, order, out_dtype=torch.bfloat16)


def test_rows_behind_the_last_sequence_and_callers_buffers():
    import torch
    note("linear rows behind")
    c = Case([40, 7], 4, 2, 64)
    pad = Case([40, 7, 30], 4, 2, 64)
    out = torch.full((77, 4, 64), 5.0, device="cuda")
    ws = torch.empty(max(1, kp.linear_chunk_workspace_size(c.cu, 2, 64)), dtype=torch.uint8, device="cuda")
    want, room = c.oracle([0, 1], [0, 1], 0.5)
    for t, x in ((pad.q, c.q), (pad.k, c.k), (pad.v, c.v)):
        t[:47] = x
        t[47:] = float("nan")  # padding is not read into anything
    got = kp.linear_chunk_attn(pad.q, pad.k, pad.v, c.state, c.decay, [0, 1], [0, 1], c.cu, scale=0.5, out=out, ws=ws)
    assert got is out and bool((out[47:] == 5.0).all())
    check(out[:47], c.state, want, room, c, [0, 1])


@pytest.mark.parametrize("B,Hq,Hkv,d", [(1, 1, 1, 64), (4, 8, 2, 64), (3, 16, 16, 128), (400, 2, 2, 64), (5, 16, 1, 128),
                                        (7, 8, 4, 64), (193, 3, 3, 128)])
def test_decode(B, Hq, Hkv, d):
    import torch
    note(f"linear decode {B} {Hq}/{Hkv} {d}")
    c = Case([1] * B, Hq, Hkv, d, slots=B + 3)
    dst = np.random.default_rng(B).permutation(B + 1).astype(np.int32)[:B]
    src = dst.copy()
    src[::3], dst[1::5] = B + 2, -1  # forks of one slot; some are not kept
    src[1::5] = -1
    for dt in (torch.float32, torch.bfloat16):
        want, room = c.oracle(src, dst, d ** -0.5)
        out = kp.linear_decode_attn(c.q, c.k, c.v, c.state, c.decay, src, dst, out_dtype=dt)
        check(out, c.state, want, room, c, dst)


def test_decode_strides_and_chunk_of_one_agree():
    import torch
    note("linear decode strides")
    c = Case([1] * 6, 8, 2, 128, fused=True)
    other = c.state.clone()
    a = kp.linear_decode_attn(c.q, c.k, c.v, c.state, c.decay, range(6), range(6))
    b = kp.linear_chunk_attn(c.q, c.k, c.v, other, c.decay, range(6), range(6), c.cu)
    want, room = Case([1] * 6, 8, 2, 128, fused=True).oracle(list(range(6)), list(range(6)), 128 ** -0.5)
    check(a, c.state, want, room, c, range(6))
    check(b, other, want, room, c, range(6))
    one = c.q[:1].expand(6, 8, 128)  # one token's queries for all sequences
    assert kp.linear_decode_attn(one, c.k, c.v, c.state, c.decay, range(6), [-1] * 6).shape == (6, 8, 128)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_not_finite(d, what, value):
    """A bad value reaches its own token and, through the state, later ones of its head and sequence: never an earlier
    token, another head or another sequence, whose bits stay."""
    import torch
    note(f"linear non-finite {d} {what} {value}")
    lens, Hq, Hkv = [150, 90], 4, 2
    for at in (0, 37, 63, 64, 149):
        c, bad = Case(lens, Hq, Hkv, d), Case(lens, Hq, Hkv, d)
        t = getattr(bad, what)
        h = 1
        t[at, h, 5] = value
        clean = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, [0, 1], [0, 1], c.cu)
        got = kp.linear_chunk_attn(bad.q, bad.k, bad.v, bad.state, bad.decay, [0, 1], [0, 1], bad.cu)
        heads = slice(1, 2) if what == "q" else slice(2, 4)
        rows = slice(at, at + 1) if what == "q" else slice(at, 150)
        hit = torch.zeros_like(got, dtype=torch.bool)
        hit[rows, heads, 5 if what == "v" else slice(None)] = True
        if what == "v":  # the whole head's later rows may change their last bits with the way that a chunk is summed
            near = hit.clone()
            near[:150, heads] = True
            assert torch.allclose(got[near & ~hit], clean[near & ~hit], rtol=1e-3, atol=1e-3)
            assert torch.equal(got[~near], clean[~near])
        else:
            assert torch.equal(got[~hit], clean[~hit])
        assert not bool(torch.isfinite(got[hit]).any())
        sh = torch.zeros_like(c.state, dtype=torch.bool)
        if what == "k":
            sh[0, 1, 5, :] = True
        elif what == "v":
            sh[0, 1, :, 5] = True
        assert torch.equal(bad.state[~sh], c.state[~sh])
        assert not bool(torch.isfinite(bad.state[sh]).any())


def test_refusals_leave_everything():
    import torch
    note("linear refusals")
    c = Case([3, 4], 4, 2, 64)
    before = c.state.clone()
    out = torch.full((7, 4, 64), 5.0, device="cuda")

    def refused(code, **kw):
        a = dict(q=c.q, k=c.k, v=c.v, state=c.state, decay=c.decay, src_slots=[0, 1], dst_slots=[0, 1], cu=c.cu, out=out)
        a.update(kw)
        with pytest.raises(code if isinstance(code, type) else kp.KvpError) as e:
            kp.linear_chunk_attn(**a)
        if not isinstance(code, type):
            assert e.value.code == code

    refused(kp.KVP_EINVAL, dst_slots=[1, 1])
    refused(kp.KVP_EINVAL, src_slots=[1, 1], dst_slots=[0, 1])
    refused(kp.KVP_ERANGE, src_slots=[0, 4])
    refused(kp.KVP_EINVAL, decay=[0.5, 1.01])
    refused(kp.KVP_EINVAL, cu=[0, 5, 3])
    refused(kp.KVP_EUNSUPPORTED, q=torch.zeros(7, 6, 64, dtype=torch.bfloat16, device="cuda"), out=None)
    refused(ValueError, decay=[0.5])
    refused(ValueError, state=c.state[:, :1].contiguous())
    refused(ValueError, state=c.state.double())
    refused(ValueError, state=c.state.transpose(2, 3))
    refused(ValueError, out=out[:5])
    refused(ValueError, out=out.half())
    refused(ValueError, k=c.k[:6])
    refused(ValueError, cu=[0, 3, 8])
    torch.cuda.synchronize()
    assert torch.equal(c.state, before) and bool((out == 5.0).all())


def test_decode_captured():
    """The slots and decays travel in the launch: the graph owns them."""
    import torch
    note("linear decode capture")
    B = 200
    c = Case([1] * B, 4, 2, 64)
    out = torch.zeros(B, 4, 64, device="cuda")
    slots = np.random.default_rng(3).permutation(B).astype(np.int32)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = c.state.clone()
    kp.linear_decode_attn(c.q, c.k, c.v, c.state, c.decay, slots, slots, out=out, stream=s)
    torch.cuda.synchronize()
    c.state.copy_(keep)
    g = torch.cuda.CUDAGraph()
    decay = c.decay.copy()
    with torch.cuda.graph(g, stream=s):
        kp.linear_decode_attn(c.q, c.k, c.v, c.state, decay, slots, slots, out=out, stream=s)
    decay[:] = 0.0
    ref = c.state.clone()
    torch.cuda.synchronize()
    assert torch.equal(c.state, keep)  # capture runs nothing
    for rep in range(4):
        for t in (c.q, c.k, c.v):
            t.copy_(torch.randn_like(t.float()))
        want = kp.linear_decode_attn(c.q, c.k, c.v, ref, c.decay, slots, slots)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(c.state, ref)


def test_chunk_on_another_stream_and_under_capture():
    import torch
    note("linear chunk stream")
    c = Case([100, 64], 2, 2, 128)
    keep = c.state.clone()
    want = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, [0, 1], [0, 1], c.cu)
    other = keep.clone()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = kp.linear_chunk_attn(c.q, c.k, c.v, other, c.decay, [0, 1], [0, 1], c.cu, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(other, c.state)
    other.copy_(keep)
    g = torch.cuda.CUDAGraph()
    one = torch.zeros(4, device="cuda")
    with torch.cuda.graph(g, stream=s):
        one.add_(1.0)
        with pytest.raises(kp.KvpError) as e:
            kp.linear_chunk_attn(c.q, c.k, c.v, other, c.decay, [0, 1], [0, 1], c.cu, out=got, stream=s)
        assert e.value.code == kp.KVP_EHIP
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(other, keep)


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (8, 2, 128)])
def test_a_session_s_steps(Hq, Hkv, d):
    """A prompt, its samples' forks, decode steps and a later turn, with rotated q and k: against one recurrence per
    sample over everything it has seen."""
    import torch
    from oracle import rotary
    note(f"linear session {Hq}/{Hkv} {d}")
    samples, rng = 3, np.random.default_rng(7)
    rope, freq = kp.Rope(d // 2), rotary.frequencies(d // 2)
    decay = np.linspace(0.95, 1.0, Hkv).astype(np.float32)
    state = torch.full((samples + 1, Hkv, d, d), 3.0, device="cuda")

    def tokens(n, pos):
        x = torch.from_numpy(rng.normal(size=(n, Hq + 2 * Hkv, d)).astype(np.float32)).to(torch.bfloat16).cuda()
        p = torch.from_numpy(np.asarray(pos, np.int32)).cuda()
        kp.kvp_rope_apply(rope, x[:, :Hq + Hkv], p, out=x[:, :Hq + Hkv])  # q and k heads in one call
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]

    seen = [[] for _ in range(samples)]
    q, k, v = tokens(100, np.arange(100))
    kp.linear_chunk_attn(q, k, v, state, decay, [-1], [samples], [0, 100])
    for s in seen:
        s.append((f64(q), f64(k), f64(v)))
    slots, pos = list(range(samples)), [100] * samples
    outs = []
    for step in range(4):
        q, k, v = tokens(samples, pos)
        src = [samples] * samples if step == 0 else slots
        outs.append(kp.linear_decode_attn(q, k, v, state, decay, src, slots))
        for i, s in enumerate(seen):
            s.append(tuple(f64(x)[i:i + 1] for x in (q, k, v)))
        pos = [p + 1 for p in pos]
    cu = [0, 33, 33, 130]  # the second sample gets no tokens in this turn
    q, k, v = tokens(130, np.concatenate([pos[i] + np.arange(cu[i + 1] - cu[i]) for i in range(3)]))
    turn = kp.linear_chunk_attn(q, k, v, state, decay, slots, slots, cu)
    for i, s in enumerate(seen):
        s.append(tuple(f64(x)[cu[i]:cu[i + 1]] for x in (q, k, v)))
    for i, s in enumerate(seen):
        q, k, v = (np.concatenate([x[j] for x in s]) for j in range(3))
        want, end = linear.sequence(q, k, v, np.zeros((Hkv, d, d)), decay.astype(np.float64), d ** -0.5)
        room, _ = linear.sequence(*(np.abs(x) for x in (q, k, v)), np.zeros((Hkv, d, d)), decay.astype(np.float64), d ** -0.5)
        tol = (2.0 ** -15 + 240 * 2.0 ** -24) * room + 2.0 ** -24 * np.abs(want)
        got = np.concatenate([f64(o)[i:i + 1] for o in outs] + [f64(turn)[cu[i]:cu[i + 1]]])
        assert np.all(np.abs(got - want[100:]) <= tol[100:])
        assert np.linalg.norm(f64(state)[i] - end) <= 2e-6 * np.linalg.norm(end)
