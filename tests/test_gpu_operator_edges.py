"""kvp_rope_apply, kv_append_rope and the linear attention calls where sizes, places and callers meet their ends: rows and
pages further apart than 32 bits of bytes, every bf16 value in an FP8 pool, lengths around the cuts of a sequence, a
workspace of exactly the size asked for, two streams at once."""
import numpy as np
import pytest

from gpu_helpers import note
from oracle import fp8
from paper_2608_11152_amd import kvpattn as kp
from test_gpu_linear import Case, check

pytestmark = pytest.mark.gpu


def far(t, stride):
    """The rows of t, `stride` elements apart in a tensor of their own."""
    import torch
    base = torch.empty((t.shape[0] - 1) * stride + t[0].numel(), dtype=t.dtype, device="cuda")
    out = base.as_strided(t.shape, (stride, t.shape[2], 1))
    out.copy_(t)
    return out


def test_linear_rows_far_apart():
    """150 tokens, 2^24 elements each from the next: the last begins 4.7 GB behind the first."""
    import torch
    note("linear far rows")
    c = Case([70, 1, 79], 4, 2, 64)
    near = [c.q, c.k, c.v]
    want, room = c.oracle([0, 1, 2], [0, 1, 2], 0.5)
    c.q, c.k, c.v = far(near[0], 1 << 24), far(near[1], (1 << 24) - 64), near[2]
    out = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, [0, 1, 2], [0, 1, 2], c.cu, scale=0.5)
    check(out, c.state, want, room, c, [0, 1, 2])
    with pytest.raises(kp.KvpError) as e:
        kp.linear_chunk_attn(far(near[0][:2], (1 << 24) + 8), near[1], near[2], c.state, c.decay, [0], [0], [0, 2])
    assert e.value.code == kp.KVP_EINVAL
    one = Case([1] * 150, 4, 2, 64)
    want, room = one.oracle(range(150), range(150), 0.5)
    out = kp.linear_decode_attn(far(one.q, 1 << 24), far(one.k, 1 << 24), one.v, one.state, one.decay, range(150), range(150),
                                scale=0.5)
    check(out, one.state, want, room, one, range(150))


def test_linear_states_far_into_their_tensor():
    """A slot that begins behind 2^32 bytes of states."""
    import torch
    note("linear far states")
    c = Case([90, 3], 2, 2, 128)
    want, room = c.oracle([0, 1], [0, 1], 0.5)
    slots = 40000  # of 131072 bytes
    states = torch.zeros(slots, 2, 128, 128, device="cuda")
    states[slots - 1], states[slots - 2] = c.state[0], c.state[1]
    at = [slots - 1, slots - 2]
    out = kp.linear_chunk_attn(c.q, c.k, c.v, states, c.decay, at, at, c.cu, scale=0.5)
    got = c.state.clone()
    got[:2] = states[at]
    check(out, got, want, room, c, [0, 1])
    assert not bool(states[:slots - 2].any())


def test_append_rope_far_rows_and_pages():
    """Tokens 2^26 elements apart, and pages behind 4 GB of a pool."""
    import torch
    note("append rope far")
    g = torch.Generator().manual_seed(1)
    T, Hq, Hkv, d = 36, 16, 16, 128
    q, k, v = (torch.randn(T, h, d, generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
    pages = 36000  # of 131072 bytes
    bt = torch.tensor([[35999, 34000, 33999]], dtype=torch.int32, device="cuda")
    rope = kp.Rope(64)
    small, large = kp.Pool(1, 3, Hkv, d), kp.Pool(1, pages, Hkv, d)
    order = torch.tensor([[2, 1, 0]], dtype=torch.int32, device="cuda")
    want_q = kp.kv_append_rope(small, 0, rope, k, v, order, [5], [0, T], q=q)
    out = far(torch.zeros_like(q), 1 << 26)
    got_q = kp.kv_append_rope(large, 0, rope, far(k, 1 << 26), far(v, 1 << 26), bt, [5], [0, T], q=far(q, 1 << 26), q_out=out)
    assert torch.equal(got_q, want_q)
    a = small.layer_raw().view(3, -1)
    b = large.layer_raw().view(pages, -1)
    assert torch.equal(b[[33999, 34000, 35999]], a)
    assert not bool(b[:33999].any()) and not bool(b[34001:35999].any())
    small.close(), large.close()


@pytest.mark.parametrize("scale", [1.0, 0.37, 3.0e38, 1.0e-38])
def test_fp8_codes_of_every_bf16_value(scale):
    """kv_append, and kv_append_rope where it does not rotate, against the oracle's quantiser: all 65536 values."""
    import torch
    note(f"fp8 codes {scale}")
    d = 128
    bits = np.arange(65536, dtype=np.uint16).reshape(512, 1, d)
    k = torch.from_numpy(bits.view(np.int16).copy()).view(torch.bfloat16).cuda()
    v = k.flip(0).contiguous()
    bt = torch.arange(32, dtype=torch.int32, device="cuda").view(1, 32)
    want_k, want_v = fp8.quantize_bf16(bits, scale), fp8.quantize_bf16(bits[::-1], scale)
    t, c = np.arange(16)[:, None], np.arange(d)[None, :]
    at_k = (((c // 64) * 4 + (c % 32) // 8) * 16 + t) * 16 + ((c // 32) % 2) * 8 + c % 8
    s = (t & ~12) | ((t & 4) << 1) | ((t & 8) >> 1)
    at_v = 16 * d + ((((c // 32) * 2 + s // 8) * 16 + c % 16) * 16 + ((c // 16) % 2) * 8 + s % 8)
    for rot in (0, 16, 10):  # 10: not made of whole units
        pool = kp.Pool(1, 32, 1, d, dtype=kp.KVP_FP8_E4M3)
        pool.set_scales(0, scale, scale)
        if rot:
            kp.kv_append_rope(pool, 0, kp.Rope(rot, interleaved=True), k, v, bt, [0], [0, 512])
        else:
            kp.kv_append(pool, 0, k, v, bt, [0], [0, 512])
        raw = pool.layer_bytes(0).cpu().numpy().reshape(32, 2 * 16 * d)
        got_k = raw[:, at_k].reshape(512, d)
        assert np.array_equal(got_k[:, rot:], want_k.reshape(512, d)[:, rot:])
        assert np.array_equal(raw[:, at_v].reshape(512, d), want_v.reshape(512, d))
        pool.close()


@pytest.mark.parametrize("n", [128, 129, 170, 171, 192, 256, 257, 320])
@pytest.mark.parametrize("Hq,Hkv,d", [(2, 2, 64), (4, 2, 128), (4, 1, 64), (16, 1, 128)])
def test_linear_lengths_around_the_cuts(n, Hq, Hkv, d):
    """Whether a sequence is cut depends on its length and the heads; the size asked for covers all, and no more of the
    workspace is written."""
    import torch
    note(f"linear cuts {n} {Hq}/{Hkv} {d}")
    c = Case([n, 5], Hq, Hkv, d)
    size = kp.linear_chunk_workspace_size(c.cu, Hkv, d)
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    want, room = c.oracle([0, 1], [0, 1], d ** -0.5)
    out = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, [0, 1], [0, 1], c.cu, ws=ws[:size] if size else None)
    check(out, c.state, want, room, c, [0, 1])
    assert bool((ws[size:] == 77).all())
    if n > 128 and Hq // Hkv == 16:
        with pytest.raises(kp.KvpError) as e:
            kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, [0, 1], [0, 1], c.cu, ws=ws[:size - 1])
        assert e.value.code == kp.KVP_EWORKSPACE


def test_two_streams_at_once():
    """Calls on two streams, enqueued in turn without waiting: each as if it were alone."""
    import torch
    note("two streams")
    lens = [[300, 40, 1], [17, 500]]
    cases = [Case(n, 4, 2, 64, seed=i) for i, n in enumerate(lens)]
    alone = []
    for c in cases:
        state = c.state.clone()
        i = list(range(len(c.lens)))
        alone.append(([kp.linear_chunk_attn(c.q, c.k, c.v, state, c.decay, i, i, c.cu) for _ in range(6)], state))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(6):
        for s, c, g in zip(streams, cases, got):
            i = list(range(len(c.lens)))
            g.append(kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, i, i, c.cu, stream=s))
    torch.cuda.synchronize()
    for (outs, state), c, g in zip(alone, cases, got):
        assert all(torch.equal(a, b) for a, b in zip(outs, g)) and torch.equal(state, c.state)


@pytest.mark.parametrize("lens", [[1000], [2048, 70], [2049], [2600, 2200], [4160]])
@pytest.mark.parametrize("Hq,Hkv,d,src", [(1, 1, 64, 0), (4, 2, 128, 0), (2, 1, 64, -1)])
def test_linear_numbers_of_parts(lens, Hq, Hkv, d, src):
    """16 to 65 parts of 64 tokens: every way that the states between them are summed."""
    import torch
    note(f"linear parts {lens} {Hq}/{Hkv} {d} {src}")
    c = Case(lens, Hq, Hkv, d, decay=[0.9997, 1.0][:Hkv])
    slots = list(range(len(lens)))
    want, room = c.oracle(slots if src == 0 else [-1] * len(lens), slots, d ** -0.5)
    out = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, slots if src == 0 else [-1] * len(lens), slots, c.cu,
                               out_dtype=torch.float32)
    check(out, c.state, want, room, c, slots)


def test_append_rope_refuses_more_heads_than_its_indices_hold():
    import torch
    note("append rope heads")
    Hq, Hkv, d = (1 << 20) + 16, 16, 64
    q = torch.zeros(1, Hq, d, dtype=torch.bfloat16, device="cuda")
    k = torch.ones(1, Hkv, d, dtype=torch.bfloat16, device="cuda")
    pool = kp.Pool(1, 2, Hkv, d)
    bt = torch.tensor([[1]], dtype=torch.int32, device="cuda")
    with pytest.raises(kp.KvpError) as e:
        kp.kv_append_rope(pool, 0, kp.Rope(64), k, k, bt, [0], [0, 1], q=q)
    assert e.value.code == kp.KVP_EUNSUPPORTED and not bool(pool.layer_raw().any())
    got = kp.kv_append_rope(pool, 0, kp.Rope(64), k, k, bt, [3], [0, 1], q=torch.ones_like(q[:, :1 << 20]))
    one = kp.kvp_rope_apply(kp.Rope(64), torch.ones_like(q[:, :1]), torch.tensor([3], dtype=torch.int32, device="cuda"))
    assert torch.equal(got, one.expand_as(got))
    pool.close()


def test_linear_more_sequences_than_one_launch_holds():
    """70000 sequences of 128 heads, 211 of them with a token: out = scale (q . k) v."""
    import torch
    note("linear many sequences")
    B, H, d = 70000, 128, 64
    lens = np.zeros(B, np.int32)
    lens[np.random.default_rng(2).choice(B, 210, replace=False)] = 1
    lens[-1] = 1
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T = int(cu[-1])
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(T, H, d, generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    state = torch.zeros(1, H, d, d, device="cuda")
    none = np.full(B, -1, np.int32)
    out = kp.linear_chunk_attn(q, k, v, state, np.full(H, 0.5), none, none, cu, scale=0.25, out_dtype=torch.float32)
    a, b, c = (t.cpu().double().numpy() for t in (q, k, v))
    want = 0.25 * (a * b).sum(-1, keepdims=True) * c
    room = 0.25 * (np.abs(a) * np.abs(b)).sum(-1, keepdims=True) * np.abs(c)
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -16 * room)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("seqs", [200, 270])  # 4 and 8 query heads a wave, interleaved
@pytest.mark.parametrize("Hq", [32, 40])
def test_append_rope_of_many_runs(interleaved, seqs, Hq):
    import torch
    note(f"append rope many {interleaved} {seqs} {Hq}")
    Hkv, d = 8, 64
    g = torch.Generator().manual_seed(seqs)
    start = np.arange(seqs, dtype=np.int32) * 7
    new = np.where(np.arange(seqs) % 9 == 0, 17, 1)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1])
    pos = torch.from_numpy(np.concatenate([np.arange(s, s + n) for s, n in zip(start, new)]).astype(np.int32)).cuda()
    q, k, v = (torch.randn(T, h, d, generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
    maxp = (int(start[-1]) + 17 + 15) // 16
    bt = torch.full((seqs, maxp), -1, dtype=torch.int32)
    pages = 0
    for i in range(seqs):
        for p in range(start[i] // 16, (start[i] + new[i] - 1) // 16 + 1):
            bt[i, p] = pages
            pages += 1
    bt = bt.cuda()
    rope = kp.Rope(32, interleaved=interleaved)
    a, b = kp.Pool(1, pages, Hkv, d), kp.Pool(1, pages, Hkv, d)
    got = kp.kv_append_rope(a, 0, rope, k, v, bt, start, cu, q=q)
    kp.kv_append(b, 0, kp.kvp_rope_apply(rope, k, pos), v, bt, start, cu)
    assert torch.equal(got, kp.kvp_rope_apply(rope, q, pos))
    assert torch.equal(a.layer_raw(), b.layer_raw())
    assert a.device_error() == kp.KVP_OK
    a.close(), b.close()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,d,rot", [(3001, 13, 128, 128), (9001, 30, 128, 64), (20011, 31, 72, 48), (300, 1000, 64, 64)])
def test_rope_of_large_calls_equals_small_ones(T, H, d, rot, interleaved, dt):
    """Calls that give a thread two or four heads: the bits of one-head calls, in place and with the gradient's sign."""
    import torch
    note(f"rope large calls {T} {H} {d} {rot} {interleaved} {dt}")
    g = torch.Generator(device="cuda").manual_seed(T)
    whole = torch.randn(T, H + 3, d, generator=g, device="cuda").to(torch.bfloat16 if dt == "bf16" else torch.float32)
    x = whole[:, 1:H + 1]
    pos = torch.randint(-5000, 1 << 20, (T,), generator=g, device="cuda", dtype=torch.int32)
    rope = kp.Rope(rot, interleaved=interleaved, magnitude=1.25)
    rest = whole[:, [0, H + 1, H + 2]].clone()
    want = torch.empty(T, H, d, dtype=x.dtype, device="cuda")
    for h in range(0, H, max(1, H // 7)):
        for t in range(0, T, 5000):
            want[t:t + 5000, h:h + 1] = kp.kvp_rope_apply(rope, x[t:t + 5000, h:h + 1], pos[t:t + 5000], grad=True)
    got = kp.kvp_rope_apply(rope, x, pos, grad=True)
    heads = list(range(0, H, max(1, H // 7)))
    assert torch.equal(got[:, heads], want[:, heads])
    kp.kvp_rope_apply(rope, x, pos, out=x, grad=True)
    assert torch.equal(x, got) and torch.equal(whole[:, [0, H + 1, H + 2]], rest)


@pytest.mark.parametrize("lens,Hq,Hkv,d", [([100, 60, 7], 16, 1, 128), ([128, 1], 64, 4, 64), ([300, 300, 300], 32, 2, 64)])
def test_linear_in_place_every_time_the_same(lens, Hq, Hkv, d):
    """Workgroups that share a sequence's query heads all read the state that one of them replaces."""
    import torch
    note(f"linear in place {lens} {Hq}/{Hkv} {d}")
    c = Case(lens, Hq, Hkv, d)
    i = list(range(len(lens)))
    before = c.state.clone()
    want, room = c.oracle(i, i, d ** -0.5)
    first = None
    for rep in range(25):
        c.state.copy_(before)
        out = kp.linear_chunk_attn(c.q, c.k, c.v, c.state, c.decay, i, i, c.cu)
        if first is None:
            first = out, c.state.clone()
            check(out, c.state, want, room, c, i)
        assert torch.equal(out, first[0]) and torch.equal(c.state, first[1])


@pytest.mark.parametrize("slots", [1300, 32768, 32769, 40000])
def test_linear_decode_slots_of_16_bits_and_more(slots):
    """1290 sequences in several launches; the first and the last slots among them."""
    import torch
    note(f"linear decode slots {slots}")
    B, Hq, Hkv, d = 1290, 2, 1, 64
    c = Case([1] * B, Hq, Hkv, d, slots=4)
    rng = np.random.default_rng(slots)
    state = torch.zeros(slots, Hkv, d, d, device="cuda")
    used = rng.permutation(np.concatenate([[0, slots - 1], 1 + rng.choice(slots - 2, B - 2, replace=False)]))
    src, dst = used.copy(), used.copy()
    src[::7], dst[3::11] = -1, -1
    at = torch.from_numpy(used).cuda()
    state[at] = torch.randn(B, Hkv, d, d, generator=torch.Generator().manual_seed(1)).cuda()
    c.state = state[at].clone()
    small = [np.where(s < 0, -1, np.arange(B)) for s in (src, dst)]
    want, room = c.oracle(*small, 0.5)
    untouched = torch.ones(slots, dtype=torch.bool, device="cuda")
    untouched[at] = False
    out = kp.linear_decode_attn(c.q, c.k, c.v, state, c.decay, src, dst, scale=0.5)
    check(out, state[at], want, room, c, small[1])
    assert not bool(state[untouched].any())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
def test_append_rope_of_rows_that_are_streamed(interleaved, fp8):
    """135 MB of rows at a fused projection's stride."""
    import torch
    note(f"append rope streamed {interleaved} {fp8}")
    Hq, Hkv, d = 32, 16, 128
    start, new = np.asarray([5, 0, 9], np.int32), [4099, 4300, 1]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1])
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(T, Hq + 2 * Hkv, d, generator=g, device="cuda").to(torch.bfloat16)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    pos = torch.from_numpy(np.concatenate([np.arange(s, s + n) for s, n in zip(start, new)]).astype(np.int32)).cuda()
    maxp = 270
    bt = torch.randperm(3 * maxp, generator=torch.Generator().manual_seed(5)).to(torch.int32).view(3, maxp).cuda()
    rope = kp.Rope(64, interleaved=interleaved)
    pools = [kp.Pool(1, 3 * maxp, Hkv, d, dtype=kp.KVP_FP8_E4M3 if fp8 else kp.KVP_BF16) for _ in range(2)]
    got = kp.kv_append_rope(pools[0], 0, rope, k, v, bt, start, cu, q=q)
    assert torch.equal(got, kp.kvp_rope_apply(rope, q, pos))
    for i in range(3):  # the same, sequence by sequence: rows that are not streamed
        lo, hi = int(cu[i]), int(cu[i + 1])
        kp.kv_append_rope(pools[1], 0, rope, k[lo:hi], v[lo:hi], bt[i:i + 1], start[i:i + 1], [0, hi - lo])
    a, b = (p.layer_bytes() if fp8 else p.layer_raw() for p in pools)
    assert torch.equal(a, b) and bool(a.any())
    for p in pools:
        p.close()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_of_rows_that_are_streamed(interleaved):
    import torch
    note(f"rope streamed {interleaved}")
    T, H, d = 17003, 33, 128
    x = torch.randn(T, H, d, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 7
    rope = kp.Rope(96, interleaved=interleaved)
    got = kp.kvp_rope_apply(rope, x, pos)
    for t in range(0, T, 4000):
        assert torch.equal(got[t:t + 4000], kp.kvp_rope_apply(rope, x[t:t + 4000], pos[t:t + 4000]))
