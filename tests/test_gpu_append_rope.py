"""kv_append_rope: the bits of kvp_rope_apply followed by kv_append (bf16 pages), the 64-bit oracle (FP8 pages), every
run shape inside a page, strides, refusals; and a session's steps with the attention that reads its pages."""
import numpy as np
import pytest

from gpu_helpers import assert_close, note
from oracle import rotary
from paper_2608_11152_amd import kvpattn as kp

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def make(start, new, Hq, Hkv, d, fused=False, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    T = int(sum(new))
    x = torch.randn(T, Hq + 2 * Hkv, d, generator=g).to(torch.bfloat16).cuda()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    maxp = max((s + n + 15) // 16 for s, n in zip(start, new)) + 1
    pages = len(start) * maxp + 3
    bt = torch.randperm(pages, generator=g).to(torch.int32)[:len(start) * maxp].view(len(start), maxp).cuda()
    pos = np.concatenate([np.arange(s, s + n) for s, n in zip(start, new)] + [np.zeros(0)]).astype(np.int32)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return q, k, v, bt, pages, torch.from_numpy(pos).cuda(), np.asarray(start, np.int32), cu


RUNS = [([0], [1]), ([15], [1]), ([7], [9]), ([3], [40]), ([16], [16]), ([0, 5, 31, 100], [1, 0, 2, 33]),
        ([1000, 17], [1, 1]), (list(range(20)), [1] * 20), ([0], [300])]


@pytest.mark.parametrize("start,new", RUNS)
@pytest.mark.parametrize("Hq,Hkv,d,rot,interleaved", [
    (8, 2, 64, 64, False), (32, 4, 128, 128, False), (4, 4, 128, 64, True), (16, 1, 128, 32, False), (2, 1, 64, 20, False),
    (5 * 8, 8, 64, 16, True), (3, 3, 128, 6, True), (16, 16, 128, 128, True)])
def test_bf16_pages_equal_rotation_then_append(start, new, Hq, Hkv, d, rot, interleaved):
    import torch
    note(f"append rope {start[:4]} {new[:4]} {Hq}/{Hkv} d={d} rot={rot} il={interleaved}")
    q, k, v, bt, pages, pos, sp, cu = make(start, new, Hq, Hkv, d, fused=rot != 64)
    rope = kp.Rope(rot, interleaved=interleaved, factor=2.0, original_len=512, high_turns=4.0)
    a, b = kp.Pool(1, pages, Hkv, d), kp.Pool(1, pages, Hkv, d)
    for pool in (a, b):
        pool.layer_raw().copy_(torch.arange(pool.layer_raw().numel(), device="cuda") % 32749)  # what is not written stays
    want_q = kp.kvp_rope_apply(rope, q, pos)
    kp.kv_append(b, 0, kp.kvp_rope_apply(rope, k, pos), v.contiguous(), bt, sp, cu)
    got_q = kp.kv_append_rope(a, 0, rope, k, v, bt, sp, cu, q=q)
    assert torch.equal(got_q, want_q)
    assert torch.equal(a.layer_raw(), b.layer_raw())
    assert a.device_error() == kp.KVP_OK
    a.close(), b.close()


@pytest.mark.parametrize("start,new", [([7], [9]), ([0, 5, 31, 100], [1, 0, 2, 33]), ([15], [1])])
@pytest.mark.parametrize("Hkv,d,rot,interleaved", [(2, 64, 64, False), (4, 128, 64, True), (1, 128, 128, False), (3, 64, 10, True)])
def test_fp8_pages_against_oracle(start, new, Hkv, d, rot, interleaved):
    """Rounded once from fp32 to E4M3.  Tolerance: half a step of E4M3 (2^-4 of the value, 2^-10 below its normal range) in
    units of the scale, the bf16 of kv_gather (2^-8 of the value), fp32 (8 steps of the pair, scale included)."""
    import torch
    note(f"append rope fp8 {start} {new} {Hkv} {d} {rot}")
    q, k, v, bt, pages, pos, sp, cu = make(start, new, Hkv, Hkv, d)
    k[0, 0, 1] = 300.0  # beyond 448 scales: saturates
    rope = kp.Rope(rot, interleaved=interleaved)
    pool = kp.Pool(1, pages, Hkv, d, dtype=kp.KVP_FP8_E4M3)
    ks, vs = 0.37, 0.05
    pool.set_scales(0, ks, vs)
    same = kp.Pool(1, pages, Hkv, d, dtype=kp.KVP_FP8_E4M3)
    same.set_scales(0, ks, vs)
    kp.kv_append_rope(pool, 0, rope, k, v, bt, sp, cu)
    kp.kv_append(same, 0, k, v, bt, sp, cu)
    lens = [s + n for s, n in zip(start, new)]
    gk, gv = kp.kv_gather(pool, 0, bt, lens)
    _, wv = kp.kv_gather(same, 0, bt, lens)
    assert torch.equal(gv, wv)  # values are stored as kv_append stores them
    at = np.concatenate([[0], np.cumsum(lens)])
    rows = np.concatenate([np.arange(at[i] + s, at[i] + s + n) for i, (s, n) in enumerate(zip(start, new))])
    got = f64(gk)[rows]
    want = rotary.rotate(f64(k), pos.cpu().numpy(), rotary.frequencies(rot), interleaved)
    clipped = np.clip(want, -448.0 * ks, 448.0 * ks)
    tol = (2.0 ** -4 + 2.0 ** -8 + 2.0 ** -12) * np.abs(clipped) + 2.0 ** -10 * ks + 8 * 2.0 ** -24 * 2 * np.abs(f64(k)).max(-1, keepdims=True)
    assert np.all(np.abs(got - clipped) <= tol)
    assert np.all(np.delete(f64(gk), rows, axis=0) == 0.0)
    pool.close(), same.close()


def test_bf16_pages_against_oracle():
    import torch
    note("append rope oracle")
    q, k, v, bt, pages, pos, sp, cu = make([3, 131000 % 4096], [50, 7], 8, 2, 128)
    pool = kp.Pool(1, pages, 2, 128)
    kp.kv_append_rope(pool, 0, kp.Rope(128, base=500000.0), k, v, bt, sp, cu)
    lens = [53, int(sp[1]) + 7]
    gk, gv = kp.kv_gather(pool, 0, bt, lens)
    rows = np.concatenate([np.arange(3, 53), np.arange(53 + int(sp[1]), 53 + int(sp[1]) + 7)])
    want = rotary.rotate(f64(k), pos.cpu().numpy(), rotary.frequencies(128, 500000.0))
    a = np.abs(f64(k))
    pair = np.concatenate([a[..., :64] + a[..., 64:]] * 2, axis=-1)
    assert np.all(np.abs(f64(gk)[rows] - want) <= 2.0 ** -8 * np.abs(want) + 8 * 2.0 ** -24 * pair)
    assert torch.equal(gv[torch.from_numpy(rows).cuda()], v)
    pool.close()


def test_queries_in_place_in_a_fused_row_and_an_output_of_their_own():
    import torch
    note("append rope in place")
    Hq, Hkv, d, T = 8, 2, 64, 21
    x = torch.randn(T, Hq + 2 * Hkv, d, device="cuda").to(torch.bfloat16)
    keep = x.clone()
    bt = torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4)
    pool = kp.Pool(1, 4, Hkv, d)
    rope = kp.Rope(d)
    pos = torch.arange(5, 5 + T, dtype=torch.int32, device="cuda")
    want = kp.kvp_rope_apply(rope, keep[:, :Hq], pos)
    out = torch.full((T + 3, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    assert kp.kv_append_rope(pool, 0, rope, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], bt, [5], [0, T], q=x[:, :Hq], q_out=out) is out
    assert torch.equal(out[:T], want) and bool((out[T:] == 7.0).all()) and torch.equal(x, keep)
    q = x[:, :Hq]
    kp.kv_append_rope(pool, 0, rope, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], bt, [5], [0, T], q=q, q_out=q)
    assert torch.equal(x[:, :Hq], want) and torch.equal(x[:, Hq:], keep[:, Hq:])
    assert kp.kv_append_rope(pool, 0, rope, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], bt, [5], [0, T]) is None
    pool.close()


def test_refusals_leave_everything():
    import torch
    note("append rope refusals")
    Hkv, d, T = 2, 64, 4
    pool = kp.Pool(2, 8, Hkv, d)
    bt = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    x = torch.randn(T, Hkv, d, device="cuda").to(torch.bfloat16)
    rope = kp.Rope(d)
    ok = dict(start_pos=[0, 16], cu_new=[0, 2, 4])

    def refused(code, k=x, v=x, layer=0, r=rope, **kw):
        with pytest.raises(kp.KvpError) as e:
            kp.kv_append_rope(pool, layer, r, k, v, bt, **{**ok, **kw})
        assert e.value.code == code

    refused(kp.KVP_EINVAL, layer=2)
    refused(kp.KVP_EINVAL, r=kp.Rope(66))
    refused(kp.KVP_ERANGE, start_pos=[0, 63])
    refused(kp.KVP_EINVAL, start_pos=[0, -1])
    refused(kp.KVP_EINVAL, cu_new=[0, 5, 4])
    refused(kp.KVP_EINVAL, cu_new=[1, 2, 4])
    refused(kp.KVP_ESHARED, group_prefix=kp.group_prefix([0, 0], [1]))
    refused(kp.KVP_EUNSUPPORTED, q=torch.zeros(T, 3, d, dtype=torch.bfloat16, device="cuda"))
    odd = torch.zeros(T, Hkv * d + 4, dtype=torch.bfloat16, device="cuda")
    refused(kp.KVP_EINVAL, k=odd[:, :Hkv * d].unflatten(1, (Hkv, d)))
    refused(kp.KVP_EINVAL, v=torch.zeros(T * Hkv * d + 1, dtype=torch.bfloat16, device="cuda")[1:].view(T, Hkv, d))
    q = torch.zeros(T, 4, d, dtype=torch.bfloat16, device="cuda")
    refused(kp.KVP_EINVAL, q=q, q_out=torch.as_strided(q, (T, 4, d), (64, d, 1)))
    for bad in (dict(k=x.float()), dict(k=x[:, :1]), dict(k=x[:3]), dict(k=x.transpose(0, 1).contiguous().transpose(0, 1)),
                dict(q_out=q), dict(q=q[:, :, :32])):
        with pytest.raises(ValueError):
            kp.kv_append_rope(pool, 0, rope, bad.pop("k", x), x, bt, **ok, **bad)
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    keep = torch.zeros(4, device="cuda")
    with torch.cuda.graph(g, stream=s):
        keep.add_(1.0)
        refused(kp.KVP_EHIP, stream=s)
    g.replay()
    torch.cuda.synchronize()
    assert not bool(pool.layer_raw(0).any()) and not bool(pool.layer_raw(1).any())
    assert kp.kv_append_rope(pool, 0, rope, x[:0], x[:0], bt[:0], [], [0]) is None
    kp.kv_append_rope(pool, 0, rope, x, x, bt, [0, 0], [0, 0, 0])  # no tokens
    torch.cuda.synchronize()
    assert not bool(pool.layer_raw(0).any())
    pool.close()


def test_a_page_outside_the_pool_is_skipped_and_reported():
    import torch
    note("append rope bad page")
    Hkv, d = 2, 64
    pool = kp.Pool(1, 4, Hkv, d)
    bt = torch.tensor([[0, 9], [-1, 1]], dtype=torch.int32, device="cuda")
    x = torch.randn(36, Hkv, d, device="cuda").to(torch.bfloat16)
    q = torch.randn(36, 4, d, device="cuda").to(torch.bfloat16)
    rope = kp.Rope(d)
    out = kp.kv_append_rope(pool, 0, rope, x, x, bt, [0, 14], [0, 18, 36], q=q)
    assert pool.device_error() == kp.KVP_ERANGE and pool.device_error() == kp.KVP_OK
    pos = torch.cat([torch.arange(0, 18), torch.arange(14, 32)]).to(torch.int32).cuda()
    assert torch.equal(out, kp.kvp_rope_apply(rope, q, pos))
    k, _ = kp.kv_gather(pool, 0, torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), [32])
    want = kp.kvp_rope_apply(rope, x, pos)
    assert torch.equal(k[:16], want[:16]) and torch.equal(k[16:], want[20:])
    pool.close()


@pytest.mark.parametrize("layer_dtype", ["bf16", "fp8"])
def test_a_session_s_steps(layer_dtype):
    """Two prompts that share pages, a chunk prefilled over each history and decode steps, all through rotated appends:
    against the oracle on keys and queries rotated in 64 bits."""
    import torch
    note(f"append rope session {layer_dtype}")
    Hq, Hkv, d, maxp = 8, 2, 64, 16
    dt = kp.KVP_FP8_E4M3 if layer_dtype == "fp8" else kp.KVP_BF16
    pool = kp.Pool(2, 40, Hkv, d, dtype=dt)
    if dt == kp.KVP_FP8_E4M3:
        pool.set_scales(1, 0.02, 0.02)
    rope, freq = kp.Rope(d, base=1000.0), rotary.frequencies(d, 1000.0)
    rng = np.random.default_rng(5)
    perm = rng.permutation(40).astype(np.int32)
    bt = np.stack([np.concatenate([perm[:4], perm[4:16]]), np.concatenate([perm[:4], perm[16:28]])])
    btd = torch.from_numpy(bt).cuda()
    hist = [[], []]  # per sequence: (rotated k, v) float64 rows
    gp = kp.group_prefix([0, 0], [4])

    def values(n, h):
        return torch.from_numpy(rng.normal(size=(n, h, d)).astype(np.float32)).to(torch.bfloat16).cuda()

    def keep(i, k, v, pos):
        hist[i] += list(zip(rotary.rotate(f64(k), pos, freq), f64(v)))

    def stored(i):
        k, v = (np.stack([r[j] for r in hist[i]]) for j in (0, 1))
        return k, v

    def attend(i, q, last, pos):
        k, v = stored(i)
        q = rotary.rotate(f64(q), pos, freq)
        out = np.empty(q.shape)
        for r in range(q.shape[0]):
            for h in range(Hq):
                s = k[:last[r] + 1, h // 4] @ q[r, h] / np.sqrt(d)
                w = np.exp(s - s.max())
                out[r, h] = (w / w.sum()) @ v[:last[r] + 1, h // 4]
        return out

    k, v = values(64, Hkv), values(64, Hkv)  # the shared prompt: four whole pages
    kp.kv_append_rope(pool, 1, rope, k, v, btd[:1], [0], [0, 64])
    for i in (0, 1):
        keep(i, k, v, np.arange(64))
    k, v, q = values(42, Hkv), values(42, Hkv), values(42, Hq)
    qr = kp.kv_append_rope(pool, 1, rope, k, v, btd, [64, 64], [0, 37, 42], q=q, group_prefix=gp)
    out = kp.prefix_chunk_prefill_attn(qr, pool, 1, btd, [64, 64], [0, 37, 42])
    keep(0, k[:37], v[:37], np.arange(64, 101))
    keep(1, k[37:], v[37:], np.arange(64, 69))
    want = np.concatenate([attend(0, q[:37], np.arange(64, 101), np.arange(64, 101)),
                           attend(1, q[37:], np.arange(64, 69), np.arange(64, 69))])
    # bf16: the repository's tolerance.  FP8 pages hold k and v to half a step of E4M3, 2^-4: scores of |s| <= 6 or so
    # move by up to 2^-4 |s| / sqrt(d) a term at random, outputs by 2^-4 of the largest value
    tol = dict(max_abs=1e-2, mean_abs=1e-3) if layer_dtype == "bf16" else dict(max_abs=0.25, mean_abs=0.02)
    assert_close(out, want, "prefill", **tol)
    lens = [101, 69]
    for step in range(3):
        k, v, q = values(2, Hkv), values(2, Hkv), values(2, Hq)
        qr = kp.kv_append_rope(pool, 1, rope, k, v, btd, lens, [0, 1, 2], q=q, group_prefix=gp)
        for i in (0, 1):
            keep(i, k[i:i + 1], v[i:i + 1], [lens[i]])
        lens = [x + 1 for x in lens]
        out = kp.paged_decode_attn(qr, pool, 1, btd, lens, group_prefix=gp)
        want = np.concatenate([attend(i, q[i:i + 1], [lens[i] - 1], [lens[i] - 1]) for i in (0, 1)])
        assert_close(out, want, f"decode {step}", **tol)
    assert pool.device_error() == kp.KVP_OK and not bool(pool.layer_bytes(0).any())
    pool.close()
