"""kv_append_rope where a call's heads, tokens and positions are at their ends."""
import numpy as np
import pytest

from gpu_helpers import note
from paper_2608_11152_amd import kvpattn as kp

pytestmark = pytest.mark.gpu


def test_more_heads_times_tokens_than_one_launch_holds():
    """65 single tokens of 2^20 query heads, a wave each: more than 2^26 waves, cut into launches."""
    import torch
    note("append rope many waves")
    B, Hq, Hkv, d = 65, 1 << 20, 16, 64
    g = torch.Generator(device="cuda").manual_seed(8)
    q = torch.empty(B, Hq, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    k, v = (torch.randn(B, Hkv, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    start = np.arange(B, dtype=np.int32) * 3
    pos = torch.from_numpy(start).cuda()
    maxp = 13
    bt = torch.randperm(B * maxp, generator=torch.Generator().manual_seed(9)).to(torch.int32).view(B, maxp).cuda()
    rope = kp.Rope(10)
    a, b = (kp.Pool(1, B * maxp, Hkv, d) for _ in range(2))
    cu = np.arange(B + 1, dtype=np.int32)
    got = kp.kv_append_rope(a, 0, rope, k, v, bt, start, cu, q=q)
    kp.kv_append(b, 0, kp.kvp_rope_apply(rope, k, pos), v, bt, start, cu)
    assert torch.equal(a.layer_raw(), b.layer_raw()) and bool(a.layer_raw().any())
    want = kp.kvp_rope_apply(rope, q, pos, out=q)
    assert torch.equal(got, want)
    a.close(), b.close()


def test_positions_beyond_31_bits_are_refused():
    """A row of 2^27 pages and more holds positions that kvp_rope_apply's do not reach; its table is never read."""
    import torch
    note("append rope far positions")
    lib, rope = kp.lib(), kp.Rope(64)
    pool = kp.Pool(1, 2, 1, 64)
    x = torch.ones(4, 1, 64, dtype=torch.bfloat16, device="cuda")
    bt = torch.zeros(1, dtype=torch.int32, device="cuda")
    cu = np.asarray([0, 4], np.int32)

    def call(start):
        sp = np.asarray([start], np.int32)
        return lib.kv_append_rope(pool.handle, 0, rope.ref(), x.data_ptr(), 64, x.data_ptr(), 64, None, 0, None, 0, 0,
                                  bt.data_ptr(), 1 << 28, sp.ctypes.data, cu.ctypes.data, 1, None, None)

    for start in (2 ** 31 - 1, 2 ** 31 - 3):
        assert call(start) == kp.KVP_ERANGE
    torch.cuda.synchronize()
    assert not bool(pool.layer_raw().any()) and pool.device_error() == kp.KVP_OK
    pool.close()


class Elsewhere:
    """A tensor that says it is on the second device."""

    def __init__(self, t):
        self.t, self.is_cuda, self.device = t, True, "cuda:1"

    def get_device(self):
        return 1

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_tensors_of_another_device_are_refused():
    import torch
    note("append rope another device")
    rope, pool = kp.Rope(64), kp.Pool(1, 4, 2, 64)
    x = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    bt = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    state = torch.zeros(1, 2, 64, 64, device="cuda")
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    far = Elsewhere
    calls = [lambda: kp.kv_append_rope(pool, 0, rope, x, x, far(bt), [0], [0, 3]),
             lambda: kp.kv_append_rope(pool, 0, rope, far(x), x, bt, [0], [0, 3]),
             lambda: kp.kv_append_rope(pool, 0, rope, x, x, bt, [0], [0, 3], q=x, q_out=far(x)),
             lambda: kp.kvp_rope_apply(rope, x, far(pos)),
             lambda: kp.kvp_rope_apply(rope, x, pos, out=far(x)),
             lambda: kp.linear_chunk_attn(x, x, x, state, [1.0, 1.0], [0], [0], [0, 3], ws=far(ws)),
             lambda: kp.linear_chunk_attn(x, x, x, far(state), [1.0, 1.0], [0], [0], [0, 3]),
             lambda: kp.linear_decode_attn(x[:1], x[:1], far(x[:1]), state, [1.0, 1.0], [0], [0])]
    for call in calls:
        with pytest.raises(ValueError, match="device|is on"):
            call()
    torch.cuda.synchronize()
    assert not bool(pool.layer_raw().any()) and not bool(state.any())
    pool.close()
