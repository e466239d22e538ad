"""The operators around a rollout session's cache: rotary positions, the append that rotates on the way, and linear
attention over a state per session, each in plain torch (`own` false) and through this library (`own` true).

The listed cases are calls of a serving engine for mixed RL rollouts, at the session counts, lengths and head shapes of
workloads.py and bench.py; draw() gives more of the same ranges.  Lengths and heads belong to a case; page placement,
positions and values come from the seed.  q, k, v ~ N(0, 1) in bf16, as in workloads.py.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

from paper_2608_11152_amd import kvpattn as kp

own = False

PAGE = 16
PLAIN_CHUNK = 128  # tokens per chunk of the plain linear attention
EXACT_BLOCK = 256  # tokens per block of its 64-bit form


# --------------------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------------------

ROPE = {"rot": 128, "interleaved": False, "base": 10000.0, "factor": 1.0, "orig": 0, "low": 1.0, "high": 32.0,
        "magnitude": 1.0}


def _rope(name, **kw):
    c = {"name": name, "op": "rope", "dtype": "bf16", "tokens": 1, "heads": 32, "gap": 0, "d": 128, "max_pos": 131072,
         "grad": False, **ROPE}
    c.update(kw)
    return c


def _append(name, **kw):
    c = {"name": name, "op": "append", "kv": "bf16", "hq": 32, "hkv": 4, "d": 128, "fused": True, "lens_seed": 1,
         "decodes": 0, "chunks": 0, "chunk_lo": 2048, "chunk_hi": 2048, "hist_lo": 1024, "hist_hi": 131072, **ROPE}
    c.update(kw)
    return c


def _chunk(name, **kw):
    c = {"name": name, "op": "chunk", "hq": 16, "hkv": 16, "d": 128, "fused": False, "lens_seed": 1, "seqs": 1, "lo": 1,
         "hi": 1, "fresh": True}
    c.update(kw)
    return c


def _token(name, **kw):
    c = {"name": name, "op": "token", "hq": 16, "hkv": 16, "d": 128, "groups": 1, "samples": 1, "fork": False}
    c.update(kw)
    return c


def listed():
    return [
        # Four sessions' queries, d = 64, 8 heads: the smallest call.
        _rope("rope_tiny", tokens=4, heads=8, d=64, rot=64, max_pos=256),
        # q and k heads of eight 2048-token turns, in place of a fused qkv row (36 of its 40 heads), frequencies scaled
        # for contexts beyond the 8192 tokens that the model was trained on.
        _rope("rope_turns", tokens=16384, heads=36, gap=4, base=500000.0, factor=16.0, orig=8192, high=4.0),
        # The gradient of fp32 queries in a training step over ragged packed samples: interleaved pairs in half of the head.
        _rope("rope_grad", tokens=5003, heads=32, dtype="f32", rot=64, interleaved=True, grad=True, max_pos=16384),
        # Four short sessions decode one token each, GQA 8/2, d = 64: the smallest append.
        _append("append_tiny", hq=8, hkv=2, d=64, rot=64, fused=False, decodes=4, hist_lo=16, hist_hi=255),
        # One token for each of 512 RLVR samples.
        _append("append_rlvr", decodes=512, hist_lo=1024, hist_hi=16384),
        # The mixed step: one token for most sessions, 2048-token chunks for eight, scaled frequencies.
        _append("append_step", decodes=32, chunks=8, base=500000.0, factor=4.0, orig=32768, magnitude=1.1386294361119891),
        # Ragged turns of middling sessions into an FP8 pool, interleaved pairs in half of the head.
        _append("append_ragged_fp8", kv="fp8", rot=64, interleaved=True, fused=False, chunks=6, chunk_lo=37, chunk_hi=1500,
                hist_lo=1000, hist_hi=24000),
        # Three short prompts, 8 query heads over 2 states, d = 64: the smallest chunk call.
        _chunk("chunk_tiny", hq=8, hkv=2, d=64, seqs=3, lo=1, hi=70),
        # First prefill of a batch of RLVR prompts: ragged, from empty states.
        _chunk("chunk_prompts", seqs=64, lo=128, hi=1024),
        # One agentic session's whole history after a weight sync: a single long sequence.
        _chunk("chunk_long", lo=131071, hi=131071, fresh=False),
        # Four sessions decode one token each: the smallest decode.
        _token("token_tiny", hq=8, hkv=2, d=64, groups=4),
        # The first token of 512 RLVR samples: each starts from its prompt's state and keeps its own.
        _token("token_rlvr", groups=64, samples=8, fork=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rope(rng, d):
    rot = rng.choice([d, d, d // 2, d // 4])
    far = rng.random() < 0.5
    return {"rot": rot, "interleaved": rng.random() < 0.4, "base": rng.choice([10000.0, 500000.0, 1000000.0]),
            "factor": rng.choice([2.0, 4.0, 8.0, 40.0]) if far else 1.0, "orig": rng.choice([0, 4096, 8192]) if far else 0,
            "high": rng.choice([4.0, 32.0]), "magnitude": 1.25 if far and rng.random() < 0.3 else 1.0}


def draw(rng):
    op = rng.choice(["rope", "append", "append", "chunk", "chunk", "token"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8, 16])
    hq = hkv * rng.choice([g for g in (1, 2, 4, 8, 16) if hkv * g <= 64])
    seed = rng.randrange(1 << 20)
    if op == "rope":
        f32 = rng.random() < 0.4
        heads = rng.choice([hq, hq + hkv])
        most = 16384 * 36 * 128 // (heads * d * (2 if f32 else 1))
        c = _rope("", dtype="f32" if f32 else "bf16", tokens=_log_int(rng, 1, min(65536, most)), heads=heads, d=d,
                  gap=rng.choice([0, hkv]), max_pos=_log_int(rng, 64, 1 << 20), grad=rng.random() < 0.4, **_draw_rope(rng, d))
    elif op == "append":
        chunk = _log_int(rng, 2, 2048)
        most = 16384 * 40 * 128 // ((hq + 2 * hkv) * d)  # tokens
        decodes = min(_log_int(rng, 1, 512), most // 2)
        c = _append("", kv=rng.choice(["bf16", "bf16", "fp8"]), hq=hq, hkv=hkv, d=d, fused=rng.random() < 0.5, lens_seed=seed,
                    decodes=decodes, chunks=rng.randrange(0, max(1, min(32, (most - decodes) // chunk)) + 1),
                    chunk_lo=max(1, int(chunk * rng.uniform(0.2, 1.0))), chunk_hi=chunk, hist_lo=1, hist_hi=65536,
                    **_draw_rope(rng, d))
    elif op == "chunk":
        n = _log_int(rng, 1, 32768)
        most = max(1, min(65536 * 32 * 128 // ((hq + hkv) * d * n), 262144 // n))
        c = _chunk("", hq=hq, hkv=hkv, d=d, fused=rng.random() < 0.5, lens_seed=seed, seqs=_log_int(rng, 1, min(96, most)),
                   lo=max(1, int(n * rng.uniform(0.2, 1.0))), hi=n, fresh=rng.random() < 0.5)
    else:
        samples = rng.choice([1, 2, 8])
        most = 8192 * 128 * 128 // (hkv * d * d * samples)
        c = _token("", hq=hq, hkv=hkv, d=d, groups=_log_int(rng, 1, max(1, min(512 // samples, most))), samples=samples,
                   fork=samples > 1 and rng.random() < 0.5)
    c.pop("name")
    return c


# --------------------------------------------------------------------------------------------------------
# structure of a case
# --------------------------------------------------------------------------------------------------------

def _appends(case):
    rng = random.Random(case["lens_seed"])
    new = [1] * case["decodes"] + [rng.randint(case["chunk_lo"], case["chunk_hi"]) for _ in range(case["chunks"])]
    return [_log_int(rng, case["hist_lo"], case["hist_hi"]) for _ in new], new


def _lens(case):
    rng = random.Random(case["lens_seed"])
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]


def _slots(case):
    """Source and destination slots of a decode step, and the slots of the state tensor: 5% of them are others' sessions.
    A fork reads the prompt's slot (one per group, behind the samples') and writes the sample's own."""
    B = case["groups"] * case["samples"]
    dst = np.arange(B, dtype=np.int32)
    src = B + dst // case["samples"] if case["fork"] else dst
    return src, dst, B + (case["groups"] if case["fork"] else 0) + 1 + B // 20


def _cu(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def _decay(hkv):
    """Rates of decay in a geometric row, from exp(-2^-0.5) at most to exp(-2^-8)."""
    return np.exp(-(2.0 ** (-8.0 * (np.arange(hkv) + 1) / hkv))).astype(np.float32)


# --------------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(gen, *shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)


def _qkv(case, tokens, gen):
    """q, k, v of the tokens: views of one fused projection's rows, or tensors of their own."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    x = _normal(gen, tokens, hq + 2 * hkv, d)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return (q, k, v) if case["fused"] else (q.contiguous(), k.contiguous(), v.contiguous())


def _tables(case, gen):
    """Only the pages that tokens land in matter: logical pages before them name any page of the pool."""
    start, new = _appends(case)
    first = [s // PAGE for s in start]
    count = [(s + n + PAGE - 1) // PAGE - f for s, n, f in zip(start, new, first)]
    pages = sum(count) + sum(count) // 4 + 8
    perm = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    bt = torch.randint(0, pages, (len(new), max(f + c for f, c in zip(first, count))), generator=gen, device="cuda",
                       dtype=torch.int32)
    at = 0
    for i, (f, c) in enumerate(zip(first, count)):
        bt[i, f:f + c] = perm[at:at + c]
        at += c
    return start, new, pages, bt


def _rope_of(case):
    """The rotation's handle, which a program makes once per model."""
    return kp.Rope(case["rot"], base=case["base"], interleaved=case["interleaved"], factor=case["factor"],
                   original_len=case["orig"], low_turns=case["low"], high_turns=case["high"], magnitude=case["magnitude"])


def prepare(case, seed):
    gen = _gen(seed)
    s = {"case": case}
    if case["op"] in ("rope", "append"):
        s["freq"] = torch.from_numpy(_frequencies(case)).cuda()
        if own:
            s["rope"] = _rope_of(case)
    if case["op"] == "rope":
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s["x"] = _normal(gen, case["tokens"], case["heads"] + case["gap"], case["d"], dtype=dt)[:, :case["heads"]]
        s["pos"] = torch.randint(0, case["max_pos"], (case["tokens"],), generator=gen, device="cuda", dtype=torch.int32)
    elif case["op"] == "append":
        start, new, pages, bt = _tables(case, gen)
        pool = kp.Pool(1, pages, case["hkv"], case["d"], dtype=kp.KVP_FP8_E4M3 if case["kv"] == "fp8" else kp.KVP_BF16)
        s["q"], s["k"], s["v"] = _qkv(case, sum(new), gen)
        s["view"] = (pool.layer_bytes().view(torch.float8_e4m3fn) if case["kv"] == "fp8"
                     else pool.layer_raw().view(torch.bfloat16))
        s["view"].owner = pool  # the view borrows the pool's memory: whoever holds the output keeps the pool
        s.update(pool=pool, bt=bt, start=np.asarray(start, dtype=np.int32), cu=_cu(new))
    elif case["op"] == "chunk":
        cu = _cu(_lens(case))
        B = len(cu) - 1
        s["q"], s["k"], s["v"] = _qkv(case, int(cu[-1]), gen)
        slots = B + 1 + B // 20
        s["state"] = _normal(gen, slots, case["hkv"], case["d"], case["d"], dtype=torch.float32)
        s["dst"] = torch.randperm(slots, generator=gen, device="cuda")[:B].to(torch.int32).cpu().numpy()
        s["src"] = np.full(B, -1, dtype=np.int32) if case["fresh"] else s["dst"]
        s.update(cu=cu, decay=_decay(case["hkv"]))
    else:
        src, dst, slots = _slots(case)
        case = {**case, "fused": False}
        s["q"], s["k"], s["v"] = _qkv(case, len(src), gen)
        s["state"] = _normal(gen, slots, case["hkv"], case["d"], case["d"], dtype=torch.float32)
        s.update(src=src, dst=dst, decay=_decay(case["hkv"]))
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        if op == "rope":
            return kp.kvp_rope_apply(s["rope"], s["x"], s["pos"], grad=s["case"]["grad"])
        if op == "append":
            q = kp.kv_append_rope(s["pool"], 0, s["rope"], s["k"], s["v"], s["bt"], s["start"], s["cu"], q=s["q"])
            return q, s["view"]
        if op == "chunk":
            out = kp.linear_chunk_attn(s["q"], s["k"], s["v"], s["state"], s["decay"], s["src"], s["dst"], s["cu"],
                                       out_dtype=torch.bfloat16)
            return out, s["state"]
        out = kp.linear_decode_attn(s["q"], s["k"], s["v"], s["state"], s["decay"], s["src"], s["dst"],
                                    out_dtype=torch.bfloat16)
        return out, s["state"]
    if op == "rope":
        return _plain_rope(s["case"], s["freq"], s["x"], s["pos"], s["case"]["grad"])
    if op == "append":
        return _plain_append(s)
    return _plain_chunk(s) if op == "chunk" else _plain_token(s)


# --------------------------------------------------------------------------------------------------------
# plain forms
# --------------------------------------------------------------------------------------------------------

def _frequencies(case):
    """Radians per position of each pair, in 64 bits: a table that a program makes once."""
    f = case["base"] ** (-2.0 * np.arange(case["rot"] // 2) / case["rot"])
    if case["orig"] == 0:
        return f / case["factor"]
    turns = case["orig"] * f / (2.0 * math.pi)
    keep = np.clip((turns - case["low"]) / (case["high"] - case["low"]), 0.0, 1.0)
    return (1.0 - keep) * f / case["factor"] + keep * f


def _plain_rope_f32(case, freq, x, pos, grad=False):
    """x [tokens, heads, d] rotated, in 32 bits; the angles in 64, since a far position times a frequency needs them."""
    angle = pos.double()[:, None] * freq[None, :]
    cos = (case["magnitude"] * torch.cos(angle)).float()[:, None, :]
    sin = (case["magnitude"] * torch.sin(angle)).float()[:, None, :]
    if grad:
        sin = -sin
    x = x.float()
    r = case["rot"]
    out = x.clone()
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        out[..., 0:r:2], out[..., 1:r:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        out[..., :r // 2], out[..., r // 2:r] = a * cos - b * sin, a * sin + b * cos
    return out


def _plain_rope(case, freq, x, pos, grad):
    return _plain_rope_f32(case, freq, x, pos, grad).to(x.dtype)


def _plain_append(s):
    case, d, hkv = s["case"], s["case"]["d"], s["case"]["hkv"]
    n = np.diff(s["cu"])
    row = torch.from_numpy(np.repeat(np.arange(len(n)), n)).cuda()
    pos = torch.from_numpy(np.repeat(s["start"] - s["cu"][:-1], n) + np.arange(s["cu"][-1])).cuda()
    q = _plain_rope(case, s["freq"], s["q"], pos, False)
    k = _plain_rope_f32(case, s["freq"], s["k"], pos)
    page, slot = s["bt"][row, pos // PAGE].long(), pos % PAGE
    z = (slot & ~12) | ((slot & 4) << 1) | ((slot & 8) >> 1)  # the slot of a token in a V block: bits 2 and 3 swapped
    T = len(pos)
    if case["kv"] == "fp8":  # the pool's scales are 1
        k8, v8 = (x.float().clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, s["v"]))
        pool = s["view"].view(torch.uint8).view(-1, hkv, 2, PAGE * d)
        kb, vb = pool[:, :, 0].view(-1, hkv, d // 64, 4, PAGE, 2, 8), pool[:, :, 1].view(-1, hkv, d // 32, 2, 16, 2, 8)
        kb[page, :, :, :, slot] = k8.reshape(T, hkv, d // 64, 2, 4, 8).transpose(3, 4)
        vb[page, :, :, z // 8, :, :, z % 8] = v8.reshape(T, hkv, d // 32, 2, 16).transpose(3, 4)
    else:
        pool = s["view"].view(-1, hkv, 2, PAGE * d)
        kb, vb = pool[:, :, 0].view(-1, hkv, d // 8, PAGE, 8), pool[:, :, 1].view(-1, hkv, d // 16, 2, 16, 8)
        kb[page, :, :, slot] = k.to(torch.bfloat16).view(T, hkv, d // 8, 8)
        vb[page, :, :, z // 8, :, z % 8] = s["v"].reshape(T, hkv, d // 16, 16)
    return q, s["view"]


def _plain_token(s):
    """S = decay S + k v^T, o = q S / sqrt(d), for one token of each session."""
    hq, hkv, d = (s["case"][x] for x in ("hq", "hkv", "d"))
    decay = torch.from_numpy(s["decay"]).cuda()
    src, dst = (torch.from_numpy(s[x]).cuda().long() for x in ("src", "dst"))
    new = s["state"][src] * decay[None, :, None, None] + s["k"].float()[..., :, None] * s["v"].float()[..., None, :]
    out = torch.matmul(s["q"].float().view(-1, hkv, hq // hkv, d), new) * (1.0 / math.sqrt(d))
    s["state"][dst] = new
    return out.view(-1, hq, d).to(torch.bfloat16), s["state"]


def _plain_chunk(s):
    """The sum over earlier tokens, cut into chunks: pairs inside a chunk, and the state before it, which is the sum of
    the earlier chunks' own sums with the decay between."""
    hq, hkv, d = (s["case"][x] for x in ("hq", "hkv", "d"))
    C, G, T = PLAIN_CHUNK, hq // hkv, s["q"].shape[0]
    lens = np.diff(s["cu"])
    per = (lens + C - 1) // C
    seq = torch.from_numpy(np.repeat(np.arange(len(lens)), per)).cuda()
    at = torch.from_numpy((np.arange(per.sum()) - np.repeat(np.cumsum(per) - per, per)) * C).cuda()  # tokens before it
    n = torch.from_numpy(np.repeat(lens, per)).cuda()
    first = torch.from_numpy(np.repeat(s["cu"][:-1], per)).cuda() + at
    size = torch.clamp(n - at, max=C)
    i = torch.arange(C, device="cuda")
    inside = i[None, :] < size[:, None]
    token = torch.where(inside, first[:, None] + i[None, :], 0)  # [chunks, C]

    def cut(x):  # [heads, chunks, C, d]
        return (x.float()[token] * inside[:, :, None, None]).permute(2, 0, 1, 3)

    k, v = cut(s["k"]).contiguous(), cut(s["v"]).contiguous()
    q = cut(s["q"]).reshape(hkv, G, len(seq), C, d)
    log = torch.log(torch.from_numpy(s["decay"]).cuda().double())[:, None]

    def power(e):  # decay^e for every head
        return torch.exp(log * e.double().flatten()[None, :]).float().view(hkv, *e.shape)

    gap = i[:, None] - i[None, :]
    pair = power(gap.clamp(min=0)) * (gap >= 0)  # [heads, C, C]
    kd = k * power((size[:, None] - 1 - i[None, :]).clamp(min=0))[..., None]
    local = torch.matmul(kd.transpose(2, 3).contiguous(), v).view(hkv, len(seq), d * d)
    src, dst = (torch.from_numpy(s[x]).cuda().long() for x in ("src", "dst"))
    old = s["state"][src.clamp(min=0)] * (src >= 0)[:, None, None, None]  # [sequences, heads, d, d]
    old = old.permute(1, 0, 2, 3).reshape(hkv, len(lens), d * d)
    end = at + size
    between = at[:, None] - end[None, :]
    earlier = (seq[:, None] == seq[None, :]) & (between >= 0)
    before = torch.matmul(power(between.clamp(min=0)) * earlier, local) + old[:, seq] * power(at)[..., None]
    total = torch.from_numpy(lens).cuda()
    rest = total[:, None] - end[None, :]
    mine = torch.arange(len(lens), device="cuda")[:, None] == seq[None, :]
    final = torch.matmul(power(rest.clamp(min=0)) * mine, local) + old * power(total)[..., None]
    s["state"][dst] = final.view(hkv, len(lens), d, d).transpose(0, 1)
    p = torch.matmul(q, k.transpose(2, 3).contiguous()[:, None]) * pair[:, None, None]
    o = torch.matmul(p, v[:, None])
    o += torch.matmul(q, before.view(hkv, 1, len(seq), d, d)) * power(i + 1)[:, None, None, :, None]
    out = torch.empty(T, hq, d, dtype=torch.bfloat16, device="cuda")
    o = (o * (1.0 / math.sqrt(d))).to(torch.bfloat16).view(hq, len(seq), C, d).permute(1, 2, 0, 3)
    out[token[inside]] = o[inside]
    return out, s["state"]


# --------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------------

def work(case):
    d = case["d"]
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"]
        return {"bytes": 2 * n * d * (4 if case["dtype"] == "f32" else 2) + 4 * case["tokens"], "flops": 3 * n * case["rot"]}
    hq, hkv = case["hq"], case["hkv"]
    if case["op"] == "append":
        T = sum(_appends(case)[1])
        return {"bytes": T * d * (4 * hq + 2 * hkv * (2 + (1 if case["kv"] == "fp8" else 2))),
                "flops": 3 * T * (hq + hkv) * case["rot"]}
    state = 4 * hkv * d * d
    if case["op"] == "chunk":
        T, B = sum(_lens(case)), case["seqs"]
        states = B * (1 if case["fresh"] else 2)
    else:
        T = B = case["groups"] * case["samples"]
        states = B + (case["groups"] if case["fork"] else B)
    return {"bytes": 4 * T * d * (hq + hkv) + states * state, "flops": T * d * d * (2 * hq + 3 * hkv)}


# --------------------------------------------------------------------------------------------------------
# the results in 64 bits, from the definitions
# --------------------------------------------------------------------------------------------------------

def _exact_rotated(case, x, pos, grad=False):
    """Each pair as a complex number, turned by e^(i position frequency)."""
    r = case["rot"]
    f = []
    for i in range(r // 2):
        w = math.exp(-2.0 * i / r * math.log(case["base"]))
        turns = case["orig"] * w / (2.0 * math.pi)
        if case["orig"] == 0 or turns <= case["low"]:
            w /= case["factor"]
        elif turns < case["high"]:
            g = (turns - case["low"]) / (case["high"] - case["low"])
            w = g * w + (1.0 - g) * w / case["factor"]
        f.append(w)
    angle = torch.outer(pos.double(), torch.tensor(f, dtype=torch.float64, device=x.device))
    turn = torch.polar(torch.full_like(angle, case["magnitude"]), -angle if grad else angle)[:, None]
    x = x.double()
    part = x[..., :r].unflatten(-1, (r // 2, 2) if case["interleaved"] else (2, r // 2))
    if not case["interleaved"]:
        part = part.transpose(-1, -2)
    part = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
    if not case["interleaved"]:
        part = part.transpose(-1, -2)
    return torch.cat([part.flatten(-2), x[..., r:]], dim=-1)


def _exact_append(case, s):
    d, hkv, fp8 = case["d"], case["hkv"], case["kv"] == "fp8"
    pool = torch.zeros(s["view"].numel(), dtype=torch.float64, device="cuda")
    c = torch.arange(d, device="cuda")
    h = torch.arange(hkv, device="cuda")[:, None]
    qs = []
    for i, p in enumerate(s["start"].tolist()):
        a, b = int(s["cu"][i]), int(s["cu"][i + 1])
        pos = p + torch.arange(b - a, device="cuda")
        qs.append(_exact_rotated(case, s["q"][a:b], pos))
        k, v = _exact_rotated(case, s["k"][a:b], pos), s["v"][a:b].double()
        page, t = s["bt"][i, pos // PAGE].long()[:, None, None], (pos % PAGE)[:, None, None]
        z = t - (t & 12) + 2 * (t & 4) + (t & 8) // 2
        if fp8:
            k, v = k.clamp(-448.0, 448.0), v.clamp(-448.0, 448.0)
            ke = (((c // 64) * 4 + (c % 32) // 8) * 16 + t) * 16 + ((c // 32) % 2) * 8 + c % 8
            ve = (((c // 32) * 2 + z // 8) * 16 + c % 16) * 16 + ((c // 16) % 2) * 8 + z % 8
        else:
            ke = ((c // 8) * 16 + t) * 8 + c % 8
            ve = (((c // 16) * 2 + z // 8) * 16 + c % 16) * 8 + z % 8
        block = (page * hkv + h) * (2 * PAGE * d)
        pool[(block + ke).flatten()] = k.flatten()
        pool[(block + PAGE * d + ve).flatten()] = v.flatten()
    return torch.cat(qs), pool


def _exact_linear(case, s, cu):
    """The recurrence, EXACT_BLOCK tokens at a time."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    decay = torch.from_numpy(s["decay"]).double().cuda()[:, None, None]
    state = s["state"].double()
    before = state.clone()
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for i in range(len(cu) - 1):
        S = before[int(s["src"][i])] if s["src"][i] >= 0 else torch.zeros_like(before[0])
        for a in range(int(cu[i]), int(cu[i + 1]), EXACT_BLOCK):
            b = min(a + EXACT_BLOCK, int(cu[i + 1]))
            k, v = (s[x][a:b].double().transpose(0, 1).contiguous() for x in ("k", "v"))
            q = s["q"][a:b].double().view(b - a, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
            t = torch.arange(b - a, dtype=torch.float64, device="cuda")
            rows = t.repeat(hq // hkv)[:, None]
            w = torch.where(rows >= t, decay ** (rows - t).clamp(min=0), 0.0)
            o = ((q @ k.transpose(1, 2).contiguous()) * w) @ v + decay ** (rows + 1) * (q @ S)
            out[a:b] = (o / math.sqrt(d)).view(hkv, hq // hkv, b - a, d).permute(2, 0, 1, 3).reshape(b - a, hq, d)
            S = decay ** (b - a) * S + (k * decay ** (b - a - 1 - t)[:, None]).transpose(1, 2).contiguous() @ v
        state[int(s["dst"][i])] = S
    return out, state


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rotated(case, s["x"], s["pos"], case["grad"])
    if case["op"] == "append":
        return _exact_append(case, s)
    return _exact_linear(case, s, s["cu"] if case["op"] == "chunk" else np.arange(len(s["src"]) + 1))
