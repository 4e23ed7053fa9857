"""What a serving program asks of the operators around the generator's attention, case by case.

A decoder next to the retrieval runs, for every layer, a norm, a product, rotary positions on the way into the 4-bit cache, the
attention, a product that adds to the residual stream, a norm, a gated product and a product back; at the end a product with the
vocabulary, whose softmax is mixed with the retrieved neighbours' distribution.  The attention is measured elsewhere; the kinds here:

* ``linear``  rows times weights, with bias, activation, gate and residual: single tokens, drafts, prompts, the vocabulary.
* ``norm``    a block's output, normed and gated, into the residual stream, and the stream's norm for the next block.
* ``rotary``  queries turned by their positions; keys turned and stored with their values in the 4-bit cache; the stored
              numbers read back.
* ``target``  the distribution that drafts are verified against: softmax of the logits, mixed with the neighbours' weights.

``own`` chooses between the plain forms below and the library's entry points.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}
BLOCK = 32                       # numbers of a head that share a power of two in the cache
TILE = 16                        # tokens of a cache tile


# ---- cases -------------------------------------------------------------------------------------------

def listed():
    return [
        # one user, one token: a block's way back into the residual stream of a small decoder; launches and latency
        dict(name="linear_one", kind="linear", T=1, K=1024, N=1024, dtype="bf16", act="none", gated=False, bias=False, res=True, out="f32"),
        # a decoding step of an ordinary serving batch: queries, keys and values of 32 and 8 heads of 128
        dict(name="linear_batch", kind="linear", T=64, K=4096, N=6144, dtype="bf16", act="none", gated=False, bias=True, res=False, out="bf16"),
        # the first half of the MLP for nine requests' last tokens and their four drafts
        dict(name="linear_draft", kind="linear", T=45, K=4096, N=11264, dtype="f16", act="silu", gated=True, bias=False, res=False, out="f16"),
        # logits of ragged drafts over a vocabulary of 50257: rows that are no whole lines
        dict(name="linear_vocabulary", kind="linear", T=90, K=1024, N=50_257, dtype="bf16", act="none", gated=False, bias=False, res=False,
             out="f32"),
        # chunks of prompts, an odd number of tokens, with bias and activation
        dict(name="linear_chunk", kind="linear", T=1387, K=4096, N=16_384, dtype="bf16", act="gelu", gated=False, bias=True, res=False, out="bf16"),
        # long prompts, back into a residual stream of 32 bits
        dict(name="linear_prompt", kind="linear", T=8192, K=16_384, N=4096, dtype="bf16", act="none", gated=False, bias=False, res=True, out="f32"),
        # one decoding step of four requests in a small decoder
        dict(name="norm_step", kind="norm", T=4, D=1024, form="rms", post=False, gate="none", bias=False, x="bf16", stream="f32", scale=1.0),
        # prompts: norms on both sides of the block, a gate for every channel, a residual scale
        dict(name="norm_prompt", kind="norm", T=8192, D=4096, form="rms", post=True, gate="channel", bias=False, x="bf16", stream="bf16", scale=0.5),
        # a decoding step of 64 requests with long contexts
        dict(name="rotary_step", kind="rotary", R=64, Hq=32, Hkv=8, d=128, T=32, rot=128, inter=False, dtype="bf16", len_lo=2000, len_hi=9000,
             s_lo=1, s_hi=1, factor=8.0, shift=100_000),
        # prompts whose heads are turned in part
        dict(name="rotary_prompt", kind="rotary", R=16, Hq=32, Hkv=8, d=128, T=32, rot=64, inter=True, dtype="bf16", len_lo=1000, len_hi=1100,
             s_lo=301, s_hi=999, factor=1.0, shift=0),
        # three drafts of four requests over a vocabulary of 50257
        dict(name="target_few", kind="target", Q=16, V=50_257, k=16, dtype="f32", out="f32", rows=False),
        # a large verification batch with a share of its own for every row
        dict(name="target_many", kind="target", Q=1300, V=32_000, k=64, dtype="bf16", out="f32", rows=True),
    ]


def _spread(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear"] * 6 + ["norm"] * 3 + ["rotary"] * 3 + ["target"] * 3)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "linear":
        T, K, N = _spread(rng, 1, 8192), 8 * _spread(rng, 8, 2048), _spread(rng, 16, 66_000)
        K = rng.choice([K, K, max(64, K // 64 * 64)])
        N = rng.choice([N, N, max(16, N // 64 * 64)])
        gated = rng.choice([False, False, True])
        wide = 2 if gated else 1
        N = max(1, min(N, int(4.0e8 / (K * wide)), int(5.5e11 / (T * K * wide)), int(2.0e8 / T)))
        return dict(kind=kind, T=T, K=K, N=N, dtype=dtype, gated=gated,
                    act=rng.choice(["silu", "gelu", "relu"]) if gated else rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]),
                    bias=rng.choice([False, True]), res=rng.choice([False, True]), out=rng.choice([dtype, dtype, "f32"]))
    if kind == "norm":
        D = rng.choice([_spread(rng, 16, 16_384), 8 * _spread(rng, 8, 2048)])
        return dict(kind=kind, T=max(1, min(_spread(rng, 1, 20_000), int(6.0e7 / D))), D=D, form=rng.choice(["rms", "rms", "layer"]),
                    post=rng.choice([False, True]), gate=rng.choice(["none", "channel", "token"]), bias=rng.choice([False, True]),
                    x=dtype, stream=rng.choice(["f32", dtype]), scale=rng.choice([1.0, 0.5]))
    if kind == "rotary":
        d, Hkv, G = rng.choice([64, 128, 128, 256]), rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([1, 2, 3, 4, 7, 8])
        while Hkv * G > 64:
            G = max(1, G // 2)
        s_hi = rng.choice([1, 8, _spread(rng, 10, 1000)])
        R = max(1, min(_spread(rng, 1, 128), int(6.0e7 / (s_hi * Hkv * (G + 2) * d))))
        return dict(kind=kind, R=R, Hq=Hkv * G, Hkv=Hkv, d=d, T=rng.choice([16, 32, 64, 128]), rot=rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)]),
                    inter=rng.choice([False, True]), dtype=rng.choice([dtype, dtype, "f32"]), len_lo=s_hi, len_hi=s_hi + _spread(rng, 1, 4000),
                    s_lo=rng.choice([0, 1, s_hi]) if s_hi > 1 else 1, s_hi=s_hi, factor=rng.choice([1.0, 1.0, 4.0, 8.0]),
                    shift=rng.choice([0, 0, _spread(rng, 10, 1_000_000)]))
    V = rng.choice([32_000, 50_257, _spread(rng, 100, 130_000)])
    k = rng.choice([1, 8, 16, 64, _spread(rng, 2, 1024)])
    return dict(kind="target", Q=max(1, min(_spread(rng, 1, 2000), int(4.0e7 / V))), V=V, k=k, dtype=rng.choice([dtype, "f32"]),
                out=rng.choice(["f32", "f32", dtype]), rows=rng.choice([False, True]))


# ---- what follows from a case alone ------------------------------------------------------------------

def _sizes(case):
    """Lengths and numbers of new tokens of every request: part of the case and not of the seed, so that work() is that of every state."""
    rng = random.Random(11)
    s = [rng.randint(case["s_lo"], case["s_hi"]) for _ in range(case["R"])]
    n = [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(case["R"])]
    s[-1], n[-1] = case["s_hi"], case["len_hi"]
    return [max(a, b) for a, b in zip(n, s)], s


def work(case):
    kind = case["kind"]
    if kind == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        rows = N * (2 if case["gated"] else 1)
        return {"bytes": (T * K + rows * K + (rows if case["bias"] else 0)) * _SIZE[case["dtype"]]
                + T * N * _SIZE[case["out"]] * (2 if case["res"] else 1), "flops": 2 * T * K * rows}
    if kind == "norm":
        T, D = case["T"], case["D"]
        per = 2 * _SIZE[case["x"]] + 2 * _SIZE[case["stream"]] + (_SIZE[case["x"]] if case["gate"] == "token" else 0)
        return {"bytes": T * D * per + 4 * D, "flops": T * D * (16 if case["post"] else 8)}
    if kind == "rotary":
        # queries read and written; keys and values read, their codes written, read again, and the numbers written
        n, es = sum(_sizes(case)[1]), _SIZE[case["dtype"]]
        kv = 2 * case["Hkv"] * case["d"]
        return {"bytes": n * (2 * case["Hq"] * case["d"] * es + 2 * kv * es + 2 * kv * 17 // 32), "flops": n * (3 * case["Hq"] * case["d"] + 8 * kv)}
    Q, V = case["Q"], case["V"]
    return {"bytes": Q * V * (_SIZE[case["dtype"]] + _SIZE[case["out"]]) + 8 * Q * case["k"], "flops": 5 * Q * V}


# ---- inputs ------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _offsets(s):
    off = [0]
    for x in s:
        off.append(off[-1] + x)
    return off


def prepare(case, seed):
    st = {"linear": _linear_state, "norm": _norm_state, "rotary": _rotary_state, "target": _target_state}[case["kind"]](case, _gen(seed))
    st["case"] = case
    return st


def _linear_state(case, g):
    T, K, N, dt = case["T"], case["K"], case["N"], _DT[case["dtype"]]
    rows = N * (2 if case["gated"] else 1)
    r = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    x = r(T, K)
    x[:, ::61] *= 4.0                                         # some channels of a decoder's states are louder
    w = torch.empty(rows, K, dtype=dt, device="cuda")
    for a in range(0, rows, 1 << 14):
        b = min(rows, a + (1 << 14))
        w[a:b] = (r(b - a, K) * K ** -0.5).to(dt)
    st = dict(x=x.to(dt), w=w, bias=(0.3 * r(rows)).to(dt) if case["bias"] else None,
              residual=r(T, N).to(_DT[case["out"]]) if case["res"] else None)
    if own:
        from paper_2401_14021_amd import binding as B
        st["ws"] = B.alloc_linear_workspace(T, N, K, gated=case["gated"])
    return st


def _norm_state(case, g):
    T, D, dt = case["T"], case["D"], _DT[case["x"]]
    r = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    loud = torch.exp(0.5 * r(D))
    st = dict(x=(r(T, D) * 2.0 + 0.5).to(dt), residual=(r(T, D) * loud + 0.25).to(_DT[case["stream"]]), weight=(1.0 + 0.1 * r(D)).to(dt),
              bias=(0.1 * r(D)).to(dt) if case["bias"] else None, post_weight=(1.0 + 0.1 * r(D)).to(dt) if case["post"] else None,
              post_bias=(0.1 * r(D)).to(dt) if case["post"] and case["bias"] else None,
              gate=None if case["gate"] == "none" else (0.5 + 0.2 * r(*([D] if case["gate"] == "channel" else [T, D]))).to(dt))
    return st


def _rotary_state(case, g):
    n, s = _sizes(case)
    dev, T, d, H, dt = "cuda", case["T"], case["d"], case["Hkv"], _DT[case["dtype"]]
    # the requests' pages lie in any order, as after long serving
    room = -(-max(n) // T) + 1
    owned = [-(-x // T) for x in n]
    total = sum(owned) + 3
    ids = torch.randperm(total, generator=g, device=dev)[:sum(owned)].to(torch.int32)
    table = torch.full((len(n), room), -1, dtype=torch.int32, device=dev)
    at = 0
    for r, p in enumerate(owned):
        table[r, :p] = ids[at:at + p]
        at += p
    refs = torch.zeros(total, dtype=torch.int32, device=dev)
    refs[ids.long()] = 1
    off = _offsets(s)
    # one row of queries, keys and values for every token, as a product leaves them
    rows = torch.randn(off[-1], case["Hq"] + 2 * H, d, generator=g, device=dev)
    rows *= torch.exp(torch.randn(off[-1], 1, 1, generator=g, device=dev) * 0.5)
    rows = rows.to(dt)
    # slow pairs are slowed down further for contexts longer than those of the training, fast ones are not
    half = case["rot"] // 2
    freqs = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
    keep = ((4096 * freqs / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
    freqs = freqs * (keep + (1 - keep) / case["factor"])
    st = dict(T=T, d=d, H=H, s=s, off=off, offsets=torch.tensor(off, device=dev), table=table, refs=refs,
              lens=torch.tensor(n, dtype=torch.int32, device=dev), pages=torch.zeros(total, H * T * 17 * d // 16, dtype=torch.uint8, device=dev),
              q=rows[:, :case["Hq"]], k=rows[:, case["Hq"]:case["Hq"] + H], v=rows[:, case["Hq"] + H:], freqs=freqs,
              amplitude=1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0,
              shift=torch.randint(0, case["shift"] + 1, (len(n),), generator=g, device=dev).to(torch.int32) if case["shift"] else None)
    if own:
        from paper_2401_14021_amd import binding as B
        st["kv"] = B.KVCache(st["pages"], table, st["lens"], refs, n_layers=1, n_heads=H, d=d, page_tokens=T)
    return st


def _target_state(case, g):
    Q, V, k = case["Q"], case["V"], case["k"]
    logits = (torch.randn(Q, V, generator=g, device="cuda") * 2.5).to(_DT[case["dtype"]])
    # neighbours agree: about half of them are one of a few tokens, some places are empty
    few = torch.randint(0, V, (Q, 4), generator=g, device="cuda")
    same = few.gather(1, torch.randint(0, 4, (Q, k), generator=g, device="cuda"))
    tokens = torch.where(torch.rand(Q, k, generator=g, device="cuda") < 0.5, same, torch.randint(0, V, (Q, k), generator=g, device="cuda"))
    empty = torch.rand(Q, k, generator=g, device="cuda") < 0.05
    weights = torch.softmax(torch.randn(Q, k, generator=g, device="cuda") * 2.0, -1)
    st = dict(logits=logits, tokens=torch.where(empty, torch.full_like(tokens, -1), tokens).to(torch.int32),
              weights=torch.where(empty, torch.zeros_like(weights), weights), temperature=0.7,
              share=torch.rand(Q, generator=g, device="cuda") * 0.8 if case["rows"] else 0.25)
    if own:
        from paper_2401_14021_amd import binding as B
        st["ws"] = B.alloc_knnlm_target_workspace(Q, V)
    return st


# ---- one pass ----------------------------------------------------------------------------------------

def run(st):
    return {"linear": _linear, "norm": _norm, "rotary": _rotary, "target": _target}[st["case"]["kind"]](st)


def _activated(y, act):
    if act == "relu":
        return torch.maximum(y, torch.zeros_like(y))
    if act == "silu":
        return y / (1.0 + torch.exp(-y))
    if act == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    return y


def _linear(st):
    case = st["case"]
    if own:
        from paper_2401_14021_amd import binding as B
        return B.ralm_linear(st["x"], st["w"], bias=st["bias"], act=case["act"], gated=case["gated"], residual=st["residual"],
                             out_dtype=_DT[case["out"]], workspace=st["ws"])
    y = st["x"].float() @ st["w"].float().t()
    if st["bias"] is not None:
        y = y + st["bias"].float()
    if case["gated"]:
        y = _activated(y[:, :case["N"]], case["act"]) * y[:, case["N"]:]
    else:
        y = _activated(y, case["act"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(_DT[case["out"]])


def _normed(y, form, weight, bias):
    if form == "layer":
        y = y - y.mean(-1, keepdim=True)
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6)
    y = y * weight.float()
    return y if bias is None else y + bias.float()


def _norm(st):
    case = st["case"]
    if own:
        from paper_2401_14021_amd import binding as B
        return B.ralm_residual_norm(st["x"], st["residual"], kind=case["form"], weight=st["weight"], bias=st["bias"], post=case["post"],
                                    post_weight=st["post_weight"], post_bias=st["post_bias"], gate=st["gate"], scale=case["scale"], eps=1e-6)
    y = st["x"].float()
    if case["post"]:
        y = _normed(y, case["form"], st["post_weight"], st["post_bias"])
    if st["gate"] is not None:
        y = y * st["gate"].float()
    h = st["residual"].float() + case["scale"] * y
    return h.to(st["residual"].dtype), _normed(h, case["form"], st["weight"], st["bias"]).to(st["x"].dtype)


def _pairs(x, half, inter):
    """The two halves of the pairs that are turned together, and what is not turned."""
    y = x[..., :2 * half]
    a, b = (y[..., 0::2], y[..., 1::2]) if inter else (y[..., :half], y[..., half:])
    return a, b, x[..., 2 * half:]


def _turned(x, cos, sin, inter):
    a, b, rest = _pairs(x.double(), cos.shape[-1], inter)
    u, v = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([u, v], -1).flatten(-2) if inter else torch.cat([u, v], -1)
    return torch.cat([y, rest], -1).to(x.dtype)


def _encode(x):
    """[..., d] -> codes [..., d] (0..15) and power bytes [..., d / 32], both uint8."""
    b = x.float().unflatten(-1, (-1, BLOCK))
    bits = b.abs().amax(-1).view(torch.int32)
    e = torch.clamp((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x400000).int(), min=1, max=252)
    m = (b * ((254 - e) << 23).view(torch.float32).unsqueeze(-1)).abs()
    code = torch.zeros_like(m, dtype=torch.uint8)
    for i, at in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += ((m >= at) if i % 2 else (m > at)).to(torch.uint8)     # ties to the even code
    return (code | torch.signbit(b).to(torch.uint8) << 3).flatten(-2), e.to(torch.uint8)


def _decode(code, e):
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    return (grid[code.long()].unflatten(-1, (-1, BLOCK)) * (e.to(torch.int32) << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)


def _rotary(st):
    """Queries turned; keys turned, and values, into the cache and back out of it."""
    case = st["case"]
    if own:
        from paper_2401_14021_amd import binding as B
        q = B.ralm_kv_append_rotary(st["kv"], 0, st["q"], st["k"], st["v"], st["offsets"], st["freqs"], interleaved=case["inter"],
                                    amplitude=st["amplitude"], shift=st["shift"])
        return (q, *B.ralm_kv_read(st["kv"], 0, st["offsets"], st["off"][-1], dtype=st["k"].dtype))
    d, H, T = st["d"], st["H"], st["T"]
    n, off, dev = st["off"][-1], st["offsets"], st["pages"].device
    # every token's request, place and angles, which are formed in 64 bits: far positions leave 32 too few
    row = torch.repeat_interleave(torch.arange(len(st["s"]), device=dev), off[1:] - off[:-1], output_size=n)
    t = st["lens"].long()[row] - off[row + 1] + torch.arange(n, device=dev)
    place = t if st["shift"] is None else t + st["shift"].long()[row]
    angle = place.double().unsqueeze(1) * st["freqs"]
    cos, sin = (torch.cos(angle) * st["amplitude"]).unsqueeze(1), (torch.sin(angle) * st["amplitude"]).unsqueeze(1)
    q = _turned(st["q"], cos, sin, case["inter"])
    kc, ke = _encode(_turned(st["k"], cos, sin, case["inter"]))
    vc, ve = _encode(st["v"])
    # the bytes of a token in its tile: keys in order, values beside those of the three tokens next to it
    pool = st["pages"].view(-1, 17 * d)
    per = T // TILE
    tile = (st["table"].long()[row, t // T].unsqueeze(1) * H + torch.arange(H, device=dev)) * per + (t % T // TILE).unsqueeze(1)
    tile, i = tile.unsqueeze(2), (t % TILE).view(-1, 1, 1)
    word, block = torch.arange(d // 2, device=dev), torch.arange(d // 32, device=dev)
    k_at, k_pow = i * (d // 2) + word, 16 * d + i * (d // 32) + block
    v_at = 8 * d + (i // 4 * 16 + word // (d // 32)) * (d // 8) + i % 4 * (d // 32) + word % (d // 32)
    v_pow = 16 * d + d // 2 + (i // 4 * (d // 32) + block) * 4 + i % 4
    pool[tile, k_at], pool[tile, v_at] = (c[..., 0::2] | c[..., 1::2] << 4 for c in (kc, vc))
    pool[tile, k_pow], pool[tile, v_pow] = ke, ve
    kc, vc = (torch.stack([x & 15, x >> 4], -1).flatten(-2) for x in (pool[tile, k_at], pool[tile, v_at]))
    return q, _decode(kc, pool[tile, k_pow]).to(st["k"].dtype), _decode(vc, pool[tile, v_pow]).to(st["v"].dtype)


def _target(st):
    case = st["case"]
    if own:
        from paper_2401_14021_amd import binding as B
        return B.ralm_knnlm_target(st["logits"], st["tokens"], st["weights"], st["share"], temperature=st["temperature"],
                                   out_dtype=_DT[case["out"]], workspace=st["ws"])
    x = st["logits"].float() / st["temperature"]
    x = torch.exp(x - x.amax(-1, keepdim=True))
    share = st["share"].unsqueeze(1) if case["rows"] else st["share"]
    p = x / x.sum(-1, keepdim=True) * (1.0 - share)
    there = st["tokens"] >= 0
    return p.scatter_add_(1, st["tokens"].clamp(min=0).long(), torch.where(there, st["weights"] * share, torch.zeros_like(st["weights"]))).to(_DT[case["out"]])


# ---- the same in 64 bits -----------------------------------------------------------------------------

def _power64(e):
    """2^e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _grid64(x):
    """Numbers -> the numbers that their 4 bits stand for, from the format's definition, in 64 bits."""
    b = x.double().unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1, keepdim=True)
    _, e = torch.frexp(top / 6.0)                       # top / 6 = f 2^e, 0.5 <= f < 1
    e = torch.where(_power64(e - 1) * 6.0 >= top, e - 1, e).clamp(min=-126, max=125)
    unit = _power64(e)
    y = b / unit
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    return ((torch.round(y / step) * step).clamp(-6, 6) * unit).flatten(-2)


def _exact_linear(st, case):
    N, x = case["N"], st["x"].double()
    out = torch.empty(case["T"], N, dtype=torch.float64, device="cuda")
    f = {"none": lambda y: y, "relu": lambda y: y.clamp(min=0), "silu": lambda y: y * torch.sigmoid(y),
         "gelu": lambda y: y * 0.5 * torch.erfc(-y / math.sqrt(2.0)),
         "gelu_tanh": lambda y: y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))}[case["act"]]

    def some(a, b):
        y = torch.mm(x, st["w"][a:b].double().t().contiguous())
        return y if st["bias"] is None else y + st["bias"][a:b].double()

    for a in range(0, N, 8192):
        b = min(N, a + 8192)
        y = f(some(a, b))
        if case["gated"]:
            y = y * some(N + a, N + b)
        out[:, a:b] = y if st["residual"] is None else y + st["residual"][:, a:b].double()
    return out


def _exact_norm(st, case):
    def norm(y, w, b):
        if case["form"] == "layer":
            var, mean = torch.var_mean(y, -1, correction=0, keepdim=True)
        else:
            var, mean = torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 / y.shape[-1], 0.0
        y = (y - mean) / torch.sqrt(var + 1e-6) * w.double()
        return y if b is None else y + b.double()

    y = st["x"].double()
    if case["post"]:
        y = norm(y, st["post_weight"], st["post_bias"])
    h = st["residual"].double() + (y if st["gate"] is None else y * st["gate"].double()) * case["scale"]
    return h, norm(h, st["weight"], st["bias"])


def _exact_rotary(st, case):
    """Every token's pairs as complex numbers times a number of its place."""
    n, half = st["off"][-1], case["rot"] // 2
    place = torch.empty(n, dtype=torch.float64, device="cuda")
    for r, S in enumerate(st["s"]):
        first = int(st["lens"][r]) - S + (0 if st["shift"] is None else int(st["shift"][r]))
        place[st["off"][r]:st["off"][r + 1]] = torch.arange(first, first + S, device="cuda")
    turn = torch.polar(torch.full((n, 1, half), st["amplitude"], dtype=torch.float64, device="cuda"), (place[:, None] * st["freqs"]).unsqueeze(1))

    def turned(x):
        y = x.double().clone()
        at = torch.arange(half, device="cuda")
        i, j = (2 * at, 2 * at + 1) if case["inter"] else (at, at + half)
        z = torch.complex(y[..., i], y[..., j]) * turn
        y[..., i], y[..., j] = z.real, z.imag
        return y

    # a key is held as what its type makes of it
    return turned(st["q"]), _grid64(turned(st["k"]).to(st["k"].dtype)), _grid64(st["v"])


def _exact_target(st, case):
    out = torch.empty(case["Q"], case["V"], dtype=torch.float64, device="cuda")
    tokens, weights = st["tokens"].long(), st["weights"].double()
    for a in range(0, case["Q"], 256):
        b = min(case["Q"], a + 256)
        share = st["share"][a:b].double().unsqueeze(1) if case["rows"] else st["share"]
        out[a:b] = torch.exp(torch.log_softmax(st["logits"][a:b].double() / st["temperature"], -1)) * (1.0 - share)
        w = weights[a:b] * share
        row = torch.arange(a, b, device="cuda")
        for j in range(case["k"]):                      # neighbour by neighbour: a token may come again
            ok = tokens[a:b, j] >= 0
            out[row[ok], tokens[a:b, j][ok]] += w[ok, j]
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"linear": _exact_linear, "norm": _exact_norm, "rotary": _exact_rotary, "target": _exact_target}[case["kind"]](st, case)
