"""What a serving program asks of the generator's operators, case by case.

The generator next to the retrieval keeps its keys and values in 4 bits, in pages that requests share.  One verification round
reserves room, appends the drafted tokens' keys and values, attends, verifies the drafts and rolls back.  The kinds of work:

* ``attend``   attention of each request's last tokens over its 4-bit cache, with or without a sliding window whose first
               tokens stay visible: single tokens, drafted tokens, chunks of a prompt.
* ``append``   keys and values into the cache and back out as the numbers that they stand for.
* ``round``    the pages of one round: fork from shared prefixes, reserve (copy on write), roll back, free.
* ``compact``  pages in use move to the front of the pool.
* ``draft``    drafted tokens against the target's probabilities from given random numbers.

``own`` chooses between the plain forms below and the library's entry points.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}
BLOCK = 32                       # numbers that share a power of two
TILE = 16                        # tokens of a cache tile
FIX = 36                         # bits behind the point of a probability


# ---- cases -------------------------------------------------------------------------------------------

def listed():
    return [
        # one user, one decoding step, a prompt with a retrieved passage: launches and latency
        dict(name="attend_one", kind="attend", R=1, Hq=32, Hkv=32, d=128, T=32, dtype="bf16", len_lo=640, len_hi=640, s_lo=1,
             s_hi=1, window=0, sinks=0),
        # a decoding step of an ordinary serving batch, grouped heads, ragged contexts
        dict(name="attend_batch", kind="attend", R=64, Hq=32, Hkv=8, d=128, T=32, dtype="bf16", len_lo=200, len_hi=4000, s_lo=1,
             s_hi=1, window=0, sinks=0),
        # a few very long contexts: the cache is all that is read
        dict(name="attend_long", kind="attend", R=6, Hq=32, Hkv=8, d=128, T=64, dtype="bf16", len_lo=100_000, len_hi=131_000,
             s_lo=1, s_hi=1, window=0, sinks=0),
        # drafted tokens of a stride of 1 to 8, narrow heads without groups, fp16, lengths from one token on
        dict(name="attend_draft", kind="attend", R=48, Hq=16, Hkv=16, d=64, T=16, dtype="f16", len_lo=1, len_hi=1500, s_lo=1,
             s_hi=8, window=0, sinks=0),
        # long streams behind a window with four first tokens
        dict(name="attend_window", kind="attend", R=32, Hq=64, Hkv=8, d=128, T=32, dtype="bf16", len_lo=3000, len_hi=30_000,
             s_lo=1, s_hi=4, window=2048, sinks=4),
        # chunks of prompts behind earlier context: matrix products
        dict(name="attend_prompt", kind="attend", R=8, Hq=32, Hkv=8, d=128, T=32, dtype="bf16", len_lo=1500, len_hi=3500,
             s_lo=700, s_hi=1500, window=0, sinks=0),
        # one token of every request of a batch goes into the cache of a layer
        dict(name="append_step", kind="append", R=64, H=8, d=128, T=32, dtype="bf16", len_lo=200, len_hi=4000, s_lo=1, s_hi=1),
        # the prompts of new requests
        dict(name="append_prompt", kind="append", R=16, H=32, d=128, T=32, dtype="bf16", len_lo=1000, len_hi=1100, s_lo=301,
             s_hi=999),
        # 128 speculations forked from 128 requests, rolled back; pages of 24 layers x 16 heads x 64
        dict(name="round_fork", kind="round", R=128, layers=24, H=16, d=64, T=16, pages=16_384, len_lo=100, len_hi=1500, s_lo=1,
             s_hi=8),
        # a pool after long serving, a third of it in use, is brought together
        dict(name="compact_pool", kind="compact", R=96, layers=24, H=16, d=64, T=16, pages=4096, len_lo=20, len_hi=430),
        # three drafts of four requests over a vocabulary of 50257
        dict(name="draft_few", kind="draft", R=4, s_lo=3, s_hi=3, V=50_257, dtype="f32", draft=True),
        # a large verification batch with ragged strides
        dict(name="draft_many", kind="draft", R=256, s_lo=1, s_hi=8, V=32_000, dtype="bf16", draft=True),
    ]


def _spread(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend"] * 6 + ["append"] * 2 + ["round", "compact", "draft", "draft"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    d = rng.choice([64, 128, 128, 256])
    T = rng.choice([16, 32, 64, 128])
    if kind == "attend":
        Hkv, G = rng.choice([1, 2, 4, 5, 8, 16, 32]), rng.choice([1, 1, 2, 3, 4, 7, 8, 12])
        while Hkv * G > 64:
            G = max(1, G // 2)
        form = rng.choice(["step", "step", "drafts", "drafts", "chunk"])
        s_lo, s_hi = {"step": (1, 1), "drafts": (rng.choice([0, 1]), rng.randint(2, 12)), "chunk": (rng.randint(1, 40), _spread(rng, 48, 1500))}[form]
        R = _spread(rng, 1, 8 if form == "chunk" else 200)
        R = max(1, min(R, int(3.0e10 / (Hkv * G * d * (s_lo + s_hi) / 2 * s_hi))))
        # the largest: as many cached tokens as six long contexts, or as many products as eight long chunks
        most = min(6.0e8 / (R * Hkv * d), 3.0e10 / (R * Hkv * G * d * (s_lo + s_hi) / 2), 120_000 if form != "chunk" else 4000)
        len_hi = _spread(rng, s_hi, max(s_hi + 1, most))
        len_lo = rng.choice([1, s_hi, len_hi])
        masked = rng.choice([False, False, True])
        return dict(kind=kind, R=R, Hq=Hkv * G, Hkv=Hkv, d=d, T=T, dtype=dtype, len_lo=min(len_lo, len_hi), len_hi=len_hi,
                    s_lo=s_lo, s_hi=s_hi, window=_spread(rng, 1, 4096) if masked else 0, sinks=rng.choice([0, 1, 4, 37]) if masked else 0)
    if kind == "append":
        R, H, s_hi = _spread(rng, 1, 128), rng.choice([1, 3, 8, 16, 32]), rng.choice([1, 8, _spread(rng, 10, 1000)])
        s_hi = max(1, min(s_hi, int(4.0e7 / (R * H * d))))
        return dict(kind=kind, R=R, H=H, d=d, T=T, dtype=rng.choice(["bf16", "f16", "f32"]), len_lo=s_hi, len_hi=s_hi + _spread(rng, 1, 1000),
                    s_lo=rng.choice([0, 1, s_hi]) if s_hi > 1 else 1, s_hi=s_hi)
    if kind in ("round", "compact"):
        layers, H = rng.choice([1, 2, 12, 24]), rng.choice([1, 4, 8, 16])
        page = layers * H * T * 17 * d // 16
        len_hi = _spread(rng, 1, 1500)
        R = _spread(rng, 1, 128)
        per = -(-(len_hi + 8) // T) + 2
        pages = 3 * R * per + 5
        if pages * page > 6.0e9:
            layers = 1
            page = H * T * 17 * d // 16
        R = max(1, min(R, int(6.0e9 / page / per / 3)))
        pages = 3 * R * per + 5
        c = dict(kind=kind, R=R, layers=layers, H=H, d=d, T=T, pages=pages, len_lo=rng.choice([1, len_hi]), len_hi=len_hi)
        return dict(c, s_lo=1, s_hi=rng.randint(1, 8)) if kind == "round" else c
    V = rng.choice([32_000, 50_257, 50_272, _spread(rng, 2, 130_000)])
    s_hi = rng.randint(1, 12)
    return dict(kind="draft", R=max(1, min(_spread(rng, 1, 256), int(1.0e8 / (V * s_hi)))), s_lo=rng.choice([0, 1, s_hi]), s_hi=s_hi, V=V,
                dtype=rng.choice(["f32", "bf16", "f16"]), draft=rng.choice([True, True, False]))


# ---- what follows from a case alone ------------------------------------------------------------------

def _sizes(case):
    """Lengths and numbers of new tokens of every request: part of the case and not of the seed, so that work() is that of every
    state.  The last request is the longest."""
    rng = random.Random(7)
    R = case["R"]
    s = [rng.randint(case.get("s_lo", 0), case.get("s_hi", 0)) for _ in range(R)]
    n = [rng.randint(case.get("len_lo", 0), case.get("len_hi", 0)) for _ in range(R)]
    if case["kind"] in ("attend", "append"):
        s[-1], n[-1] = case["s_hi"], case["len_hi"]
        n = [max(a, b) for a, b in zip(n, s)]
    return n, s


def _offsets(s):
    off = [0]
    for x in s:
        off.append(off[-1] + x)
    return off


def _page_bytes(case):
    H = case.get("Hkv", case.get("H"))
    return case.get("layers", 1) * H * case["T"] * 17 * case["d"] // 16


def _visible(case):
    """Per request, the tokens that any of its queries sees, and the pairs of query and token."""
    n, s = _sizes(case)
    w, f = case["window"], case["sinks"]
    tokens, pairs = [], []
    for N, S in zip(n, s):
        if S == 0:
            tokens.append(0), pairs.append(0)
            continue
        lo = max(0, N - S - w + 1) if w else 0
        tokens.append(N - lo + min(f, lo) if w else N)
        if w:
            pairs.append(sum(p + 1 - max(0, p - w + 1) + min(f, max(0, p - w + 1)) for p in range(N - S, N)))
        else:
            pairs.append(sum(range(N - S + 1, N + 1)))
    return tokens, pairs


def work(case):
    kind = case["kind"]
    n, s = _sizes(case)
    if kind == "attend":
        tokens, pairs = _visible(case)
        return {"bytes": sum(tokens) * case["Hkv"] * 17 * case["d"] // 16 + 2 * sum(s) * case["Hq"] * case["d"] * _SIZE[case["dtype"]],
                "flops": 4 * sum(pairs) * case["Hq"] * case["d"]}
    if kind == "append":
        # the numbers read, their codes written; the codes read, the numbers written
        x = sum(s) * case["H"] * case["d"]
        return {"bytes": 2 * x * (2 * _SIZE[case["dtype"]]) + 2 * sum(s) * case["H"] * 17 * case["d"] // 16, "flops": 8 * x}
    if kind == "round":
        # a page that is partly filled is copied for its fork; the counts and the tables are read
        copies = sum(1 for N in n if N % case["T"])
        return {"bytes": 2 * copies * _page_bytes(case) + 4 * case["pages"] + 16 * case["R"] * _max_pages(case), "flops": 0}
    if kind == "compact":
        used = sum(-(-N // case["T"]) for N in n)
        return {"bytes": 2 * round(used * (1 - used / case["pages"])) * _page_bytes(case) + 8 * case["pages"], "flops": 0}
    return {"bytes": case["R"] * case["V"] * _SIZE[case["dtype"]] * (2 if case["draft"] else 1), "flops": 4 * case["R"] * case["V"]}


def _max_pages(case):
    n, s = _sizes(case)
    return -(-(max(n) + max(s)) // case["T"]) + 1


# ---- the format in plain form ------------------------------------------------------------------------

def _encode(x):
    """[..., d] -> codes [..., d] (0..15) and power bytes [..., d / 32], both uint8."""
    b = x.float().unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1)
    bits = top.view(torch.int32)
    e = torch.clamp((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x400000).int(), min=1, max=252)
    e = torch.where(torch.isfinite(top), e, torch.full_like(e, 255))
    y = b * ((254 - e.clamp(max=253)) << 23).view(torch.float32).unsqueeze(-1)
    m = y.abs()
    code = torch.zeros_like(m, dtype=torch.uint8)
    for k, at in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += ((m >= at) if k % 2 else (m > at)).to(torch.uint8)     # ties to the even code
    code |= torch.signbit(b).to(torch.uint8) << 3
    code = torch.where((e == 255).unsqueeze(-1), torch.zeros_like(code), code)
    return code.flatten(-2), e.to(torch.uint8)


def _decode(code, e):
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    p = torch.where(e == 255, torch.full_like(e, 0, dtype=torch.int32), e.to(torch.int32)) << 23
    p = torch.where(e == 255, torch.full((), float("nan"), device=code.device), p.view(torch.float32))
    return (grid[code.long()].unflatten(-1, (-1, BLOCK)) * p.unsqueeze(-1)).flatten(-2)


def _tile(k, v):
    """[n, 16, d] keys and values -> the bytes of n cache tiles [n, 17 d]."""
    n, _, d = k.shape
    kc, ke = _encode(k)
    vc, ve = _encode(v)
    kb = (kc[..., 0::2] | kc[..., 1::2] << 4).reshape(n, 8 * d)
    # values: four tokens beside each other for every sixteenth of the head
    vb = (vc[..., 0::2] | vc[..., 1::2] << 4).reshape(n, 4, 4, 16, d // 32).transpose(2, 3).reshape(n, 8 * d)
    return torch.cat([kb, vb, ke.reshape(n, d // 2), ve.reshape(n, 4, 4, d // 32).transpose(2, 3).reshape(n, d // 2)], 1)


def _untile(tiles, d):
    """[n, 17 d] bytes -> codes and power bytes of keys and values, [n, 16, ..]."""
    n = tiles.shape[0]
    kb, vb, ke, ve = tiles.split([8 * d, 8 * d, d // 2, d // 2], 1)
    kb = kb.reshape(n, 16, d // 2)
    vb = vb.reshape(n, 4, 16, 4, d // 32).transpose(2, 3).reshape(n, 16, d // 2)
    kc = torch.stack([kb & 15, kb >> 4], -1).reshape(n, 16, d)
    vc = torch.stack([vb & 15, vb >> 4], -1).reshape(n, 16, d)
    return kc, ke.reshape(n, 16, d // 32), vc, ve.reshape(n, 4, d // 32, 4).transpose(2, 3).reshape(n, 16, d // 32)


def _tiles_of(st, layer, r, tiles):
    """Indexes of a request's tiles of every head in the pool seen as [tiles, 17 d]: [H, len(tiles)]."""
    H, per, L = st["H"], st["T"] // TILE, st["layers"]
    page = st["table"][r].long()[tiles // per]
    head = torch.arange(H, device=page.device)
    return ((page.unsqueeze(0) * L + layer) * H + head.unsqueeze(1)) * per + (tiles % per).unsqueeze(0)


def _cached(st, layer, r, a, b):
    """Codes and power bytes of the tokens a .. b-1 of a request: K and V, [H, b - a, ..]."""
    t = torch.arange(a // TILE, -(-b // TILE), device=st["table"].device)
    at = _tiles_of(st, layer, r, t)
    pool = st["pages"].view(-1, 17 * st["d"])
    skip = a - a // TILE * TILE
    return [x.reshape(st["H"], -1, x.shape[-1])[:, skip:skip + b - a] for x in _untile(pool[at.reshape(-1)], st["d"])]


# ---- inputs ------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _pool(case, seed, n, room):
    """A pool whose requests' pages lie in any order, as after long serving; room: pages in the table per request."""
    dev, T, d = "cuda", case["T"], case["d"]
    H, L = case.get("Hkv", case.get("H")), case.get("layers", 1)
    owned = [-(-x // T) for x in n]
    total = case.get("pages", sum(owned) + 3)
    g = _gen(seed)
    ids = torch.randperm(total, generator=g, device=dev)[:sum(owned)].to(torch.int32)
    table = torch.full((len(n), room), -1, dtype=torch.int32, device=dev)
    at = 0
    for r, p in enumerate(owned):
        table[r, :p] = ids[at:at + p]
        at += p
    refs = torch.zeros(total, dtype=torch.int32, device=dev)
    refs[ids.long()] = 1
    st = dict(case=case, T=T, d=d, H=H, layers=L, table=table, refs=refs,
              lens=torch.tensor(n, dtype=torch.int32, device=dev))
    st["pages"] = torch.empty(total, L * H * T * 17 * d // 16, dtype=torch.uint8, device=dev)
    return st, g


def _handle(st):
    if own:
        from paper_2401_14021_amd import binding as B
        st["kv"] = B.KVCache(st["pages"], st["table"], st["lens"], st["refs"], n_layers=st["layers"], n_heads=st["H"], d=st["d"],
                             page_tokens=st["T"])
    return st


def prepare(case, seed):
    kind = case["kind"]
    n, s = _sizes(case)
    dev = "cuda"
    if kind == "draft":
        g, V, dt = _gen(seed), case["V"], _DT[case["dtype"]]
        off = _offsets(s)
        Qt, R = off[-1], case["R"]
        # the target's rows: peaked, as a language model's; the draft's are near them
        rows = torch.randn(Qt + R, V, generator=g, device=dev) * 2.5
        target = torch.softmax(rows, -1).to(dt)
        mine = torch.tensor([off[r] + r + i for r in range(R) for i in range(s[r])], dtype=torch.long, device=dev)
        near = rows[mine] + torch.randn(Qt, V, generator=g, device=dev) * 0.7
        del rows
        draft = torch.softmax(near, -1).to(dt)
        # drafts drawn from the draft's own distribution: the largest of logits plus Gumbel numbers
        gumbel = -torch.log(-torch.log(torch.rand(Qt, V, generator=g, device=dev).clamp(1e-7, 1 - 1e-7)))
        ids = (near + gumbel).argmax(-1).to(torch.int32) if Qt else torch.empty(0, dtype=torch.int32, device=dev)
        del near, gumbel
        return dict(case=case, s=s, off=off, offsets=torch.tensor(off, device=dev), ids=ids, target=target,
                    draft=draft if case["draft"] else None, u=torch.rand(Qt, generator=g, device=dev),
                    u_next=torch.rand(R, generator=g, device=dev))
    if kind == "attend":
        st, g = _pool(case, seed, n, _max_pages(case))
        # every tile of the pool holds keys and values; some channels of the keys are larger, as they are behind
        # rotary positions
        d = case["d"]
        pool = st["pages"].view(-1, 17 * d)
        loud = torch.ones(d, device=dev)
        loud[::17] = 3.0
        for a in range(0, pool.shape[0], 1 << 14):
            m = min(1 << 14, pool.shape[0] - a)
            kv = torch.randn(2, m, TILE, d, generator=g, device=dev)
            pool[a:a + m] = _tile(kv[0] * loud, kv[1])
        off = _offsets(s)
        st.update(s=s, n=n, off=off, offsets=torch.tensor(off, device=dev), max_q=max(s), max_len=max(n),
                  q=torch.randn(off[-1], case["Hq"], d, generator=g, device=dev).to(_DT[case["dtype"]]))
        st = _handle(st)
        if own:
            from paper_2401_14021_amd import binding as B
            st["ws"] = B.alloc_kv_attention_workspace(st["kv"], case["Hq"], off[-1], max_q=st["max_q"], max_len=st["max_len"],
                                                      window=case["window"], sinks=case["sinks"])
        return st
    if kind == "append":
        st, g = _pool(case, seed, n, _max_pages(case))
        st["pages"].zero_()
        off = _offsets(s)
        dt = _DT[case["dtype"]]
        k, v = (torch.randn(off[-1], st["H"], st["d"], generator=g, device=dev) for _ in range(2))
        # tokens of different loudness
        k *= torch.exp(torch.randn(off[-1], 1, 1, generator=g, device=dev) * 0.5)
        st.update(s=s, n=n, off=off, offsets=torch.tensor(off, device=dev), k=k.to(dt), v=v.to(dt))
        return _handle(st)
    if kind == "round":
        # rows 0 .. R-1 of the table hold the requests, rows R .. 2R-1 their speculations
        R = case["R"]
        st, g = _pool(case, seed, n + [0] * R, _max_pages(case))
        st["src"] = torch.arange(R, dtype=torch.int32, device=dev)
        st["dst"] = st["src"] + R
        st["grow"] = torch.tensor([0] * R + s, dtype=torch.int32, device=dev)
        st["back"] = torch.tensor(n + [0] * R, dtype=torch.int32, device=dev)
    else:
        st, g = _pool(case, seed, n, _max_pages(case))
    # whole numbers from 0 to 255 that stand for a page's bytes
    flat = st["pages"].view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        m = min(1 << 28, flat.numel() - a)
        flat[a:a + m].random_(0, 256, generator=g)
    st = _handle(st)
    if own:
        from paper_2401_14021_amd import binding as B
        st["ws"] = B.alloc_kv_pages_workspace(st["kv"])
    return st


# ---- one pass ----------------------------------------------------------------------------------------

def run(st):
    return {"attend": _attend, "append": _append, "round": _round, "compact": _compact, "draft": _draft}[st["case"]["kind"]](st)


def _seen(case, a, b, p0, s, dev):
    """[s, b - a]: whether the query at p0 + i sees the token a + j."""
    p = torch.arange(p0, p0 + s, device=dev).unsqueeze(1)
    j = torch.arange(a, b, device=dev).unsqueeze(0)
    ok = j <= p
    if case["window"]:
        ok &= (j > p - case["window"]) | (j < case["sinks"])
    return ok


def _attend(st):
    case = st["case"]
    if own:
        from paper_2401_14021_amd import binding as B
        return B.ralm_kv_attention(st["kv"], 0, st["q"], st["offsets"], max_q=st["max_q"], max_len=st["max_len"],
                                   window=case["window"], sinks=case["sinks"], workspace=st["ws"])
    out = torch.zeros_like(st["q"])
    G, d, w = case["Hq"] // case["Hkv"], case["d"], case["window"]
    for r, (N, S) in enumerate(zip(st["n"], st["s"])):
        if S == 0:
            continue
        lo = max(0, N - S - w + 1) if w else 0
        parts = [(lo, N)] if min(case["sinks"], lo) == 0 else [(0, min(case["sinks"], lo)), (lo, N)]
        kv = [_cached(st, 0, r, a, b) for a, b in parts]
        K = torch.cat([_decode(x[0], x[1]) for x in kv], 1)
        Vv = torch.cat([_decode(x[2], x[3]) for x in kv], 1)
        ok = torch.cat([_seen(case, a, b, N - S, S, K.device) for a, b in parts], 1)
        o = st["off"][r]
        q = st["q"][o:o + S].float().reshape(S, case["Hkv"], G, d).permute(1, 2, 0, 3).reshape(case["Hkv"], G * S, d).contiguous()
        x = torch.bmm(q, K.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
        x = x.view(case["Hkv"], G, S, -1).masked_fill(~ok, float("-inf"))
        x = torch.exp(x - x.amax(-1, keepdim=True))
        x = x / x.sum(-1, keepdim=True)
        y = torch.bmm(x.view(case["Hkv"], G * S, -1), Vv.contiguous())
        out[o:o + S] = y.view(case["Hkv"], G, S, d).permute(2, 0, 1, 3).reshape(S, case["Hq"], d).to(out.dtype)
    return out


def _append(st):
    """Into the cache of layer 0, and the same tokens back out of it."""
    if own:
        from paper_2401_14021_amd import binding as B
        B.ralm_kv_append(st["kv"], 0, st["k"], st["v"], st["offsets"])
        return B.ralm_kv_read(st["kv"], 0, st["offsets"], st["off"][-1], dtype=st["k"].dtype)
    pool = st["pages"].view(-1, 17 * st["d"])
    d, H = st["d"], st["H"]
    n, off = st["off"][-1], st["offsets"]
    kc, ke = _encode(st["k"])
    vc, ve = _encode(st["v"])
    kb, vb = (c[..., 0::2] | c[..., 1::2] << 4 for c in (kc, vc))                    # [n, H, d / 2]
    # every token's request and place
    row = torch.repeat_interleave(torch.arange(len(st["s"]), device=pool.device), off[1:] - off[:-1], output_size=n)
    t = st["lens"].long()[row] - off[row + 1] + torch.arange(n, device=pool.device)
    page = st["table"].long()[row, t // st["T"]]
    head = torch.arange(H, device=pool.device)
    per = st["T"] // TILE
    tile = ((page * st["layers"]).unsqueeze(1) * H + head) * per + (t % st["T"] // TILE).unsqueeze(1)
    tile, i = tile.unsqueeze(2), (t % TILE).view(-1, 1, 1)
    word = torch.arange(d // 2, device=pool.device)
    block = torch.arange(d // 32, device=pool.device)
    # where the bytes of a token lie in its tile, keys in order, values beside those of the three tokens next to it
    k_at, k_pow = i * (d // 2) + word, 16 * d + i * (d // 32) + block
    v_at = 8 * d + (i // 4 * 16 + word // (d // 32)) * (d // 8) + i % 4 * (d // 32) + word % (d // 32)
    v_pow = 16 * d + d // 2 + (i // 4 * (d // 32) + block) * 4 + i % 4
    pool[tile, k_at], pool[tile, v_at], pool[tile, k_pow], pool[tile, v_pow] = kb, vb, ke, ve
    kb, vb, ke, ve = pool[tile, k_at], pool[tile, v_at], pool[tile, k_pow], pool[tile, v_pow]
    kc, vc = (torch.stack([x & 15, x >> 4], -1).flatten(-2) for x in (kb, vb))
    return _decode(kc, ke).to(st["k"].dtype), _decode(vc, ve).to(st["v"].dtype)


def _round(st):
    """Fork, reserve, roll back: the tables as they stood in the middle, and the state behind it, which is that before it."""
    if own:
        from paper_2401_14021_amd import binding as B
        kv = st["kv"]
        B.ralm_kv_fork(kv, st["src"], st["dst"])
        granted = B.ralm_kv_reserve(kv, st["grow"], workspace=st["ws"])
        middle = kv.table.clone(), kv.lens.clone(), kv.refs.clone()
        B.ralm_kv_truncate(kv, st["back"])
        return granted, middle, kv.table, kv.lens, kv.refs, kv.pages
    T = st["T"]
    table, lens, refs, pages = st["table"], st["lens"], st["refs"], st["pages"]
    place = torch.arange(table.shape[1], device=table.device)
    # fork: the speculation shares the request's pages
    src, dst = st["src"].long(), st["dst"].long()
    held = (place * T).unsqueeze(0) < lens[src].unsqueeze(1)
    table[dst] = torch.where(held, table[src], torch.full_like(table[src], -1))
    lens[dst] = lens[src]
    shared = table[dst].clamp(min=0).long()
    refs.index_add_(0, shared.reshape(-1), held.reshape(-1).to(torch.int32))
    # reserve: new pages behind the last one, a copy of a last page that is shared and partly filled
    grow = st["grow"]
    have, want = (lens + T - 1) // T, (lens + grow + T - 1) // T
    last = table.gather(1, (have - 1).clamp(min=0).unsqueeze(1).long()).squeeze(1)
    copy = (grow > 0) & (lens % T != 0) & (refs[last.clamp(min=0).long()] > 1)
    need = want - have + copy.int()
    upto = torch.cumsum(need, 0)
    free = refs == 0
    granted = ((grow == 0) | (need == 0) | (upto <= free.sum())).int()
    copy &= granted.bool()
    need = need * granted
    base = upto - need
    order = torch.argsort((~free).to(torch.int8), stable=True).to(torch.int32)       # free pages, lowest first
    fresh = ((place.unsqueeze(0) >= have.unsqueeze(1)) & (place.unsqueeze(0) < want.unsqueeze(1)) & granted.bool().unsqueeze(1))
    fresh |= copy.unsqueeze(1) & (place.unsqueeze(0) == (have - 1).unsqueeze(1))
    rank = base.unsqueeze(1) + torch.cumsum(fresh.int(), 1) - 1
    new = order[rank.clamp(0, order.numel() - 1).long()]
    old = table.clone()
    table.copy_(torch.where(fresh, new, table))
    at = torch.where(fresh, new, torch.zeros_like(new)).long().reshape(-1)
    refs.index_add_(0, at, fresh.reshape(-1).to(torch.int32))
    moved = fresh & (place.unsqueeze(0) == (have - 1).unsqueeze(1)) & copy.unsqueeze(1)
    refs.index_add_(0, old.clamp(min=0).long().reshape(-1), -moved.reshape(-1).to(torch.int32))
    pages[table[moved].long()] = pages[old[moved].long()]
    lens += grow * granted
    middle = table.clone(), lens.clone(), refs.clone()
    # roll back: what lies behind the new lengths goes back to the pool
    lens.copy_(torch.minimum(lens, st["back"]))
    gone = ((place * T).unsqueeze(0) >= lens.unsqueeze(1)) & (table >= 0)
    refs.index_add_(0, table.clamp(min=0).long().reshape(-1), -gone.reshape(-1).to(torch.int32))
    table.masked_fill_(gone, -1)
    return granted, middle, table, lens, refs, pages


def _compact(st):
    """Into a table and counts of their own: the old ones stay valid for calls that are under way."""
    if own:
        from paper_2401_14021_amd import binding as B
        table, refs, used = B.ralm_kv_compact(st["kv"], workspace=st["ws"])
        return table, refs, used, st["kv"].pages
    table, refs, pages = st["table"], st["refs"], st["pages"]
    used = refs > 0
    n = used.sum()
    page = torch.arange(refs.numel(), device=refs.device)
    movers, holes = page[used & (page >= n)], page[~used & (page < n)]
    goes = page.clone()
    goes[movers] = holes
    pages[holes] = pages[movers]
    new = torch.where(table >= 0, goes[table.clamp(min=0).long()].to(torch.int32), table)
    counts = torch.zeros_like(refs)
    counts[goes[used]] = refs[used]
    return new, counts, n.to(torch.int32), pages


def _fixed(p):
    return torch.floor(p.float().clamp(0, 1).double() * float(1 << FIX)).long()


def _draft(st):
    case = st["case"]
    if own:
        from paper_2401_14021_amd import binding as B
        return B.ralm_verify_draft(st["ids"], st["target"], st["u"], st["u_next"], st["offsets"], draft_probs=st["draft"])
    R, Qt, V = case["R"], st["off"][-1], case["V"]
    off = st["offsets"]
    first, count = off[:-1], off[1:] - off[:-1]
    dev = off.device
    step = torch.arange(max(max(st["s"]), 1), device=dev).unsqueeze(0)
    there = step < count.unsqueeze(1)
    n = torch.zeros(R, dtype=torch.long, device=dev)
    if Qt:
        at = (first.unsqueeze(1) + step).clamp(max=Qt - 1)
        x = st["ids"].long()[at]
        row = at + torch.arange(R, device=dev).unsqueeze(1)
        P = _fixed(st["target"][row, x])
        Q = torch.full_like(P, 1 << FIX) if st["draft"] is None else _fixed(st["draft"][at, x])
        m = torch.floor(st["u"] * float(1 << 24)).long()[at]
        good = there & (m * Q < (P << 24))
        n = torch.cumprod(good.long(), 1).sum(1)
    rest = n < count
    w = _fixed(st["target"][first + torch.arange(R, device=dev) + n])
    if Qt:
        q_row = (first + n).clamp(max=Qt - 1)
        if st["draft"] is not None:
            Q = _fixed(st["draft"][q_row])
        else:
            Q = torch.zeros_like(w).scatter_(1, st["ids"].long()[q_row].unsqueeze(1), 1 << FIX)
        less = torch.clamp(w - Q, min=0)
        use = rest & (less.sum(1) > 0)
        w = torch.where(use.unsqueeze(1), less, w)
    upto = torch.cumsum(w, 1)
    total = upto[:, -1]
    t = (torch.floor(st["u_next"] * float(1 << 24)).long() * total) >> 24
    token = (upto <= t.unsqueeze(1)).sum(1)
    token = torch.where(total > 0, token, torch.full_like(token, -1))
    return n.to(torch.int32), token.to(torch.int32)


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


def _draft64(st):
    """Draft by draft and entry by entry, in whole numbers on the host."""
    one = 1 << FIX

    def whole(row):
        return np.minimum(np.floor(np.maximum(row, 0.0) * one), one).astype(np.int64)

    target = st["target"].double().cpu().numpy()
    draft = None if st["draft"] is None else st["draft"].double().cpu().numpy()
    ids, u, u_next = (st[k].double().cpu().numpy() for k in ("ids", "u", "u_next"))
    counts, tokens = [], []
    for r, S in enumerate(st["s"]):
        a = st["off"][r]
        n = 0
        while n < S:
            x = int(ids[a + n])
            p = int(whole(target[a + r + n, x]))
            q = one if draft is None else int(whole(draft[a + n, x]))
            if int(u[a + n] * 2 ** 24) * q >= p << 24:
                break
            n += 1
        p = whole(target[a + r + n])
        w = p
        if n < S:
            q = np.zeros_like(p) if draft is None else whole(draft[a + n])
            if draft is None:
                q[int(ids[a + n])] = one
            w = np.maximum(p - q, 0)
            w = w if w.any() else p
        total = int(w.sum())
        t = int(u_next[r] * 2 ** 24) * total >> 24
        counts.append(n)
        tokens.append(int(np.searchsorted(np.cumsum(w), t, side="right")) if total else -1)
    return torch.tensor(counts, dtype=torch.int32), torch.tensor(tokens, dtype=torch.int32)


def exact(case, seed):
    kind = case["kind"]
    if kind == "append":
        st = prepare(case, seed)
        return _grid64(st["k"]), _grid64(st["v"])
    if kind == "draft":
        return _draft64(prepare(case, seed))
    if kind != "attend":
        return None                                     # whole numbers that are moved, none computed
    st = prepare(case, seed)
    d, G, dev = case["d"], case["Hq"] // case["Hkv"], "cuda"
    scale = 1.0 / math.sqrt(d)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=dev)
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=dev)

    def numbers(code, power):
        mag = levels[(code & 7).long()] * (1.0 - 2.0 * (code >> 3).double())
        return mag * _power64(power.int().repeat_interleave(BLOCK, -1) - 127)

    for r in range(case["R"]):
        N, S, o = st["n"][r], st["s"][r], st["off"][r]
        if S == 0:
            continue
        # the visible tokens one by one, from the mask's definition
        j = torch.arange(N, device=dev)
        p = torch.arange(N - S, N, device=dev)
        seen = (j.unsqueeze(0) <= p.unsqueeze(1))
        if case["window"] > 0:
            seen &= ((p.unsqueeze(1) - j.unsqueeze(0) < case["window"]) | (j.unsqueeze(0) < case["sinks"]))
        some = seen.any(0).nonzero().squeeze(1)
        tile = _tiles_of(st, 0, r, some // TILE)
        for h in range(case["Hkv"]):
            whole = st["pages"].view(-1, 17 * d)[torch.unique(tile[h])]
            back = torch.searchsorted(torch.unique(tile[h]), tile[h])
            kc, ke, vc, ve = (x[back, some % TILE] for x in _untile(whole, d))
            K, Vv = numbers(kc, ke), numbers(vc, ve)
            for g in range(G):
                x = st["q"][o:o + S, h * G + g].double() @ K.T.contiguous() * scale
                x = torch.where(seen[:, some], x, torch.full_like(x, float("-inf")))
                x = torch.exp(x - x.max(1, keepdim=True).values)
                out[o:o + S, h * G + g] = (x @ Vv) / x.sum(1, keepdim=True)
    return out
