"""Rotary positions on the way into the 4-bit cache (ralm_kv_append_rotary).

Angles and turns are formed in 64 bits on both sides, from the same angle, and rounded alike: queries are equal, and the cache's bytes are those that
ralm_kv_append stores of the turned keys."""
import ctypes
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2401_14021_amd import binding
    return binding


def turned(x, place, freqs, inter, amplitude):
    """[n, heads, d] by the formula."""
    if freqs.numel() == 0:
        return x.clone()
    a = place.double().view(-1, 1, 1) * freqs.double()
    c, s = torch.cos(a) * amplitude, torch.sin(a) * amplitude
    half = freqs.numel()
    y = x.double()
    u, v = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if inter else (y[..., :half], y[..., half:2 * half])
    p, q = u * c - v * s, v * c + u * s
    z = torch.stack([p, q], -1).flatten(-2) if inter else torch.cat([p, q], -1)
    return torch.cat([z, y[..., 2 * half:]], -1).float().to(x.dtype)


def setup(b, lens, H, d, T=32, layers=2):
    kv = b.KVCache.empty(len(lens), max(max(lens), 1) + T, sum(-(-n // T) for n in lens) + 2, n_layers=layers, n_heads=H, d=d, page_tokens=T)
    kv.pages.zero_()
    b.ralm_kv_reserve(kv, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    return kv


def places(lens, counts, shift):
    out = []
    for r, (n, s) in enumerate(zip(lens, counts)):
        out += [n - s + i + (0 if shift is None else int(shift[r])) for i in range(s)]
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def offsets(counts):
    return torch.cumsum(torch.tensor([0] + counts), 0).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 0), (64, 2), (64, 40), (128, 128), (128, 64), (128, 20), (128, 126), (256, 256), (256, 72), (256, 16)])
@pytest.mark.parametrize("inter", [False, True])
def test_against_append_of_turned_keys(b, d, rot, inter, dtype):
    lens, counts = [1, 40, 33, 700, 5], [1, 7, 33, 130, 0]
    H, Hq = 3, 6
    g = torch.Generator().manual_seed(d * 1000 + rot)
    n = sum(counts)
    rows = (torch.randn(n, Hq + 2 * H, d, generator=g) * 3).to(DT[dtype]).cuda()
    q, k, v = rows.split([Hq, H, H], 1)
    kv = setup(b, lens, H, d)
    freqs = b.ralm_rotary_frequencies(rot)
    shift = torch.tensor([0, 100_000, 3, 17, 1_000_000], dtype=torch.int32, device="cuda")
    off = offsets(counts)
    for amplitude, sh in ((1.0, None), (1.2079, shift)):
        at = places(lens, counts, sh)
        kv.pages.zero_()
        b.ralm_kv_append(kv, 1, turned(k, at, freqs, inter, amplitude), v, off)
        want = kv.pages.clone()
        kv.pages.zero_()
        got = b.ralm_kv_append_rotary(kv, 1, q, k, v, off, freqs, interleaved=inter, amplitude=amplitude, shift=sh)
        assert torch.equal(got, turned(q, at, freqs, inter, amplitude))
        assert torch.equal(kv.pages, want) and bool(want.any())
        kv.pages.zero_()
        assert b.ralm_kv_append_rotary(kv, 1, None, k, v, off, freqs, interleaved=inter, amplitude=amplitude, shift=sh) is None
        assert torch.equal(kv.pages, want)
        own = q.clone(memory_format=torch.contiguous_format)                    # queries in place
        assert b.ralm_kv_append_rotary(kv, 1, own, k, v, off, freqs, interleaved=inter, amplitude=amplitude, shift=sh, q_out=own) is own
        assert torch.equal(own, got) and torch.equal(kv.pages, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot", [(64, 36), (128, 100), (256, 244), (256, 256), (256, 2)])
@pytest.mark.parametrize("inter", [False, True])
def test_many_heads(b, d, rot, inter, dtype):
    """Tokens of more pieces than a workgroup has threads, of queries and of keys; some of them without a place."""
    H, Hq, n = 33, 71, 21
    g = torch.Generator().manual_seed(rot)
    q, k, v = (torch.randn(n, h, d, generator=g).to(DT[dtype]).cuda() for h in (Hq, H, H))
    kv, freqs, off = setup(b, [19, 40], H, d), b.ralm_rotary_frequencies(rot), torch.tensor([0, 4, 20], device="cuda")
    kv.table[1, 0] = -1                                                           # the first tokens of the second request
    at = torch.tensor(list(range(15, 19)) + list(range(24, 40)) + [0], dtype=torch.float64, device="cuda")
    b.ralm_kv_append(kv, 0, turned(k, at, freqs, inter, 1.0), v, off)
    want = kv.pages.clone()
    kv.pages.zero_()
    out = torch.full_like(q, 7.0)
    b.ralm_kv_append_rotary(kv, 0, q, k, v, off, freqs, interleaved=inter, q_out=out)
    assert torch.equal(out[:20], turned(q, at, freqs, inter, 1.0)[:20]) and bool((out[20] == 7.0).all())
    assert torch.equal(kv.pages, want) and bool(want.any())


def test_far_places(b):
    """Places near 2^31: an angle of fp32 would be off by hundreds of turns' worth of steps."""
    kv = setup(b, [64], 2, 128)
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(64, h, 128, generator=g).cuda() for h in (4, 2, 2))
    shift = torch.tensor([2 ** 31 - 1 - 64], dtype=torch.int32, device="cuda")
    freqs = b.ralm_rotary_frequencies(128)
    got = b.ralm_kv_append_rotary(kv, 0, q, k, v, offsets([64]), freqs, shift=shift)
    want = turned(q, places([64], [64], shift), freqs, False, 1.0)
    # equal but for a rounding of the cosine of an angle of 2^31 (2^-53 of it is 2^-22)
    assert float((got - want).abs().max()) < 1e-5
    shift.fill_(-64)                                                              # places below 0 turn the other way
    back = b.ralm_kv_append_rotary(kv, 0, q, k, v, offsets([64]), freqs, shift=shift)
    assert torch.equal(back, turned(q, places([64], [64], shift), freqs, False, 1.0))


def test_rows_and_places_that_are_none(b):
    """Rows of no request and tokens without a place: queries of the first are not written, those of the second are; nothing is stored."""
    kv = setup(b, [40, 3], 2, 64)
    g = torch.Generator().manual_seed(1)
    n = 12
    q, k, v = (torch.randn(n, h, 64, generator=g).bfloat16().cuda() for h in (2, 2, 2))
    off = torch.tensor([2, 5, 10], dtype=torch.int64, device="cuda")              # rows 0, 1, 10, 11 are nobody's; request 1 has 3 tokens of its 5
    freqs = b.ralm_rotary_frequencies(64)
    out = torch.full_like(q, 7.0)
    b.ralm_kv_append_rotary(kv, 0, q, k, v, off, freqs, q_out=out)
    at = torch.tensor([37, 38, 39, -2, -1, 0, 1, 2], dtype=torch.float64, device="cuda")
    assert torch.equal(out[2:10], turned(q[2:10], at, freqs, False, 1.0))
    assert bool((out[:2] == 7.0).all()) and bool((out[10:] == 7.0).all())
    got = kv.pages.clone()
    kv.pages.zero_()
    b.ralm_kv_append(kv, 0, torch.cat([k[:2], turned(k[2:10], at, freqs, False, 1.0), k[10:]]), v, off)
    assert torch.equal(got, kv.pages)
    kv.table.fill_(-1)                                                            # no pages at all
    kv.pages.zero_()
    b.ralm_kv_append_rotary(kv, 0, q, k, v, off, freqs, q_out=out)
    assert not bool(kv.pages.any())
    kv.table.fill_(10 ** 6)                                                       # entries that are no pages
    b.ralm_kv_append_rotary(kv, 0, q, k, v, off, freqs, q_out=out)
    assert not bool(kv.pages.any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan(b, dtype):
    """A pair with an infinity or NaN spoils itself: its query's numbers, its key's block of 32, and nothing beside them."""
    kv = setup(b, [2], 1, 64)
    k = torch.ones(2, 1, 64, dtype=DT[dtype], device="cuda")
    k[0, 0, 3], k[1, 0, 40] = float("inf"), float("nan")
    freqs = b.ralm_rotary_frequencies(64)
    q = b.ralm_kv_append_rotary(kv, 0, k, k, k, offsets([2]), freqs)
    bad = ~torch.isfinite(q)
    assert bad[0, 0].nonzero().flatten().tolist() == [3, 35] and bad[1, 0].nonzero().flatten().tolist() == [8, 40]
    keys, values = b.ralm_kv_read(kv, 0, offsets([2]), 2, dtype=torch.float32)
    assert bool(keys.isnan().all())                                               # both blocks of both keys hold one
    assert values[0, 0].isnan().sum() == 32 and values[1, 0].isnan().sum() == 32


def test_graph_of_growing_requests(b):
    """A captured step: room is reserved, keys are turned by the places that the lengths tell at the time of the replay."""
    kv, eager = (setup(b, [5, 20], 2, 64, T=16) for _ in range(2))
    for c in (kv, eager):
        c.table.fill_(-1), c.refs.zero_(), c.lens.zero_()
        b.ralm_kv_reserve(c, torch.tensor([3, 11], dtype=torch.int32, device="cuda"))
    g = torch.Generator().manual_seed(6)
    q, k, v = (torch.randn(2, h, 64, generator=g).bfloat16().cuda() for h in (4, 2, 2))
    grow, off, freqs = torch.ones(2, dtype=torch.int32, device="cuda"), offsets([1, 1]), b.ralm_rotary_frequencies(64)
    ws, out = b.alloc_kv_pages_workspace(kv), torch.empty_like(q)
    warm = setup(b, [8, 8], 2, 64, T=16)
    b.ralm_kv_reserve(warm, grow, workspace=ws)
    b.ralm_kv_append_rotary(warm, 0, q, k, v, off, freqs, q_out=out)
    granted = torch.empty_like(grow)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.ralm_kv_reserve(kv, grow, workspace=ws, granted=granted)
        b.ralm_kv_append_rotary(kv, 0, q, k, v, off, freqs, q_out=out)
    for i in range(6):
        q.normal_(), k.normal_(), v.normal_()
        graph.replay()
        b.ralm_kv_reserve(eager, grow)
        want = b.ralm_kv_append_rotary(eager, 0, q, k, v, off, freqs)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(kv.lens, eager.lens)
        total = int(kv.lens.sum())
        both = [b.ralm_kv_read(c, 0, offsets(kv.lens.tolist()), total) for c in (kv, eager)]
        at = torch.tensor([2 + i + 1, 10 + i + 1], dtype=torch.float64, device="cuda")
        assert torch.equal(out, turned(q, at, freqs, False, 1.0))
        last = torch.tensor([int(kv.lens[0]) - 1, total - 1], device="cuda")
        assert all(torch.equal(x[last], y[last]) for x, y in zip(*both))


def test_frequencies(b):
    """Plain and scaled: fast pairs as they are, slow ones divided, a ramp between them."""
    f = b.ralm_rotary_frequencies(64, 10000.0, device="cpu")
    want = torch.tensor([10000.0 ** (-j / 32) for j in range(32)], dtype=torch.float64)
    assert torch.allclose(f, want, rtol=1e-15, atol=0)
    assert torch.allclose(b.ralm_rotary_frequencies(64, 10000.0, factor=4.0, device="cpu"), want / 4, rtol=1e-15, atol=0)
    s = b.ralm_rotary_frequencies(64, 10000.0, factor=4.0, context=4096, low=1.0, high=32.0, device="cpu")
    turns = 4096 * want / (2 * math.pi)
    m = ((turns - 1) / 31).clamp(0, 1)
    assert torch.allclose(s, want * (m + (1 - m) / 4), rtol=1e-14, atol=0)
    assert torch.equal(s[turns >= 32], f[turns >= 32]) and bool((turns < 1).any()) and bool((turns > 32).any())
    assert b.ralm_rotary_frequencies(0, device="cpu").shape == (0,)
