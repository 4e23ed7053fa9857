"""The 4-bit paged cache: append, read and attention against the plain forms in 64 bits, at the lengths, head layouts and masks where
they can go wrong."""
import numpy as np
import pytest
import torch

import kv_plain

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2401_14021_amd import binding
    binding.lib()
    return binding


def make_cache(B, lens, H, d, T, layers=1, seed=0, fill=255, spare=2):
    """A cache whose pages lie in any order and hold `fill` where nothing was written (255: powers that are NaN)."""
    rng = np.random.default_rng(seed)
    owned = [-(-n // T) for n in lens]
    total = sum(owned) + 5
    ids = rng.permutation(total)
    table = np.full((len(lens), max(owned) + spare), -1, np.int32)
    refs = np.zeros(total, np.int32)
    at = 0
    for r, p in enumerate(owned):
        table[r, :p] = ids[at:at + p]
        refs[ids[at:at + p]] = 1
        at += p
    page = B.ralm_kv_page_bytes(layers, H, d, T)
    pages = torch.full((total, page), fill, dtype=torch.uint8, device="cuda")
    return B.KVCache(pages, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                     torch.from_numpy(refs).cuda(), n_layers=layers, n_heads=H, d=d, page_tokens=T)


def offsets_of(s):
    return torch.tensor([0] + list(np.cumsum(s)), dtype=torch.int64, device="cuda")


def fill_cache(B, kv, lens, layer, dtype, seed, nan_at=()):
    """Random keys and values for all tokens; returns what they stand for, per request [n, H, d]."""
    rng = np.random.default_rng(seed)
    n, H, d = sum(lens), kv.n_heads, kv.d
    loud = np.exp(rng.normal(size=(n, H, 1)))
    k, v = (torch.from_numpy((rng.normal(size=(n, H, d)) * loud).astype(np.float32)).to(DT[dtype]) for _ in range(2))
    for token, what in nan_at:
        (k if what == "k" else v)[token, 0, 5] = float("nan")
    B.ralm_kv_append(kv, layer, k.cuda(), v.cuda(), offsets_of(lens))
    K, V = kv_plain.four_bits(k.double().numpy()), kv_plain.four_bits(v.double().numpy())
    cut = np.cumsum(lens)[:-1]
    return np.split(K, cut), np.split(V, cut)


# ---- append and read -----------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_append_and_read(B, d, dtype):
    lens, H, T = [1, 0, 15, 16, 17, 70, 33], 3, 32
    kv = make_cache(B, lens, H, d, T, layers=3, seed=d)
    K, V = fill_cache(B, kv, lens, 1, dtype, seed=d + 1)
    k, v = B.ralm_kv_read(kv, 1, offsets_of(lens), sum(lens), dtype=torch.float32)
    assert np.array_equal(k.double().cpu().numpy(), np.concatenate(K))
    assert np.array_equal(v.double().cpu().numpy(), np.concatenate(V))
    # bf16 holds every number of the format
    k16, v16 = B.ralm_kv_read(kv, 1, offsets_of(lens), sum(lens), dtype=torch.bfloat16)
    assert torch.equal(k16.float(), k) and torch.equal(v16.float(), v)
    # from a place of their own on, and tokens that have no place
    start = torch.tensor([0, 0, 3, 15, 2, 60, 400], dtype=torch.int32, device="cuda")
    take = [1, 0, 5, 1, 9, 10, 2]
    k, v = B.ralm_kv_read(kv, 1, offsets_of(take), sum(take), start=start, dtype=torch.float16)
    want = [K[r][int(start[r]):int(start[r]) + take[r]] for r in range(6)] + [np.zeros((2, H, d))]
    assert np.array_equal(k.double().cpu().numpy(), np.concatenate(want).astype(np.float16))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_append_values_at_the_edges_of_the_format(B, d):
    """Ties, largest numbers of a block at and around 6 * 2^e, zeros, subnormal numbers, infinities and NaN."""
    rng = np.random.default_rng(5)
    n, H = 64, 2
    x = np.zeros((n, H, d), np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.2499999, 0.7500001, 4.9999995, 5.0000005], np.float32)
    for t in range(n):
        x[t] = rng.choice(ties, size=(H, d)) * rng.choice([-1, 1], size=(H, d)) * np.float32(2.0 ** rng.integers(-30, 30))
    x[3] = 0.0
    x[4] = -0.0
    x[5] = rng.normal(size=(H, d)) * 1e-39                  # subnormal
    x[6] = rng.normal(size=(H, d)) * 1e38
    x[7, 0, 3] = np.inf
    x[8, 1, d - 1] = np.nan
    x[9, 0, :32] = 3.4e38
    lens = [n]
    for dtype in ("f32", "bf16"):
        kv = make_cache(B, lens, H, d, 16, seed=3)
        a = torch.from_numpy(x).to(DT[dtype])
        B.ralm_kv_append(kv, 0, a.cuda(), (-a).cuda(), offsets_of(lens))
        k, v = B.ralm_kv_read(kv, 0, offsets_of(lens), n, dtype=torch.float32)
        want = kv_plain.four_bits(a.double().numpy())
        np.testing.assert_array_equal(k.double().cpu().numpy(), want)
        np.testing.assert_array_equal(v.double().cpu().numpy(), -want)


@pytest.mark.parametrize("d", [64, 128])
def test_append_of_fp16_at_the_edges_of_the_type(B, d):
    """Subnormal numbers, the largest one, ties at every power, infinities and NaN."""
    rng = np.random.default_rng(6)
    n, H = 48, 2
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 4.0, 0.5])
    x = np.stack([rng.choice(ties, size=(H, d)) * rng.choice([-1, 1], size=(H, d)) * 2.0 ** (t % 30 - 16) for t in range(n)]).astype(np.float16)
    x[0] = 2.0 ** -24 * rng.integers(-9, 10, size=(H, d))       # subnormal
    x[1, 0, :32] = 65504.0
    x[2] = -0.0
    x[3, 1, 7] = np.inf
    x[4, 0, d - 1] = np.nan
    kv = make_cache(B, [n], H, d, 16, seed=8)
    a = torch.from_numpy(x).cuda()
    B.ralm_kv_append(kv, 0, a, -a, offsets_of([n]))
    k, v = B.ralm_kv_read(kv, 0, offsets_of([n]), n, dtype=torch.float32)
    want = kv_plain.four_bits(x.astype(np.float64))
    np.testing.assert_array_equal(k.double().cpu().numpy(), want)
    np.testing.assert_array_equal(v.double().cpu().numpy(), -want)


def test_append_writes_its_own_tokens_only(B):
    """A few tokens behind others, from a fused tensor's strided parts; rows of no request and places outside the table are left out."""
    H, d, T, layers = 2, 128, 32, 2
    lens = [40, 7, 33]
    kv = make_cache(B, lens, H, d, T, layers=layers, seed=1, fill=0x33)
    before = kv.pages.clone()
    s = [3, 7, 1]
    fused = torch.randn(11, H * 5, d, device="cuda", dtype=torch.bfloat16)
    k, v = fused[:, H:2 * H], fused[:, 3 * H:4 * H]
    off = offsets_of(s)
    B.ralm_kv_append(kv, 1, k, v, off)                                    # 11 rows; the requests own 11
    changed = (kv.pages != before).view(kv.pages.shape[0], layers, -1)
    assert not changed[:, 0].any()
    want = kv_plain.four_bits(k.double().cpu().numpy())
    got, _ = B.ralm_kv_read(kv, 1, off, 11, dtype=torch.float32)
    assert np.array_equal(got.double().cpu().numpy(), want)
    # the tokens in front of them: as they were
    front = offsets_of([37, 0, 32])
    k0, v0 = B.ralm_kv_read(kv, 1, front, 69, start=torch.zeros(3, dtype=torch.int32, device="cuda"), dtype=torch.float32)
    new = kv.pages.clone()
    kv.pages.copy_(before)
    k1, v1 = B.ralm_kv_read(kv, 1, front, 69, start=torch.zeros(3, dtype=torch.int32, device="cuda"), dtype=torch.float32)
    assert torch.equal(k0, k1) and torch.equal(v0, v1)
    # offsets that own fewer rows than there are, and a table without pages
    kv.table[1] = -1
    kv.table[2] = 10_000_000
    B.ralm_kv_append(kv, 1, k, v, offsets_of([3, 5, 1]))
    torch.cuda.synchronize()
    owned = set(kv.table[0, :2].tolist())
    rows = (kv.pages != before).any(1).nonzero().squeeze(1).tolist()
    assert set(rows) <= owned and not torch.equal(new, before)


# ---- attention -----------------------------------------------------------------------------------------

def check_attention(B, lens, s, Hq, Hkv, d, T, dtype, window=0, sinks=0, layers=1, layer=0, hints=None, seed=0, nan_at=(), scale=None,
                    kv_dtype="f32"):
    kv = make_cache(B, lens, Hkv, d, T, layers=layers, seed=seed)
    K, V = fill_cache(B, kv, lens, layer, kv_dtype, seed + 1, nan_at)
    rng = np.random.default_rng(seed + 2)
    n = sum(s)
    q = torch.from_numpy(rng.normal(size=(n, Hq, d)).astype(np.float32)).to(DT[dtype])
    lse = torch.empty(n, Hq, dtype=torch.float32, device="cuda")
    out = B.ralm_kv_attention(kv, layer, q.cuda(), offsets_of(s), max_q=hints[0] if hints else max(s), max_len=hints[1] if hints else max(lens),
                              scale=scale, window=window, sinks=sinks, lse=lse)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    o = 0
    for r in range(len(lens)):
        a = s[r] - lens[r] if s[r] > lens[r] else 0                       # queries in front of the first token see nothing
        qr = q[o:o + s[r]].double().numpy()
        want, want_lse, mag, size = kv_plain.attention(qr[a:], K[r], V[r], scale or d ** -0.5, window, sinks)
        assert (got[o:o + a] == 0).all() and (got_lse[o:o + a] == -np.inf).all()
        y, x = got[o + a:o + s[r]], got_lse[o + a:o + s[r]]
        nan = np.isnan(want)
        assert np.array_equal(np.isnan(y), nan), (r, np.argwhere(np.isnan(y) != nan)[:5])
        tol = kv_plain.attention_tolerance(dtype, want, mag, size, d)
        bad = np.abs(y - want) > tol
        assert not bad[~nan].any(), (r, np.argwhere(bad & ~nan)[:5], np.abs(y - want)[~nan].max())
        ok = ~np.isnan(want_lse)
        lt = 2.0 * (d + 4) * 2.0 ** -24 * size[0] + 2.0 ** -20 * (1 + np.abs(want_lse))
        assert (np.abs(x - want_lse)[ok & np.isfinite(want_lse)] <= lt[ok & np.isfinite(want_lse)]).all()
        assert np.array_equal(np.isnan(x), ~ok)
        o += s[r]
    return kv, q, out


EDGE = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 127, 128, 129, 200]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (8, 2), (7, 1), (24, 2)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_single_tokens(B, d, Hq, Hkv, dtype):
    check_attention(B, EDGE, [1] * len(EDGE), Hq, Hkv, d, 32, dtype, seed=d + Hq)


@pytest.mark.parametrize("T", [16, 64, 256])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_drafted_tokens_and_pages_that_end_inside_a_step(B, d, T):
    s = [0, 1, 3, 8, 5, 2, 8, 7, 6, 1, 4, 8, 3, 2, 1, 8, 5, 4]
    check_attention(B, EDGE, s, 6, 2, d, T, "bf16", layers=3, layer=2, seed=T)     # some have more queries than tokens
    check_attention(B, EDGE, s, 16, 4, d, T, "f16", seed=T + 1, kv_dtype="f16")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_chunks(B, d, dtype):
    check_attention(B, [150, 65, 300, 1], [150, 33, 129, 1], 4, 2, d, 32, dtype, seed=d)
    check_attention(B, [90, 17], [75, 17], 5, 1, d, 16, dtype, seed=d + 1)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 4), (16, 16), (33, 40), (64, 3), (1000, 4), (7, 1000)])
@pytest.mark.parametrize("s", [1, 6, 70])
def test_window_and_first_tokens(B, window, sinks, s):
    lens = [1, 5, 16, 37, 90, 161, 250]
    check_attention(B, lens, [min(s, n) for n in lens], 4, 2, 128, 16, "bf16", window=window, sinks=sinks, seed=window + s)
    check_attention(B, lens, [min(s, n) for n in lens], 3, 3, 64, 32, "f16", window=window, sinks=sinks, seed=window + s + 1)


@pytest.mark.parametrize("Hq,s", [(2, 1), (8, 4), (4, 40)])
def test_long_contexts_in_parts(B, Hq, s):
    """Few requests: contexts are split over workgroups and their sums joined."""
    for d, T in ((128, 64), (64, 16), (256, 128)):
        check_attention(B, [5000, 3, 2049], [s, 1, min(s, 9)], Hq, 2, d, T, "bf16", seed=Hq + d)
        check_attention(B, [4000, 900], [s, s], Hq, 1, d, T, "f16", window=700, sinks=5, seed=Hq + d + 1)


@pytest.mark.parametrize("R,Hkv", [(2, 160), (33, 8), (37, 9), (64, 5), (65, 4), (130, 2)])
def test_more_workgroups_than_cus(B, R, Hkv):
    """Up to 64 requests are handed out by their lengths: equal ones, empty ones, requests without queries."""
    rng = np.random.default_rng(R)
    lens = rng.choice([0, 1, 40, 40, 100, 300], size=R).tolist()
    s = [min(n, int(rng.integers(0, 3))) for n in lens]
    s[0], lens[0] = 2, max(lens[0], 2)
    check_attention(B, lens, s, Hkv, Hkv, 64, 16, "bf16", seed=R)
    check_attention(B, lens, s, Hkv, Hkv, 64, 16, "f16", window=30, sinks=3, seed=R)


@pytest.mark.parametrize("R,Hkv", [(5, 12), (64, 1), (66, 1)])
def test_chunks_of_more_workgroups_than_cus(B, R, Hkv):
    rng = np.random.default_rng(R)
    lens = rng.choice([30, 90, 90, 161], size=R).tolist()
    s = [min(n, int(rng.integers(20, 80))) for n in lens]
    check_attention(B, lens, s, 12 * Hkv, Hkv, 64, 16, "bf16", hints=(1000, 200), seed=R)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 50])
def test_chunks_by_waves_with_rows_of_their_own(B, d, dtype, window):
    """No hint how many queries a request has: the launch is that of many rows, of which waves have all, some or none."""
    rng = np.random.default_rng(d + window)
    lens = [200, 16, 75, 130, 33, 90, 64]
    s = [min(n, int(rng.integers(20, 76))) for n in lens]
    check_attention(B, lens, s, 40, 10, d, 32, dtype, window=window, sinks=3, seed=d, hints=(0, 200), nan_at=[(100, "v"), (150, "k"), (190, "v")])


def test_hints_that_are_too_small_or_missing_change_no_result(B):
    lens, s = [700, 20, 3001], [40, 9, 3]
    for hints in ((0, 0), (1, 1), (1, 3001), (40, 16), (0, 1), (2, 0), (1 << 30, 1 << 30)):
        kv, q, out = check_attention(B, lens, s, 4, 2, 128, 32, "bf16", hints=hints)
        same = B.ralm_kv_attention(kv, 0, q.cuda(), offsets_of(s), max_q=hints[0], max_len=hints[1])
        assert torch.equal(same, out)


@pytest.mark.parametrize("s", [1, 3, 40])
def test_nan_in_masked_places(B, s):
    """Keys and values that are NaN reach the rows that see them, and no others; pages are full of NaN behind the last token."""
    lens = [100, 77]
    for d in (64, 128, 256):
        for dtype in ("bf16", "f16"):
            # token 3: outside the window; tokens 98, 99 and 176: the last ones, which only the last queries see
            check_attention(B, lens, [s, s], 4, 2, d, 32, dtype, window=50, sinks=2, seed=s + d, nan_at=[(3, "k"), (4, "v"), (99, "v"), (176, "k")])
            check_attention(B, lens, [s, s], 4, 2, d, 32, dtype, seed=s + d, nan_at=[(98, "v"), (150, "v")])
            check_attention(B, lens, [s, s], 4, 2, d, 32, dtype, seed=s + d, nan_at=[(20, "k")])


def test_large_and_tiny_numbers(B):
    """Scores far apart (all weight on one token), equal ones, and a cache beyond fp16's range under fp16 queries."""
    kv = make_cache(B, [64], 1, 64, 16)
    for factor in (1e-30, 1.0, 1e6):
        rng = np.random.default_rng(1)
        k, v = (torch.from_numpy(rng.normal(size=(64, 1, 64)).astype(np.float32) * np.float32(factor)) for _ in range(2))
        B.ralm_kv_append(kv, 0, k.cuda(), v.cuda(), offsets_of([64]))
        K, V = (kv_plain.four_bits(x.double().numpy()) for x in (k, v))
        q = torch.from_numpy(rng.normal(size=(2, 1, 64)).astype(np.float32)).bfloat16()
        out = B.ralm_kv_attention(kv, 0, q.cuda(), offsets_of([2]))
        want, _, mag, size = kv_plain.attention(q.double().numpy(), K, V, 64 ** -0.5)
        tol = kv_plain.attention_tolerance("bf16", want, mag, size, 64)
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


def test_places_that_are_no_pages_are_not_attended_to(B):
    def spoil(kv):
        kv.table[0, 1] = -1
        kv.table[1, 0] = 1 << 30
    lens = [96, 40]
    kv = make_cache(B, lens, 2, 128, 32, seed=4)
    K, V = fill_cache(B, kv, lens, 0, "f32", 5)
    spoil(kv)
    q = torch.randn(2, 4, 128, device="cuda").bfloat16()
    out = B.ralm_kv_attention(kv, 0, q, offsets_of([1, 1]))
    for r, keep in ((0, np.r_[0:32, 64:96]), (1, np.r_[32:40])):
        want, _, mag, size = kv_plain.attention(q[r:r + 1].double().cpu().numpy(), K[r][keep], V[r][keep], 128 ** -0.5)
        tol = kv_plain.attention_tolerance("bf16", want, mag, size, 128)
        assert (np.abs(out[r:r + 1].double().cpu().numpy() - want) <= tol).all()


def test_offsets_beyond_32_bits(B):
    """Pages that lie more than 4 GiB behind the pool's begin."""
    H, d, T, layers = 32, 128, 256, 8
    page = B.ralm_kv_page_bytes(layers, H, d, T)
    n_pages = int(9.0e9 / page)
    kv = B.KVCache.empty(2, 3 * T, n_pages, n_layers=layers, n_heads=H, d=d, page_tokens=T)
    kv.table[0, :3] = torch.tensor([n_pages - 1, 3, n_pages - 2], dtype=torch.int32)
    kv.lens[0] = 600
    k, v = (torch.randn(600, H, d, device="cuda").bfloat16() for _ in range(2))
    off = offsets_of([600, 0])
    B.ralm_kv_append(kv, layers - 1, k, v, off)
    K, V = (kv_plain.four_bits(x[:, :2].double().cpu().numpy()) for x in (k, v))
    gk, gv = B.ralm_kv_read(kv, layers - 1, off, 600, dtype=torch.float32)
    assert np.array_equal(gk[:, :2].double().cpu().numpy(), K) and np.array_equal(gv[:, :2].double().cpu().numpy(), V)
    q = torch.randn(1, H, d, device="cuda").bfloat16()
    out = B.ralm_kv_attention(kv, layers - 1, q, offsets_of([1, 0]))
    want, _, mag, size = kv_plain.attention(q[:, :2].double().cpu().numpy(), K, V, d ** -0.5)
    assert (np.abs(out[:, :2].double().cpu().numpy() - want) <= kv_plain.attention_tolerance("bf16", want, mag, size, d)).all()


def test_strided_queries_and_outputs(B):
    lens, s = [50, 9], [4, 9]
    kv, q, out = check_attention(B, lens, s, 4, 2, 128, 32, "bf16")
    wide = torch.zeros(13, 10, 136, device="cuda", dtype=torch.bfloat16)
    wide[:, 3:7, :128] = q.cuda()
    into = torch.full((13, 8, 144), 7.0, device="cuda", dtype=torch.bfloat16)
    B.ralm_kv_attention(kv, 0, wide[:, 3:7, :128], offsets_of(s), max_q=9, max_len=50, out=into[:, 2:6, :128])
    assert torch.equal(into[:, 2:6, :128], out)
    into[:, 2:6, :128] = 7.0
    assert (into == 7.0).all()


def test_rows_of_no_request_are_not_written(B):
    kv, q, out = check_attention(B, [50, 9], [4, 9], 4, 2, 128, 32, "bf16")
    off = torch.tensor([2, 4, 10], device="cuda")
    got = torch.full_like(out, 3.0)
    B.ralm_kv_attention(kv, 0, q.cuda(), off, out=got)
    assert (got[:2] == 3.0).all() and (got[10:] == 3.0).all() and not (got[2:10] == 3.0).all()


def test_no_queries_at_all(B):
    kv = make_cache(B, [5], 1, 64, 16)
    assert B.ralm_kv_attention(kv, 0, torch.empty(0, 1, 64, device="cuda", dtype=torch.bfloat16), offsets_of([0])).shape == (0, 1, 64)
    B.ralm_kv_append(kv, 0, torch.empty(0, 1, 64, device="cuda"), torch.empty(0, 1, 64, device="cuda"), offsets_of([0]))


def test_on_another_stream_and_replayed_from_a_graph(B):
    lens, s = [2500, 130], [3, 8]
    kv, q, out = check_attention(B, lens, s, 8, 2, 128, 32, "bf16")
    q, off = q.cuda(), offsets_of(s)
    k, v = (torch.randn(11, 2, 128, device="cuda").bfloat16() for _ in range(2))
    ws = B.alloc_kv_attention_workspace(kv, 8, 11, max_q=8, max_len=2500)
    got = torch.empty_like(out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.ralm_kv_attention(kv, 0, q, off, max_q=8, max_len=2500, out=got, workspace=ws)
    side.synchronize()
    assert torch.equal(got, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ralm_kv_append(kv, 0, k, v, off)
        B.ralm_kv_attention(kv, 0, q, off, max_q=8, max_len=2500, out=got, workspace=ws)
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        k.copy_(torch.randn(k.shape, generator=g, device="cuda"))
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        B.ralm_kv_append(kv, 0, k, v, off)
        want = B.ralm_kv_attention(kv, 0, q, off, max_q=8, max_len=2500)
        assert torch.equal(got, want), seed


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_nan_keys_that_are_all_a_wave_or_part_sees(B, d, dtype):
    """3841 tokens are 241 tiles in parts of 24: the newest token is alone in the last one.  Outputs and lse of the rows that see a NaN
    key are NaN, whoever summed it up."""
    for s in (1, 3):
        check_attention(B, [3841], [s], 8, 2, d, 32, dtype, seed=s + d, nan_at=[(3840, "k")])
    check_attention(B, [3841], [1], 8, 2, d, 32, dtype, seed=d, nan_at=[(t, "k") for t in range(3841)])
    check_attention(B, [1, 100], [1, 1], 4, 2, d, 32, dtype, seed=d, nan_at=[(0, "k")] + [(1 + t, "k") for t in range(96, 100)])


@pytest.mark.parametrize("lens", [[3841], [700, 90]])
def test_queries_that_are_nan(B, lens):
    """Their rows are NaN, and no others: those stay within the bounds of their own roundings."""
    H, d, s = 2, 128, [2] * len(lens)
    kv = make_cache(B, lens, H, d, 32, seed=1)
    K, V = fill_cache(B, kv, lens, 0, "f32", 2)
    q = torch.randn(sum(s), 8, d, generator=torch.Generator().manual_seed(3)).bfloat16()
    bad = q.clone()
    bad[0, 3, 7] = float("nan")
    lse = torch.empty(q.shape[:2], device="cuda")
    got = B.ralm_kv_attention(kv, 0, bad.cuda(), offsets_of(s), max_q=2, max_len=max(lens), lse=lse).double().cpu().numpy()
    assert np.isnan(got[0, 3]).all() and np.isnan(got).sum() == d and torch.isnan(lse[0, 3]) and int(torch.isnan(lse).sum()) == 1
    for r in range(len(lens)):
        want, _, mag, size = kv_plain.attention(q[2 * r:2 * r + 2].double().numpy(), K[r], V[r], d ** -0.5)
        off = np.abs(got[2 * r:2 * r + 2] - want) > kv_plain.attention_tolerance("bf16", want, mag, size, d)
        assert not off.any()                                              # comparisons with NaN are false


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_nan_values_where_a_parts_factor_vanishes(B, d, dtype):
    """The newest token is alone in the last part, and its scores lie hundreds below the largest: its weight is 0 in fp32, its value NaN."""
    check_attention(B, [3841], [1], 8, 2, d, 32, dtype, seed=d, scale=10.0, nan_at=[(3840, "v")])
    check_attention(B, [3841], [3], 8, 2, d, 32, dtype, seed=d, scale=10.0, nan_at=[(3840, "v")])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_read_does_not_write_rows_of_no_request(B, d, dtype):
    """Into buffers of the caller's: rows in front of the first offset and behind the last stay as they are, tokens without a place become zeros."""
    lens, H = [20, 0, 33], 3
    kv = make_cache(B, lens, H, d, 16, seed=d)
    K, V = fill_cache(B, kv, lens, 0, "f32", seed=d + 1)
    off = torch.tensor([4, 9, 9, 12], device="cuda")
    start = torch.tensor([15, 0, 31], dtype=torch.int32, device="cuda")
    kv.table[2, 2] = -1                                                   # token 32 of the last request has no place
    k, v = (torch.full((17, H, d), 7.0, device="cuda", dtype=DT[dtype]) for _ in range(2))
    B.ralm_kv_read(kv, 0, off, 17, start=start, k=k, v=v)
    for got, held in ((k, K), (v, V)):
        assert (got[:4] == 7.0).all() and (got[12:] == 7.0).all()
        want = np.concatenate([held[0][15:], held[2][31:32], np.zeros((2, H, d))])
        assert np.array_equal(got[4:12].double().cpu().numpy(), torch.from_numpy(want).to(DT[dtype]).double().numpy())


def test_many_requests_without_hints(B):
    """As many row tiles as all queries could make, times all requests, are more workgroups than a launch has: they are gone through in turn."""
    R = 1 << 14
    rng = np.random.default_rng(3)
    lens = rng.integers(1, 4, size=R).tolist()
    s = [min(n, int(k)) for n, k in zip(lens, rng.integers(0, 3, size=R))]
    lens[77], s[77] = 90, 70
    check_attention(B, lens, s, 1, 1, 64, 16, "bf16", hints=(0, 0), seed=5)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 50])
def test_chunks_by_waves_with_rows_of_their_own_by_the_hint(B, d, dtype, window):
    """A hint of 256 queries in every request: the launch is that of many rows, of which waves have all, some or none."""
    rng = np.random.default_rng(d + window)
    lens = [200, 16, 75, 130, 33, 90, 64]
    s = [min(n, int(rng.integers(50, 76))) for n in lens]
    assert sum(s) >= 256                                                  # a hint beyond all queries says nothing
    check_attention(B, lens, s, 40, 10, d, 32, dtype, window=window, sinks=3, seed=d, hints=(256, 200), nan_at=[(100, "v"), (150, "k"), (190, "v")])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_chunk_among_single_tokens_without_a_hint(B, dtype):
    """The launch is that for the mean: the chunk's row tiles are more than there are workgroups for them."""
    lens = [1, 300, 17, 33, 90, 2, 64, 150] * 40
    s = [1] * len(lens)
    s[1], lens[1] = 290, 300
    check_attention(B, lens, s, 8, 2, 64, 32, dtype, seed=9, hints=(0, 0))
    check_attention(B, lens, s, 8, 2, 64, 32, dtype, seed=9, hints=(0, 0), window=40, sinks=2)
