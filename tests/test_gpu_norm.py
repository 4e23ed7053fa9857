"""Norms of the residual stream (ralm_residual_norm) against the formulas in 64 bits.

A sum over a row is at most 32 additions in a thread, 6 across a wave and 16 across waves: less than 64 roundings of 2^-24, as are a mean's and a
variance's.  A normed number moves by that share of itself and of the row's mean magnitude in units of the spread."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2401_14021_amd import binding
    return binding


def norm64(y, kind, w, bias, eps, err=0.0):
    """(norm, how far fp32 may be off) of rows y that may themselves be off by err."""
    mean = y.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(y[:, :1])
    c = y - mean
    r = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    w = torch.ones_like(y[0]) if w is None else w.double()
    o = torch.zeros_like(y[0]) if bias is None else bias.double()
    out = c * r * w + o
    # a wrong mean moves every number, a wrong spread scales them; err moves a number by itself, the mean and the spread by at most its root mean square
    scale = (c.abs() + y.abs().mean(-1, keepdim=True)) * r * w.abs()
    e = err + torch.zeros_like(y)
    rms = e.square().mean(-1, keepdim=True).sqrt()
    return out, 160 * U * (scale + o.abs()) + (e + rms + c.abs() * r * rms) * r * w.abs() * 1.1


def formula(x, res, kind, w, bias, post, pw, pb, gate, scale, eps):
    y, e = x.double(), 0.0
    if post:
        y, e = norm64(y, kind, pw, pb, eps)
    k = scale * (1.0 if gate is None else gate.double())
    y, e = y * k, (e * k.abs() if gate is not None else e * abs(scale))
    s = y if res is None else res.double() + y
    e = e + 4 * U * (y.abs() + s.abs())
    out, oe = norm64(s, kind, w, bias, eps, e)
    return s, e, out, oe


def near(got, want, err):
    dt = got.dtype
    step = torch.finfo(dt).eps / 2
    tiny = torch.finfo(dt).tiny * torch.finfo(dt).eps
    return bool(((got.double() - want).abs() <= err + step * (want.abs() + err) + tiny).all())


SIZES = [(1, 1), (3, 2), (5, 63), (4, 64), (2, 100), (7, 512), (6, 513), (3, 768), (4, 1024), (1, 1032), (2, 2048), (3, 2049), (2, 4096), (3, 4104), (1, 5000),
         (2, 8192), (2, 8200), (1, 16384), (2, 16391), (1, 32768), (300, 96), (1001, 24)]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("T,D", SIZES)
def test_formulas(b, T, D, kind):
    g = torch.Generator().manual_seed(T * 100_003 + D)
    r = lambda *n: torch.randn(*n, generator=g)  # noqa: E731
    for i, (xd, sd, od, pd) in enumerate([("bf16", "f32", "bf16", "bf16"), ("f16", "f16", "f16", "f32"), ("f32", "f32", "f32", "f32"), ("bf16", "bf16", "f32", "f16")]):
        x, res = (r(T, D) * 2 + 0.5).to(DT[xd]).cuda(), (r(T, D) * 3 - 1).to(DT[sd]).cuda()
        w, bias, pw, pb = ((1 + 0.2 * r(D)).to(DT[pd]).cuda() if i != 2 else None, (0.3 * r(D)).to(DT[pd]).cuda() if i & 1 else None,
                           (1 + 0.2 * r(D)).to(DT[pd]).cuda(), (0.3 * r(D)).to(DT[pd]).cuda() if i > 1 else None)
        gate = [None, r(D), r(T, D), None][i]
        gate = None if gate is None else gate.to(DT[xd]).cuda()
        for post in (False, True):
            s, out = b.ralm_residual_norm(x, res, kind=kind, weight=w, bias=bias, post=post, post_weight=pw if post else None,
                                          post_bias=pb if post else None, gate=gate, scale=0.5, eps=1e-5, out_dtype=DT[od])
            assert s.dtype == DT[sd] and out.dtype == DT[od]
            s64, se, o64, oe = formula(x, res, kind, w, bias, post, pw, pb, gate, 0.5, 1e-5)
            assert near(s, s64, se) and near(out, o64, oe), (i, post)


@pytest.mark.parametrize("T,D", [(5, 100), (3, 1024), (2, 4096), (2, 10_000)])
def test_parts_alone_in_place_and_strides(b, T, D):
    g = torch.Generator().manual_seed(D)
    x, res = torch.randn(T, D, generator=g).bfloat16().cuda(), torch.randn(T, D, generator=g).bfloat16().cuda()
    s, out = b.ralm_residual_norm(x, res)
    only, none = b.ralm_residual_norm(x, res, want_out=False)
    assert none is None and torch.equal(only, s)
    none, only = b.ralm_residual_norm(x, res, want_sum=False)
    assert none is None and torch.equal(only, out)
    s0, o0 = b.ralm_residual_norm(x)                                             # no residual: the norm of x
    assert torch.equal(s0, x)
    _, _, want, err = formula(x, None, "rms", None, None, False, None, None, None, 1.0, 1e-6)
    assert near(o0, want, err)
    stream, y = res.clone(), x.clone()                                           # the stream and x in place
    b.ralm_residual_norm(y, stream, sum=stream, out=y)
    assert torch.equal(stream, s) and torch.equal(y, out)
    for pad in (1, 8):                                                           # rows further apart, NaN between them
        wide = torch.full((2, T, D + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[0, :, :D], wide[1, :, :D] = x, res
        big = torch.full((2, T + 2, D + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        b.ralm_residual_norm(wide[0, :, :D], wide[1, :, :D], sum=big[0, 1:T + 1, :D], out=big[1, 1:T + 1, :D])
        assert torch.equal(big[0, 1:T + 1, :D], s) and torch.equal(big[1, 1:T + 1, :D], out)
        big[:, 1:T + 1, :D] = 7.0
        assert bool((big == 7.0).all())
    gate = torch.randn(1, D, generator=g).bfloat16().cuda()
    a, c = b.ralm_residual_norm(x, res, gate=gate.expand(T, -1)), b.ralm_residual_norm(x, res, gate=gate[0])
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_edges_of_the_numbers(b, kind):
    """Rows of zeros (eps alone is under the root), constant rows, one number, a large mean, infinities and NaN in rows of their own."""
    D = 1024
    x = torch.zeros(6, D, device="cuda")
    x[1] = 3.0
    x[2, 7] = 5.0
    x[3] = 4096.0 + torch.arange(D, device="cuda") % 2
    x[4, 0] = float("inf")
    x[5, D - 1] = float("nan")
    s, out = b.ralm_residual_norm(x, kind=kind, eps=1e-6)
    assert torch.equal(out[0], torch.zeros(D, device="cuda"))
    _, _, want, err = formula(x[:4], None, kind, None, None, False, None, None, None, 1.0, 1e-6)
    assert near(out[:4], want, err)
    assert bool(out[4].isnan().any()) and bool(out[5].isnan().all()) and bool(out[:4].isfinite().all())
    if kind == "layer":   # neighbours 4096 and 4097: +-1 behind the mean, which a difference of mean squares would lose
        assert float((out[3].abs() - 1.0).abs().max()) < 1e-3


def test_graph_replays(b):
    g = torch.Generator().manual_seed(1)
    x, res = torch.randn(9, 1500, generator=g).bfloat16().cuda(), torch.randn(9, 1500, generator=g).cuda()
    stream, out = res.clone(), torch.empty_like(x)
    b.ralm_residual_norm(x, res, kind="layer", post=True, sum=stream, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.ralm_residual_norm(x, stream, kind="layer", post=True, sum=stream, out=out)
    stream.copy_(res)
    eager = res.clone()
    for _ in range(4):
        graph.replay()
        _, want = b.ralm_residual_norm(x, eager, kind="layer", post=True, sum=eager)
        torch.cuda.synchronize()
        assert torch.equal(stream, eager) and torch.equal(out, want)


def test_no_rows(b):
    s, out = b.ralm_residual_norm(torch.empty(0, 64, device="cuda"))
    assert s.shape == out.shape == (0, 64)
