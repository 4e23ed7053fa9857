"""Products with epilogues (ralm_linear) against the formula in 64 bits.

Whole numbers: products and sums of small whole numbers are exact in fp32 in any order, so fp32 outputs must be equal and 16-bit ones the
rounding of the exact sum.  Other numbers: a sum of K products in fp32 is off by at most K 2^-24 of the sum of their magnitudes,
whatever its order; the activations have slopes of at most 1.13 and add less than 8 roundings."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2401_14021_amd import binding
    return binding


def whole(g, n, m, top, dt):
    return torch.randint(-top, top + 1, (n, m), generator=g).to(dt).cuda()


def pitched(t, pad):
    """The same matrix with rows further apart; NaN in between."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


# rows around the lines between kernels and tiles; outputs and depths with remainders of every kind
SHAPES = [(1, 1, 8), (1, 64, 64), (1, 1024, 1024), (2, 17, 24), (3, 130, 72), (5, 257, 136), (8, 4099, 64), (15, 96, 1096), (16, 128, 512),
          (17, 33, 200), (31, 1000, 128), (32, 512, 4096), (33, 48, 520), (45, 300, 328), (48, 2049, 8), (63, 65, 56), (64, 256, 2048), (65, 255, 64),
          (96, 511, 264), (100, 1, 1024), (127, 129, 8), (128, 384, 640), (129, 1027, 72), (200, 2000, 192), (255, 256, 1000), (256, 512, 512),
          (257, 513, 264), (300, 4096, 128), (700, 130, 2056), (1025, 640, 64), (2050, 257, 40)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_whole_numbers(b, T, N, K, dtype):
    g = torch.Generator().manual_seed(T * 7919 + N * 31 + K)
    dt = DT[dtype]
    x, w = whole(g, T, K, 3, dt), whole(g, N, K, 3, dt)
    want = x.double() @ w.double().T.contiguous()
    assert torch.equal(b.ralm_linear(x, w, out_dtype=torch.float32).double(), want)
    bias, res = whole(g, 1, N, 9, dt)[0], whole(g, T, N, 99, torch.float32)
    got = b.ralm_linear(x, w, bias=bias, act="relu", residual=res)
    assert torch.equal(got.double(), (want + bias.double()).clamp(min=0) + res.double())
    # 16-bit outputs: small enough that the sum is rounded once from an exact fp32 number
    got = b.ralm_linear(x, w, bias=bias, residual=res.to(dt))
    assert got.dtype == dt and torch.equal(got, (want + bias.double() + res.to(dt).double()).float().to(dt))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_whole_numbers_gated(b, T, N, K, dtype):
    g = torch.Generator().manual_seed(T * 31 + N * 7919 + K)
    dt = DT[dtype]
    x, w = whole(g, T, K, 1, dt), whole(g, 2 * N, K, 1, dt)
    bias = whole(g, 1, 2 * N, 5, dt)[0]
    y = x.double() @ w.double().T.contiguous() + bias.double()
    want = y[:, :N].clamp(min=0) * y[:, N:]
    assert float(want.abs().max()) < 2 ** 24
    assert torch.equal(b.ralm_linear(x, w, bias=bias, act="relu", gated=True, out_dtype=torch.float32).double(), want)
    res = whole(g, T, N, 99, torch.float32)
    assert torch.equal(b.ralm_linear(x, w, bias=bias, act="relu", gated=True, residual=res).double(), want + res.double())


# sizes that reach every tile, with whole and broken strips, the depth in one part and in several
TILES = [(259, 131, 64), (280, 129, 8), (286, 137, 768), (271, 137, 728), (194, 4761, 384), (133, 5493, 368), (20, 2209, 5888), (17, 2767, 4312),
         (661, 7659, 128), (665, 7429, 72), (4489, 133, 3584), (2734, 157, 5048), (2083, 5817, 192), (3877, 2081, 248), (285, 7411, 3200),
         (137, 5471, 5896), (1709, 8131, 384), (2718, 4465, 328), (3796, 1061, 3392), (1181, 3567, 3256),
         (665, 5475, 4608), (1297, 3267, 4384), (16, 8192, 2048), (16, 1027, 16384), (48, 4099, 4096), (200, 2051, 4096)]
TILES_GATED = [(259, 131, 64), (280, 129, 8), (24, 131, 6144), (21, 157, 5640), (72, 4291, 384), (69, 5105, 368), (18, 1725, 3904), (17, 1509, 4424),
               (661, 3917, 128), (484, 5299, 72), (130, 1851, 5120), (1878, 147, 5384), (836, 4761, 256), (668, 8191, 136), (141, 5733, 2432),
               (154, 5473, 2448), (4283, 1417, 384), (1183, 5497, 328), (1207, 1669, 3648), (194, 5641, 5304), (201, 5773, 4560), (201, 5723, 5248),
               (16, 4096, 8192), (45, 4099, 4096)]


@pytest.mark.parametrize("T,N,K,gated", [(*s, False) for s in TILES] + [(*s, True) for s in TILES_GATED])
def test_every_tile(b, T, N, K, gated):
    """Whole numbers again, from operands whose rows lie apart with NaN between them: what is read behind a row's end would show."""
    g = torch.Generator(device="cuda").manual_seed(T + N + K)
    rows = 2 * N if gated else N
    draw = lambda n, m, top: torch.randint(-top, top + 1, (n, m), generator=g, device="cuda").bfloat16()
    x, w, bias, res = draw(T, K, 1), draw(rows, K, 1), draw(1, rows, 5)[0], draw(T, N, 99).float()
    y = x.double() @ w.double().T.contiguous() + bias.double()
    want = y[:, :N].clamp(min=0) * y[:, N:] if gated else y.clamp(min=0)
    assert float(want.abs().max()) < 2 ** 23
    big = torch.full((T + 1, N + 5), 7.0, device="cuda")
    out = big[:T, 1:N + 1]
    b.ralm_linear(pitched(x, 8), pitched(w, 24), bias=bias, act="relu", gated=gated, residual=res, out=out)
    assert torch.equal(out.double(), want + res.double())
    out.fill_(7.0)
    assert bool((big == 7.0).all())
    assert torch.equal(b.ralm_linear(x, w, bias=bias, act="relu", gated=gated), want.float().bfloat16())


@pytest.mark.parametrize("T,N,K", [(1, 131, 72), (20, 77, 264), (64, 300, 136), (130, 259, 200), (520, 300, 520)])
@pytest.mark.parametrize("gated", [False, True])
def test_strides(b, T, N, K, gated):
    """Rows that are further apart, with NaN between them; an output inside a larger one, of which nothing else is written; outputs and
    residuals that are aligned to nothing but their type."""
    g = torch.Generator().manual_seed(3)
    rows = 2 * N if gated else N
    x, w = whole(g, T, K, 1, torch.bfloat16), whole(g, rows, K, 1, torch.bfloat16)
    res = whole(g, T, N, 9, torch.float32)
    y = x.double() @ w.double().T.contiguous()
    want = (y[:, :N] * y[:, N:] if gated else y) + res.double()
    for out_dtype in (torch.float32, torch.bfloat16):
        big = torch.full((T + 2, N + 7), 7.0, dtype=out_dtype, device="cuda")
        out = big[1:T + 1, 3:N + 3]
        b.ralm_linear(pitched(x, 8), pitched(w, 24), gated=gated, residual=pitched(res.to(out_dtype), 1), out=out)
        assert torch.equal(out, want.float().to(out_dtype))
        out.fill_(7.0)
        assert bool((big == 7.0).all())


@pytest.mark.parametrize("T", [1, 30, 64, 200, 600])
def test_in_place_residual_and_repeated_inputs(b, T):
    g = torch.Generator().manual_seed(5)
    x, w = whole(g, T, 128, 2, torch.float16), whole(g, 200, 128, 2, torch.float16)
    res = whole(g, T, 200, 50, torch.float32)
    want = x.double() @ w.double().T.contiguous() + res.double()
    stream = res.clone()
    assert b.ralm_linear(x, w, residual=stream, out=stream) is stream and torch.equal(stream.double(), want)
    one = x[:1].expand(T, -1)                                   # a view that repeats a row
    assert torch.equal(b.ralm_linear(one, w, out_dtype=torch.float32), b.ralm_linear(one.contiguous(), w, out_dtype=torch.float32))
    assert torch.equal(b.ralm_linear(x.t().contiguous().t(), w, out_dtype=torch.float32).double(), want - res.double())
    with pytest.raises(AssertionError):
        b.ralm_linear(x, w, out=torch.empty(1, 200, dtype=torch.float16, device="cuda").expand(max(T, 2), -1)[:T] if T > 1 else torch.empty(1, 1, device="cuda"))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T,dtype", [(1, "bf16"), (7, "f16"), (40, "bf16"), (90, "f16"), (333, "bf16")])
def test_activations(b, T, dtype, act, gated):
    N, K = 301, 520
    g = torch.Generator().manual_seed(11)
    dt = DT[dtype]
    rows = 2 * N if gated else N
    x = torch.randn(T, K, generator=g).to(dt).cuda()
    w = (torch.randn(rows, K, generator=g) * 3 * K ** -0.5).to(dt).cuda()      # sums with a spread of 3
    bias = torch.randn(rows, generator=g).to(dt).cuda()
    res = torch.randn(T, N, generator=g).cuda()
    s = x.double() @ w.double().T.contiguous() + bias.double()
    err = (K + 2) * 2.0 ** -24 * (x.double().abs() @ w.double().abs().T.contiguous() + bias.double().abs())
    y = s[:, :N]
    f = {"none": y, "relu": y.clamp(min=0), "silu": y * torch.sigmoid(y), "gelu": y * 0.5 * torch.erfc(-y * 0.5 ** 0.5),
         "gelu_tanh": y * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (y + 0.044715 * y ** 3))}[act]
    # the argument of an exponential or error function of y is rounded too: 8 roundings of it move the result by 8 2^-24 times |y|^2 at most 2 |y|
    tol = 1.13 * err[:, :N] + 8 * 2.0 ** -24 * (f.abs() + y.abs() * (1 + y * y * torch.exp(-y.abs())))
    if gated:
        up = s[:, N:]
        tol = tol * (up.abs() + err[:, N:]) + f.abs() * err[:, N:]
        f = f * up
    want = f + res.double()
    tol = tol + 3 * 2.0 ** -24 * (f.abs() + want.abs())
    got = b.ralm_linear(x, w, bias=bias, act=act, gated=gated, residual=res)
    assert bool(((got.double() - want).abs() <= tol).all())
    half = b.ralm_linear(x, w, bias=bias, act=act, gated=gated)                  # one rounding to 16 bits more
    assert bool(((half.double() - f).abs() <= tol + torch.finfo(dt).eps / 2 * (f.abs() + tol) + torch.finfo(dt).tiny * 2.0 ** -10).all())


@pytest.mark.parametrize("T", [1, 70])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_activations_far_out(b, T, act):
    """Beyond every exponential's range an activation is its argument or nothing, and infinite where that is."""
    x, w = torch.zeros(T, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda")
    x[:, 0], w[:, 0] = 1.0, torch.tensor([float("inf"), 1e30, 200.0, -1e30, -200.0])
    got, sums = b.ralm_linear(x, w, act=act, out_dtype=torch.float32), w[:, 0].float()
    assert torch.equal(got[:, :3], sums[:3].expand(T, -1))
    assert torch.equal(got[:, 3:], (sums[3:] if act == "none" else torch.zeros(2, device="cuda")).expand(T, -1))


@pytest.mark.parametrize("T", [1, 20, 64, 150, 400])
def test_infinities_and_nan_stay_in_their_rows(b, T):
    g = torch.Generator().manual_seed(2)
    N, K = 150, 136                                             # a depth that ends inside a strip
    x, w = whole(g, T, K, 2, torch.bfloat16), whole(g, N, K, 2, torch.bfloat16)
    w[w == 0] = 1.0
    clean = b.ralm_linear(x, w, out_dtype=torch.float32)
    y = x.clone()
    y[0, 5], w2 = float("nan"), w.clone()
    if T > 1:
        y[T - 1, K - 1] = float("inf")
    w2[N - 1, K - 1] = float("inf")
    x1 = x.clone()
    x1[x1 == 0] = 1.0
    got = b.ralm_linear(y, w, out_dtype=torch.float32)
    assert bool(got[0].isnan().all()) and torch.equal(got[1:T - 1], clean[1:T - 1])
    if T > 1:
        assert bool(got[T - 1].isinf().all())
    got = b.ralm_linear(x1, w2, out_dtype=torch.float32)
    assert bool(got[:, N - 1].isinf().all()) and torch.equal(got[:, :N - 1], b.ralm_linear(x1, w, out_dtype=torch.float32)[:, :N - 1])


@pytest.mark.parametrize("T,N,K", [(1, 512, 1024), (16, 500, 2048), (50, 777, 4096), (120, 640, 2048), (700, 513, 512)])
def test_same_from_call_to_call_and_in_graphs(b, T, N, K):
    """Two captured graphs with workspaces of their own, replayed in turn with eager calls between them."""
    g = torch.Generator().manual_seed(9)
    w = torch.randn(N, K, generator=g).bfloat16().cuda()
    xs = [torch.randn(T, K, generator=g).bfloat16().cuda() for _ in range(3)]
    want = [b.ralm_linear(x, w, act="gelu") for x in xs]
    graphs = []
    for i in range(2):
        buf, out, ws = xs[i].clone(), torch.empty_like(want[0]), b.alloc_linear_workspace(T, N, K)
        gr = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        with torch.cuda.graph(gr, stream=side):
            b.ralm_linear(buf, w, act="gelu", out=out, workspace=ws)
        graphs.append((gr, buf, out))
    for k in range(4):
        for i, (gr, buf, out) in enumerate(graphs):
            j = (i + k) % 3
            buf.copy_(xs[j])
            gr.replay()
            assert torch.equal(b.ralm_linear(xs[(j + 1) % 3], w, act="gelu"), want[(j + 1) % 3])
            torch.cuda.synchronize()
            assert torch.equal(out, want[j])


def test_streams(b):
    """Calls on two streams at once, each with a workspace of its own."""
    g = torch.Generator().manual_seed(4)
    w = torch.randn(1000, 2048, generator=g).bfloat16().cuda()
    x = [torch.randn(n, 2048, generator=g).bfloat16().cuda() for n in (20, 60)]
    want = [b.ralm_linear(y, w) for y in x]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = b.ralm_linear(x[i], w)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_no_rows(b):
    w = torch.ones(16, 64, dtype=torch.bfloat16, device="cuda")
    assert b.ralm_linear(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), w).shape == (0, 16)


def test_wide_outputs_and_far_rows(b):
    """More than 2^31 bytes of output: offsets beyond 32 bits."""
    T, N, K = 4200, 131_077, 8
    x = torch.ones(T, K, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = (torch.arange(T, device="cuda") % 97).bfloat16()
    w = torch.ones(N, K, dtype=torch.bfloat16, device="cuda")
    w[:, 1] = (torch.arange(N, device="cuda") % 89).bfloat16()
    out = b.ralm_linear(x, w, out_dtype=torch.float32)
    for t in (0, 1, 4095, 4096, T - 1):
        assert torch.equal(out[t], (t % 97) + 6.0 + torch.arange(N, device="cuda") % 89)
