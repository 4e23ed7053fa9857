"""The target of a verification (ralm_knnlm_target) against its formula in 64 bits.

A probability of z = (logit - largest) / T is off by the rounding of z (3 roundings, 3 2^-24 |z| of the probability), of the exponential (2), of the sum of a row
(8 in a piece, one per join of a piece, wave and workgroup: less than 64 + V / 8192) and of the mixture (4); the neighbours' sum by k 2^-24."""
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


def formula(logits, tokens, weights, share, T):
    x = logits.double() / T
    top = x.max(-1, keepdim=True).values
    z = torch.where(torch.isinf(x), torch.zeros_like(x), x - top)
    p = torch.softmax(x, -1)
    p = torch.where(torch.isnan(p), torch.zeros_like(p), p)                       # nothing but -inf
    Q, V = logits.shape
    sh = share.double().view(-1, 1) if isinstance(share, torch.Tensor) else torch.full((Q, 1), float(torch.tensor(share)), dtype=torch.float64, device=x.device)
    near = torch.zeros_like(p)
    ok = (tokens >= 0) & (tokens < V)
    near.scatter_add_(1, tokens.long().clamp(0, V - 1), torch.where(ok, weights.double(), torch.zeros_like(weights.double())))
    want = (1 - sh) * p + sh * near
    err = p * U * (5 * z.abs() + 2 * 64 + V / 4096) + sh * near * U * (tokens.shape[1] + 4) + 4 * U * want
    return want, err


def near(got, want, err):
    dt = got.dtype
    return bool(((got.double() - want).abs() <= err + torch.finfo(dt).eps / 2 * (want + err) + torch.finfo(dt).tiny * torch.finfo(dt).eps).all())


def inputs(Q, V, k, dtype, seed, same=4):
    g = torch.Generator().manual_seed(seed)
    logits = (torch.randn(Q, V, generator=g) * 3).to(DT[dtype]).cuda()
    few = torch.randint(0, V, (Q, same), generator=g)
    tokens = few.gather(1, torch.randint(0, same, (Q, max(k, 1)), generator=g))[:, :k].to(torch.int32)
    other = torch.randint(-1, V, (Q, k), generator=g, dtype=torch.int32)
    tokens = torch.where(torch.rand(Q, k, generator=g) < 0.5, tokens, other)
    return logits, tokens.cuda(), torch.rand(Q, k, generator=g).cuda(), torch.rand(Q, generator=g).cuda()


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("Q,V,k", [(1, 1, 1), (1, 7, 0), (3, 8, 5), (2, 9, 1), (5, 100, 16), (4, 1023, 64), (300, 513, 8), (3, 8193, 1024), (2, 32000, 20), (7, 50257, 16),
                                   (1, 131_075, 33), (2, 300_001, 4), (1, 1 << 20, 7)])
def test_formula(b, Q, V, k, dtype, out):
    logits, tokens, weights, share = inputs(Q, V, k, dtype, Q * 1000 + V)
    for s, T in ((share, 0.7), (0.25, 1.0), (0.0, 3.0), (1.0, 1.0)):
        want, err = formula(logits, tokens, weights, s, T)
        got = b.ralm_knnlm_target(logits, tokens, weights, s, temperature=T, out_dtype=DT[out])
        assert got.dtype == DT[out] and near(got, want, err)


@pytest.mark.parametrize("V", [1000, 40_003])
def test_strides_and_in_place(b, V):
    logits, tokens, weights, share = inputs(3, V, 9, "f32", 5)
    want = b.ralm_knnlm_target(logits, tokens, weights, share)
    wide = torch.full((3, V + 5), float("nan"), device="cuda")
    wide[:, :V] = logits
    big = torch.full((5, V + 3), 7.0, device="cuda")
    b.ralm_knnlm_target(wide[:, :V], tokens, weights, share, out=big[1:4, 1:V + 1])
    assert torch.equal(big[1:4, 1:V + 1], want)
    big[1:4, 1:V + 1] = 7.0
    assert bool((big == 7.0).all())
    own = logits.clone()
    assert b.ralm_knnlm_target(own, tokens, weights, share, out=own) is own and torch.equal(own, want)
    one = logits[:1].expand(3, -1)
    assert torch.equal(b.ralm_knnlm_target(one, tokens, weights, share), b.ralm_knnlm_target(one.contiguous(), tokens, weights, share))


@pytest.mark.parametrize("V", [100, 70_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_infinities_and_nan(b, V, dtype):
    logits, tokens, weights, _ = inputs(7, V, 6, dtype, 3)
    logits[1, :V // 2] = float("-inf")                                            # half of the vocabulary is forbidden
    logits[2] = float("-inf")                                                     # all of it
    logits[3] = torch.finfo(DT[dtype]).min                                        # masks of the type's lowest value: an even distribution
    logits[4, 5] = float("nan")
    logits[5, V - 1] = float("inf")
    logits[6] = -1e30 if dtype == "f32" else logits[6]
    logits[6, 3] = 1e30
    got = b.ralm_knnlm_target(logits, tokens, weights, 0.5)
    ok = [0, 1, 2, 3, 6]
    want, err = formula(logits[ok], tokens[ok], weights[ok], 0.5, 1.0)
    assert near(got[ok], want, err)
    assert bool(got[4].isnan().all()) and bool(got[5].isnan().all())


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("Q,V,k", [(128, 10_001, 16), (131, 16_385, 65), (130, 20_003, 100), (129, 32_768, 16), (128, 50_257, 5), (133, 65_535, 3)])
def test_rows_of_one_workgroup(b, Q, V, k, dtype, out):
    """Long rows, enough of them for one to be a workgroup's: masks and what is no number among them, rows that lie apart, in place."""
    logits, tokens, weights, share = inputs(Q, V, k, dtype, V)
    logits[1, :V // 2] = float("-inf")
    logits[2] = float("-inf")
    logits[3] = torch.finfo(DT[dtype]).min
    logits[4, 5] = float("nan")
    logits[5, V - 1] = float("inf")
    rest = torch.tensor([i for i in range(Q) if i not in (4, 5)], device="cuda")
    want, err = formula(logits[rest], tokens[rest], weights[rest], share[rest], 0.7)
    big = torch.full((Q, V + 3), 7.0, dtype=DT[out], device="cuda")
    got = b.ralm_knnlm_target(logits, tokens, weights, share, temperature=0.7, out=big[:, 1:V + 1])
    assert near(got[rest], want, err) and bool(got[4:6].isnan().all())
    if dtype == out:
        own = logits.clone()
        assert b.ralm_knnlm_target(own, tokens, weights, share, temperature=0.7, out=own) is own and torch.equal(own[rest], got[rest])
    got.fill_(7.0)
    assert bool((big == 7.0).all())


def test_a_tokens_weights_add_up_in_order(b):
    """All neighbours are one token: the sum is that of fp32 additions in their order, call after call."""
    k = 1024
    g = torch.Generator().manual_seed(8)
    w = torch.rand(1, k, generator=g) * torch.exp(3 * torch.randn(1, k, generator=g))
    tokens = torch.full((1, k), 3, dtype=torch.int32, device="cuda")
    logits = torch.full((1, 11), float("-inf"), device="cuda")
    s = torch.zeros((), dtype=torch.float32)
    for x in w[0]:
        s = s + x
    for _ in range(3):
        got = b.ralm_knnlm_target(logits, tokens, w.cuda(), 1.0)
        assert float(got[0, 3]) == float(s) and float(got.sum()) == float(s)


@pytest.mark.parametrize("Q,V", [(2, 50_257), (40, 3000), (1, 300_000)])
def test_graph_replays(b, Q, V):
    logits, tokens, weights, share = inputs(Q, V, 16, "bf16", 1)
    other = inputs(Q, V, 16, "bf16", 2)[0]
    ws, out = b.alloc_knnlm_target_workspace(Q, V), torch.empty(Q, V, device="cuda")
    want = [b.ralm_knnlm_target(x, tokens, weights, share) for x in (logits, other)]
    buf = logits.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.ralm_knnlm_target(buf, tokens, weights, share, out=out, workspace=ws)
    for i in range(4):
        buf.copy_((logits, other)[i % 2])
        graph.replay()
        assert torch.equal(b.ralm_knnlm_target(other, tokens, weights, share), want[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want[i % 2])


def test_no_rows(b):
    e = torch.empty(0, 3, device="cuda")
    assert b.ralm_knnlm_target(torch.empty(0, 50, device="cuda"), e.to(torch.int32), e, 0.5).shape == (0, 50)
