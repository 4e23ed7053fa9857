"""Activations of ralm_linear apart from its sums: every sum is exact, so that what differs from the formula in 64 bits is the activation's own error.

A sum is y = a + b of two 16-bit numbers, by weights (a, b, 0, ..) and rows (1, 1, 0, ..).  Roundings, each at most 2^-24 of what is rounded; rcp and exp2 of the hardware
are good to 2:

  gelu       y Phi(y), Phi(-|y|) = exp(-y^2 / 2) t P(t), t = 1 / (1 + p |y|).  t 3 (its effect on t P(t) below 1.3 times as much); the Horner steps, whose partial sums
             add up to 4 times the last one at t = 1 where they weigh most, 4, the product with t 1; the exponential 2 and its correction 1; three products and a difference 4:
             16 in all.  16-bit outputs may take 128 (2^-17), 1/64 of bf16's half step and 1/16 of fp16's, and the step itself.
  gelu_tanh  y / (1 + exp(-v)), v = 2 sqrt(2 / pi) (y + 0.044715 y^3): v by 6 roundings, its product with log2 e 1.5 more, which exp takes as 7.5 |v|; then 2 + 1 + 2 + 1
  silu       y / (1 + exp(-y)): 1.5 |y|, and 6

Below 2^-118 the exponentials are nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2401_14021_amd import binding
    return binding


def sums():
    """[-13, 13] by steps of 1/512, and powers of two around nothing."""
    small = 2.0 ** -torch.arange(1, 15, dtype=torch.float64)
    return torch.cat([torch.arange(-13 * 512, 13 * 512 + 1, dtype=torch.float64) / 512, small, -small]).cuda()


def formula(act, y):
    """The activation, and the roundings of 2^-24 of it that fp32 may take."""
    v = 2 * (2 / torch.pi) ** 0.5 * (y + 0.044715 * y ** 3)
    six = torch.full_like(y, 6.0)
    return {"none": (y, 0 * y), "relu": (y.clamp(min=0), 0 * y), "silu": (y * torch.sigmoid(y), six + 1.5 * y.abs()),
            "gelu": (y * 0.5 * torch.erfc(-y * 0.5 ** 0.5), 0 * y + 16), "gelu_tanh": (y * torch.sigmoid(v), six + 7.5 * v.abs())}[act]


def off_by(act, y, got, step=0.0, least=0.0):
    """The largest error in units of what is allowed; step: of the output's own rounding, least: of its smallest numbers."""
    f, roundings = formula(act, y)
    if step and act == "gelu":
        roundings = roundings + 112
    return float(((got.double() - f).abs() / (f.abs() * (roundings * 2.0 ** -24 + step) + 2.0 ** -118 + least)).max())


def call(b, y, T, K, dt, act, gated, out_dtype):
    high = y.to(dt)                             # 8 or 11 of y's 13 bits
    low = (y - high.double()).to(dt)
    assert torch.equal(high.double() + low.double(), y)
    w = torch.zeros(len(y), K, dtype=dt, device="cuda")
    w[:, 0], w[:, K - 1] = high, low
    if gated:
        up = torch.zeros_like(w)
        up[:, 0] = 1.0
        w = torch.cat([w, up])
    x = torch.zeros(T, K, dtype=dt, device="cuda")
    x[:, 0] = x[:, K - 1] = 1.0
    return b.ralm_linear(x, w, act=act, gated=gated, out_dtype=out_dtype)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T,K,dtype", [(1, 8, "bf16"), (3, 136, "f16"), (64, 4096, "bf16"), (70, 72, "f16"), (300, 8, "bf16")])
def test_exact_sums(b, T, K, dtype, gated, act):
    y, dt = sums(), DT[dtype]
    got = call(b, y, T, K, dt, act, gated, torch.float32)
    assert bool((got == got[:1]).all())
    assert off_by(act, y, got[0]) <= 1
    got = call(b, y, T, K, dt, act, gated, dt)
    assert off_by(act, y, got[0], torch.finfo(dt).eps / 2, torch.finfo(dt).tiny * torch.finfo(dt).eps / 2) <= 1


def test_the_two_gelus_differ_by_more(b):
    """One in the place of the other would not pass, nor one that is off by 2^-14 of its value."""
    y = sums()
    f = formula("gelu", y)[0]
    assert off_by("gelu_tanh", y, f) > 30 and off_by("gelu", y, formula("gelu_tanh", y)[0]) > 30
    assert off_by("gelu", y, f * (1 + 2.0 ** -14)) > 30 and off_by("gelu", y, f) <= 1
