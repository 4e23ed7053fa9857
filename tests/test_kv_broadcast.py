"""Views that repeat rows or heads (a stride of 0 in torch, which the C ABI reads as "dense"): what the library is handed describes the
tensor's numbers, and outputs that repeat memory are refused.  Without a GPU: the library is a stub that reads the memory it is told of."""
import ctypes
import os

import numpy as np
import pytest
import torch


@pytest.fixture
def b(monkeypatch):
    from paper_2401_14021_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2401_14021_amd import build
        build.build()
    real = binding.lib()
    stub = Stub(real)
    monkeypatch.setattr(binding, "lib", lambda: stub)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    binding.stub = stub
    yield binding
    del binding.stub


def numbers(p, shape, strides):
    """fp32 numbers at p; no stride may be one that the C ABI replaces by another."""
    assert all(s > 0 or n <= 1 for n, s in zip(shape, strides)), f"strides {strides} of shape {shape} are not the tensor's for the library"
    out = np.empty(shape, np.float32)
    for at in np.ndindex(*shape[:-1]):
        line = p + 4 * sum(i * s for i, s in zip(at, strides))
        out[at] = np.ctypeslib.as_array((ctypes.c_float * shape[-1]).from_address(line))
    return out


class Stub:
    """Keeps what the calls would read."""

    def __init__(self, real):
        self.real, self.seen = real, None

    def __getattr__(self, name):
        return getattr(self.real, name)

    def ralm_kv_append(self, kv, layer, k, v, dt, kt, kh, vt, vh, off, n, stream):
        H, d = kv._obj.n_heads, kv._obj.d
        self.seen = numbers(k, (n, H, d), (kt, kh)), numbers(v, (n, H, d), (vt, vh))
        return 0

    def ralm_kv_read(self, *a):
        self.seen = True
        return 0

    def ralm_kv_attention(self, kv, layer, q, dt, qt, qh, heads, off, Qt, *rest):
        d = kv._obj.d
        bits = numbers(q, (Qt, heads, d // 2), (qt // 2, qh // 2))       # two 16-bit numbers in the place of one
        self.seen = torch.from_numpy(bits).view(torch.bfloat16)
        return 0

    def ralm_verify_draft(self, ids, q, qs, p, ps, dt, V, u, un, Qt, off, R, *rest):
        self.seen = numbers(p, (Qt + R, V), (ps,)), None if q is None else numbers(q, (Qt, V), (qs,))
        return 0


def cache(b, H=4, d=64, R=2):
    i32 = torch.int32
    page = b.ralm_kv_page_bytes(1, H, d, 16)
    return b.KVCache(torch.zeros(4 * page, dtype=torch.uint8), torch.full((R, 2), -1, dtype=i32), torch.zeros(R, dtype=i32),
                     torch.zeros(4, dtype=i32), n_layers=1, n_heads=H, d=d, page_tokens=16)


OFF = torch.tensor([0, 2, 5])
VIEWS = [(lambda x: x[:, :1].expand(5, 4, 64)), (lambda x: x[:1].expand(5, 4, 64)), (lambda x: x[:1, :1].expand(5, 4, 64)),
         (lambda x: x[:, :, :1].expand(5, 4, 64)), (lambda x: x)]


@pytest.mark.parametrize("view", VIEWS)
@pytest.mark.parametrize("other", VIEWS[-2:])
def test_keys_and_values(b, view, other):
    k, v = view(torch.randn(5, 4, 64)), other(torch.randn(5, 4, 64))
    for x, y in ((k, v), (v, k)):
        b.ralm_kv_append(cache(b), 0, x, y, OFF)
        assert np.array_equal(b.stub.seen[0], x.numpy()) and np.array_equal(b.stub.seen[1], y.numpy())


def test_one_token_and_one_head(b):
    x = torch.randn(1, 1, 64)
    for k in (x, x.as_strided((1, 1, 64), (0, 0, 1))):                   # a dimension of one is no repetition
        b.ralm_kv_append(cache(b, H=1), 0, k, k, torch.tensor([0, 1, 1]))
        assert np.array_equal(b.stub.seen[0], x.numpy())
    k = torch.randn(1, 4, 64)
    b.ralm_kv_append(cache(b), 0, k, k[:, :1].expand(1, 4, 64), torch.tensor([0, 1, 1]))
    assert np.array_equal(b.stub.seen[0], k.numpy()) and np.array_equal(b.stub.seen[1], k[:, :1].expand(1, 4, 64).numpy())


@pytest.mark.parametrize("view", VIEWS)
def test_queries(b, view):
    q = view(torch.randn(5, 4, 64).bfloat16())
    out = b.ralm_kv_attention(cache(b), 0, q, OFF, workspace=torch.empty(1 << 12, dtype=torch.uint8))
    assert torch.equal(b.stub.seen, q) and out.shape == q.shape and out.is_contiguous()


def test_outputs(b):
    dense = torch.zeros(5, 4, 64)
    for bad in (dense[:1].expand(5, 4, 64), dense[:, :1].expand(5, 4, 64)):
        b.stub.seen = None
        for k, v in ((bad, dense), (dense, bad)):
            with pytest.raises(AssertionError):
                b.ralm_kv_read(cache(b), 0, OFF, 5, k=k, v=v)
        with pytest.raises(AssertionError):
            b.ralm_kv_attention(cache(b), 0, dense.bfloat16(), OFF, out=bad.bfloat16().as_strided(bad.shape, bad.stride()),
                                workspace=torch.empty(1 << 12, dtype=torch.uint8))
        assert b.stub.seen is None
    b.ralm_kv_read(cache(b), 0, OFF, 5, k=dense, v=dense)
    assert b.stub.seen


@pytest.mark.parametrize("broadcast_p", [False, True])
@pytest.mark.parametrize("broadcast_q", [False, True])
def test_probabilities(b, broadcast_p, broadcast_q):
    R = Qt = 3
    V = 10
    p = torch.rand(V).expand(Qt + R, V) if broadcast_p else torch.rand(Qt + R, V)
    q = torch.rand(V).expand(Qt, V) if broadcast_q else torch.rand(Qt, V)
    ids, u = torch.zeros(Qt, dtype=torch.int32), torch.rand(3)
    for draft in (q, None):
        b.ralm_verify_draft(ids, p, u, u, torch.arange(R + 1), draft_probs=draft)
        assert np.array_equal(b.stub.seen[0], p.numpy())
        assert b.stub.seen[1] is None if draft is None else np.array_equal(b.stub.seen[1], q.numpy())
    # a single row is no repetition
    b.ralm_verify_draft(ids[:1], p[:2], u[:1], u[:1], torch.arange(2), draft_probs=torch.rand(V).expand(1, V))
    assert np.array_equal(b.stub.seen[0], p[:2].numpy())
