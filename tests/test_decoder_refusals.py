"""Argument errors of the operators around the generator's attention: a status before anything is launched, without a GPU."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2401_14021_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2401_14021_amd import build
        build.build()
    binding.lib()
    return binding


P = 0x10000   # fake, aligned, never dereferenced
NULL, SHAPE, K_, DTYPE, ALIGN, WORKSPACE, RANGE = 1, 2, 3, 4, 5, 6, 7
F32, BF16, F16 = 0, 1, 2


def test_linear(b):
    L = b.lib()

    def at(x=P, xs=0, T=4, w=P, ws=0, N=128, K=64, dt=BF16, bias=None, act=0, gated=0, res=None, rs=0, out=2 * P, os_=0, odt=BF16, work=P, n=1 << 40):
        return L.ralm_linear(x, xs, T, w, ws, N, K, dt, bias, act, gated, res, rs, out, os_, odt, work, n, None)
    assert at(x=None) == NULL and at(w=None) == NULL and at(out=None) == NULL
    assert at(T=-1) == SHAPE and at(T=(1 << 22) + 1) == SHAPE and at(N=0) == SHAPE and at(N=(1 << 20) + 1) == SHAPE
    assert at(N=(1 << 19) + 1, gated=1) == SHAPE and at(K=0) == SHAPE and at(K=12) == SHAPE and at(K=(1 << 17) + 8) == SHAPE
    assert at(T=1 << 22, N=(1 << 14) + 1) == SHAPE and at(T=1 << 17, N=1 << 19, K=8, gated=1) == SHAPE   # 2^32 work-items
    assert at(dt=F32) == DTYPE and at(dt=7) == DTYPE and at(odt=F16) == DTYPE and at(odt=9) == DTYPE
    assert at(act=-1) == RANGE and at(act=5) == RANGE and at(gated=2) == RANGE
    assert at(xs=56) == SHAPE and at(ws=56) == SHAPE and at(os_=127) == SHAPE and at(res=P, rs=100) == SHAPE
    assert at(xs=(1 << 22) + 8) == SHAPE and at(ws=(1 << 22) + 8) == SHAPE
    assert at(xs=68) == ALIGN and at(ws=68) == ALIGN and at(x=P + 8) == ALIGN and at(w=P + 2) == ALIGN
    assert at(out=P + 1) == ALIGN and at(out=P + 2, odt=F32) == ALIGN and at(res=P + 2, odt=F32) == ALIGN and at(bias=P + 1) == ALIGN
    assert at(res=2 * P, rs=136) == SHAPE                                  # in place with another stride
    assert at(out=P) == SHAPE and at(x=3 * P, out=P) == SHAPE and at(bias=2 * P) == SHAPE   # other inputs in place
    assert at(T=0, x=None, w=None, out=None) == 0
    need = L.ralm_linear_workspace_bytes(4, 128, 64, 0)
    assert L.ralm_linear_workspace_bytes(4, 128, 60, 0) == 0 and need >= 0
    for T, N, K in ((1, 1024, 8192), (40, 1024, 8192), (64, 4096, 4096), (100, 500, 16384)):
        need = L.ralm_linear_workspace_bytes(T, N, K, 0)
        if need:
            assert at(T=T, N=N, K=K, work=None) == WORKSPACE and at(T=T, N=N, K=K, work=P + 8) == WORKSPACE and at(T=T, N=N, K=K, n=need - 1) == WORKSPACE


def test_norm(b):
    L = b.lib()

    def at(**kw):
        f = dict(T=3, D=64, kind=0, eps=1e-6, scale=1.0, x=P, x_dtype=BF16, param_dtype=F32, sum=2 * P, sum_dtype=F32, out=3 * P, out_dtype=BF16)
        f.update(kw)
        return L.ralm_residual_norm(ctypes.byref(b.ralm_norm_t(**f)), None)
    assert L.ralm_residual_norm(None, None) == NULL
    assert at(x=None) == NULL and at(sum=None, out=None) == NULL
    assert at(T=-1) == SHAPE and at(T=(1 << 22) + 1) == SHAPE and at(D=0) == SHAPE and at(D=32769) == SHAPE
    assert at(kind=2) == RANGE and at(post=2) == RANGE and at(gate=P, gate_rows=3) == RANGE
    assert at(eps=-1.0) == RANGE and at(eps=float("nan")) == RANGE and at(scale=float("inf")) == RANGE
    assert at(x_dtype=3) == DTYPE and at(param_dtype=-1) == DTYPE and at(sum_dtype=4) == DTYPE and at(out_dtype=8) == DTYPE
    assert at(x_stride=63) == SHAPE and at(sum_stride=63) == SHAPE and at(out_stride=1) == SHAPE and at(residual=P, residual_stride=60) == SHAPE
    assert at(gate=P, gate_rows=1, gate_stride=5) == SHAPE
    assert at(x=P + 1) == ALIGN and at(sum=P + 2) == ALIGN and at(out=P + 1) == ALIGN and at(residual=P + 2) == ALIGN and at(weight=P + 2) == ALIGN
    assert at(bias=P + 1) == ALIGN and at(post_weight=P + 3) == ALIGN and at(post_bias=P + 2) == ALIGN and at(gate=P + 1) == ALIGN
    assert at(out=2 * P) == SHAPE and at(residual=3 * P, sum=None, out_dtype=F32) == SHAPE
    assert at(residual=2 * P, residual_stride=72) == SHAPE                 # in place with another stride
    assert at(sum=P) == SHAPE and at(sum=P, sum_dtype=BF16, x_stride=72) == SHAPE and at(out=P, out_dtype=F32) == SHAPE and at(out=P, out_stride=72) == SHAPE
    assert at(T=1 << 22, D=16392) == SHAPE                                 # 2^32 work-items
    assert at(weight=2 * P) == SHAPE and at(bias=3 * P) == SHAPE and at(gate=2 * P, x=P) == SHAPE and at(post=1, post_weight=3 * P) == SHAPE
    assert at(T=0, x=None) == 0


def test_append_rotary(b):
    L = b.lib()
    f = dict(pages=P, n_pages=100, n_layers=2, n_heads=4, d=128, page_tokens=32, table=P, lens=P, refs=None, R=8, max_pages=16)
    kv = ctypes.byref(b.ralm_kv_t(*[f[n] for n, _ in b.ralm_kv_t._fields_]))

    def at(kv=kv, layer=0, q=P, qs=(0, 0), heads=8, qo=2 * P, os_=(0, 0), k=P, v=P, dt=BF16, st=(0, 0, 0, 0), freqs=P, rot=128, inter=0, amp=1.0, off=P, n=4):
        return L.ralm_kv_append_rotary(kv, layer, q, *qs, heads, qo, *os_, k, v, dt, *st, freqs, rot, inter, amp, None, off, n, None)
    assert at(kv=None) == NULL and at(k=None) == NULL and at(v=None) == NULL and at(off=None) == NULL and at(freqs=None) == NULL and at(qo=None) == NULL
    assert at(layer=2) == RANGE and at(n=-1) == RANGE and at(inter=2) == RANGE and at(amp=float("nan")) == RANGE and at(amp=float("inf")) == RANGE
    assert at(rot=-2) == SHAPE and at(rot=3) == SHAPE and at(rot=130) == SHAPE and at(heads=0) == SHAPE and at(heads=5000) == SHAPE
    assert at(dt=3) == DTYPE and at(freqs=P + 4) == ALIGN and at(q=P + 8) == ALIGN and at(qo=P + 8) == ALIGN and at(k=P + 8) == ALIGN
    assert at(qs=(1028, 128)) == ALIGN and at(os_=(1024, 100)) == ALIGN and at(st=(512, 124, 0, 0)) == ALIGN
    assert at(qo=P, qs=(2048, 128)) == SHAPE
    assert at(n=0, k=None, v=None, q=None) == 0
    bad = dict(f, d=96)
    assert at(kv=ctypes.byref(b.ralm_kv_t(*[bad[n] for n, _ in b.ralm_kv_t._fields_]))) == SHAPE


def test_frequencies(b):
    L = b.lib()
    buf = (ctypes.c_double * 32)()
    at = lambda p=buf, rot=64, base=1e4, factor=1.0, ctx=0.0, lo=1.0, hi=32.0: L.ralm_rotary_frequencies(p, rot, base, factor, ctx, lo, hi)
    assert at() == 0 and buf[0] == 1.0 and abs(buf[16] - 0.01) < 1e-17
    assert at(rot=-2) == SHAPE and at(rot=5) == SHAPE and at(p=None) == NULL and at(p=None, rot=0) == 0
    assert at(base=0.5) == RANGE and at(base=float("inf")) == RANGE and at(factor=0.0) == RANGE and at(factor=float("nan")) == RANGE and at(ctx=-1.0) == RANGE
    assert at(ctx=1.0, lo=2.0, hi=2.0) == RANGE and at(ctx=1.0, lo=-1.0) == RANGE


def test_target(b):
    L = b.lib()

    def at(x=P, xs=0, Q=2, V=100, dt=F32, T=1.0, tok=P, w=P, k=4, share=None, all_=0.5, out=2 * P, os_=0, odt=F32, work=P, n=1 << 40):
        return L.ralm_knnlm_target(x, xs, Q, V, dt, T, tok, w, k, share, all_, out, os_, odt, work, n, None)
    assert at(x=None) == NULL and at(tok=None) == NULL and at(w=None) == NULL and at(out=None) == NULL
    assert at(Q=-1) == SHAPE and at(Q=(1 << 20) + 1) == SHAPE and at(V=0) == SHAPE and at(V=(1 << 20) + 1) == SHAPE
    assert at(k=-1) == K_ and at(k=1025) == K_ and at(dt=3) == DTYPE and at(odt=3) == DTYPE
    assert at(T=0.0) == RANGE and at(T=-1.0) == RANGE and at(T=float("nan")) == RANGE and at(T=float("inf")) == RANGE and at(T=1e-42) == RANGE
    assert at(all_=-0.1) == RANGE and at(all_=1.1) == RANGE and at(all_=float("nan")) == RANGE
    assert at(xs=99) == SHAPE and at(os_=99) == SHAPE and at(out=P, os_=104) == SHAPE and at(out=P, odt=BF16) == SHAPE
    assert at(x=P + 2) == ALIGN and at(out=P + 1, odt=BF16) == ALIGN and at(tok=P + 2) == ALIGN and at(w=P + 2) == ALIGN and at(share=P + 2) == ALIGN
    assert at(Q=0, x=None, out=None) == 0
    assert at(Q=1 << 19, V=1 << 17) == SHAPE and at(Q=1 << 20, V=65537) == SHAPE   # 2^32 work-items
    for V in (1000, 8193, 50257, 65536, 70000, 1 << 20):                   # room for Q rows is room for fewer
        sizes = [L.ralm_knnlm_target_workspace_bytes(Q, V) for Q in (1, 2, 100, 127, 128, 129, 1000, 5000)]
        assert sizes == sorted(sizes)
    need = L.ralm_knnlm_target_workspace_bytes(1, 1 << 20)
    if need:
        assert at(Q=1, V=1 << 20, work=None) == WORKSPACE and at(Q=1, V=1 << 20, work=P + 8) == WORKSPACE and at(Q=1, V=1 << 20, n=need - 1) == WORKSPACE
    assert L.ralm_knnlm_target_workspace_bytes(0, 0) == 0


def test_tensors_that_are_not_on_the_gpu(b):
    """The binding refuses them by itself: a kernel would fault on their addresses."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(b.RalmError):
        b.ralm_linear(x, x)
    with pytest.raises(b.RalmError):
        b.ralm_residual_norm(x)
    with pytest.raises(b.RalmError):
        b.ralm_knnlm_target(x, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), 0.5)


def test_shapes_and_types_in_the_binding(b):
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for bad in (dict(w=x.float()), dict(w=x[:, :32]), dict(w=x[:3], gated=True), dict(w=x, bias=x[0]), dict(w=x, residual=x),
                dict(w=x, out=torch.zeros(4, 5, dtype=torch.bfloat16)), dict(w=x, out=torch.zeros(1, 4, dtype=torch.bfloat16).expand(4, 4))):
        with pytest.raises((AssertionError, b.RalmError)):
            b.ralm_linear(x, **bad)
    for bad in (dict(residual=x[:3]), dict(weight=x[0, :8]), dict(gate=x[:2]), dict(out=x.t()), dict(post_weight=x[0]), dict(want_sum=False, sum=x)):
        with pytest.raises((AssertionError, b.RalmError)):
            b.ralm_residual_norm(x, **bad)
