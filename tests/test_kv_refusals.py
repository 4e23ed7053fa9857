"""Argument errors of the generator's operators: a status before anything is launched, without a GPU."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2401_14021_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2401_14021_amd import build
        build.build()
    binding.lib()
    return binding


P = 0x10000   # fake, aligned, never dereferenced
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, RANGE = 1, 2, 4, 5, 6, 7


def desc(b, **kw):
    f = dict(pages=P, n_pages=100, n_layers=2, n_heads=4, d=128, page_tokens=32, table=P, lens=P, refs=P, R=8, max_pages=16)
    f.update(kw)
    return ctypes.byref(b.ralm_kv_t(*[f[n] for n, _ in b.ralm_kv_t._fields_]))


BAD_CACHES = [(dict(pages=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(d=96), SHAPE), (dict(d=0), SHAPE),
              (dict(page_tokens=8), SHAPE), (dict(page_tokens=48), SHAPE), (dict(page_tokens=512), SHAPE), (dict(n_layers=0), SHAPE),
              (dict(n_heads=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=(1 << 22) + 1), SHAPE), (dict(R=0), SHAPE),
              (dict(R=(1 << 16) + 1), SHAPE), (dict(max_pages=0), SHAPE), (dict(max_pages=(1 << 25) + 1), SHAPE),
              (dict(R=1 << 16, max_pages=1 << 15), SHAPE), (dict(pages=P + 8), ALIGN)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_caches(b, kw, status):
    L, kv = b.lib(), desc(b, **kw)
    assert L.ralm_kv_append(kv, 0, P, P, 1, 0, 0, 0, 0, P, 4, None) == status
    assert L.ralm_kv_read(kv, 0, P, 4, None, P, P, 1, 0, 0, 0, 0, None) == status
    assert L.ralm_kv_attention(kv, 0, P, 1, 0, 0, 8, P, 4, 1, 64, 1.0, 0, 0, P, 0, 0, None, P, 1 << 30, None) == status
    assert L.ralm_kv_reserve(kv, P, P, P, 1 << 30, None) == status
    assert L.ralm_kv_fork(kv, P, P, None, 2, None) == status
    assert L.ralm_kv_truncate(kv, P, None) == status
    assert L.ralm_kv_copy_pages(kv, P, P, 2, None) == status
    assert L.ralm_kv_compact(kv, P, P, P, P, 1 << 30, None) == status
    assert L.ralm_kv_attention_workspace_bytes(kv, 8, 4, 1, 64, 0, 0) == 0 and L.ralm_kv_pages_workspace_bytes(kv) == 0
    assert L.ralm_last_error()


def test_page_bytes(b):
    L = b.lib()
    assert L.ralm_kv_page_bytes(2, 4, 128, 32) == 2 * 4 * 32 * 136 and L.ralm_kv_page_bytes(1, 1, 64, 16) == 16 * 68
    for bad in ((0, 1, 64, 16), (1, 0, 64, 16), (1, 1, 80, 16), (1, 1, 64, 24), (1, 1, 64, 0)):
        assert L.ralm_kv_page_bytes(*bad) == 0


def test_append_and_read(b):
    L, kv = b.lib(), desc(b)
    ap = lambda k=P, v=P, layer=0, dt=1, st=(0, 0, 0, 0), off=P, n=4: L.ralm_kv_append(kv, layer, k, v, dt, *st, off, n, None)
    assert ap(k=None) == NULL and ap(v=None) == NULL and ap(off=None) == NULL
    assert ap(layer=-1) == RANGE and ap(layer=2) == RANGE and ap(n=-1) == RANGE and ap(n=(1 << 22) + 1) == RANGE
    assert ap(dt=3) == DTYPE and ap(k=P + 8) == ALIGN and ap(v=P + 2) == ALIGN
    assert ap(st=(512, 124, 0, 0)) == ALIGN and ap(st=(0, 0, 516, 128)) == ALIGN and ap(st=(64, 128, 0, 0)) == ALIGN
    assert ap(n=0, k=None, v=None) == 0                                   # nothing to do
    assert L.ralm_kv_read(kv, 0, None, 4, None, P, P, 1, 0, 0, 0, 0, None) == NULL
    assert L.ralm_kv_read(kv, 0, P, 4, None, P, P, 9, 0, 0, 0, 0, None) == DTYPE


def test_attention(b):
    L, kv = b.lib(), desc(b, max_pages=256)
    big = L.ralm_kv_attention_workspace_bytes(kv, 8, 4, 1, 8192, 0, 0)
    assert big > 256                                                       # a few long contexts: split
    assert L.ralm_kv_attention_workspace_bytes(kv, 8, 4, 1, 300, 0, 0) == 256

    def at(layer=0, q=P, dt=1, qs=(0, 0), heads=8, off=P, Qt=4, mq=1, ml=8192, scale=1.0, w=0, f=0, out=P, os_=(0, 0), ws=P, n=big):
        return L.ralm_kv_attention(kv, layer, q, dt, *qs, heads, off, Qt, mq, ml, scale, w, f, out, *os_, None, ws, n, None)
    assert at(q=None) == NULL and at(out=None) == NULL and at(off=None) == NULL
    assert at(layer=2) == RANGE and at(layer=-1) == RANGE and at(Qt=-1) == RANGE and at(mq=-1) == RANGE and at(ml=-1) == RANGE
    assert at(w=-1) == RANGE and at(f=-1) == RANGE
    assert at(scale=0.0) == RANGE and at(scale=-1.0) == RANGE and at(scale=float("nan")) == RANGE and at(scale=float("inf")) == RANGE
    assert at(heads=6) == SHAPE and at(heads=0) == SHAPE and at(heads=2) == SHAPE and at(heads=8192) == SHAPE
    assert at(heads=1024, Qt=(1 << 20) + 1, n=1 << 62) == SHAPE             # more than 2^30 rows
    assert at(dt=0) == DTYPE and at(dt=5) == DTYPE
    assert at(q=P + 8) == ALIGN and at(out=P + 4) == ALIGN and at(qs=(1028, 128)) == ALIGN and at(os_=(1024, 100)) == ALIGN
    assert at(ws=None) == WORKSPACE and at(ws=P + 8) == WORKSPACE and at(n=big - 1) == WORKSPACE
    assert at(Qt=0, q=None, out=None, ws=None) == 0                         # nothing to do


def test_pages(b):
    L, kv = b.lib(), desc(b)
    n = L.ralm_kv_pages_workspace_bytes(kv)
    assert n > 0
    no_refs = desc(b, refs=None)
    assert L.ralm_kv_reserve(no_refs, P, P, P, n, None) == NULL and L.ralm_kv_compact(no_refs, P, P, P, P, n, None) == NULL
    assert L.ralm_kv_fork(no_refs, P, P, None, 1, None) == NULL and L.ralm_kv_truncate(no_refs, P, None) == NULL
    assert L.ralm_kv_reserve(kv, None, P, P, n, None) == NULL
    assert L.ralm_kv_reserve(kv, P, P, None, n, None) == WORKSPACE and L.ralm_kv_reserve(kv, P, P, P + 4, n, None) == WORKSPACE
    assert L.ralm_kv_reserve(kv, P, P, P, n - 1, None) == WORKSPACE
    assert L.ralm_kv_fork(kv, None, P, None, 1, None) == NULL and L.ralm_kv_fork(kv, P, None, None, 1, None) == NULL
    assert L.ralm_kv_fork(kv, P, P, None, -1, None) == RANGE and L.ralm_kv_fork(kv, None, None, None, 0, None) == 0
    assert L.ralm_kv_truncate(kv, None, None) == NULL
    assert L.ralm_kv_copy_pages(kv, None, P, 1, None) == NULL and L.ralm_kv_copy_pages(kv, P, P, -1, None) == RANGE
    assert L.ralm_kv_copy_pages(kv, None, None, 0, None) == 0
    assert L.ralm_kv_compact(kv, None, P, P, P, n, None) == NULL and L.ralm_kv_compact(kv, P, None, P, P, n, None) == NULL
    assert L.ralm_kv_compact(kv, P, P, None, P, n, None) == NULL and L.ralm_kv_compact(kv, P, P, P, P, n - 1, None) == WORKSPACE


def test_drafts(b):
    L = b.lib()
    n = L.ralm_verify_draft_workspace_bytes(4, 1000)
    assert n > 0
    for bad in ((0, 1000), (4, 0), (4, (1 << 20) + 1), ((1 << 16) + 1, 10)):
        assert L.ralm_verify_draft_workspace_bytes(*bad) == 0

    def vd(ids=P, dp=P, ds=0, tp=P, ts=0, dt=0, V=1000, u=P, un=P, Qt=6, off=P, R=4, acc=P, nxt=P, ws=P, size=n):
        return L.ralm_verify_draft(ids, dp, ds, tp, ts, dt, V, u, un, Qt, off, R, acc, nxt, ws, size, None)
    for name in ("ids", "tp", "u", "un", "off", "acc", "nxt"):
        assert vd(**{name: None}) == NULL, name
    assert vd(R=0) == SHAPE and vd(R=(1 << 16) + 1) == SHAPE and vd(V=0) == SHAPE and vd(V=(1 << 20) + 1) == SHAPE
    assert vd(Qt=-1) == RANGE and vd(dt=3) == DTYPE and vd(ts=999) == SHAPE and vd(ds=10) == SHAPE
    assert vd(tp=P + 2) == ALIGN and vd(dp=P + 1, dt=1) == ALIGN
    assert vd(ws=None) == WORKSPACE and vd(ws=P + 8) == WORKSPACE and vd(size=n - 1) == WORKSPACE


def test_attention_of_many_requests_without_hints(b):
    """Any R is served, whatever is known of the queries; only more pairs of request and head than a launch has workgroups are refused."""
    L = b.lib()
    for heads in (1, 8, 127):
        kv = desc(b, R=1 << 16, n_heads=heads, max_pages=64)
        for max_q in (0, 1, 1 << 16):
            assert L.ralm_kv_attention_workspace_bytes(kv, heads, 1 << 16, max_q, 0, 0, 0) == 256, (heads, max_q)
    assert L.ralm_kv_attention_workspace_bytes(desc(b, R=1 << 16, n_heads=128, max_pages=64), 128, 1 << 16, 1, 0, 0, 0) == 0
    assert L.ralm_kv_attention_workspace_bytes(desc(b, R=(1 << 16) - 1, n_heads=128, max_pages=64), 128, 1 << 16, 0, 0, 0, 0) == 256
    assert L.ralm_kv_attention_workspace_bytes(desc(b, R=3, n_heads=1), 4096, 1 << 18, 0, 0, 0, 0) == 256


@pytest.mark.parametrize("R,heads,q_heads,d,q", [(32, 8, 32, 128, 1), (16, 4, 16, 64, 2), (20, 4, 16, 256, 5), (6, 8, 32, 128, 1), (1, 8, 8, 128, 9)])
def test_a_batch_of_equal_requests_is_planned_alike_without_the_hint(b, R, heads, q_heads, d, q):
    """The workspace says into how many parts contexts are split."""
    L, kv = b.lib(), desc(b, R=R, n_heads=heads, d=d, max_pages=1 << 12)
    with_hint = L.ralm_kv_attention_workspace_bytes(kv, q_heads, R * q, q, 60000, 0, 0)
    assert with_hint > 256
    for nothing in (0, R * q + 1):
        assert L.ralm_kv_attention_workspace_bytes(kv, q_heads, R * q, nothing, 60000, 0, 0) == with_hint
