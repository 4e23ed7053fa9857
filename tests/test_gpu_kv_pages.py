"""Forking, reserving, rolling back and compacting pages of the 4-bit cache: whole numbers, against the definitions."""
import numpy as np
import pytest
import torch

import kv_plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2401_14021_amd import binding
    binding.lib()
    return binding


def new_cache(B, R, max_pages, n_pages, T=16, layers=1, H=1, d=64, seed=0):
    kv = B.KVCache.empty(R, max_pages * T, n_pages, n_layers=layers, n_heads=H, d=d, page_tokens=T)
    g = torch.Generator(device="cuda").manual_seed(seed)
    kv.pages.random_(0, 256, generator=g)
    return kv


def state(kv):
    return tuple(t.cpu().numpy().copy() for t in (kv.table, kv.lens, kv.refs))


def check_state(kv):
    """Every count is the number of places that hold the page, and a request's places are those of its length."""
    table, lens, refs = state(kv)
    count = np.zeros_like(refs)
    for r, n in enumerate(lens):
        held = -(-int(n) // kv.page_tokens)
        assert (table[r, :held] >= 0).all() and (table[r, held:] == -1).all(), r
        assert len(set(table[r, :held])) == held
        np.add.at(count, table[r, :held], 1)
    np.testing.assert_array_equal(count, refs)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def check_reserve(B, kv, grow):
    table, lens, refs = state(kv)
    pages = kv.pages.cpu().numpy().copy()
    want = kv_plain.reserve(table, lens, refs, grow, kv.page_tokens)
    granted = B.ralm_kv_reserve(kv, i32(grow))
    got = state(kv)
    for a, b in zip(got, want[:3]):
        np.testing.assert_array_equal(a, b)
    np.testing.assert_array_equal(granted.cpu().numpy(), want[3])
    for src, dst in want[4]:
        pages[dst] = pages[src]
    np.testing.assert_array_equal(kv.pages.cpu().numpy(), pages)
    check_state(kv)
    return want[3]


@pytest.mark.parametrize("R,max_pages,n_pages", [(1, 4, 3), (5, 8, 30), (70, 6, 300), (300, 30, 9000), (700, 20, 20000), (1024, 12, 65536), (1025, 9, 20000),
                                                 (60, 700, 65537), (1300, 30, 70000)])
def test_rounds_of_forks_reservations_and_rollbacks(B, R, max_pages, n_pages):
    rng = np.random.default_rng(R)
    kv = new_cache(B, R, max_pages, n_pages)
    T = kv.page_tokens
    for step in range(8):
        grow = rng.integers(-1, 3 * T, size=R) * (rng.random(R) < 0.8)
        if step == 3:
            grow[:] = rng.integers(0, 5, size=R)
        if step == 5:
            grow[rng.integers(0, R)] = max_pages * T + 1              # outgrows the table
        check_reserve(B, kv, grow)
        table, lens, refs = state(kv)
        # empty some requests and fork others into them
        gone = rng.random(R) < 0.3
        back = np.where(gone, 0, np.maximum(lens - rng.integers(0, 2 * T, size=R), -3))
        B.ralm_kv_truncate(kv, i32(back))
        lens = np.minimum(lens, np.maximum(back, 0))
        np.testing.assert_array_equal(kv.lens.cpu().numpy(), lens)
        check_state(kv)
        empty, full = np.nonzero(lens == 0)[0], np.nonzero(lens > 0)[0]
        if len(empty) and len(full):
            dst = empty[:max(1, len(empty) // 2)]
            src = rng.choice(full, size=len(dst))
            keep = rng.integers(0, lens[src].max() + 5, size=len(dst))
            table, _, _ = state(kv)
            B.ralm_kv_fork(kv, i32(src), i32(dst), None if step % 2 else i32(keep))
            kept = lens[src] if step % 2 else np.minimum(lens[src], keep)
            np.testing.assert_array_equal(kv.lens.cpu().numpy()[dst], kept)
            for s_, d_, n in zip(src, dst, kept):
                held = -(-int(n) // T)
                np.testing.assert_array_equal(kv.table.cpu().numpy()[d_, :held], table[s_, :held])
            check_state(kv)


def test_a_full_pool_serves_requests_in_order(B):
    kv = new_cache(B, 6, 10, 7)
    granted = check_reserve(B, kv, [33, 16, 80, 1, 0, 17])           # 3 + 1 pages, then five that are not there
    assert granted.tolist() == [1, 1, 0, 0, 1, 0]
    granted = check_reserve(B, kv, [15, 0, 48, 16, 0, 0])            # room in the last page; the last three pages
    assert granted.tolist() == [1, 1, 1, 0, 1, 1]
    B.ralm_kv_truncate(kv, i32([0, 16, 48, 0, 0, 0]))
    check_reserve(B, kv, [0, 0, 0, 16, 16, 16])


def test_both_owners_of_a_shared_page_grow(B):
    kv = new_cache(B, 3, 4, 12, layers=2, H=3, d=128)
    check_reserve(B, kv, [20, 0, 0])
    B.ralm_kv_fork(kv, i32([0, 0]), i32([1, 2]), i32([20, 16]))
    check_reserve(B, kv, [1, 1, 1])                                  # 0 and 1 copy the page, 2 begins one
    refs = kv.refs.cpu().numpy()
    assert sorted(refs[refs > 0].tolist()) == [1, 1, 1, 3]


def test_forks_that_are_left_out(B):
    kv = new_cache(B, 4, 4, 12)
    check_reserve(B, kv, [20, 5, 0, 0])
    before = state(kv)
    B.ralm_kv_fork(kv, i32([0, -1, 7, 0, 2]), i32([1, 2, 3, 9, 2]))  # not empty, out of range (three times), itself
    for a, b in zip(state(kv), before):
        np.testing.assert_array_equal(a, b)
    B.ralm_kv_fork(kv, i32([]), i32([]))


@pytest.mark.parametrize("shape", [(16, 1, 1, 64), (32, 2, 3, 128), (256, 4, 2, 256), (16, 24, 16, 64)])
def test_copies_of_pages(B, shape):
    T, layers, H, d = shape
    kv = new_cache(B, 2, 2, 40, T=T, layers=layers, H=H, d=d)
    rng = np.random.default_rng(1)
    ids = rng.permutation(40)
    src, dst = ids[:11], ids[11:22]
    want = kv.pages.cpu().numpy().copy()
    want[dst] = want[src]
    B.ralm_kv_copy_pages(kv, i32(np.r_[src, [-1, 3, 40]]), i32(np.r_[dst, [5, -1, 6]]))
    np.testing.assert_array_equal(kv.pages.cpu().numpy(), want)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("R,n_pages,share", [(1, 1, 0.0), (3, 9, 0.5), (40, 1000, 0.3), (200, 4096, 0.2), (500, 13000, 0.5), (900, 65536, 0.1),
                                             (900, 65537, 0.1), (3, 70001, 0.0)])
def test_compact(B, R, n_pages, share, in_place):
    rng = np.random.default_rng(R)
    max_pages = max(1, n_pages // R)
    kv = new_cache(B, R, max_pages, n_pages, seed=R)
    T = kv.page_tokens
    # requests with pages anywhere, some of them shared
    ids = rng.permutation(n_pages)
    table, lens, refs = state(kv)
    at = 0
    for r in range(R):
        n = int(rng.integers(0, max_pages + 1) * rng.random())
        if r and rng.random() < share:
            n = min(n, -(-int(lens[r - 1]) // T))
            table[r, :n] = table[r - 1, :n]
        else:
            n = min(n, n_pages - at)
            table[r, :n] = ids[at:at + n]
            at += n
        lens[r] = n * T
        np.add.at(refs, table[r, :n], 1)
    for t, x in ((kv.table, table), (kv.lens, lens), (kv.refs, refs)):
        t.copy_(torch.from_numpy(x))
    check_state(kv)
    pages = kv.pages.cpu().numpy().copy()
    used = int((refs > 0).sum())
    movers, holes = np.nonzero((refs > 0) & (np.arange(n_pages) >= used))[0], np.nonzero((refs == 0) & (np.arange(n_pages) < used))[0]
    goes = np.arange(n_pages)
    goes[movers] = holes
    want_table = np.where(table >= 0, goes[np.maximum(table, 0)], table)
    want_refs = np.zeros_like(refs)
    want_refs[goes[refs > 0]] = refs[refs > 0]
    got = B.ralm_kv_compact(kv, table=kv.table if in_place else None, refs=kv.refs if in_place else None)
    np.testing.assert_array_equal(got[0].cpu().numpy(), want_table)
    np.testing.assert_array_equal(got[1].cpu().numpy(), want_refs)
    assert int(got[2]) == used
    pages[holes] = pages[movers]
    np.testing.assert_array_equal(kv.pages.cpu().numpy(), pages)
    if in_place:
        check_state(kv)
    else:
        np.testing.assert_array_equal(kv.table.cpu().numpy(), table)
        np.testing.assert_array_equal(kv.refs.cpu().numpy(), refs)
    # nothing is left to move
    kv2 = B.KVCache(kv.pages, got[0], kv.lens, got[1], n_layers=1, n_heads=1, d=64, page_tokens=T)
    again = B.ralm_kv_compact(kv2)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1]) and np.array_equal(kv.pages.cpu().numpy(), pages)


def test_a_table_entry_without_a_count_stays_where_it_is(B):
    kv = new_cache(B, 2, 4, 20)
    check_reserve(B, kv, [16, 16])
    kv.table[0, 1], kv.table[0, 2], kv.table[1, 3] = 17, 1 << 30, 19
    kv.refs[19] = 1
    table, refs, used = B.ralm_kv_compact(kv)
    assert int(used) == 3 and table[0].tolist() == [0, 17, 1 << 30, -1] and table[1].tolist() == [1, -1, -1, 2]
    assert refs[:4].tolist() == [1, 1, 1, 0]


def test_a_round_replays_from_a_graph(B):
    kv = new_cache(B, 8, 8, 60, layers=2, H=2, d=128)
    check_reserve(B, kv, [20, 33, 5, 16, 0, 0, 0, 0])
    src, dst = i32([0, 1, 2, 3]), i32([4, 5, 6, 7])
    grow, back = i32([0, 0, 0, 0, 3, 20, 1, 7]), i32([20, 33, 5, 16, 0, 0, 0, 0])
    ws = B.alloc_kv_pages_workspace(kv)
    granted = torch.empty_like(grow)
    mid = [torch.empty_like(t) for t in (kv.table, kv.lens, kv.refs)]

    def go():
        B.ralm_kv_fork(kv, src, dst)
        B.ralm_kv_reserve(kv, grow, workspace=ws, granted=granted)
        for m, t in zip(mid, (kv.table, kv.lens, kv.refs)):
            m.copy_(t)
        B.ralm_kv_truncate(kv, back)

    go()
    want, end = [m.clone() for m in mid], state(kv)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(4):
        for m in mid:
            m.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(mid, want))
        for a, b in zip(state(kv), end):
            np.testing.assert_array_equal(a, b)
        check_state(kv)
