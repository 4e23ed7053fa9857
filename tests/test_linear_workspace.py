"""The workspace of a product (host, no GPU): what is said to be enough for T rows is enough for fewer."""
import os
import time

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2401_14021_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2401_14021_amd import build
        build.build()
    return binding.lib()


SIZES = [(6144, 4096, 0), (4096, 16384, 0), (11264, 4096, 1), (8192, 8192, 0), (500, 16384, 0), (1000, 6656, 0), (129, 1024, 1), (50257, 1024, 0),
         (1, 131072, 0), (2049, 40000, 1), (4096, 8, 0)]


@pytest.mark.parametrize("N,K,gated", SIZES)
def test_enough_for_fewer_rows(L, N, K, gated):
    most = before = 0
    for T in list(range(1, 3000)) + list(range(3000, 20000, 37)):
        room, need = L.ralm_linear_workspace_bytes(T, N, K, gated) if T < 600 or T % 7 == 0 else None, L.ralm_linear_workspace_bytes_exact(T, N, K, gated)
        most = max(most, need)
        if room is not None:
            assert room >= most and room >= before, T
            assert room <= most * 1.25 + 64 * 16 * 4 * 2 * (N + 3), T      # and hardly more: the rows of a tile
            before = room


def test_some_products_need_none_and_some_need_less_than_fewer_rows(L):
    exact, room = L.ralm_linear_workspace_bytes_exact, L.ralm_linear_workspace_bytes
    assert exact(64, 6144, 4096, 0) > 0 and exact(1024, 6144, 4096, 0) == 0 < room(1024, 6144, 4096, 0)
    assert room(4096, 4096, 8, 0) == 0 and room(0, 64, 64, 0) == 0 and room(-1, 64, 64, 0) == 0 and exact(4, 64, 60, 0) == 0


def test_the_binding_allocates_for_fewer_rows(L):
    from paper_2401_14021_amd import binding as b
    assert b.alloc_linear_workspace(1024, 6144, 4096, device="cpu").numel() == L.ralm_linear_workspace_bytes(1024, 6144, 4096, 0)
    assert b.alloc_linear_workspace(1024, 1024, 64, device="cpu") is None


def test_the_search_ends_soon(L):
    begin = time.perf_counter()
    L.ralm_linear_workspace_bytes(1 << 22, 1, 131072, 0)
    assert time.perf_counter() - begin < 2


@pytest.mark.gpu
def test_one_workspace_for_all_batches():
    import torch
    from paper_2401_14021_amd import binding as b
    N, K, most = 1500, 4096, 1024
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.randint(-2, 3, (N, K), generator=g, device="cuda").bfloat16()
    x = torch.randint(-2, 3, (most, K), generator=g, device="cuda").bfloat16()
    want = x.double() @ w.double().T.contiguous()
    room = b.alloc_linear_workspace(most, N, K)
    split = 0
    for T in (1, 16, 17, 64, 100, 255, 256, 257, 300, 448, 640, 700, 960, 1023, 1024):
        split += b.lib().ralm_linear_workspace_bytes_exact(T, N, K, 0) > 0
        room.fill_(255)
        assert torch.equal(b.ralm_linear(x[:T], w, out_dtype=torch.float32, workspace=room).double(), want[:T])
    assert split > 4
    small = torch.empty(64, dtype=torch.uint8, device="cuda")
    with pytest.raises(b.RalmError):
        b.ralm_linear(x[:64], w, workspace=small)
