"""Verification of drafted tokens: whole numbers, against the definition; and that the tokens are distributed as the target's."""
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


def check(B, ids, target, u, u_next, off, draft=None):
    got = B.ralm_verify_draft(torch.tensor(ids, dtype=torch.int32, device="cuda"), target.cuda(), torch.tensor(u, dtype=torch.float32, device="cuda"),
                              torch.tensor(u_next, dtype=torch.float32, device="cuda"), torch.tensor(off, dtype=torch.int64, device="cuda"),
                              draft_probs=None if draft is None else draft.cuda())
    want = kv_plain.verify_draft(ids, target.double().numpy(), np.float32(u), np.float32(u_next), off,
                                 None if draft is None else draft.double().numpy())
    np.testing.assert_array_equal(got[0].cpu().numpy(), want[0])
    np.testing.assert_array_equal(got[1].cpu().numpy(), want[1])
    return want


def rows(rng, n, V, sharp=2.0):
    x = np.exp(rng.normal(size=(n, V)) * sharp)
    return x / x.sum(1, keepdims=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 255, 256, 1023, 1024, 1025, 4099])
@pytest.mark.parametrize("drafted", [True, False])
def test_against_the_definition(B, V, dtype, drafted):
    rng = np.random.default_rng(V)
    s = [0, 1, 3, 8, 2, 0, 5]
    off = np.concatenate([[0], np.cumsum(s)])
    Qt, R = int(off[-1]), len(s)
    target = rows(rng, Qt + R, V)
    mine = [int(off[r]) + r + i for r in range(R) for i in range(s[r])]
    near = target[mine] * np.exp(rng.normal(size=(Qt, V)) * 0.3)
    near /= near.sum(1, keepdims=True)
    ids = np.array([rng.choice(V, p=p) for p in near])
    target, near = (torch.from_numpy(x).to(DT[dtype]) for x in (target, near))
    check(B, ids, target, rng.random(Qt) * (1.0 if drafted else 0.2), rng.random(R), off, near if drafted else None)


def test_many_drafts_of_one_request(B):
    """More drafts than a wave has lanes, all accepted but one."""
    rng = np.random.default_rng(2)
    for stop in (0, 63, 64, 65, 149, 150):
        s, V = 150, 50
        off = [0, s]
        target = torch.from_numpy(rows(rng, s + 1, V)).float()
        draft = target[:-1].clone()
        ids = rng.integers(0, V, size=s)
        u = np.full(s, 0.5)
        if stop < s:
            target[stop, ids[stop]] = 0.0
        want = check(B, ids, target, u, [0.3], off, draft)
        assert want[0][0] == stop


def test_rows_and_random_numbers_at_the_edges(B):
    V, nan = 1500, float("nan")
    last = 1.0 - 2.0 ** -24
    one = torch.zeros(V)
    cases = []
    p = torch.zeros(2, V)
    p[:, V - 1] = 1.0
    cases.append((p, p[:1], V - 1, last, last))            # certain on both sides: accepted, the last token next
    cases.append((p, p[:1], 0, 0.0, 0.5))                  # no probability on either side: not accepted
    cases.append((torch.zeros(2, V), p[:1], 3, 0.0, 0.5))  # a target of zeros: no token
    cases.append((p.clone().fill_(nan), p[:1], 3, 0.0, 0.5))
    cases.append((p, p[:1], -1, 0.0, 0.2))                 # drafts that are no tokens
    cases.append((p, p[:1], V, 0.0, 0.2))
    cases.append((p, p[:1], 1 << 30, 0.0, 0.2))
    q = torch.full((1, V), 1.0)
    cases.append((torch.full((2, V), 1.0 / V), q, 7, 0.9, 0.999))      # nothing is left beside the draft: the target alone
    t = torch.full((2, V), 2.0 ** -40)
    t[:, 11] = 2.0 ** -36
    cases.append((t, t[:1], 5, 0.5, last))                  # below the last place
    t = torch.full((2, V), -1.0)
    t[:, 1024] = 7.0
    cases.append((t, t[:1], 1024, 0.5, 0.0))                # outside [0, 1]
    for target, draft, x, u, v in cases:
        for dr in (draft, None):
            check(B, [x], target, [u], [v], [0, 1], dr)
    assert one.sum() == 0


def test_strided_rows_and_a_workspace_of_the_callers(B):
    rng = np.random.default_rng(4)
    V, s = 777, [2, 4]
    off = [0, 2, 6]
    target, draft = torch.from_numpy(rows(rng, 8, V)).float(), torch.from_numpy(rows(rng, 6, V)).float()
    ids, u, un = rng.integers(0, V, size=6), rng.random(6), rng.random(2)
    want = check(B, ids, target, u, un, off, draft)
    wide = torch.zeros(8, 1000, device="cuda")
    wide[:, 3:3 + V] = target.cuda()
    wd = torch.zeros(6, 801, device="cuda")
    wd[:, 1:1 + V] = draft.cuda()
    args = [torch.tensor(x, dtype=t, device="cuda") for x, t in ((ids, torch.int32), (u, torch.float32), (un, torch.float32), (off, torch.int64))]
    ws = torch.empty(int(B.lib().ralm_verify_draft_workspace_bytes(2, V)), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        ws.random_(0, 256)
        got = B.ralm_verify_draft(args[0], wide[:, 3:3 + V], args[1], args[2], args[3], draft_probs=wd[:, 1:1 + V], workspace=ws)
        assert np.array_equal(got[0].cpu(), want[0]) and np.array_equal(got[1].cpu(), want[1])


def test_a_large_vocabulary_and_all_types_agree(B):
    """2^20 entries; probabilities that bf16 holds give the same tokens in every type."""
    V, R = 1 << 20, 5
    g = torch.Generator().manual_seed(1)
    target = torch.softmax(torch.randn(2 * R, V, generator=g) * 3, -1).bfloat16()
    draft = torch.softmax(torch.randn(R, V, generator=g) * 3, -1).bfloat16()
    ids = draft.float().multinomial(1, generator=g).squeeze(1).to(torch.int32)
    u, un, off = torch.rand(R, generator=g), torch.rand(R, generator=g), torch.arange(R + 1)
    got = {}
    for name in ("bf16", "f32"):
        got[name] = B.ralm_verify_draft(ids.cuda(), target.to(DT[name]).cuda(), u.cuda(), un.cuda(), off.cuda(), draft_probs=draft.to(DT[name]).cuda())
    assert torch.equal(got["bf16"][0], got["f32"][0]) and torch.equal(got["bf16"][1], got["f32"][1])
    one = float(1 << 36)
    for r in range(R):
        n = int(got["f32"][0][r])
        w = torch.floor(target[2 * r + n].double().clamp(0, 1) * one).long()
        if n == 0:
            w = (w - torch.floor(draft[r].double() * one).long()).clamp(min=0)
        t = int(float(un[r]) * 2 ** 24) * int(w.sum()) >> 24
        assert int((w.cumsum(0) <= t).sum()) == int(got["f32"][1][r])


@pytest.mark.parametrize("certain", [False, True])
def test_tokens_are_distributed_as_the_targets(B, certain):
    """One draft per request from q, verified against p: the first token that comes out has p's distribution.  200000 draws: a frequency's
    standard deviation is at most sqrt(1/4 / 200000) = 0.0011, and six of them are allowed."""
    V, R = 7, 65536
    g = torch.Generator(device="cuda").manual_seed(3)
    p = torch.tensor([0.4, 0.05, 0.2, 0.0, 0.1, 0.2, 0.05], device="cuda")
    q = torch.tensor([0.1, 0.3, 0.05, 0.1, 0.2, 0.2, 0.05], device="cuda")
    count = torch.zeros(V, device="cuda", dtype=torch.long)
    rounds = 4
    for _ in range(rounds):
        ids = torch.full((R,), 2, device="cuda", dtype=torch.int32) if certain else \
            q.expand(R, V).multinomial(1, generator=g).squeeze(1).to(torch.int32)
        n, nxt = B.ralm_verify_draft(ids, p.expand(2 * R, V).contiguous(), torch.rand(R, generator=g, device="cuda"),
                                     torch.rand(R, generator=g, device="cuda"), torch.arange(R + 1, device="cuda"),
                                     draft_probs=None if certain else q.expand(R, V).contiguous())
        count += torch.bincount(torch.where(n == 1, ids, nxt).long(), minlength=V)
    assert (count.double() / (rounds * R) - p.double()).abs().max() < 6 * (0.25 / (rounds * R)) ** 0.5


def test_a_round_replays_from_a_graph(B):
    rng = np.random.default_rng(9)
    V, off = 3000, torch.tensor([0, 3, 4, 9], device="cuda")
    target, draft = torch.empty(12, V, device="cuda"), torch.empty(9, V, device="cuda")
    ids, u, un = torch.empty(9, dtype=torch.int32, device="cuda"), torch.empty(9, device="cuda"), torch.empty(3, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")

    def fill():
        target.copy_(torch.from_numpy(rows(rng, 12, V)))
        draft.copy_(torch.from_numpy(rows(rng, 9, V)))
        ids.copy_(torch.from_numpy(rng.integers(0, V, size=9)))
        u.copy_(torch.from_numpy(rng.random(9)))
        un.copy_(torch.from_numpy(rng.random(3)))

    fill()
    B.ralm_verify_draft(ids, target, u, un, off, draft_probs=draft, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n, nxt = B.ralm_verify_draft(ids, target, u, un, off, draft_probs=draft, workspace=ws)
    for _ in range(4):
        fill()
        graph.replay()
        torch.cuda.synchronize()
        a, b = n.clone(), nxt.clone()
        want = B.ralm_verify_draft(ids, target, u, un, off, draft_probs=draft)
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])
