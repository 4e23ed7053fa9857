"""A decoder's layers on the library's operators, as a serving program strings them together: norms, gated products, rotary positions into the 4-bit cache, attention,
the vocabulary, the neighbours' target and the verification of drafts, eagerly and as one captured graph, against the same arithmetic in 64 bits.

Between the operators numbers are rounded to bf16 (2^-9 of a number, at random); the plain form rounds at the same places.  A sum of products then differs where a rounding fell
the other way: the bound on the states is 2^-5 of their size, several such steps in two layers, and what a wrong row, place or weight would miss by is their whole size."""
import pytest
import torch

pytestmark = pytest.mark.gpu
WIDTH, HEADS, KV, D, HIDDEN, VOCABULARY, LAYERS = 256, 4, 2, 64, 320, 1003, 2


@pytest.fixture(scope="module")
def b():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2401_14021_amd import binding
    return binding


class Layers:
    def __init__(self, b, interleaved):
        g = torch.Generator().manual_seed(3)

        def weights(n, m):
            return (torch.randn(m, n, generator=g) * n ** -0.5).bfloat16().cuda()

        self.b, self.interleaved = b, interleaved
        self.qkv = [(weights(WIDTH, (HEADS + 2 * KV) * D), (0.1 * torch.randn((HEADS + 2 * KV) * D, generator=g)).bfloat16().cuda()) for _ in range(LAYERS)]
        self.out = [weights(HEADS * D, WIDTH) for _ in range(LAYERS)]
        self.up = [weights(WIDTH, 2 * HIDDEN) for _ in range(LAYERS)]
        self.down = [weights(HIDDEN, WIDTH) for _ in range(LAYERS)]
        self.norms = [[(1 + 0.1 * torch.randn(WIDTH, generator=g)).bfloat16().cuda() for _ in range(2)] for _ in range(LAYERS)]
        self.post = [(1 + 0.1 * torch.randn(WIDTH, generator=g)).bfloat16().cuda() for _ in range(LAYERS)]
        self.head = weights(WIDTH, VOCABULARY)
        self.embed = torch.randn(VOCABULARY, WIDTH, generator=g).bfloat16().cuda()
        self.freqs = b.ralm_rotary_frequencies(32, 10000.0, factor=4.0, context=64, low=1.0, high=8.0)

    def run(self, kv, tokens, offsets, max_q, max_len):
        b, n = self.b, tokens.shape[0]
        x = self.embed[tokens.long()].float()
        _, y = b.ralm_residual_norm(x, weight=self.norms[0][0], want_sum=False, out_dtype=torch.bfloat16)
        for i in range(LAYERS):
            w, bias = self.qkv[i]
            q, k, v = b.ralm_linear(y, w, bias=bias).view(n, -1, D).split([HEADS, KV, KV], 1)
            q = b.ralm_kv_append_rotary(kv, i, q, k, v, offsets, self.freqs, interleaved=self.interleaved, amplitude=1.1)
            y = b.ralm_kv_attention(kv, i, q, offsets, max_q=max_q, max_len=max_len)
            # the block's output is normed before it joins the stream, and the stream for the next block, in one call
            _, y = b.ralm_residual_norm(b.ralm_linear(y.view(n, -1), self.out[i]), x, sum=x, post=True, post_weight=self.post[i], weight=self.norms[i][1], scale=0.5)
            x = b.ralm_linear(b.ralm_linear(y, self.up[i], act="silu", gated=True), self.down[i], residual=x, out=x)
            _, y = b.ralm_residual_norm(x, weight=self.norms[i + 1][0] if i + 1 < LAYERS else None, want_sum=False, out_dtype=torch.bfloat16)
        return x, b.ralm_linear(y, self.head, out_dtype=torch.float32)

    def plain(self, kv, tokens, offsets):
        """In 64 bits, rounded where the operators round; keys and values as the cache holds them."""
        def rounded(y):
            return y.float().bfloat16().double()

        def norm(y, w):
            return y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * (1.0 if w is None else w.double())

        def mm(y, w):
            return y @ w.double().T.contiguous()

        n, half = tokens.shape[0], self.freqs.numel()
        off, lens = offsets.tolist(), kv.lens.tolist()
        place = torch.cat([torch.arange(N - (e - a), N) for N, a, e in zip(lens, off[:-1], off[1:])]).cuda().double()
        cos, sin = (f(place.view(-1, 1, 1) * self.freqs) * 1.1 for f in (torch.cos, torch.sin))

        def turned(z):
            u, v = (z[..., 0:2 * half:2], z[..., 1:2 * half:2]) if self.interleaved else (z[..., :half], z[..., half:2 * half])
            p, q = u * cos - v * sin, v * cos + u * sin
            return rounded(torch.cat([torch.stack([p, q], -1).flatten(-2) if self.interleaved else torch.cat([p, q], -1), z[..., 2 * half:]], -1))

        x = self.embed[tokens.long()].double()
        y = rounded(norm(x, self.norms[0][0]))
        for i in range(LAYERS):
            w, bias = self.qkv[i]
            q = turned(rounded(mm(y, w) + bias.double()).view(n, -1, D)[:, :HEADS])
            total = torch.cumsum(torch.tensor([0] + lens), 0).cuda()
            K, V = (z.double() for z in self.b.ralm_kv_read(kv, i, total, sum(lens), dtype=torch.float32))
            rows = []
            for r, (a, e) in enumerate(zip(off[:-1], off[1:])):
                k, v = (z[int(total[r]):int(total[r + 1])].repeat_interleave(HEADS // KV, 1) for z in (K, V))
                for t in range(a, e):
                    seen = lens[r] - (e - t) + 1
                    p = torch.softmax((k[:seen] * q[t]).sum(-1) * D ** -0.5, 0)
                    rows.append((p.unsqueeze(-1) * v[:seen]).sum(0).reshape(-1))
            y = rounded(torch.stack(rows))
            x = x + 0.5 * norm(rounded(mm(y, self.out[i])), self.post[i])
            y = rounded(norm(x, self.norms[i][1]))
            x = x.float().double()
            z = mm(y, self.up[i])
            x = (x + mm(rounded(torch.nn.functional.silu(z[:, :HIDDEN]) * z[:, HIDDEN:]), self.down[i])).float().double()
            y = rounded(norm(x, self.norms[i + 1][0] if i + 1 < LAYERS else None))
        return x, mm(y, self.head)


def cache(b, R):
    kv = b.KVCache.empty(R, 128, 64, n_layers=LAYERS, n_heads=KV, d=D, page_tokens=16)
    kv.pages.zero_()
    return kv


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("prompt,drafts", [([40, 7, 1], [1, 1, 1]), ([33, 70, 16], [5, 1, 3])])
def test_layers(b, prompt, drafts, interleaved):
    net = Layers(b, interleaved)
    g = torch.Generator().manual_seed(7)
    kv = cache(b, len(prompt))
    for counts in (prompt, drafts):                                               # prompts, then a step behind them
        grow = torch.tensor(counts, dtype=torch.int32, device="cuda")
        assert bool(b.ralm_kv_reserve(kv, grow).all())
        off = torch.cumsum(torch.tensor([0] + counts), 0).cuda()
        tokens = torch.randint(0, VOCABULARY, (sum(counts),), generator=g).cuda()
        x, logits = net.run(kv, tokens, off, max(counts), 128)
        want, want_logits = net.plain(kv, tokens, off)
        assert float((x.double() - want).abs().max()) < 2 ** -5 * float(want.abs().max())
        assert float((logits.double() - want_logits).abs().max()) < 2 ** -5 * float(want_logits.abs().max())


def test_a_step_as_one_graph(b):
    """Reserve, layers, target, verification and rollback captured once and replayed as requests grow; an eager run of its own beside it."""
    net = Layers(b, False)
    R, k, drafts = 3, 8, 2
    g = torch.Generator().manual_seed(11)
    states = []
    for _ in range(2):
        kv = cache(b, R)
        prompt = [20, 5, 33]
        b.ralm_kv_reserve(kv, torch.tensor(prompt, dtype=torch.int32, device="cuda"))
        net.run(kv, torch.arange(sum(prompt), device="cuda") % VOCABULARY, torch.cumsum(torch.tensor([0] + prompt), 0).cuda(), 33, 128)
        states.append(kv)
    captured, eager = states
    n = R * (drafts + 1)
    off, q_off = torch.arange(R + 1, device="cuda") * (drafts + 1), torch.arange(R + 1, device="cuda") * drafts
    grow = torch.full((R,), drafts + 1, dtype=torch.int32, device="cuda")
    tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
    near, weights = torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda")
    share, u, u_next = torch.zeros(n, device="cuda"), torch.zeros(R * drafts, device="cuda"), torch.zeros(R, device="cuda")

    def step(kv, ws):
        before = kv.lens.clone()
        b.ralm_kv_reserve(kv, grow, workspace=ws)
        x, logits = net.run(kv, tokens, off, drafts + 1, 128)
        target = b.ralm_knnlm_target(logits, near, weights, share, temperature=0.8)
        ids = tokens.view(R, drafts + 1)[:, 1:].reshape(-1)
        accepted, token = b.ralm_verify_draft(ids, target, u, u_next, q_off)
        b.ralm_kv_truncate(kv, before + 1 + accepted)
        return x, target, accepted, token

    ws = [b.alloc_kv_pages_workspace(kv) for kv in states]
    spare = cache(b, R)
    b.ralm_kv_reserve(spare, torch.full((R,), 9, dtype=torch.int32, device="cuda"))
    step(spare, ws[0])                                                            # the first launches set the kernels' attributes
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(captured, ws[0])
    for i in range(5):
        tokens.copy_(torch.randint(0, VOCABULARY, (n,), generator=g))
        near.copy_(torch.randint(-1, VOCABULARY, (n, k), generator=g))
        weights.copy_(torch.rand(n, k, generator=g))
        for t in (share, u, u_next):
            t.copy_(torch.rand(t.shape, generator=g))
        graph.replay()
        want = step(eager, ws[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(outs, want)) and torch.equal(captured.lens, eager.lens)
        assert bool(want[1].isfinite().all())
