"""A small neighbour language model on the library's entry points: retrieval, speculation and the generator's cache together.

A decoder of random weights stands in for the language model; everything around it is what a serving program does.  The datastore
holds the decoder's own hidden states over a corpus and the tokens that followed.  Requests share a prompt: it is run once and
its pages are forked.  A round then

1. looks the current state up in the request's speculation cache and drafts the tokens that followed the entry that it finds,
2. reserves room (copying pages that are still shared) and runs the decoder on the drafts: norms of the residual stream, products with their epilogues,
   keys turned by their places on the way into the 4-bit cache, attention,
3. retrieves the neighbours of every state exactly, and mixes their distribution with the decoder's,
4. verifies the drafts against that target from given random numbers,
5. rolls the context back behind the last accepted one and updates the speculation cache.

    python examples/neighbour_generator.py
"""
from __future__ import annotations

import os
import sys
from typing import Optional

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2401_14021_amd import binding as B  # noqa: E402


class Decoder:
    """Two layers, grouped heads of 64; keys and values live in a paged 4-bit cache."""

    def __init__(self, vocabulary: int = 512, width: int = 256, layers: int = 2, heads: int = 4, kv_heads: int = 2, seed: int = 0,
                 window: int = 0, sinks: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weights(n, m):
            """[m, n]: a row for every output."""
            return (torch.randn(n, m, generator=g, device="cuda") * n ** -0.5).bfloat16().t().contiguous()

        self.V, self.width, self.layers, self.H, self.Hkv, self.d = vocabulary, width, layers, heads, kv_heads, 64
        self.window, self.sinks = window, sinks
        self.embed = torch.randn(vocabulary, width, generator=g, device="cuda").bfloat16()
        self.qkv = [weights(width, (heads + 2 * kv_heads) * 64) for _ in range(layers)]
        self.out = [weights(heads * 64, width) for _ in range(layers)]
        self.mlp = [(weights(width, 4 * width), weights(4 * width, width)) for _ in range(layers)]
        self.head = weights(width, vocabulary)
        self.freqs = B.ralm_rotary_frequencies(64)

    def cache(self, requests: int, tokens: int, pages: int) -> B.KVCache:
        return B.KVCache.empty(requests, tokens, pages, n_layers=self.layers, n_heads=self.Hkv, d=self.d, page_tokens=16)

    def run(self, kv: B.KVCache, tokens: torch.Tensor, places: Optional[torch.Tensor], offsets: torch.Tensor, max_q: int, max_len: int):
        """The requests' last tokens (room for them is reserved): hidden states and logits of each, fp32.  ``places``: where they stand in their
        texts; None: where they stand in the cache."""
        n = tokens.shape[0]
        shift = None
        if places is not None:
            first, end = offsets[:-1], offsets[1:]
            shift = (places[first.clamp(max=n - 1)] - (kv.lens - (end - first))).to(torch.int32)

        def normed(x):
            return B.ralm_residual_norm(x, want_sum=False, out_dtype=torch.bfloat16)[1]

        x = self.embed[tokens.long()].float()                                    # the residual stream
        for i in range(self.layers):
            q, k, v = B.ralm_linear(normed(x), self.qkv[i]).view(n, -1, 64).split([self.H, self.Hkv, self.Hkv], 1)
            q = B.ralm_kv_append_rotary(kv, i, q, k, v, offsets, self.freqs, shift=shift)
            y = B.ralm_kv_attention(kv, i, q, offsets, max_q=max_q, max_len=max_len, window=self.window, sinks=self.sinks)
            B.ralm_linear(y.view(n, -1), self.out[i], residual=x, out=x)
            up, down = self.mlp[i]
            B.ralm_linear(B.ralm_linear(normed(x), up, act="relu"), down, residual=x, out=x)
        state = normed(x)
        return state.float(), B.ralm_linear(state, self.head, out_dtype=torch.float32)


class Generator:
    """The speculative loop over one decoder, its datastore and a batch of requests."""

    def __init__(self, model: Decoder, requests: int, max_tokens: int = 512, corpus: int = 2048, k: int = 16, share: float = 0.3,
                 sharpness: float = 1.0, seed: int = 1):
        self.model, self.R, self.k, self.share, self.sharpness = model, requests, k, share, sharpness
        self.max_tokens = max_tokens
        self.kv = model.cache(requests, max_tokens, requests * (max_tokens // 16) + 8)
        self.pages_ws = B.alloc_kv_pages_workspace(self.kv)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        # the datastore: states of a corpus in which a phrase comes again and again, one token in ten another, and what followed
        phrase = torch.randint(0, model.V, (97,), generator=self.gen, device="cuda", dtype=torch.int32)
        tokens = phrase[torch.arange(corpus, device="cuda") % 97]
        noise = torch.randint(0, model.V, (corpus,), generator=self.gen, device="cuda", dtype=torch.int32)
        tokens = torch.where(torch.rand(corpus, generator=self.gen, device="cuda") < 0.1, noise, tokens)
        book = model.cache(1, corpus, corpus // 16)
        B.ralm_kv_reserve(book, torch.tensor([corpus], dtype=torch.int32, device="cuda"))
        states, _ = model.run(book, tokens, None, torch.tensor([0, corpus], device="cuda"), corpus, corpus)
        self.values = torch.roll(tokens, -1).contiguous()
        self.store = B.Datastore.from_fp32(states)
        self.cache_ids = torch.full((requests, 256), -1, dtype=torch.int32, device="cuda")
        self.cache_len = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.cache_head = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.corpus = tokens

    def _step(self, tokens: torch.Tensor, counts: list):
        """Runs counts[r] more tokens of every request: states and the target's distributions behind each of them."""
        grow = torch.tensor(counts, dtype=torch.int32, device="cuda")
        granted = B.ralm_kv_reserve(self.kv, grow, workspace=self.pages_ws)
        if not bool(granted.all()):
            raise RuntimeError("the cache has no room for these requests")
        off = torch.cumsum(torch.tensor([0] + counts, device="cuda"), 0)
        states, logits = self.model.run(self.kv, tokens, None, off, max(counts), self.max_tokens)
        ids, scores = B.ralm_retrieve_topk_ex(states, self.store, self.k)
        near, weights, _, _ = B.ralm_knnlm_probs(ids, scores, self.values, temperature=4.0, want_top=False)
        target = B.ralm_knnlm_target(logits, near, weights, self.share, temperature=1.0 / self.sharpness, out=logits)
        return states, target, ids, off

    def prompt(self, tokens: torch.Tensor):
        """One prompt for all requests: run once, its pages forked; the first token of each is drawn from it."""
        n = tokens.shape[0]
        _, target, ids, _ = self._step(tokens, [n] + [0] * (self.R - 1))
        others = torch.arange(1, self.R, dtype=torch.int32, device="cuda")
        B.ralm_kv_fork(self.kv, torch.zeros_like(others), others)
        # every request draws its own first token from the last row, and begins with the neighbours of the prompt's last state
        u = torch.rand(self.R, generator=self.gen, device="cuda")
        none = torch.zeros(self.R + 1, dtype=torch.int64, device="cuda")
        empty = torch.empty(0, dtype=torch.int32, device="cuda")
        _, first = B.ralm_verify_draft(empty, target[-1:].expand(self.R, -1).contiguous(), u[:0], u, none)
        self._remember(ids[-1:].expand(self.R, -1).contiguous(), torch.arange(self.R + 1, device="cuda"), None)
        self.last = first
        self.texts = [[t] for t in first.tolist()]
        self.state = None

    def _remember(self, ids, off, accepted):
        B.ralm_cache_insert(self.cache_ids, self.cache_len, self.cache_head, ids, off, self.store.N, p=min(8, self.k), n_next=4,
                            first_mismatch=accepted)

    def round(self, stride: int) -> int:
        """Up to stride drafts per request are verified at once; returns how many were accepted."""
        R = self.R
        if self.state is None or stride == 0:
            drafts = torch.empty(R, 0, dtype=torch.int32, device="cuda")
        else:
            one = torch.arange(R + 1, device="cuda")
            found, _ = B.ralm_cache_lookup(self.cache_ids, self.cache_len, self.state, one, self.store)
            # the entry stands for the state that the last token was drawn from: the drafts follow that token
            after = found.clamp(min=0).unsqueeze(1) + 1 + torch.arange(stride, device="cuda")
            drafts = self.values[after.clamp(max=self.store.N - 1).long()]
        s = drafts.shape[1]
        before = self.kv.lens.clone()
        tokens = torch.cat([self.last.unsqueeze(1), drafts], 1).reshape(-1)
        states, target, ids, off = self._step(tokens, [s + 1] * R)
        accepted, token = B.ralm_verify_draft(drafts.reshape(-1).contiguous(), target, torch.rand(R * s, generator=self.gen, device="cuda"),
                                              torch.rand(R, generator=self.gen, device="cuda"), torch.arange(R + 1, device="cuda") * s)
        B.ralm_kv_truncate(self.kv, before + 1 + accepted)
        self._remember(ids, off, accepted + 1)
        self.state = states.view(R, s + 1, -1)[torch.arange(R, device="cuda"), accepted.long()].contiguous()
        self.last = token
        for r, (n, t) in enumerate(zip(accepted.tolist(), token.tolist())):
            self.texts[r] += drafts[r, :n].tolist() + [t]
        return int(accepted.sum())

    def compact(self) -> int:
        """Brings the cache's pages together; the number in use."""
        _, _, used = B.ralm_kv_compact(self.kv, table=self.kv.table, refs=self.kv.refs, workspace=self.pages_ws)
        return int(used)


def main():
    gen = Generator(Decoder(window=192, sinks=4), requests=8, share=0.9)
    gen.prompt(gen.corpus[100:180])
    rounds, drafted, accepted = 24, 0, 0
    for i in range(rounds):
        stride = 4 if i else 0
        accepted += gen.round(stride)
        drafted += stride * gen.R
    torch.cuda.synchronize()
    print(f"{rounds} rounds, {sum(map(len, gen.texts))} tokens, {accepted} of {drafted} drafts accepted; "
          f"{gen.compact()} of {gen.kv.refs.numel()} pages in use")


if __name__ == "__main__":
    main()
