"""Verification rounds over a paged cache: the operators around the verifier, run together as a server would.

A toy target model (random weights, a few attention layers without positions) serves several requests.  Every request
sends K drafted tokens per round and the drafter's distribution; one round is

    PagedCache.extend          pages, slots and lengths for the K + 1 window rows of every request
    PagedCache.append          per layer: the window's keys and values into their slots
    PagedCache.attend          per layer: the window over everything cached
    Verifier.verify            the LM head and the decision head on the final hidden states: what is accepted
    verify_residual            the token behind the accepted drafts, drawn from max(P - Q, 0) or, for a full accept, from P
    PagedCache.commit          the kept lengths; pages of rejected drafts go back to the pool (a request that the pool had no
                               pages for keeps its old length)

Lengths, verdicts and pages stay on the device; the host sees tokens only when it prints them.  With --cache-bits 8 keys and values are
kept as e4m3 codes with a scale for each token and head (append_q8, attend_q8).

    python examples/paged_round.py [--requests 4] [--rounds 6] [--drafts 5] [--cache-bits 16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_17701_b200 as wisv  # noqa: E402


class ToyTarget:
    """Pre-norm attention layers with grouped key heads, and an LM head; bf16 weights, fp32 residual stream."""

    def __init__(self, *, vocab=2000, hidden=512, heads=8, kv_heads=2, head_dim=64, layers=2, seed=0, device="cuda:0"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(*shape, scale):
            return (torch.randn(shape, generator=g, device=device) * scale).bfloat16()

        self.heads, self.kv_heads, self.head_dim, self.device = heads, kv_heads, head_dim, device
        self.embed = weight(vocab, hidden, scale=1.0)
        self.qkv = [weight(hidden, (heads + 2 * kv_heads) * head_dim, scale=hidden ** -0.5) for _ in range(layers)]
        self.out = [weight(heads * head_dim, hidden, scale=(heads * head_dim) ** -0.5) for _ in range(layers)]
        self.lm_head = weight(vocab, hidden, scale=2.0 * hidden ** -0.5)

    @staticmethod
    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def forward(self, tokens, attention):
        """Final hidden states of `tokens`; attention(layer, q, k, v) -> [T, heads, head_dim]."""
        x = self.embed[tokens.long()].float()
        for i, (w, o) in enumerate(zip(self.qkv, self.out)):
            rows = (self.norm(x).bfloat16() @ w).view(len(tokens), -1, self.head_dim)
            h, kv = self.heads, self.kv_heads
            y = attention(i, rows[:, :h], rows[:, h:h + kv], rows[:, h + kv:])
            x = x + (y.reshape(len(tokens), -1) @ o).float()
        return self.norm(x)


class Server:
    """The target with its paged cache and the verifier; every method only enqueues work."""

    def __init__(self, model, *, requests, drafts, page_size=16, max_tokens=256, drafter_hidden=64, seed=1,
                 cache_bits=16):
        dev = model.device
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        self.model, self.B, self.K = model, requests, drafts
        blocks = -(-max_tokens // page_size)
        self.cache = wisv.PagedCache(n_heads=model.heads, n_kv_heads=model.kv_heads, head_dim=model.head_dim,
                                     page_size=page_size, n_pages=requests * blocks, max_requests=requests,
                                     max_blocks=blocks, device=dev)
        shape = (requests * blocks, page_size, model.kv_heads, model.head_dim)
        if cache_bits == 8:
            self.pools = [self.cache.quant_pages() for _ in model.qkv]
        else:
            self.pools = [(torch.empty(shape, dtype=torch.bfloat16, device=dev), torch.empty(shape, dtype=torch.bfloat16, device=dev))
                          for _ in model.qkv]
        vocab, hidden = model.lm_head.shape
        d_j, d_c = 128, 2
        w1 = (torch.randn((d_j, drafter_hidden + hidden + d_c), generator=g, device=dev) * 0.05).bfloat16()
        b1, w2 = torch.zeros(d_j, device=dev), torch.randn(d_j, generator=g, device=dev)
        self.verifier = wisv.Verifier(model.lm_head, w1, b1, w2, 0.0, H_d=drafter_hidden, d_c=d_c, tau=0.5,
                                      max_requests=requests, max_rows=requests * (drafts + 1))

    def forward(self, tokens, layout, max_new):
        """The new tokens through all layers: their keys and values cached, their hidden states returned."""
        def attention(i, q, k, v):
            if isinstance(self.pools[i], wisv.QuantPages):
                self.cache.append_q8(k, v, self.pools[i], layout.slot_map)
                return self.cache.attend_q8(q, self.pools[i], layout.kv_len, B=self.B, max_new=max_new, q_off=layout.q_off)
            k_pages, v_pages = self.pools[i]
            self.cache.append(k, v, k_pages, v_pages, layout.slot_map)
            return self.cache.attend(q, k_pages, v_pages, layout.kv_len, B=self.B, max_new=max_new, q_off=layout.q_off)
        return self.model.forward(tokens, attention)

    def prompt(self, tokens, lengths):
        """Prompts of `lengths` (a list) whose tokens lie one after another; all but the last token of each is cached."""
        n_new = torch.tensor(lengths, dtype=torch.int32, device=self.model.device)
        layout = self.cache.extend(B=self.B, n_new=n_new, T=sum(lengths))
        self.forward(tokens, layout, max(lengths))
        self.commit(layout, layout.kv_len - 1)                     # the last token is the first row of the next window

    def commit(self, layout, new_len):
        """Keeps new_len tokens of the requests that the round served and the old length of the others; returns who was served.
        (A request that got no pages has kv_len 0: nothing of its window is cached.)"""
        served = layout.kv_len > 0
        self.cache.commit(torch.where(served, new_len, self.cache.seq_len[:self.B]), B=self.B)
        return served

    def round(self, last, drafts, draft_probs, draft_hidden, csi, u, u_draw, semantic=True):
        """One window per request: `last` [B] the newest token, `drafts` [B, K].  Returns (accepted [B], next token [B]); a request
        that got no pages is not served: -1 accepted, and its newest token again."""
        B, K = self.B, self.K
        tokens = torch.cat([last[:, None], drafts], 1).reshape(-1)
        layout = self.cache.extend(B=B, n_new=K + 1)
        hidden = self.forward(tokens, layout, K + 1).contiguous()
        flat = drafts.reshape(-1).contiguous()
        probs = torch.softmax(hidden.bfloat16().float() @ self.model.lm_head.float().T, -1)
        accepted = None
        if semantic:                                               # the decision head may keep drafts that sampling rejects
            accepted = self.verifier.verify(hidden, flat, draft_hidden, csi, B=B, K=K, extras=False,
                                            draft_q=draft_probs.gather(1, flat.long()[:, None])[:, 0].contiguous(),
                                            uniforms=u).accept_len
        res = wisv.verify_residual(probs, flat, u, u_draw, B=B, K=K, draft_probs=draft_probs, accept_len=accepted)
        served = self.commit(layout, self.cache.seq_len[:B] + res.accept_len + 1)
        return torch.where(served, res.accept_len, -1), torch.where(served, res.token, last)

    def close(self):
        self.verifier.close()
        self.cache.close()


def serve(requests=4, rounds=6, drafts=5, seed=0, semantic=True, device="cuda:0", cache_bits=16):
    """Runs the rounds and returns (server, the tokens of each request, tokens accepted per round)."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    model = ToyTarget(device=device)
    server = Server(model, requests=requests, drafts=drafts, cache_bits=cache_bits)
    vocab = model.embed.shape[0]
    lengths = [7 + 9 * b for b in range(requests)]
    text = [torch.randint(0, vocab, (n,), generator=g, device=device, dtype=torch.int32) for n in lengths]
    server.prompt(torch.cat(text), lengths)
    last = torch.stack([t[-1] for t in text])
    history = []
    for _ in range(rounds):
        # a stand-in for the drafters: distributions over the vocabulary and tokens drawn from them
        q = torch.softmax(4.0 * torch.randn((requests * drafts, vocab), generator=g, device=device), -1)
        draft = torch.multinomial(q, 1, generator=g).int().view(requests, drafts)
        rand = lambda n: torch.rand(n, generator=g, device=device)  # noqa: E731
        csi = torch.stack([30 * rand(requests), 100 * rand(requests)], 1)
        hidden = torch.randn((requests * drafts, 64), generator=g, device=device)
        accepted, token = server.round(last, draft, q, hidden, csi, rand(requests * drafts), rand(requests), semantic)
        for b in range(requests):                                  # (for the printout only: the cache does not need it)
            if accepted[b] >= 0:
                text[b] = torch.cat([text[b], draft[b, :accepted[b]], token[b:b + 1]])
        last = token
        history.append(accepted.clone())
    return server, text, torch.stack(history)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--rounds", type=int, default=6)
    ap.add_argument("--drafts", type=int, default=5)
    ap.add_argument("--cache-bits", type=int, default=16, choices=(16, 8))
    a = ap.parse_args()
    server, text, accepted = serve(a.requests, a.rounds, a.drafts, cache_bits=a.cache_bits)
    print("accepted drafts per round (rows) and request (columns; -1: no pages):\n%s" % accepted.cpu())
    print("kept tokens %s, free pages %d of %d" % (server.cache.seq_len.tolist(), server.cache.n_free.item(),
                                                   server.cache.n_pages))
    for b, t in enumerate(text):
        print("request %d: %s" % (b, t.tolist()))
    server.close()


if __name__ == "__main__":
    main()
