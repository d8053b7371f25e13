"""The example's rounds: what is cached, accepted and emitted agrees with a model that caches nothing."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def dense_hidden(model, tokens):
    """Final hidden states of one sequence without a cache, attention in 64 bits."""
    n, G = len(tokens), model.heads // model.kv_heads

    def attention(i, q, k, v):
        k, v = (x.double().repeat_interleave(G, 1) for x in (k, v))
        s = torch.einsum("nhd,lhd->hnl", q.double(), k) * model.head_dim ** -0.5
        s.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1), float("-inf"))
        return torch.einsum("hnl,lhd->nhd", torch.softmax(s, 2), v).to(q.dtype)
    return model.forward(tokens, attention)


@pytest.mark.parametrize("semantic", [True, False])
def test_rounds_agree_with_a_model_without_a_cache(semantic):
    from paged_round import serve
    server, text, accepted = serve(requests=4, rounds=6, drafts=5, semantic=semantic)
    cache, model = server.cache, server.model
    assert cache.device_error() == 0 and server.verifier.device_error() == 0
    # all but the newest token are kept, on no more pages than that takes
    assert cache.seq_len.tolist() == [len(t) - 1 for t in text]
    held = [-(-(len(t) - 1) // 16) for t in text]
    assert cache.n_blocks.tolist() == held and cache.n_free.item() == cache.n_pages - sum(held)
    used = torch.cat([cache.block_table[b, :h] for b, h in enumerate(held)] + [cache.free_list[:cache.n_free.item()]])
    assert used.sort().values.tolist() == list(range(cache.n_pages))
    # the next token's hidden state over the cache, against the whole sequence at once
    last = torch.stack([t[-1] for t in text])
    layout = cache.extend(B=4, n_new=1)
    got = server.forward(last, layout, 1)
    for b, t in enumerate(text):
        want = dense_hidden(model, t)[-1]
        # two layers of bf16 products (2^-8 a rounding, a few of them in a row) on states of size 1
        assert (got[b] - want).abs().max() < 0.1 and (got[b] - want).norm() < 0.02 * want.norm()
    cache.commit(torch.zeros(4, dtype=torch.int32, device=last.device), B=4)
    assert cache.n_free.item() == cache.n_pages and (cache.block_table == -1).all()
    if semantic:
        assert accepted.max() > 0                                  # the decision head keeps some drafts of random drafters
    server.close()


def test_a_request_that_gets_no_pages_keeps_its_length():
    """Rounds beyond what a request's row of the table can hold: it is not served, and nothing that was not cached is kept."""
    from paged_round import serve
    server, text, accepted = serve(requests=2, rounds=250, drafts=5)
    cache, model = server.cache, server.model
    most = cache.max_blocks * cache.page_size
    assert (accepted < 0).any() and (accepted >= 0).any()          # a round that is not served is marked
    for b, t in enumerate(text):
        kept = len(t) - 1
        assert cache.seq_len[b].item() == kept and most - 6 < kept <= most
        assert len(t) == 7 + 9 * b + sum(a + 1 for a in accepted[:, b].tolist() if a >= 0)
    # the keys of the first layer are those of the whole sequence
    for b, t in enumerate(text):
        rows = {}

        def attention(i, q, k, v):
            rows.setdefault(i, k)
            return torch.zeros_like(q)
        model.forward(t, attention)
        pos = torch.arange(len(t) - 1, device=t.device)
        got = server.pools[0][0][cache.block_table[b].long()[pos // 16], pos % 16]
        # the same products of other batch sizes: a rounding of bf16 apart
        assert (got.float() - rows[0][:-1].float()).abs().max() <= 2.0 ** -6 * rows[0].float().abs().max()
    server.close()
