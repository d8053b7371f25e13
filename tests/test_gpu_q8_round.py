"""The example's rounds over a cache in 8 bits: what is cached, read back and attended to agrees with a model that caches nothing."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def rounded(x):
    """Keys or values [n, heads, d] as the cache keeps them: codes of the nearest e4m3 number to 448 x / max|x|, times max|x| / 448."""
    t = x.double().abs().amax(-1, keepdim=True).clamp(min=1e-300)
    return (x.double() * 448 / t).float().to(torch.float8_e4m3fn).double() * t / 448


@pytest.mark.parametrize("drafts", [5, 20])
def test_rounds_agree_with_a_model_without_a_cache(drafts):
    from paged_round import serve
    server, text, _ = serve(requests=4, rounds=6, drafts=drafts, cache_bits=8)
    cache, model = server.cache, server.model
    assert cache.device_error() == 0 and server.verifier.device_error() == 0
    assert cache.seq_len.tolist() == [len(t) - 1 for t in text]
    G = model.heads // model.kv_heads
    # keys and values of the first layer, read back, are those of the whole sequence quantised: the products are of other batch
    # sizes, a rounding of bf16 apart (2^-8), and each may be one code off for it (2^-3 between codes, of their size)
    for b, t in enumerate(text):
        rows = {}

        def attention(i, q, k, v):
            rows.setdefault(i, (k, v))
            return torch.zeros_like(q)
        model.forward(t, attention)
        start = torch.zeros(1, dtype=torch.int32, device=t.device)
        got = cache.read_q8(server.pools[0], B=1, n=len(t) - 1, start=start, block_table=cache.block_table[b:b + 1])
        for x, y in zip(got, rows[0]):
            y = y[:-1].double()
            assert ((x.double() - y).abs() <= 2.0 ** -3 * y.abs() + 2.0 ** -8 * y.abs().amax(-1, keepdim=True)).all()
    # the next token's hidden state over the cache, against the whole sequence at once with keys and values rounded alike
    last = torch.stack([t[-1] for t in text])
    layout = cache.extend(B=4, n_new=1)
    got = server.forward(last, layout, 1)

    def dense(i, q, k, v):
        n = len(q)
        k, v = (rounded(x).repeat_interleave(G, 1) for x in (k, v))
        s = torch.einsum("nhd,lhd->hnl", q.double(), k) * model.head_dim ** -0.5
        s.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1), float("-inf"))
        return torch.einsum("hnl,lhd->nhd", torch.softmax(s, 2), v).to(q.dtype)
    for b, t in enumerate(text):
        want = model.forward(t, dense)[-1]
        # bf16 products (2^-8 a rounding, a few in a row) on states of size 1, and codes that fall the other way for them
        assert (got[b] - want).norm() < 0.03 * want.norm()
    server.close()
