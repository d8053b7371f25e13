"""Attention over the paged cache where masks and special values meet: what a row does not see does not reach it.

Row i of a request sees keys 0 .. kv_len - n + i.  A weight is exp(score - max): a score of -inf gives 0, and one of +inf or NaN makes the
row NaN, as it does in the softmax.  Finite entries are held to the tolerance derived in test_gpu_paged.py.
"""
import pytest
import torch

from test_gpu_paged import DEV, build, check, dev, reference

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def place(cache, pool, b, key, head, column, value):
    """Writes one element of a request's key or value."""
    page = pool.shape[1]
    pool[int(cache.block_table[b, key // page]), key % page, head, column] = value


@pytest.mark.parametrize("n, L", [(40, 300), (9, 709), (300, 300)])
def test_large_values_do_not_reach_rows_that_do_not_see_them(n, L):
    """Values near the type's largest number: times anything but 0 they would show."""
    H, kv, d = 8, 2, 128
    cache, q, kp, vp, q_off = build(n_new=[n], kv_len=[L], H=H, kv=kv, d=d, page=16, dtype="bf16", seed=n)
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, [L], q_off, d ** -0.5)
    first = n // 3                                                 # new tokens from here on hold large values
    for key in range(L - n + first, L):
        place(cache, vp, 0, key, slice(None), slice(None), 3e38)
    for hint in (n, 1):
        out = cache.attend(q, kp, vp, dev([L]), B=1, max_new=hint, q_off=dev(q_off))
        check(out[:first], None, [x[:first] for x in ref], "bf16", L)
    cache.close()


# n_new, kv_len, H, kv, d, dtype, the keys that get an infinite element
SCORES = {
    "whole items": ([300], [300], 4, 2, 128, "bf16", [0, 1, 2, 16, 17, 33, 63, 64, 65, 80, 250, 299]),
    "shared items": ([9], [709], 32, 8, 128, "bf16", [0, 1, 5, 48, 64, 130, 657, 700, 704, 708]),
    "one row": ([1, 1], [500, 64], 8, 8, 64, "fp16", [0, 2, 17, 63, 48]),
    "two tiles": ([70], [600], 14, 2, 64, "fp16", [0, 16, 18, 529, 544, 592]),
}


@pytest.mark.parametrize("name", SCORES)
def test_infinite_scores(name):
    """One infinite element in one key: +inf scores make the row NaN, -inf scores have no weight."""
    n_new, kv_len, H, kv, d, dtype, keys = SCORES[name]
    g, scale = H // kv, d ** -0.5
    for key in keys:
        cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=H, kv=kv, d=d, page=16, dtype=dtype, seed=key + 1)
        b = len(n_new) - 1 if key < kv_len[-1] else 0
        head = key % kv
        place(cache, kp, b, key, head, 3, INF)
        lse = torch.empty(q.shape[0], H, dtype=torch.float32, device=DEV)
        out = cache.attend(q, kp, vp, dev(kv_len), B=len(n_new), max_new=max(n_new), q_off=dev(q_off), lse=lse)
        # in 64 bits: rows whose query has a positive third element are NaN, for the others the key is not there
        rows = torch.zeros(q.shape[0], H, dtype=torch.bool, device=DEV)
        lo, hi = int(q_off[b]) + max(0, key - (kv_len[b] - n_new[b])), int(q_off[b + 1])
        rows[lo:hi, head * g:(head + 1) * g] = True
        bad = rows & (q[:, :, 3] >= 0)
        finite = kp.nan_to_num(0.0, 0.0, 0.0)
        place(cache, finite, b, key, head, 3, 0.0)
        want, mag, want_lse = reference(q, finite, vp.nan_to_num(0.0), cache.block_table, kv_len, q_off, scale)
        gone = rows & ~bad
        if gone.any():
            page = kp.shape[1]
            pg = cache.block_table[b, :-(-kv_len[b] // page)].long()
            k, v = (x[pg].reshape(-1, kv, d)[:kv_len[b], head].double() for x in (finite, vp.nan_to_num(0.0)))
            for r, h in gone.nonzero().tolist():
                s = k[:kv_len[b] - n_new[b] + r - int(q_off[b]) + 1] @ q[r, h].double() * scale
                s[key] = -INF
                p = torch.softmax(s, 0).nan_to_num(0.0)
                want[r, h], mag[r, h] = p @ v[:len(s)], p @ v[:len(s)].abs()
                want_lse[r, h] = torch.logsumexp(s, 0)
        assert torch.equal(torch.isnan(out).any(2), bad) and torch.equal(torch.isnan(out).all(2), bad), key
        assert torch.equal(torch.isnan(lse), bad), key
        zero = torch.zeros((), dtype=torch.float64, device=DEV)
        check(out.masked_fill(bad[:, :, None], 0.0), lse.masked_fill(bad, 0.0),
              (torch.where(bad[:, :, None], zero, want), mag, torch.where(bad, zero, want_lse)), dtype, max(kv_len))
        assert cache.device_error() == 0
        cache.close()
