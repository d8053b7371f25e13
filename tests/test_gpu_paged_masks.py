"""Attention over the paged cache where masks and special values meet: what a row does not see does not reach it.

Row i of a request sees keys 0 .. kv_len - n + i.  A weight is exp(score - max): a score of -inf gives 0, and one of +inf or NaN makes the
row NaN, as it does in the softmax.  An infinite or NaN value reaches the rows that see its key, in its own column.  Finite entries are
held to the tolerance derived in test_gpu_paged.py.
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


def check_special(out, special, ref, dtype, keys):
    """Entries where `special` (float64, 0 elsewhere) is infinite or NaN equal it, the others are within tolerance."""
    odd = ~torch.isfinite(special)
    o = out.double()
    assert torch.equal(torch.isnan(o), torch.isnan(special))
    inf = torch.isinf(special)
    assert torch.equal(torch.isinf(o), inf) and torch.equal(o[inf], special[inf])
    want, mag, _ = ref
    check(torch.where(odd, torch.zeros_like(out), out), None, (torch.where(odd, 0.0, want), mag, None), dtype, keys)


# n_new, kv_len, H, kv, d, page, dtype, and (request, key, key head, column, value) of the odd values
VALUES = {
    # one window of 9 rows, shared by several blocks; the third, fourth and last new token
    "window": ([9], [709], 32, 8, 128, 16, "bf16", [(0, 702, 1, 5, NAN), (0, 703, 1, 6, INF), (0, 703, 0, 0, -INF), (0, 708, 7, 127, NAN)]),
    # the boundary of two 64-key jobs and of two key tiles lies between the new tokens
    "edges": ([20, 20], [138, 74], 8, 2, 64, 16, "fp16", [(0, 127, 0, 1, NAN), (0, 128, 1, 2, INF), (1, 63, 0, 3, -INF), (1, 64, 1, 4, NAN)]),
    # a prompt chunk: pairs of row tiles share a key tile, the odd value is masked for one of them or for both
    "chunk": ([300], [1000], 8, 2, 128, 64, "bf16", [(0, 700, 0, 0, NAN), (0, 731, 0, 1, INF), (0, 732, 1, 2, -INF), (0, 763, 1, 3, NAN),
                                                   (0, 764, 0, 4, NAN), (0, 765, 0, 5, INF), (0, 899, 1, 6, NAN), (0, 999, 1, 7, NAN)]),
    # infinities of both signs in one column: the rows that see one, then both (NaN)
    "signs": ([40], [40], 4, 4, 64, 16, "bf16", [(0, 10, 2, 9, INF), (0, 20, 2, 9, -INF), (0, 12, 3, 9, -INF), (0, 22, 3, 9, -INF), (0, 0, 1, 63, INF)]),
    # a cached value, which every row sees, beside new ones
    "cached": ([5, 70], [400, 1500], 28, 4, 128, 32, "fp16", [(0, 17, 0, 7, INF), (1, 1429, 2, 8, NAN), (1, 1430, 3, 8, NAN), (1, 1470, 3, 9, -INF)]),
    # more rows than keys: rows without a key stay zero
    "fewer": ([6, 300], [3, 120], 8, 2, 128, 16, "bf16", [(0, 0, 0, 3, NAN), (0, 2, 1, 4, INF), (1, 0, 0, 5, NAN), (1, 64, 1, 6, -INF), (1, 119, 1, 7, NAN)]),
    # 64 query heads to a key head: two tokens to a row tile
    "group": ([7], [260], 64, 1, 64, 256, "bf16", [(0, 254, 0, 11, NAN), (0, 255, 0, 12, INF), (0, 256, 0, 13, -INF), (0, 259, 0, 14, NAN)]),
}


@pytest.mark.parametrize("name", VALUES)
@pytest.mark.parametrize("heads_first", [False, True])
def test_odd_values_reach_the_rows_that_see_them_and_no_others(name, heads_first):
    n_new, kv_len, H, kv, d, page, dtype, odd = VALUES[name]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=H, kv=kv, d=d, page=page, dtype=dtype, heads_first=heads_first, seed=11)
    special = torch.zeros(q.shape[0], H, d, dtype=torch.float64, device=DEV)
    for b, key, head, column, _ in odd:                            # the finite part: the odd entries as zeros
        place(cache, vp, b, key, head, column, 0.0)
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, kv_len, q_off, d ** -0.5)
    for b, key, head, column, value in odd:
        place(cache, vp, b, key, head, column, value)
        first = max(0, key - (kv_len[b] - n_new[b]))               # the first row of the request that sees the key
        g = H // kv
        special[q_off[b] + first:q_off[b + 1], head * g:(head + 1) * g, column] += value
    for hint in (max(n_new), 1, 4 * max(n_new) + 3):
        out = cache.attend(q, kp, vp, dev(kv_len), B=len(n_new), max_new=hint, q_off=dev(q_off))
        check_special(out, special, ref, dtype, max(kv_len))
    assert cache.device_error() == 0
    cache.close()


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


@pytest.mark.parametrize("H, kv, d, dtype", [(8, 2, 128, "bf16"), (14, 2, 64, "fp16")])
def test_rows_outside_all_windows_are_zero(H, kv, d, dtype):
    """A batch padded to a fixed number of rows: those before the first window and behind the last."""
    n_new, kv_len = [4, 70], [100, 900]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=H, kv=kv, d=d, page=16, dtype=dtype, seed=2)
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, kv_len, q_off, d ** -0.5)
    for before, behind in ((0, 1), (3, 0), (2, 400)):
        T = before + q.shape[0] + behind
        wide = torch.full((T, H, d), NAN, dtype=q.dtype, device=DEV)
        wide[before:before + q.shape[0]] = q
        big = torch.full((T + 1, H + 1, d + 8), NAN, dtype=q.dtype, device=DEV)
        lse = torch.full((T, H), NAN, dtype=torch.float32, device=DEV)
        out = cache.attend(wide, kp, vp, dev(kv_len), B=2, max_new=70, q_off=dev(q_off) + before, out=big[:T, :H, :d], lse=lse,
                           clear_rest=True)
        inside = torch.zeros(T, dtype=torch.bool, device=DEV)
        inside[before:before + q.shape[0]] = True
        assert (out[~inside] == 0).all() and (lse[~inside] == -INF).all()
        check(out[inside], lse[inside], ref, dtype, 900)
        big[:T, :H, :d] = NAN
        assert torch.isnan(big).all()                              # nothing beside the output was written
    # an output that the call makes is whole without being asked for; no window has a row
    out = cache.attend(q, kp, vp, dev(kv_len), B=2, max_new=1, q_off=dev([0, 0, 0]))
    assert (out == 0).all() and cache.device_error() == 0
    cache.close()


def test_calls_that_share_an_output_leave_each_others_rows_alone():
    """Two calls over parts of one packed batch, in either order, the offsets those of the whole."""
    n_new, kv_len = [4, 70, 1, 9], [100, 900, 33, 40]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=8, kv=2, d=128, page=16, dtype="bf16", seed=6)
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, kv_len, q_off, 128 ** -0.5)
    for parts in (((0, 2), (2, 4)), ((2, 4), (0, 2)), ((1, 2), (0, 1), (2, 4))):
        out, lse = torch.full_like(q, NAN), torch.full(q.shape[:2], NAN, dtype=torch.float32, device=DEV)
        for lo, hi in parts:
            cache.attend(q, kp, vp, dev(kv_len[lo:hi]), B=hi - lo, max_new=70, q_off=dev(q_off[lo:hi + 1]), out=out, lse=lse,
                         block_table=cache.block_table[lo:hi])
        check(out, lse, ref, "bf16", 900)
    cache.close()
