"""The paged cache against plain models of it: a list of pages in Python, attention in 64 bits.

Tolerance of an attention output o = sum_j p_j v_j with p the softmax: the kernel rounds the numerators of p to the cache's type
(relative half step h: 2^-8 for bf16, 2^-11 for fp16, plus 2^-25 absolute where an fp16 numerator is subnormal, against a
largest numerator of at least 1) and the result once more; scores are sums of at most 128 exact products in fp32, so
their error is some 1e-5 of their own size at most and enters p relatively.  Hence
    |error| <= h |o| + (h + 2e-4) sum_j p_j |v_j| + keys 2^-25 max|v| (fp16).
"""
import numpy as np
import pytest
import torch

import paper_2604_17701_b200 as wisv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NO_PAGES, BAD_LENGTH = 32, 128
TYPES = {"bf16": (torch.bfloat16, wisv.DT_BF16, 2.0 ** -8), "fp16": (torch.float16, wisv.DT_F16, 2.0 ** -11)}


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device=DEV)


# ------------------------------------------------------------------------------------------------ pages
class Pool:
    """The bookkeeping with Python lists."""

    def __init__(self, page, n_pages, B, width):
        self.page, self.width, self.size = page, width, n_pages
        self.free = list(range(n_pages - 1, -1, -1))
        self.table = [[] for _ in range(B)]
        self.len = [0] * B

    def extend(self, n_new):
        B, page = len(n_new), self.page
        need, fits = [], []
        for b, n in enumerate(n_new):
            want = -(-(self.len[b] + n) // page)
            fits.append(want <= self.width)
            need.append(max(0, want - len(self.table[b])) if fits[-1] else 0)
        upto = np.cumsum(need)
        good = [f and (c == 0 or u <= len(self.free)) for f, c, u in zip(fits, need, upto)]
        N = sum(c for c, g in zip(need, good) if g)
        taken, self.free = self.free[len(self.free) - N:], self.free[:len(self.free) - N]
        slots, pos, kv = [], [], []
        for b, n in enumerate(n_new):
            if good[b]:
                self.table[b] += taken[:need[b]]
                taken = taken[need[b]:]
            for i in range(n):
                x = self.len[b] + i
                pos.append(x)
                slots.append(self.table[b][x // page] * page + x % page if good[b] else -1)
            kv.append(self.len[b] + n if good[b] else 0)
        return dict(q_off=np.concatenate([[0], np.cumsum(n_new)]), kv_len=kv, slot_map=slots, positions=pos,
                    status=[0 if g else NO_PAGES for g in good])

    def commit(self, new_len):
        status = []
        for b, n in enumerate(new_len):
            most = len(self.table[b]) * self.page
            status.append(BAD_LENGTH if n < 0 or n > most else 0)
            n = min(max(n, 0), most)
            keep = -(-n // self.page)
            self.free += self.table[b][keep:]
            self.table[b] = self.table[b][:keep]
            self.len[b] = n
        return status

    def check(self, cache):
        B = len(self.len)
        assert cache.n_free.item() == len(self.free)
        assert cache.free_list[:len(self.free)].tolist() == self.free
        assert cache.seq_len[:B].tolist() == self.len
        assert cache.n_blocks[:B].tolist() == [len(t) for t in self.table]
        want = np.full((B, self.width), -1)
        for b, t in enumerate(self.table):
            want[b, :len(t)] = t
        assert np.array_equal(cache.block_table[:B].cpu().numpy(), want)


def make_cache(**kw):
    base = dict(n_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=64, max_requests=8, max_blocks=16, device=DEV)
    return wisv.PagedCache(**{**base, **kw})


@pytest.mark.parametrize("B, page, width, n_max, tight", [
    (1, 16, 8, 9, False), (3, 16, 8, 40, False), (8, 32, 16, 65, True), (65, 16, 12, 17, True), (130, 64, 4, 30, True),
    (512, 16, 10, 17, False), (1500, 16, 6, 7, True), (4096, 128, 2, 3, False)])
def test_rounds_match_the_list_model(B, page, width, n_max, tight):
    rng = np.random.default_rng(B)
    n_pages = B * width // (3 if tight else 1)
    cache = make_cache(page_size=page, n_pages=n_pages, max_requests=B, max_blocks=width)
    pool = Pool(page, n_pages, B, width)
    seen = 0
    for step in range(8):
        n_new = rng.integers(0, n_max + 1, B)
        if step == 2:
            n_new[rng.integers(0, B)] = width * page + 1            # longer than a row of the table
        want = pool.extend([int(x) for x in n_new])
        lay = cache.extend(B=B, n_new=dev(n_new), T=int(n_new.sum()))
        for k, v in want.items():
            assert getattr(lay, k).tolist() == [int(x) for x in v], k
        seen |= max(want["status"])
        kv = np.array(want["kv_len"])
        # keep part of the windows, finish a few requests, ask for impossible lengths now and then
        new_len = np.where(kv > 0, kv - (rng.random(B) * (n_new + 1)).astype(int), np.array(pool.len))
        new_len = np.where(rng.random(B) < 0.15, 0, np.maximum(new_len, 0))
        if step == 5:
            new_len[0], new_len[-1] = -4, 1 << 29
        status = cache.commit(dev(new_len), B=B)
        assert status.tolist() == pool.commit([int(x) for x in new_len])
        pool.check(cache)
    assert seen == NO_PAGES or not tight
    cache.close()


def test_prompt_chunks_are_laid_out_by_a_cluster():
    cache = make_cache(page_size=32, n_pages=1000, max_requests=5, max_blocks=400)
    pool = Pool(32, 1000, 5, 400)
    for n_new in ([5000, 0, 1, 3000, 70], [1, 2, 3, 4, 5]):
        want = pool.extend(n_new)
        lay = cache.extend(B=5, n_new=dev(n_new), T=sum(n_new))
        for k, v in want.items():
            assert getattr(lay, k).tolist() == [int(x) for x in v], k
        assert cache.commit(lay.kv_len, B=5).tolist() == pool.commit([int(x) for x in want["kv_len"]])
        pool.check(cache)
    cache.commit(dev([0] * 5), B=5)
    pool.commit([0] * 5)
    pool.check(cache)
    cache.close()


def test_uniform_windows_withdrawn_rounds_and_reused_outputs():
    cache = make_cache()
    lay = cache.extend(B=3, n_new=20)
    cache.commit(lay.kv_len, B=3)
    before = [t.clone() for t in (cache.free_list, cache.n_free, cache.block_table, cache.n_blocks, cache.seq_len)]
    lay2 = cache.extend(B=3, n_new=30, out=None)
    assert lay2.positions.tolist() == [20 + i for _ in range(3) for i in range(30)]
    again = cache.commit(cache.seq_len.clone(), B=3)
    assert again.tolist() == [0, 0, 0]
    for x, y in zip(before, (cache.free_list, cache.n_free, cache.block_table, cache.n_blocks, cache.seq_len)):
        assert torch.equal(x, y)
    slots = lay2.slot_map.clone()
    assert cache.extend(B=3, n_new=30, out=lay2) is lay2 and torch.equal(lay2.slot_map, slots)
    cache.close()


def test_rows_past_the_sum_and_bad_lengths_are_flagged():
    cache = make_cache()
    cache.seq_len[1] = -3
    lay = cache.extend(B=3, n_new=dev([2, 3, -1]), T=8)
    assert lay.q_off.tolist() == [0, 2, 5, 5]
    assert lay.status.tolist() == [0, BAD_LENGTH, BAD_LENGTH]
    assert lay.slot_map.tolist()[5:] == [-1] * 3 and lay.positions.tolist()[5:] == [-1] * 3
    # fewer rows than the sum: nothing is written past them
    buf = torch.full((4,), 77, dtype=torch.int64, device=DEV)
    pos = torch.full((4,), 77, dtype=torch.int32, device=DEV)
    out = wisv.WindowLayout(torch.empty(2, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV),
                            buf, pos, None)
    cache.extend(B=1, n_new=dev([4]), T=2, out=out)
    assert buf.tolist()[2:] == [77, 77] and pos.tolist()[2:] == [77, 77]
    cache.close()


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("kv, d, page, dtype, T, heads_first, fused", [
    (2, 64, 16, "bf16", 1, False, True), (8, 128, 16, "fp16", 9, True, False), (4, 128, 64, "bf16", 77, False, True),
    (1, 64, 256, "fp16", 300, True, True), (3, 128, 32, "bf16", 1000, False, False)])
def test_append_copies_rows_to_their_slots(kv, d, page, dtype, T, heads_first, fused):
    dt, code, _ = TYPES[dtype]
    torch.manual_seed(T)
    pages = T // page + 3
    cache = make_cache(n_heads=kv, n_kv_heads=kv, head_dim=d, page_size=page, n_pages=pages, dtype=code)
    rows = torch.randn(T, 5 + 2 * kv, d, device=DEV).to(dt)
    k, v = rows[:, 5:5 + kv], rows[:, 5 + kv:]
    if not fused:
        k, v = k.contiguous(), v.contiguous()
    shape = (pages, kv, page, d) if heads_first else (pages, page, kv, d)
    pools = [torch.full(shape, 7.0, dtype=dt, device=DEV) for _ in range(2)]
    kp, vp = (x.transpose(1, 2) if heads_first else x for x in pools)
    slots = torch.randperm(pages * page, device=DEV)[:T]
    slots[T // 2:T // 2 + 1] = -1
    if T > 5:
        slots[5] = pages * page                                     # outside the pool: skipped
    cache.append(k, v, kp, vp, slots)
    want_k, want_v = (torch.full((pages * page, kv, d), 7.0, dtype=dt, device=DEV) for _ in range(2))
    ok = (slots >= 0) & (slots < pages * page)
    want_k[slots[ok]], want_v[slots[ok]] = k[ok], v[ok]
    assert torch.equal(kp.reshape(-1, kv, d), want_k) and torch.equal(vp.reshape(-1, kv, d), want_v)
    cache.close()


# ------------------------------------------------------------------------------------------------ attend
def reference(q, k_pages, v_pages, table, kv_len, q_off, scale):
    """Output, its tolerance's sum p|v|, and log-sum-exp, in 64 bits, request by request."""
    T, H, d = q.shape
    page, kv = k_pages.shape[1], k_pages.shape[2]
    G = H // kv
    out = torch.zeros(T, H, d, dtype=torch.float64, device=DEV)
    mag, lse = torch.zeros_like(out), torch.full((T, H), float("-inf"), dtype=torch.float64, device=DEV)
    for b in range(len(kv_len)):
        lo, n, L = q_off[b], q_off[b + 1] - q_off[b], kv_len[b]
        if n == 0 or L == 0:
            continue
        pg = table[b, :-(-L // page)].long()
        inside = (pg >= 0) & (pg < k_pages.shape[0])
        k, v = (x[pg.clamp(0, k_pages.shape[0] - 1)].double() * inside[:, None, None, None] for x in (k_pages, v_pages))
        k, v = (x.reshape(-1, kv, d)[:L].repeat_interleave(G, 1) for x in (k, v))
        s = torch.einsum("nhd,lhd->hnl", q[lo:lo + n].double(), k) * scale
        last = L - n + torch.arange(n, device=DEV)
        s.masked_fill_(torch.arange(L, device=DEV)[None, None] > last[None, :, None], float("-inf"))
        lse[lo:lo + n] = torch.logsumexp(s, 2).T
        p = torch.softmax(s, 2).nan_to_num(0.0)
        out[lo:lo + n] = torch.einsum("hnl,lhd->nhd", p, v)
        mag[lo:lo + n] = torch.einsum("hnl,lhd->nhd", p, v.abs())
    return out, mag, lse


def build(*, n_new, kv_len, H, kv, d, page, dtype, heads_first=False, spread=1.0, poison=True, seed=0, extra=0):
    """A cache filled for these lengths; everything past them (rest of a page, unused pages) is NaN."""
    dt, code, _ = TYPES[dtype]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    B, T = len(n_new), int(sum(n_new))
    blocks = [-(-x // page) for x in kv_len]
    n_pages, width = sum(blocks) + 3, max(blocks) + 1
    cache = wisv.PagedCache(n_heads=H, n_kv_heads=kv, head_dim=d, page_size=page, n_pages=n_pages, max_requests=B,
                            max_blocks=width, dtype=code, device=DEV)
    perm = np.random.default_rng(seed).permutation(n_pages)
    table, at = np.full((B, width), -1), 0
    for b, c in enumerate(blocks):
        table[b, :c] = perm[at:at + c]
        at += c
    cache.block_table.copy_(dev(table))
    shape = (n_pages, kv, page, d) if heads_first else (n_pages, page, kv, d)
    pools = []
    for _ in range(2):
        x = torch.empty(shape, dtype=dt, device=DEV).normal_(generator=g)
        pools.append(x.transpose(1, 2) if heads_first else x)
    if poison:
        live = torch.zeros(n_pages, page, dtype=torch.bool, device=DEV)
        for b, L in enumerate(kv_len):
            s = np.arange(L)
            live[dev(table[b][s // page], torch.int64), dev(s % page, torch.int64)] = True
        for x in pools:
            x[~live] = float("nan")
    rows = torch.empty((T, H + 2 * kv, d), dtype=dt, device=DEV).normal_(0, spread, generator=g)
    q_off = np.concatenate([[0], np.cumsum(n_new)]).astype(int)
    return cache, rows[:, :H], pools[0], pools[1], q_off


def check(out, lse, ref, dtype, keys, v_max=6.0):
    dt, _, h = TYPES[dtype]
    want, mag, want_lse = ref
    tol = h * want.abs() + (h + 2e-4) * mag + 1e-9
    if dtype == "fp16":
        tol = tol + keys * 2.0 ** -25 * v_max + 2.0 ** -25           # subnormal numerators, subnormal results
    off = (out.double() - want).abs()
    assert torch.isfinite(out).all()
    assert (off <= tol).all(), "worst %.3g of its tolerance" % float((off / tol).max())
    if lse is not None:
        fin = torch.isfinite(want_lse)
        assert torch.equal(torch.isfinite(lse), fin) and (lse[~fin] == float("-inf")).all()
        # fp32 score sums and a sum of ex2.approx terms (2^-22 each): 1e-5 of a score of size 30 at most
        assert ((lse.double() - want_lse).abs()[fin] <= 3e-4).all()


CASES = [
    # n_new, kv_len, H, kv, d, page, dtype, heads_first
    ([1], [1], 4, 1, 64, 16, "bf16", False),
    ([1], [1], 8, 2, 128, 16, "fp16", True),
    ([9], [709], 32, 8, 128, 16, "bf16", False),
    ([1, 1, 1], [127, 128, 129], 8, 8, 128, 32, "fp16", False),
    ([1] * 5, [1, 2, 31, 33, 2000], 28, 4, 128, 64, "bf16", True),
    ([2, 0, 5, 17], [2, 40, 1030, 17], 14, 2, 64, 16, "bf16", False),
    ([0, 0, 3], [0, 100, 5], 4, 4, 64, 256, "fp16", True),
    ([65, 3, 64], [65, 1500, 640], 28, 4, 128, 32, "bf16", False),
    ([300], [300], 4, 2, 128, 16, "bf16", False),
    ([257, 1, 130], [1000, 500, 131], 8, 1, 64, 128, "fp16", False),
    ([513, 40], [4000, 900], 6, 2, 128, 64, "bf16", True),
    ([33], [9000], 64, 1, 128, 32, "bf16", False),
    ([5] * 33, list(range(5, 1061, 32)), 24, 8, 128, 16, "fp16", False),
    ([100], [3100], 40, 1, 64, 16, "fp16", True),
    ([1] * 200, [17 + 3 * i for i in range(200)], 8, 8, 64, 16, "bf16", False),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_attend_matches_64_bits(case):
    n_new, kv_len, H, kv, d, page, dtype, heads_first = CASES[case]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=H, kv=kv, d=d, page=page, dtype=dtype,
                                    heads_first=heads_first, seed=case)
    lse = torch.empty(q.shape[0], H, dtype=torch.float32, device=DEV)
    out = cache.attend(q, kp, vp, dev(kv_len), B=len(n_new), max_new=max(n_new), q_off=dev(q_off), lse=lse)
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, kv_len, q_off, d ** -0.5)
    check(out, lse, ref, dtype, max(kv_len))
    assert cache.device_error() == 0
    # max_new only lays out the work
    for hint in (1, 7, 4 * max(n_new) + 3):
        other = cache.attend(q, kp, vp, dev(kv_len), B=len(n_new), max_new=hint, q_off=dev(q_off))
        check(other, None, ref, dtype, max(kv_len))
    assert cache.device_error() == 0
    cache.close()


@pytest.mark.parametrize("spread", [0.0, 8.0, 40.0])
def test_flat_and_peaked_scores(spread):
    """All scores equal; and scores of many tens, where the running maximum keeps growing along the keys."""
    n_new, kv_len = [7, 130], [700, 2000]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=4, kv=1, d=128, page=16, dtype="bf16", spread=spread, seed=3)
    if spread:
        # later keys ever larger, so that every block of keys raises the maximum of some rows
        for b, L in enumerate(kv_len):
            pos = torch.arange(L, device=DEV)
            pg = cache.block_table[b].long()[pos // 16]
            kp[pg, pos % 16] *= (0.05 + pos / L)[:, None, None].to(kp.dtype)
    out = cache.attend(q, kp, vp, dev(kv_len), B=2, max_new=130, q_off=dev(q_off))
    want, mag, _ = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, kv_len, q_off, 128 ** -0.5)
    h = 2.0 ** -8
    # scores reach some hundreds: their fp32 sums are good to 1e-6 of that, which p shows relatively
    tol = h * want.abs() + (h + 2e-4 + 2e-5 * spread) * mag + 1e-9
    assert ((out.double() - want).abs() <= tol).all()
    cache.close()


def test_rows_that_see_no_key_are_zero():
    n_new, kv_len = [6, 4, 300, 5], [3, 0, 120, 5]            # more rows than keys; none at all; both
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=8, kv=2, d=128, page=16, dtype="bf16")
    lse = torch.empty(q.shape[0], 8, dtype=torch.float32, device=DEV)
    out = cache.attend(q, kp, vp, dev(kv_len), B=4, max_new=300, q_off=dev(q_off), lse=lse)
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, kv_len, q_off, 128 ** -0.5)
    check(out, lse, ref, "bf16", 300)
    assert (out[:3] == 0).all() and (out[6:10] == 0).all() and (out[10:190] == 0).all() and (lse[:3] == float("-inf")).all()
    cache.close()


def test_strides_scale_tables_and_missing_pages():
    """Padded outputs and interleaved pools, another scale, a table of the caller's, uniform windows without q_off, entries outside
    the pool (read as zero keys and values)."""
    B, n, kv_len, H, kv, d, page = 3, 6, [200, 100, 333], 8, 2, 128, 16
    cache, q, kp, vp, q_off = build(n_new=[n] * B, kv_len=kv_len, H=H, kv=kv, d=d, page=page, dtype="bf16", seed=5)
    both = torch.empty(kp.shape[0], 2, page, kv, d + 8, dtype=kp.dtype, device=DEV)
    ip, jp = both[:, 0, :, :, :d], both[:, 1, :, :, :d]
    ip.copy_(kp), jp.copy_(vp)
    table = torch.full((B + 1, 40), -7, dtype=torch.int32, device=DEV)
    table[:B, :cache.block_table.shape[1]] = cache.block_table
    table[0, 2], table[2, 5] = -1, 10 ** 6
    wide = torch.full((n * B, H + 3, d + 16), 9.0, dtype=q.dtype, device=DEV)
    out = cache.attend(q, ip, jp, dev(kv_len), B=B, max_new=n, block_table=table[:, :30], scale=0.2,
                       out=wide[:, 1:H + 1, 8:d + 8])
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), table, kv_len, q_off, 0.2)
    check(out, None, ref, "bf16", 333)
    wide[:, 1:H + 1, 8:d + 8] = 9.0
    assert (wide == 9.0).all()                                 # nothing beside the output was written
    cache.close()


def test_lengths_past_the_table_are_cut():
    cache, q, kp, vp, q_off = build(n_new=[4], kv_len=[64], H=4, kv=4, d=64, page=16, dtype="fp16")
    table = cache.block_table[:, :4].contiguous()
    out = cache.attend(q, kp, vp, dev([1000]), B=1, max_new=4, block_table=table)
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), table, [64], q_off, 64 ** -0.5)
    check(out, None, ref, "fp16", 64)
    cache.close()


def test_other_streams_graphs_and_repeats():
    n_new, kv_len = [9, 1, 30], [900, 40, 3000]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=32, kv=8, d=128, page=16, dtype="bf16")
    args = (q, kp, vp, dev(kv_len))
    kw = dict(B=3, max_new=30, q_off=dev(q_off))
    first = cache.attend(*args, **kw)
    torch.cuda.synchronize()
    for _ in range(3):                                         # the same bits every time
        assert torch.equal(cache.attend(*args, **kw), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = cache.attend(*args, **kw, stream=side)
    side.synchronize()
    assert torch.equal(out, first)
    buf = torch.zeros_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(*args, **kw, out=buf)
    for _ in range(2):
        buf.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(buf, first)
    # the graph reads lengths when it runs
    args[3].copy_(dev([800, 40, 2900]))
    graph.replay()
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, [800, 40, 2900], q_off, 128 ** -0.5)
    check(buf, None, ref, "bf16", 3000)
    assert cache.device_error() == 0
    cache.close()


def test_pools_past_four_gigabytes():
    """Page offsets that do not fit 32 bits, for the copy and for the attention."""
    page, kv, d, n_pages = 256, 8, 128, 8300                   # 2.2e9 elements, 4.35 GB per pool
    cache = wisv.PagedCache(n_heads=32, n_kv_heads=kv, head_dim=d, page_size=page, n_pages=n_pages, max_requests=2,
                            max_blocks=8, device=DEV)
    kp = torch.empty(n_pages, page, kv, d, dtype=torch.bfloat16, device=DEV)
    vp = torch.empty_like(kp)
    cache.free_list.copy_(torch.arange(n_pages, dtype=torch.int32, device=DEV))       # the highest pages first
    torch.manual_seed(1)
    lay = cache.extend(B=2, n_new=300)
    assert lay.slot_map.max().item() == n_pages * page - 1 - (512 - 300)
    k, v = (torch.randn(600, kv, d, device=DEV).bfloat16() for _ in range(2))
    cache.append(k, v, kp, vp, lay.slot_map)
    assert torch.equal(kp.view(-1, kv, d)[lay.slot_map], k) and torch.equal(vp.view(-1, kv, d)[lay.slot_map], v)
    q = torch.randn(600, 32, d, device=DEV).bfloat16()
    out = cache.attend(q, kp, vp, lay.kv_len, B=2, max_new=300, q_off=lay.q_off)
    ref = reference(q, kp, vp, cache.block_table, [300, 300], [0, 300, 600], d ** -0.5)
    check(out, None, ref, "bf16", 300)
    cache.close()


def test_refusals():
    cache = make_cache(n_heads=8, n_kv_heads=2, head_dim=64)
    q = torch.zeros(4, 8, 64, dtype=torch.bfloat16, device=DEV)
    kp = torch.zeros(64, 16, 2, 64, dtype=torch.bfloat16, device=DEV)
    n = dev([4])
    cache.attend(q, kp, kp, n, B=1, max_new=4)
    for bad in (dict(q=q.half()), dict(q=q[:, :4]), dict(q=q.cpu()), dict(k_pages=kp[:3]), dict(v_pages=kp.transpose(1, 2)),
                dict(kv_len=n.long()), dict(kv_len=n.cpu()), dict(scale=-1.0), dict(scale=float("nan")),
                dict(q_off=dev([0])), dict(out=torch.zeros_like(q)[:2]), dict(lse=torch.zeros(4, 8, dtype=torch.float64, device=DEV)),
                dict(block_table=cache.block_table.long())):
        with pytest.raises(ValueError):
            cache.attend(**{**dict(q=q, k_pages=kp, v_pages=kp, kv_len=n, B=1, max_new=4), **bad})
    for bad, code in ((dict(max_new=0), -2), (dict(max_new=3), -2), (dict(B=9, kv_len=dev([0] * 9), q_off=dev([0] * 10)), -4),
                      (dict(q=torch.zeros(4 * 8 * 64 + 8, dtype=torch.bfloat16, device=DEV)[1:2049].view(4, 8, 64)), -3),
                      (dict(q=torch.zeros(4, 8, 65, dtype=torch.bfloat16, device=DEV)[:, :, :64]), -3)):
        with pytest.raises(wisv.WisvError) as e:
            cache.attend(**{**dict(q=q, k_pages=kp, v_pages=kp, kv_len=n, B=1, max_new=4, block_table=None), **bad})
        assert e.value.code == code
    for call in (lambda: cache.extend(B=9, n_new=1), lambda: cache.commit(dev([0] * 9), B=9)):
        with pytest.raises(wisv.WisvError) as e:
            call()
        assert e.value.code == -4
    with pytest.raises(ValueError):
        cache.extend(B=1, n_new=n)                              # the sum of a device tensor is the caller's to give
    with pytest.raises(ValueError):
        cache.commit(n.long(), B=1)
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    for bad in ((k, k[:3], kp, kp, n), (k.half(), k, kp, kp, n), (k, k, kp, kp, dev([0, 1, 2, 3]))):
        with pytest.raises(ValueError):
            cache.append(*bad)
    cache.append(k[:0], k[:0], kp, kp, torch.empty(0, dtype=torch.int64, device=DEV))
    assert cache.attend(q[:0], kp, kp, n, B=1, max_new=4, q_off=dev([0, 0])).shape == (0, 8, 64)
    assert cache.device_error() == 0
    cache.close()


def test_a_workspace_of_the_callers():
    import ctypes as C
    from paper_2604_17701_b200 import paged
    lib = paged._lib()
    cfg = paged._CacheConfig(8, 2, 64, 16, 64, 8, 16, wisv.DT_BF16)
    need, h = C.c_int64(), C.c_void_p()
    assert lib.wisv_cache_workspace(C.byref(cfg), C.byref(need)) == 0 and need.value > 0
    buf = torch.full((need.value + 256,), 255, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for shift, size, code in ((8, need.value, -3), (0, need.value - 1, -4), (0, need.value, 0)):
        cfg.workspace, cfg.workspace_bytes = buf.data_ptr() + shift, size
        assert lib.wisv_cache_create(C.byref(cfg), C.byref(h)) == code
        assert bool(h.value) == (code == 0)
    flags = C.c_int32(9)
    assert lib.wisv_cache_error(h, None, C.byref(flags)) == 0 and flags.value == 0     # cleared at create
    assert lib.wisv_cache_destroy(h) == 0
    cfg.workspace, cfg.workspace_bytes = None, 0                                       # one of its own
    assert lib.wisv_cache_create(C.byref(cfg), C.byref(h)) == 0 and lib.wisv_cache_destroy(h) == 0


def test_stale_workspace_does_not_matter():
    """Everything a call reads of its workspace it has written itself (the arrival counters and the error word excepted)."""
    n_new, kv_len = [9, 300], [3000, 1000]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=32, kv=8, d=128, page=16, dtype="bf16")
    args = (q, kp, vp, dev(kv_len))
    kw = dict(B=2, max_new=300, q_off=dev(q_off))
    first = cache.attend(*args, **kw)
    cache._workspace[1024:] = 255                              # NaN in every partial result
    assert torch.equal(cache.attend(*args, **kw), first)
    cache.close()


def test_offsets_that_overlap_are_reported():
    """Row offsets that run back and forth make more work than the line of key tiles can count: nothing runs, an error bit says so,
    and the cache stays usable."""
    B, T = 4096, 1 << 20
    cache = make_cache(n_heads=1, n_kv_heads=1, page_size=256, max_requests=B, max_blocks=4096, n_pages=4)
    q = torch.zeros(T, 1, 64, dtype=torch.bfloat16, device=DEV)
    kp = torch.zeros(4, 256, 1, 64, dtype=torch.bfloat16, device=DEV)
    off = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    off[1::2] = T
    # 2048 times all rows, each over up to 2^20 keys: 3e10 key tiles
    cache.attend(q, kp, kp, torch.full((B,), 1 << 20, dtype=torch.int32, device=DEV), B=B, max_new=128, q_off=off)
    assert cache.device_error() == 4 and cache.device_error() == 0
    out = cache.attend(q[:5], kp, kp, dev([5]), B=1, max_new=5)
    assert torch.isfinite(out).all() and cache.device_error() == 0
    cache.close()


def test_nan_keys_reach_the_rows_that_see_them_and_no_others():
    n_new, kv_len = [6, 40], [500, 300]
    for where in (3, 64, 65, 200, 297):                        # cached keys; the third new token of the second request
        cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=4, kv=2, d=128, page=16, dtype="bf16", seed=where)
        pg = int(cache.block_table[1, where // 16])
        kp[pg, where % 16, 1] = float("nan")
        out = cache.attend(q, kp, vp, dev(kv_len), B=2, max_new=40, q_off=dev(q_off))
        bad = torch.isnan(out).all(2)
        assert torch.equal(bad, torch.isnan(out).any(2))
        want = torch.zeros_like(bad)
        first = max(0, where - (300 - 40))                     # the first new row whose keys include it
        want[6 + first:, 2:] = True
        assert torch.equal(bad, want), where
        assert cache.device_error() == 0
        cache.close()


@pytest.mark.parametrize("rows, d, dtype", [(1, 128, "fp16"), (1, 64, "bf16"), (40, 128, "bf16")])
def test_batches_that_fill_memory_bandwidth(rows, d, dtype):
    """Every block works at a stretch of some twenty tiles of several requests, one or two row tiles each, keys and values arriving
    later than they are asked for: whatever runs ahead has to stop for what it needs."""
    rng = np.random.default_rng(rows + d)
    B, H, kv, page = 96, 16, 4, 32
    n_new = [1] * B if rows == 1 else [int(x) for x in rng.integers(1, rows + 1, B)]
    kv_len = [int(x) for x in rng.integers(64, 5000, B)]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=H, kv=kv, d=d, page=page, dtype=dtype, seed=rows)
    args = dict(B=B, max_new=max(n_new), q_off=dev(q_off))
    length = dev(kv_len)
    outs = [cache.attend(q, kp, vp, length, **args) for _ in range(6)]
    ref = reference(q, kp.nan_to_num(0.0), vp.nan_to_num(0.0), cache.block_table, kv_len, q_off, d ** -0.5)
    check(outs[0], None, ref, dtype, max(kv_len))
    for o in outs[1:]:
        assert torch.equal(o, outs[0])
    assert cache.device_error() == 0
    cache.close()


def test_another_current_device_is_refused():
    """The calls check the current device against the one at create; as a second device need not be there, the number kept
    behind the configuration is changed instead."""
    import ctypes as C
    from paper_2604_17701_b200 import paged
    cache = make_cache()
    q = torch.zeros(4, 8, 64, dtype=torch.bfloat16, device=DEV)
    kp = torch.zeros(64, 16, 2, 64, dtype=torch.bfloat16, device=DEV)
    k, n, slots = q[:, :2], dev([4]), dev([0, 1, 2, 3], torch.int64)
    calls = [lambda: cache.extend(B=1, n_new=1), lambda: cache.commit(dev([0]), B=1), lambda: cache.append(k, k, kp, kp, slots),
             lambda: cache.attend(q, kp, kp, n, B=1, max_new=4), lambda: cache.device_error()]
    kept = C.c_int32.from_address(cache._h.value + C.sizeof(paged._CacheConfig))
    assert kept.value == torch.cuda.current_device()
    for call in calls:
        call()
        kept.value += 1
        with pytest.raises(wisv.WisvError) as e:
            call()
        kept.value -= 1
        assert e.value.code == -1
    cache.close()


def test_attention_right_behind_the_call_that_lays_pages_out():
    """extend hands out pages, commit takes them back, and attend reads the table in the next launch, with nothing between."""
    B, page, H, kv, d = 96, 16, 8, 2, 64
    cache = make_cache(n_heads=H, n_kv_heads=kv, head_dim=d, page_size=page, n_pages=B * 16, max_requests=B, max_blocks=16)
    torch.manual_seed(0)
    kp, vp = (torch.randn(B * 16, page, kv, d, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn(B * 20, H, d, device=DEV).bfloat16()
    outs, layouts, tables = [], [], []
    order = torch.randperm(B * 16, device=DEV).int()
    for step in range(8):
        cache.free_list.copy_(order.roll(step * 7))                # other pages every time
        lay = cache.extend(B=B, n_new=20)
        outs.append(cache.attend(q, kp, vp, lay.kv_len, B=B, max_new=20, q_off=lay.q_off))
        layouts.append(lay.kv_len.clone())
        tables.append(cache.block_table.clone())
        cache.commit(torch.zeros(B, dtype=torch.int32, device=DEV) if step % 2 else lay.kv_len - 7, B=B)
    off = [20 * b for b in range(B + 1)]
    for out, kv_len, table in zip(outs, layouts, tables):
        check(out, None, reference(q, kp, vp, table, kv_len.tolist(), off, d ** -0.5), "bf16", 256)
    cache.close()
