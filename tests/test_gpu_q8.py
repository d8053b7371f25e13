"""The paged cache in 8 bits against plain models in 64 bits.

Codes.  x and the largest |x| of its head, t, have at most 11 bits, so 448 x / t in 64 bits is a border between two e4m3 numbers only where
it is one exactly, and rounding it is the definition: codes must be equal.  Scales are one division in fp32 (2^-24, relative, or half a step of
2^-149 where the result is subnormal).

Attention.  With p the softmax, c and b the codes and scales of the values, v = c b.  A numerator P of p, times b, is cut into parts that are added
up again (by way of fp16, 2^-11 at most): two parts leave a bf16 cache at most 2^-8 of it, three an fp16 one 2^-13.  Below that is
the last part's half step, 2^-14 at most in units in which a column's largest P b is 1 or more; it meets every code.  Queries lose at
most 2^-17 of the largest element A of their tile in each element, which enters a score as scale 2^-17 A sum_d |k_d|; sums are fp32, 2e-4
covers them as in the 16-bit test.  The result is rounded once.  With h = 2^-11 + 2^-8 (2^-13 for fp16) and r = eps / 2:
    |error| <= r |o| + (h + 2e-4 + 2 dq) sum_j p_j |v_j| + 2^-13.9 max_j (p_j b_j) sum_j |c_j|,   dq = scale 2^-17 A max_j sum_d |k_jd|.
"""
import math

import pytest
import torch

import paper_2604_17701_b200 as wisv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn
TYPES = {"bf16": (torch.bfloat16, wisv.DT_BF16, 2.0 ** -8), "fp16": (torch.float16, wisv.DT_F16, 2.0 ** -11)}
NAN, INF = float("nan"), float("inf")


def dev(a, dtype=torch.int32):
    return torch.tensor(a, dtype=dtype, device=DEV)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def values(codes):
    return codes.float().double()


def pools(cache, heads_first):
    """Pools of NaN codes and scales: what nothing has been written to."""
    n, page, kv, d = cache._pool
    shape = (n, kv, page, d) if heads_first else (n, page, kv, d)
    made = [torch.full(shape, 0x7F, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)]
    if heads_first:
        made = [x.transpose(1, 2) for x in made]
    made += [torch.full((n, kv, page), NAN, device=DEV).transpose(1, 2) for _ in range(2)]
    return wisv.QuantPages(*made)


def quantise(x):
    """(codes as numbers in 64 bits, scales) of rows x [..., d] in 16 bits, by the definition."""
    t = x.abs().amax(-1, keepdim=True).double()
    fine = torch.isfinite(t)
    y = torch.where(fine & (t > 0), x.double() * 448 / torch.where(t > 0, t, 1.0), 0.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, torch.where(fine, t / 448, NAN)[..., 0]


class Case:
    """Requests with cached keys and values (written by append_q8 from 16-bit rows) and queries."""

    def __init__(self, n_new, kv_len, H, kv, d, page, dtype, heads_first=True, seed=0, k_size=0.4, edit=None, spare=3):
        tdt, code, _ = TYPES[dtype]
        B, width = len(n_new), max(1, -(-max(kv_len) // page))
        need = [-(-n // page) for n in kv_len]
        n_pages = sum(need) + spare
        self.cache = wisv.PagedCache(n_heads=H, n_kv_heads=kv, head_dim=d, page_size=page, n_pages=n_pages, max_requests=B, max_blocks=width,
                                     dtype=code, device=DEV)
        g, order, at = gen(seed), torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).int(), 0
        slots, self.k, self.v = [], [], []
        for b, n in enumerate(kv_len):
            self.cache.block_table[b, :need[b]] = order[at:at + need[b]].to(DEV)
            at += need[b]
            i = torch.arange(n, device=DEV)
            slots.append(self.cache.block_table[b].long()[i // page] * page + i % page)
            for rows in (self.k, self.v):
                rows.append((normal(g, n, kv, d) * torch.exp(k_size * normal(g, n, kv, 1))).to(tdt))
        if edit:
            edit(self)
        self.pages = pools(self.cache, heads_first)
        self.cache.append_q8(torch.cat(self.k), torch.cat(self.v), self.pages, torch.cat(slots))
        self.n_new, self.kv_len, self.dtype, self.group = n_new, kv_len, dtype, H // kv
        off = [0]
        for n in n_new:
            off.append(off[-1] + n)
        self.off, self.T = off, off[-1]
        self.q = normal(g, off[-1], H, d).to(tdt)

    def attend(self, q=None, **kw):
        args = dict(B=len(self.n_new), max_new=max(max(self.n_new), 1), q_off=dev(self.off))
        return self.cache.attend_q8(self.q if q is None else q, self.pages, dev(self.kv_len), **{**args, **kw})

    def reference(self, q=None, scale=None):
        """(output, tolerance, lse, tolerance of lse) in 64 bits."""
        q = self.q if q is None else q
        d = q.shape[2]
        scale = d ** -0.5 if scale is None else scale
        h = 2.0 ** -11 + (2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -13)
        outs, tols, lses, ltols = [], [], [], []
        for b, (n, L) in enumerate(zip(self.n_new, self.kv_len)):
            (kc, ks), (vc, vs) = (tuple(x.repeat_interleave(self.group, 1) for x in quantise(rows[b])) for rows in (self.k, self.v))
            k, rows = kc * ks[..., None], q[self.off[b]:self.off[b + 1]].double()
            s = torch.einsum("nhd,lhd->nhl", rows, k) * scale
            hide = torch.arange(L, device=DEV)[None] > (L - n + torch.arange(n, device=DEV))[:, None]
            s = s.masked_fill(hide[:, None], -INF)
            lse = torch.logsumexp(s, -1) if L else torch.full((n, s.shape[1]), -INF, dtype=torch.float64, device=DEV)
            p = torch.where(torch.isneginf(lse)[..., None], 0.0, torch.exp(s - lse[..., None]))
            seen = torch.where(hide[:, None], 0.0, p)
            # (what a row does not see is taken out, so that NaN there does not count)
            vz, bz = torch.nan_to_num(vc * vs[..., None], nan=0.0), torch.nan_to_num(vs, nan=0.0)
            o = torch.einsum("nhl,lhd->nhd", torch.nan_to_num(seen, nan=0.0), vz)
            bad = ((torch.isnan(ks) | torch.isnan(vs)).T[None] & ~hide[:, None]).any(-1) | torch.isnan(lse)
            mag = torch.einsum("nhl,lhd->nhd", torch.nan_to_num(seen, nan=0.0), vz.abs())
            most = (torch.nan_to_num(seen, nan=0.0) * bz.T[None]).amax(-1) if L else torch.zeros(s.shape[:2], dtype=torch.float64, device=DEV)
            codes = torch.einsum("nhl,lhd->nhd", (~hide[:, None]).double().expand_as(s).contiguous(), vc.abs())
            A = torch.nan_to_num(rows, nan=0.0, posinf=0.0, neginf=0.0).abs().amax(dim=(0, 2)) if n else torch.zeros(s.shape[1], dtype=torch.float64, device=DEV)
            A = A.view(-1, self.group).amax(1).repeat_interleave(self.group)                        # (tiles hold the heads of a key head)
            dq = scale * 2.0 ** -17 * A * (torch.nan_to_num(k, nan=0.0).abs().sum(-1).amax(0) if L else 0.0)
            tol = TYPES[self.dtype][2] * o.abs() + (h + 2e-4 + 2 * dq)[:, None] * mag + 2.0 ** -13.9 * most[..., None] * codes
            outs.append(torch.where(bad[..., None], NAN, o))
            tols.append(tol)
            lses.append(torch.where(bad, NAN, lse))
            ltols.append((dq + 5e-5)[None].expand(n, -1))
        return torch.cat(outs), torch.cat(tols), torch.cat(lses), torch.cat(ltols)


def check(out, lse, ref):
    want, tol, want_lse, ltol = ref
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    fine = ~torch.isnan(want)
    off = (out.double() - want)[fine].abs()
    assert (off <= tol[fine]).all(), "worst %.3g of the tolerance" % (off / tol[fine].clamp(min=1e-300)).max().item()
    if lse is not None:
        assert torch.equal(torch.isnan(lse), torch.isnan(want_lse)) and torch.equal(torch.isneginf(lse), torch.isneginf(want_lse))
        fine = torch.isfinite(want_lse)
        assert ((lse.double() - want_lse)[fine].abs() <= ltol[fine]).all()


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("kv, d, page, dtype, T, heads_first, fused", [
    (1, 64, 16, "bf16", 1, True, False), (2, 128, 16, "fp16", 9, False, True), (8, 128, 64, "bf16", 700, True, True),
    (3, 64, 256, "fp16", 333, False, False), (5, 128, 32, "bf16", 65, True, False), (7, 64, 128, "bf16", 1000, False, True)])
def test_append_rounds_to_the_nearest_code(kv, d, page, dtype, T, heads_first, fused):
    tdt, code, _ = TYPES[dtype]
    n_pages = T // page + 5
    cache = wisv.PagedCache(n_heads=kv, n_kv_heads=kv, head_dim=d, page_size=page, n_pages=n_pages, max_requests=1, max_blocks=n_pages, dtype=code)
    g = gen(T)
    rows = normal(g, T, 3 * kv if fused else 2 * kv, d)
    whole = torch.randint(-60, 61, rows.shape, generator=g, device=DEV).float()                      # (quotients of whole numbers: ties)
    rows = torch.where(torch.rand((T, 1, 1), generator=g, device=DEV) < 0.5, rows, whole)
    lo, hi = (-140, 110) if dtype == "bf16" else (-24, 9)
    size = torch.randint(lo, hi, (T, rows.shape[1], 1), generator=g, device=DEV).float()
    rows = (rows * torch.where(torch.rand(size.shape, generator=g, device=DEV) < 0.3, torch.exp2(size), 1.0)).to(tdt)
    if T > 60:
        rows[3, :, 1], rows[4, :, d - 1], rows[5, :, 0], rows[6] = NAN, INF, -INF, 0.0
    k, v = (rows[:, kv:2 * kv], rows[:, 2 * kv:]) if fused else (rows[:, :kv].contiguous(), rows[:, kv:].contiguous())
    pages = pools(cache, heads_first)
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(1))[:T].to(DEV)
    given = slots.clone()
    given[::7] = torch.where(torch.arange(len(given[::7]), device=DEV) % 2 == 0, -1, n_pages * page)  # nothing is written for these
    cache.append_q8(k, v, pages, given)
    there = (given >= 0) & (given < n_pages * page)
    for x, codes, scales in ((k, pages.k, pages.k_scale), (v, pages.v, pages.v_scale)):
        want, scale = quantise(x)
        at, o = slots // page, slots % page
        got, got_scale = values(codes[at, o]), scales[at, o].double()
        assert torch.isnan(got[~there]).all() and torch.isnan(got_scale[~there]).all()
        assert torch.equal(got[there], want[there])
        assert torch.equal(torch.isnan(got_scale[there]), torch.isnan(scale[there]))
        off = (got_scale - scale)[there].abs()
        assert (torch.nan_to_num(off, nan=0.0) <= 2.0 ** -24 * torch.nan_to_num(scale[there], nan=0.0) + 2.0 ** -150).all()
    assert int(torch.isnan(values(pages.k)).all(-1).sum()) == (n_pages * page - int(there.sum())) * kv   # and nothing else was written
    cache.close()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("lens, kv, d, page, heads_first", [
    ([1], 1, 64, 16, True), ([709], 8, 128, 16, False), ([5, 0, 300, 0, 33], 3, 64, 64, True), ([0, 7], 2, 128, 256, False),
    ([40] * 70 + [0, 900], 2, 64, 32, True), ([11, 2, 0], 65, 128, 16, True)])
def test_read_returns_what_codes_and_scales_stand_for(lens, kv, d, page, heads_first, dtype):
    c = Case([1] * len(lens), lens, kv, kv, d, page, dtype, heads_first, seed=5)
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    got = c.cache.read_q8(c.pages, B=len(lens), off=dev(off), T=off[-1])
    for rows, x in zip((c.k, c.v), got):
        codes, scale = quantise(torch.cat(rows))
        assert torch.equal(x, (codes.float() * (scale.float())[..., None]).to(x.dtype))              # code * scale in fp32, rounded once
    c.cache.close()


def test_read_of_parts_other_tables_and_rows_of_nobody():
    c = Case([1, 1, 1], [100, 60, 80], 4, 2, 64, 16, "bf16", seed=6)
    whole = c.cache.read_q8(c.pages, B=3, off=dev([0, 100, 160, 240]), T=240)
    # from a token of its own for each request, uniform
    part = c.cache.read_q8(c.pages, B=3, n=20, start=dev([70, 0, 33]))
    for x, y in zip(part, whole):
        assert torch.equal(x, torch.cat([y[70:90], y[100:120], y[193:213]]))
    # rows before the first offset and behind the last: zeros in rows made here, left alone in rows that are given, strided ones too
    rows = [torch.full((70, 5, 64), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    given = tuple(x[:, 1:3] for x in rows)
    made = c.cache.read_q8(c.pages, B=2, off=dev([10, 30, 60]), T=70)
    c.cache.read_q8(c.pages, B=2, off=dev([10, 30, 60]), T=70, out=given)
    for m, g, r, y in zip(made, given, rows, whole):
        assert torch.equal(m[10:30], y[:20]) and torch.equal(m[30:60], y[100:130])
        assert (m[:10] == 0).all() and (m[60:] == 0).all()
        assert torch.equal(g[10:60], m[10:60]) and (g[:10] == 7).all() and (g[60:] == 7).all() and (r[:, 0] == 7).all() and (r[:, 3:] == 7).all()
    # entries outside the pool, tokens before the first and past the table: zeros
    table = c.cache.block_table[:2].clone()
    table[0, 1], table[0, 2] = -5, 1 << 20
    x = c.cache.read_q8(c.pages, B=2, n=130, block_table=table)[0]
    assert torch.equal(x[:16], whole[0][:16]) and (x[16:48] == 0).all() and torch.equal(x[48:100], whole[0][48:100]) and (x[112:130] == 0).all()
    assert (c.cache.read_q8(c.pages, B=1, n=8, start=dev([-8]))[0] == 0).all()
    c.cache.close()


# ------------------------------------------------------------------------------------------------ attention
SHAPES = {
    # n_new, kv_len, H, kv, d, page, dtype, heads first
    "one token": ([1], [1], 1, 1, 128, 16, "bf16", True),
    "one token, 64": ([1], [129], 4, 4, 64, 16, "fp16", False),
    "window": ([9], [709], 32, 8, 128, 16, "bf16", True),
    "window fp16": ([9], [709], 32, 8, 64, 64, "fp16", False),
    "long": ([1], [20000], 8, 2, 128, 64, "bf16", True),
    "long fp16": ([2], [17001], 16, 1, 128, 128, "fp16", True),
    "ragged": ([5, 17, 1, 0, 16, 9], [300, 2000, 128, 77, 16, 1111], 8, 2, 128, 32, "bf16", False),
    "ragged fp16": ([5, 17, 1, 0, 16, 9], [300, 2000, 128, 77, 16, 1111], 14, 2, 128, 32, "fp16", True),
    "few keys": ([6, 1, 40, 3], [3, 0, 11, 3], 8, 2, 64, 16, "bf16", True),
    "wide group": ([7, 3], [260, 90], 64, 1, 64, 256, "bf16", True),
    "group of 40": ([2, 1, 5], [300, 45, 129], 40, 1, 128, 16, "fp16", True),
    "pairs": ([20, 30], [500, 40], 8, 2, 128, 16, "bf16", True),
    "rows": ([65, 70], [1500, 900], 28, 4, 128, 32, "bf16", True),
    "rows fp16": ([65, 130, 3], [1500, 900, 70], 14, 2, 64, 32, "fp16", False),
    "chunk": ([300, 1], [1000, 40], 8, 2, 128, 64, "bf16", True),
    "chunk fp16": ([515], [777], 8, 1, 128, 128, "fp16", False),
    "chunk of few keys": ([300], [120], 8, 2, 64, 16, "bf16", True),
    "batch": ([1] * 70, list(range(0, 1400, 20)), 16, 4, 128, 16, "bf16", True),
    "a long window among single tokens": ([1] * 40 + [300, 0, 90] + [1] * 50, [30 + 7 * i for i in range(40)] + [1000, 5, 90] + [200] * 50, 8, 2, 128, 16, "bf16", True),
    "a thousand requests": ([1] * 1000, [1 + i % 150 for i in range(1000)], 2, 1, 64, 16, "fp16", True),
    "large batch": ([2] * 300, [64 + i for i in range(300)], 4, 2, 64, 32, "fp16", True),
}


@pytest.mark.parametrize("name", SHAPES)
def test_attend_matches_64_bits(name):
    c = Case(*SHAPES[name], seed=len(name))
    ref = c.reference()
    hints = sorted({1, max(c.n_new), 9, 33, 400})
    for hint in hints:                                             # a hint for the layout of the work, not a limit
        lse = torch.full((c.T, c.q.shape[1]), 5.0, device=DEV)
        out = c.attend(max_new=hint, lse=lse)
        assert c.cache.device_error() == 0
        check(out, lse, ref)
        assert torch.equal(out.view(torch.int16), c.attend(max_new=hint).view(torch.int16))         # (bits: the same every time)
    c.cache.close()


@pytest.mark.parametrize("rows", ["window", "rows", "ragged fp16"])
@pytest.mark.parametrize("spread", [0.0, 1e-3, 8.0, 60.0])
def test_flat_and_peaked_scores(rows, spread):
    c = Case(*SHAPES[rows], seed=2)
    q = (c.q.float() * spread).to(c.q.dtype)
    lse = torch.empty(c.T, q.shape[1], device=DEV)
    out = c.attend(q, lse=lse)
    want, tol, want_lse, ltol = c.reference(q)
    # (scores of hundreds: fp32 sums are off by 2^-22 of their size)
    check(out, lse, (want, tol, want_lse, ltol + want_lse.abs().nan_to_num(posinf=0, neginf=0) * 2.0 ** -20))
    c.cache.close()


@pytest.mark.parametrize("name", ["window", "window fp16", "rows", "chunk fp16"])
def test_growing_scores(name):
    """Keys that grow along the cache: every tile has a new largest score."""
    def edit(c):
        for k in c.k:
            k.copy_((k.float().abs() * torch.linspace(0.05, 1.5, k.shape[0], device=DEV)[:, None, None]).to(k.dtype))
    c = Case(*SHAPES[name], seed=3, edit=edit)
    q = c.q.abs()
    check(c.attend(q), None, c.reference(q))
    c.cache.close()


@pytest.mark.parametrize("name", ["window", "rows"])
@pytest.mark.parametrize("what", ["sink", "zeros", "tiny", "huge", "apart"])
def test_sizes_of_values(name, what):
    """An attention sink without values, heads of zeros, and values at the ends of the type: l and the reference of P must cope."""
    def edit(c):
        for k, v in zip(c.k, c.v):
            if what == "sink":                                     # the first token takes nearly all of the weight and has no values
                k[0] = 3.0
                v[0] = 0.0
            elif what == "zeros":
                v[::3] = 0.0
                v[:200] = 0.0
            elif what == "tiny":
                v.copy_((v.float() * 1e-22).to(v.dtype))
            elif what == "huge":
                v.copy_((v.float() * 1e36).to(v.dtype))
            else:
                v.copy_((v.float() * torch.exp2(torch.randint(-12, 13, v.shape[:2] + (1,), device=DEV, generator=gen(8)).float())).to(v.dtype))
    c = Case(*SHAPES[name], seed=4, edit=edit)
    q = c.q
    if what == "sink":
        q = (q.float().abs() * 0.6).to(q.dtype)
    lse = torch.empty(c.T, q.shape[1], device=DEV)
    check(c.attend(q, lse=lse), lse, c.reference(q))
    c.cache.close()


@pytest.mark.parametrize("name", ["window", "window fp16", "ragged", "rows fp16"])
def test_special_queries_and_tokens_reach_the_rows_that_see_them(name):
    def edit(c):
        c.v[0][-2, 0, 5], c.k[0][-1, -1, 3] = NAN, INF             # seen by the last rows alone
    c = Case(*SHAPES[name], seed=7, edit=edit)
    q = c.q.clone()
    q[0, 0, 1], q[1, -1, 2] = NAN, INF                             # rows of their own
    ref = c.reference(torch.nan_to_num(q, nan=0.0, posinf=0.0))
    want, want_lse = ref[0].clone(), ref[2].clone()
    for t, h in ((0, 0), (1, -1 % q.shape[1])):
        sees = torch.isfinite(want_lse[t, h]) | torch.isnan(want_lse[t, h])
        if sees:
            want[t, h], want_lse[t, h] = NAN, NAN
    assert torch.isnan(want).any() and not torch.isnan(want).all()
    lse = torch.empty(c.T, q.shape[1], device=DEV)
    check(c.attend(q, lse=lse), lse, (want, ref[1], want_lse, ref[3]))
    c.cache.close()


def test_rows_of_very_different_size_share_a_tile():
    c = Case([9], [709], 32, 8, 128, 16, "bf16", seed=9)
    size = torch.exp2(torch.arange(32, device=DEV) % 4 * -2.0)     # heads of a key head 64 times apart
    q = (c.q.float() * size[None, :, None]).to(c.q.dtype)
    check(c.attend(q), None, c.reference(q))
    c.cache.close()


@pytest.mark.parametrize("name", ["window", "rows"])
def test_overflowing_scores_make_their_rows_nan(name):
    def edit(c):
        c.k[0][5] = 3e38
    c = Case(*SHAPES[name], seed=10, edit=edit)
    q = c.q.clone()
    q[:] = 0.0
    q[0] = 3e38                                                    # its score with key 5 is infinite
    out = c.attend(q)
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1:]).all()
    c.cache.close()


def test_outputs_offsets_scale_and_tables_of_the_callers():
    c = Case([9, 4], [300, 77], 8, 2, 64, 16, "bf16", seed=11)
    want = c.attend()
    q = torch.zeros((20, 8, 64), dtype=torch.bfloat16, device=DEV)
    q[3:16] = c.q
    off = dev([3, 12, 16])
    out = torch.full((20, 24, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    got, lse = out[:, 8:16], torch.full((20, 8), 7.0, device=DEV)
    c.cache.attend_q8(q, c.pages, dev(c.kv_len), B=2, max_new=9, q_off=off, out=got, lse=lse)
    assert torch.equal(got[3:16], want) and (out[:3] == 7).all() and (out[16:] == 7).all() and (out[:, :8] == 7).all() and (out[:, 16:] == 7).all()
    assert (lse[:3] == 7).all() and (lse[16:] == 7).all() and torch.isfinite(lse[3:16]).all()
    made = c.cache.attend_q8(q, c.pages, dev(c.kv_len), B=2, max_new=9, q_off=off)
    assert torch.equal(made[3:16], want) and (made[:3] == 0).all() and (made[16:] == 0).all()
    c.cache.attend_q8(q, c.pages, dev(c.kv_len), B=2, max_new=9, q_off=off, out=got, lse=lse, clear_rest=True)
    assert (got[:3] == 0).all() and torch.isneginf(lse[:3]).all() and torch.isneginf(lse[16:]).all()
    # queries cut out of a fused projection, another table, another scale
    fused = torch.zeros((13, 12, 64), dtype=torch.bfloat16, device=DEV)
    fused[:, :8] = c.q
    table = torch.full((5, 40), 1 << 28, dtype=torch.int32, device=DEV)
    table[:2, :c.cache.max_blocks] = c.cache.block_table
    lse2 = torch.empty((13, 8), device=DEV)
    check(c.attend(fused[:, :8], block_table=table, scale=0.31, lse=lse2), lse2, c.reference(scale=0.31))
    # pages that are not there read as zeros: weight, but no value
    table[0, 2] = -1
    gone = c.attend(block_table=table)
    k, v, (n, L) = c.k[0].clone(), c.v[0].clone(), (9, 300)
    c.k[0][32:48], c.v[0][32:48] = 0.0, 0.0
    check(gone, None, c.reference())
    # uniform windows need no offsets
    u = Case([4, 4], [90, 20], 8, 2, 64, 16, "bf16", seed=12)
    assert torch.equal(u.attend(), u.cache.attend_q8(u.q, u.pages, dev(u.kv_len), B=2, max_new=4))
    c.cache.close()
    u.cache.close()


def test_other_streams_and_graphs():
    cases = [Case(*SHAPES[n], seed=13) for n in ("ragged", "rows", "batch")]
    stream = torch.cuda.Stream()
    for c in cases:
        want = c.attend()
        q_off, kv_len = dev(c.off), dev(c.kv_len)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            assert torch.equal(c.attend(), want)
        graph, out, kv = torch.cuda.CUDAGraph(), torch.zeros_like(want), [torch.empty((c.T, c.k[0].shape[1], c.q.shape[2]), dtype=c.q.dtype, device=DEV) for _ in range(2)]
        call = dict(B=len(c.n_new), max_new=max(c.n_new), q_off=q_off, out=out)
        c.cache.attend_q8(c.q, c.pages, kv_len, stream=stream, **call)
        with torch.cuda.graph(graph, stream=stream):
            c.cache.attend_q8(c.q, c.pages, kv_len, **call)
            c.cache.read_q8(c.pages, B=len(c.n_new), off=q_off, T=c.T, out=tuple(kv))
        for lengths in (c.kv_len, [max(n - 3, 0) for n in c.kv_len]):
            kv_len.copy_(dev(lengths))                             # lengths live on the device: the graph stays as it is
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, c.attend() if lengths is c.kv_len else c.cache.attend_q8(c.q, c.pages, kv_len, B=len(c.n_new), max_new=max(c.n_new), q_off=q_off))
        c.cache.close()


def test_stale_workspace_does_not_matter_and_16_bit_calls_share_it():
    c = Case([9, 30], [3000, 900], 8, 2, 128, 16, "bf16", seed=14)
    want = c.attend()
    n = c.cache.n_pages
    kp, vp = (normal(gen(i), n, 16, 2, 128).bfloat16() for i in (1, 2))
    sixteen = c.cache.attend(c.q, kp, vp, dev(c.kv_len), B=2, max_new=30, q_off=dev(c.off))
    for _ in range(3):                                             # one after the other on one workspace
        assert torch.equal(c.attend(), want)
        assert torch.equal(c.cache.attend(c.q, kp, vp, dev(c.kv_len), B=2, max_new=30, q_off=dev(c.off)), sixteen)
    counters = 256 + 4 * torch.cuda.get_device_properties(0).multi_processor_count
    c.cache._workspace[(counters + 255) // 256 * 256:].view(torch.float32).fill_(NAN)
    assert torch.equal(c.attend(), want)
    c.cache.close()


def test_pools_past_four_gigabytes():
    c = wisv.PagedCache(n_heads=8, n_kv_heads=8, head_dim=128, page_size=256, n_pages=17000, max_requests=1, max_blocks=4)
    pages = c.quant_pages()                                        # 4.46 GB of codes each
    c.block_table[0, :2] = dev([16999, 16500])
    k, v = (normal(gen(i), 300, 8, 128).bfloat16() for i in (3, 4))
    i = torch.arange(300, device=DEV)
    c.append_q8(k, v, pages, c.block_table[0].long()[i // 256] * 256 + i % 256)
    got = c.read_q8(pages, B=1, n=300)
    for x, y in zip((k, v), got):
        codes, scale = quantise(x)
        assert torch.equal(y, (codes.float() * scale.float()[..., None]).bfloat16())
    q = normal(gen(5), 2, 8, 128).bfloat16()
    out = c.attend_q8(q, pages, dev([300]), B=1, max_new=2).double()
    K, V = (x.double() for x in got)
    s = torch.einsum("nhd,lhd->nhl", q.double(), K) * 128 ** -0.5
    s[0, :, 299] = -INF
    assert (out - torch.einsum("nhl,lhd->nhd", torch.softmax(s, -1), V)).abs().max() < 0.02
    c.close()


# ------------------------------------------------------------------------------------------------ failures and refusals
@pytest.mark.parametrize("name", ["window", "ragged", "pairs", "rows", "chunk fp16"])
def test_waits_give_up_and_later_calls_are_right(name):
    """(Block 0 always has key tiles: the line of work starts with those of the first item.  Others may have none: an item of 6 tiles weighs 14 units,
    and a block's 2 units may be among the 8 behind the tiles.)"""
    c, block = Case(*SHAPES[name], seed=15), 0
    first, other = c.attend(), c.attend(c.q * -2)
    assert c.cache.device_error() == 0
    for read in (True, False):
        c.cache.debug_waits(2_000_000, block)                      # about 1 ms; this block gets no values
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        c.attend()
        end.record()
        if read:
            assert c.cache.device_error() == 1 and c.cache.device_error() == 0
        c.cache.debug_waits()
        assert torch.equal(c.attend(), first) and torch.equal(c.attend(c.q * -2), other)
        end.synchronize()
        assert begin.elapsed_time(end) < 500
    assert c.cache.device_error() == 1                             # the unread one
    c.cache.close()


def test_refusals():
    c = Case([2], [40], 8, 2, 64, 16, "bf16", seed=16)
    cache, pages, kv_len = c.cache, c.pages, dev([40])
    other = wisv.PagedCache(n_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=9, max_requests=1, max_blocks=4)
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device=DEV)
    slots = torch.arange(4, device=DEV)
    good = dict(B=1, max_new=2)
    for call in (lambda: cache.attend_q8(c.q, other.quant_pages(), kv_len, **good), lambda: cache.attend_q8(c.q.half(), pages, kv_len, **good),
                 lambda: cache.attend_q8(c.q[:, :7], pages, kv_len, **good), lambda: cache.attend_q8(c.q, pages, kv_len.long(), **good),
                 lambda: cache.attend_q8(c.q, pages, kv_len, scale=-1.0, **good), lambda: cache.attend_q8(c.q, pages, kv_len, lse=torch.empty(2, 8), **good),
                 lambda: cache.attend_q8(c.q, pages, kv_len, block_table=torch.zeros((1, 4), device=DEV), **good),
                 lambda: cache.append_q8(k, k[:3], pages, slots), lambda: cache.append_q8(k.float(), k, pages, slots),
                 lambda: cache.append_q8(k, k, pages, slots.int()), lambda: cache.append_q8(k, k, other.quant_pages(), slots),
                 lambda: cache.read_q8(pages, B=1), lambda: cache.read_q8(pages, B=1, off=dev([0, 4])),
                 lambda: cache.read_q8(pages, B=1, n=4, out=(k, k[:3])), lambda: cache.read_q8(pages, B=1, n=4, start=torch.zeros(1, device=DEV)),
                 lambda: wisv.QuantPages(pages.k.view(torch.uint8), pages.v, pages.k_scale, pages.v_scale),
                 lambda: wisv.QuantPages(pages.k, pages.v[:1], pages.k_scale, pages.v_scale),
                 lambda: wisv.QuantPages(pages.k, pages.v, pages.k_scale.contiguous(), pages.v_scale),
                 lambda: wisv.QuantPages(pages.k, pages.v, pages.k_scale, pages.v_scale.double())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(AttributeError):
        pages.k = pages.v                                          # the addresses are taken once
    for call, code in ((lambda: cache.attend_q8(c.q, pages, kv_len, B=1, max_new=3), -2), (lambda: cache.attend_q8(c.q, pages, dev([40, 1]), B=2, max_new=1), -4),
                       (lambda: cache.read_q8(pages, B=2, n=2), -4), (lambda: cache.read_q8(pages, B=1, n=2, T=3), -2),
                       (lambda: cache.attend_q8(torch.zeros(2 * 8 * 64 + 4, dtype=torch.bfloat16, device=DEV)[4:].view(2, 8, 64), pages, kv_len, **good), -3),
                       (lambda: cache.append_q8(torch.zeros((4, 2, 68), dtype=torch.bfloat16, device=DEV)[:, :, :64], k, pages, slots), -3)):
        with pytest.raises(wisv.WisvError) as e:
            call()
        assert e.value.code == code
    # pools whose pieces are not 16-byte aligned
    n = cache.n_pages
    raw = torch.zeros(n * 16 * 2 * 72, dtype=torch.uint8, device=DEV).view(E4M3).view(n, 16, 2, 72)[..., :64]
    loose = torch.zeros((n, 2, 18), device=DEV)[..., :16].transpose(1, 2)
    for bad in (wisv.QuantPages(raw, pages.v, pages.k_scale, pages.v_scale), wisv.QuantPages(pages.k, pages.v, loose, pages.v_scale)):
        for call in (lambda: cache.append_q8(k, k, bad, slots), lambda: cache.read_q8(bad, B=1, n=4), lambda: cache.attend_q8(c.q, bad, kv_len, **good)):
            with pytest.raises(wisv.WisvError) as e:
                call()
            assert e.value.code == -3
    assert cache.attend_q8(c.q[:0], pages, kv_len, B=1, max_new=1, q_off=dev([0, 0])).shape == (0, 8, 64)         # nothing to do
    assert cache.read_q8(pages, B=1, n=0)[0].shape == (0, 2, 64)
    cache.append_q8(k[:0], k[:0], pages, slots[:0])
    assert cache.device_error() == 0 and not math.isnan(float(c.attend().float().sum()))
    cache.close()
    other.close()
