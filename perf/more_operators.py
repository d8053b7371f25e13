"""Workloads of the operators of a paged cache held in 8 bits, with their plain forms.

Keys and values are kept as e4m3 codes with one 32-bit scale for each token and key head, half the bytes of a 16-bit cache:

* ``append``  the new keys and values of one layer, quantised as they are written into their slots;
* ``read``    tokens of the cache as 16-bit rows again (a prefix that is handed on, or used at full width);
* ``attend``  attention of every request's new tokens over the codes (causal among the new tokens), from one token per
              request to prompt chunks.

``run`` computes them with elementary torch operations (``own = False``) or through the package (``own = True``).
"""
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TOP = 448.0                     # the largest e4m3 number
E4M3 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one window's keys and values, cut out of a fused q/k/v projection: only latency counts
        dict(name="append_b1_k8", op="append", T=9, kv=8, q=32, d=128, dtype="bf16", page=16, pages=512, fused=True,
             heads_first=True),
        # the windows of 512 requests at head size 64
        dict(name="append_b512_d64", op="append", T=5633, kv=8, q=32, d=64, dtype="fp16", page=16, pages=4096, fused=True,
             heads_first=False),
        # a prompt chunk's keys and values, projections kept apart
        dict(name="append_chunk_8k", op="append", T=8192, kv=8, q=32, d=128, dtype="bf16", page=64, pages=1024, fused=False,
             heads_first=True),
        # one request's prefix read back
        dict(name="read_b1", op="read", B=1, lo=709, hi=709, kv=8, q=32, d=128, dtype="bf16", page=16, heads_first=True),
        # the prefixes of 64 requests, of ragged lengths
        dict(name="read_b64_ragged", op="read", B=64, lo=200, hi=4100, kv=8, q=32, d=128, dtype="fp16", page=16,
             heads_first=False),
        # one request at the 8B shape, K = 8: the smallest call
        dict(name="attend_b1_k8", op="attend", B=1, n_lo=9, n_hi=9, len_lo=700, len_hi=700, q=32, kv=8, d=128, page=16,
             dtype="bf16", heads_first=True),
        # one token over one long context: the work has to be cut along the cache
        dict(name="attend_b1_long", op="attend", B=1, n_lo=1, n_hi=1, len_lo=131071, len_hi=131071, q=32, kv=8, d=128, page=64,
             dtype="bf16", heads_first=True),
        # plain decoding of 64 requests, one token each (the round after a full rejection)
        dict(name="attend_b64_decode", op="attend", B=64, n_lo=1, n_hi=1, len_lo=65, len_hi=16000, q=32, kv=8, d=128, page=64,
             dtype="fp16", heads_first=True),
        # a verification batch of ragged windows at the 8B shape, token-major pages
        dict(name="attend_b64_ragged", op="attend", B=64, n_lo=5, n_hi=17, len_lo=200, len_hi=8200, q=32, kv=8, d=128, page=16,
             dtype="bf16", heads_first=False),
        # windows of 64 drafts, 7 query heads to a key head, long contexts
        dict(name="attend_b8_k64_long", op="attend", B=8, n_lo=65, n_hi=65, len_lo=9001, len_hi=20001, q=28, kv=4, d=128,
             page=32, dtype="bf16", heads_first=True),
        # windows at head size 64
        dict(name="attend_b48_d64", op="attend", B=48, n_lo=3, n_hi=9, len_lo=33, len_hi=9000, q=32, kv=8, d=64, page=32,
             dtype="fp16", heads_first=True),
        # two prompt chunks of 2048 tokens on top of a cached prefix: bound by the tensor cores
        dict(name="attend_chunk_2k", op="attend", B=2, n_lo=2048, n_hi=2048, len_lo=6000, len_hi=8192, q=32, kv=8, d=128,
             page=64, dtype="bf16", heads_first=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng: random.Random):
    op = rng.choice(["append", "read", "attend", "attend", "attend"])
    kv = rng.choice([2, 4, 8])
    both = dict(kv=kv, q=kv * rng.choice([1, 4, 7] if kv < 8 else [1, 4]), d=rng.choice([64, 128, 128]),
                page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "fp16"]), heads_first=rng.random() < 0.6)
    if op == "append":
        T = _log_int(rng, 1, 8192)
        return dict(both, op=op, T=T, pages=T // both["page"] + rng.randint(1, 99), fused=rng.random() < 0.5)
    if op == "read":
        B = _log_int(rng, 1, 64)
        hi = _log_int(rng, 40, min(20000, 130000 // B))
        return dict(both, op=op, B=B, lo=rng.randint(0, hi), hi=hi)
    chunk = rng.random() < 0.25
    B = _log_int(rng, 1, 3) if chunk else _log_int(rng, 1, 64)
    hi = _log_int(rng, 40, min(40000, 500000 // B))
    n_hi = min(hi, _log_int(rng, 100, max(101, min(2048, 28000000 // (B * hi)))) if chunk else _log_int(rng, 1, 65))
    return dict(both, op=op, B=B, n_lo=rng.randint(max(1, n_hi // 4), n_hi), n_hi=n_hi, len_lo=rng.randint(0, hi), len_hi=hi)


# ------------------------------------------------------------------------------------------------ inputs
def _spread(lo, hi, B, seed):
    """B whole numbers spread evenly over [lo, hi], in an order that the seed decides (their sum does not depend on it)."""
    v = lo + (np.arange(B) * 2 + 1) * (hi - lo + 1) // (2 * B)
    return np.random.default_rng(seed).permutation(np.minimum(v, hi)).astype(np.int32)


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _tables(lens, page, width, n_pages, seed):
    """A block table for requests of these lengths over shuffled pages."""
    perm = np.random.default_rng(seed + 1).permutation(n_pages).astype(np.int32)
    need = (lens.astype(np.int64) + page - 1) // page
    held = np.arange(width)[None] < need[:, None]
    table = np.full((len(lens), width), -1, np.int32)
    table[held] = perm[:int(need.sum())]
    return table


def _rows(g, shape, dtype):
    """Keys or values as a projection leaves them: every token and head has a size of its own."""
    x = torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)
    return x.mul_(torch.empty(shape[:-1] + (1,), dtype=dtype, device=DEV).normal_(std=0.4, generator=g).exp_())


def _quantise(x):
    """The e4m3 codes and the scales of rows x [..., d]: scale = max|x| / 448, codes = x / scale rounded to the nearest number, ties
    to even (the quotients in 64 bits, since those of 16-bit numbers lie next to a border or on it); a row with an infinite
    element or NaN has the scale NaN and codes of 0."""
    top = x.abs().amax(-1, keepdim=True).double()
    fine = torch.isfinite(top)
    y = torch.where(fine & (top > 0), x.double() * TOP / top, 0.0)
    return y.float().to(E4M3), torch.where(fine, top.float() / TOP, float("nan"))[..., 0]


def _pool(g, n_pages, c):
    """Codes [n_pages, page, kv, d] and scales [n_pages, page, kv] of random keys or values, in the case's layout."""
    x = _rows(g, (n_pages, c["kv"], c["page"], c["d"]), DTYPES[c["dtype"]])
    top = x.abs().amax(-1, keepdim=True).float()
    codes = (x.float() * (TOP / top)).clamp(-TOP, TOP).to(E4M3).transpose(1, 2)
    scales = (top / TOP)[..., 0].transpose(1, 2)
    return codes if c["heads_first"] else codes.contiguous(), scales


def _empty_pool(c):
    shape = (c["pages"], c["kv"], c["page"], c["d"])
    codes = torch.zeros(shape, device=DEV).to(E4M3).transpose(1, 2)
    return codes if c["heads_first"] else codes.contiguous(), torch.zeros(shape[:3], device=DEV).transpose(1, 2)


def _cache(**kw):
    import paper_2604_17701_b200 as wisv
    names = {"bf16": wisv.DT_BF16, "fp16": wisv.DT_F16}
    return wisv.PagedCache(**{**kw, "dtype": names[kw["dtype"]], "device": DEV})


def _quant_pages(s):
    import paper_2604_17701_b200 as wisv
    return wisv.QuantPages(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"])


def prepare(case, seed):
    return {"append": _prepare_append, "read": _prepare_read, "attend": _prepare_attend}[case["op"]](case, seed)


def _prepare_append(c, seed):
    g, T, dt = _gen(seed), c["T"], DTYPES[c["dtype"]]
    rows = _rows(g, (T, c["q"] + 2 * c["kv"], c["d"]), dt)
    k, v = rows[:, c["q"]:c["q"] + c["kv"]], rows[:, c["q"] + c["kv"]:]
    if not c["fused"]:
        k, v = k.contiguous(), v.contiguous()
    # runs of up to a page, as requests have them, on shuffled pages
    order = np.random.default_rng(seed).permutation(c["pages"])
    slots = (order[:, None].astype(np.int64) * c["page"] + np.arange(c["page"])).reshape(-1)[:T]
    (kc, ks), (vc, vs) = _empty_pool(c), _empty_pool(c)
    s = dict(case=c, k=k, v=v, k_codes=kc, k_scale=ks, v_codes=vc, v_scale=vs, slot_map=_dev(slots, torch.int64))
    if own:
        s["cache"] = _cache(n_heads=c["q"], n_kv_heads=c["kv"], head_dim=c["d"], page_size=c["page"], n_pages=c["pages"],
                            max_requests=1, max_blocks=c["pages"], dtype=c["dtype"])
        s["pages"] = _quant_pages(s)
    return s


def _filled(c, seed, lens):
    """A cache of requests of these lengths: its block table and pools."""
    g, width = _gen(seed), max(1, -(-int(lens.max()) // c["page"]))
    n_pages = int(((lens.astype(np.int64) + c["page"] - 1) // c["page"]).sum()) + 3
    (kc, ks), (vc, vs) = _pool(g, n_pages, c), _pool(g, n_pages, c)
    s = dict(case=c, k_codes=kc, k_scale=ks, v_codes=vc, v_scale=vs, max_len=int(lens.max()),
             block_table=_dev(_tables(lens, c["page"], width, n_pages, seed)))
    if own:
        s["cache"] = cache = _cache(n_heads=c["q"], n_kv_heads=c["kv"], head_dim=c["d"], page_size=c["page"], n_pages=n_pages,
                                    max_requests=c["B"], max_blocks=width, dtype=c["dtype"])
        cache.block_table.copy_(s["block_table"])
        s["pages"] = _quant_pages(s)
    return s


def _prepare_read(c, seed):
    lens = _spread(c["lo"], c["hi"], c["B"], seed)
    off = np.concatenate([[0], np.cumsum(lens)])
    return dict(_filled(c, seed, lens), T=int(off[-1]), off=_dev(off))


def _attend_lengths(c, seed):
    n_new = _spread(c["n_lo"], c["n_hi"], c["B"], seed + 7)
    return n_new, _spread(c["len_lo"], c["len_hi"], c["B"], seed) + n_new


def _prepare_attend(c, seed):
    n_new, kv_len = _attend_lengths(c, seed)
    q_off = np.concatenate([[0], np.cumsum(n_new)])
    T = int(q_off[-1])
    # queries as the projection leaves them: the first heads of a fused q/k/v row
    qkv = torch.empty((T, c["q"] + 2 * c["kv"], c["d"]), dtype=DTYPES[c["dtype"]], device=DEV).normal_(generator=_gen(seed + 1))
    return dict(_filled(c, seed, kv_len), T=T, max_new=int(n_new.max()), q=qkv[:, :c["q"]], kv_len=_dev(kv_len), q_off=_dev(q_off))


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"append": _run_append, "read": _run_read, "attend": _run_attend}[s["case"]["op"]](s)


def _run_append(s):
    if own:
        s["cache"].append_q8(s["k"], s["v"], s["pages"], s["slot_map"])
    else:
        page, slot = s["case"]["page"], s["slot_map"]
        at, off = slot // page, slot % page
        kc, ks = _quantise(s["k"])
        vc, vs = _quantise(s["v"])
        s["k_codes"].view(torch.uint8)[at, off] = kc.view(torch.uint8)
        s["v_codes"].view(torch.uint8)[at, off] = vc.view(torch.uint8)
        s["k_scale"][at, off] = ks
        s["v_scale"][at, off] = vs
    return dict(k_codes=s["k_codes"], v_codes=s["v_codes"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def _run_read(s):
    c = s["case"]
    if own:
        return s["cache"].read_q8(s["pages"], B=c["B"], off=s["off"], T=s["T"])
    off, t = s["off"].long(), torch.arange(s["T"], device=DEV)
    b = torch.searchsorted(off, t, right=True) - 1
    i = t - off[b]
    at, i = s["block_table"][b, i // c["page"]].long(), i % c["page"]
    dt = DTYPES[c["dtype"]]
    return ((s["k_codes"].view(torch.uint8)[at, i].view(E4M3).float() * s["k_scale"][at, i][..., None]).to(dt),
            (s["v_codes"].view(torch.uint8)[at, i].view(E4M3).float() * s["v_scale"][at, i][..., None]).to(dt))


def _run_attend(s):
    c = s["case"]
    if own:
        return s["cache"].attend_q8(s["q"], s["pages"], s["kv_len"], B=c["B"], max_new=s["max_new"], q_off=s["q_off"])
    B, n, L, kv, G, d = c["B"], s["max_new"], s["max_len"], c["kv"], c["q"] // c["kv"], c["d"]
    pages = s["block_table"].clamp(min=0).long()
    length = s["kv_len"][:, None]
    here = (torch.arange(L, device=DEV)[None] < length)[:, :, None, None]
    k = (s["k_codes"].view(torch.uint8)[pages].view(E4M3).float() * s["k_scale"][pages][..., None]).reshape(B, -1, kv, d)[:, :L]
    v = (s["v_codes"].view(torch.uint8)[pages].view(E4M3).float() * s["v_scale"][pages][..., None]).reshape(B, -1, kv, d)[:, :L]
    v = torch.where(here, v, 0.0)
    off = s["q_off"].long()
    new = off[1:] - off[:-1]
    i = torch.arange(n, device=DEV)
    at = (off[:-1, None] + i).clamp(max=s["T"] - 1)
    q = s["q"][at].float().reshape(B, n, kv, G, d).permute(0, 2, 3, 1, 4).reshape(B, kv, G * n, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(d ** -0.5).reshape(B, kv, G, n, L)
    last = length - new[:, None] + i                                       # the last key that row i sees
    score.masked_fill_((torch.arange(L, device=DEV) > last[:, :, None])[:, None, None], float("-inf"))
    score.sub_(score.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.reshape(B, kv, G * n, L), v.permute(0, 2, 1, 3)).reshape(B, kv, G, n, d)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, n, kv * G, d)
    return out[(i[None] < new[:, None])].to(DTYPES[c["dtype"]])


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(c):
    row = c["kv"] * (2 * c["d"] + 8)                                       # codes and scales of one token's keys and values
    if c["op"] == "append":
        return {"bytes": c["T"] * (c["kv"] * c["d"] * 4 + row + 8), "flops": 0}
    if c["op"] == "read":
        return {"bytes": float(_spread(c["lo"], c["hi"], c["B"], 0).sum()) * (row + c["kv"] * c["d"] * 4), "flops": 0}
    n_new = _spread(c["n_lo"], c["n_hi"], c["B"], 7).astype(np.int64)
    lens = _spread(c["len_lo"], c["len_hi"], c["B"], 0).astype(np.int64)
    new, kept, B = float(n_new.sum()), float(lens.sum()), c["B"]
    seen = new / B * kept + float((n_new * (n_new + 1) // 2).sum())        # keys that the query rows of one head see
    return {"bytes": (kept + new) * row + new * c["q"] * c["d"] * 4, "flops": 4.0 * seen * c["q"] * c["d"]}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    if case["op"] == "append":
        s, out = _prepare_append(case, seed), {}
        page, slot = case["page"], s["slot_map"]
        for name in ("k", "v"):
            x = s[name].double()
            top = x.abs().amax(-1)
            scale = top / 448
            y = x * 448 / torch.where(top > 0, top, 1.0)[..., None]
            # steps of an eighth of the power of two below, of 2^-9 under 2^-6
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
            codes = s[name + "_codes"].float().double()
            codes[slot // page, slot % page] = (torch.round(y / step) * step).clamp(-448, 448)
            scales = s[name + "_scale"].double()
            scales[slot // page, slot % page] = scale
            out[name + "_codes"], out[name + "_scale"] = codes, scales
        return dict(k_codes=out["k_codes"], v_codes=out["v_codes"], k_scale=out["k_scale"], v_scale=out["v_scale"])
    s = (_prepare_read if case["op"] == "read" else _prepare_attend)(case, seed)
    table = s["block_table"].cpu().numpy().astype(np.int64)
    page, kv, d = case["page"], case["kv"], case["d"]

    def tokens(b, n):
        """The first n keys and values of a request in 64 bits, [n, kv, d]."""
        pages = _dev(table[b], torch.int64)[:-(-n // page)]
        both = []
        for name in ("k", "v"):
            codes = s[name + "_codes"].view(torch.uint8)[pages].view(E4M3).float().double()
            both.append((codes * s[name + "_scale"][pages].double()[..., None]).reshape(-1, kv, d)[:n])
        return both

    if case["op"] == "read":
        off = s["off"].tolist()
        got = [tokens(b, off[b + 1] - off[b]) for b in range(case["B"])]
        return torch.cat([k for k, _ in got]), torch.cat([v for _, v in got])
    n_new, kv_len = _attend_lengths(case, seed)
    out, at = [], 0
    for b in range(case["B"]):
        n, L = int(n_new[b]), int(kv_len[b])
        k, v = tokens(b, L)
        hide = torch.arange(L, device=DEV)[None] > (L - n + torch.arange(n, device=DEV))[:, None]
        heads = []
        for h in range(case["q"]):
            g = h // (case["q"] // kv)
            x = s["q"][at:at + n, h].double() @ k[:, g].T / float(d) ** 0.5
            heads.append(torch.softmax(x.masked_fill(hide, float("-inf")), 1) @ v[:, g])
        out.append(torch.stack(heads, 1))
        at += n
    return torch.cat(out)
