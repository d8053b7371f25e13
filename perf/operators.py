"""Workloads of the paged-cache and residual-verification operators, with their plain forms.

Four operators serve the part of a verification round that surrounds the LM head:

* ``pages``   block tables and slot maps of a round built from request lengths, and the return of the pages that
              the round did not keep;
* ``append``  the new keys and values of one layer written into the paged cache;
* ``attend``  attention of every request's new tokens over its paged cache (causal among the new tokens);
* ``residual`` verification of drafted tokens against the target's probabilities with given random numbers, and the
              draw of the correction (or bonus) token from the residual distribution.

``run`` computes them with elementary torch operations (``own = False``) or through the package (``own = True``).
"""
import random

import numpy as np
import torch

own = False

DEV = "cuda"
FIX = float(1 << 44)            # the residual draw adds weights in units of 2^-44
NO_PAGES = 32                   # status bit of a request whose pages could not be had
NO_MASS = 64                    # status bit of a request whose distribution has no weight
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one request, a window of 8 drafts and its bonus row: the round's bookkeeping where only latency counts
        dict(name="pages_b1_k8", op="pages", B=1, n_lo=9, n_hi=9, len_lo=700, len_hi=700, page=16, width=64, spare=64),
        # the largest verification batch, windows of 4 to 16 drafts, contexts up to 8 k tokens
        dict(name="pages_b512_ragged", op="pages", B=512, n_lo=5, n_hi=17, len_lo=1, len_hi=8000, page=16, width=512,
             spare=2000),
        # one window's keys and values, cut out of a fused q/k/v projection
        dict(name="append_b1_k8", op="append", T=9, kv=8, q=32, d=128, dtype="bf16", page=16, pages=512, fused=True),
        # a prompt chunk's keys and values, projections kept apart
        dict(name="append_chunk_8k", op="append", T=8192, kv=8, q=32, d=128, dtype="bf16", page=64, pages=1024,
             fused=False),
        # one request at the 8B shape, K = 8: the smallest call
        dict(name="attend_b1_k8", op="attend", B=1, n_lo=9, n_hi=9, len_lo=700, len_hi=700, q=32, kv=8, d=128, page=16,
             dtype="bf16", heads_first=False),
        # plain decoding of 64 requests, one token each (the round after a full rejection)
        dict(name="attend_b64_decode", op="attend", B=64, n_lo=1, n_hi=1, len_lo=65, len_hi=8000, q=32, kv=8, d=128,
             page=64, dtype="fp16", heads_first=True),
        # a verification batch of ragged windows at the 8B shape
        dict(name="attend_b64_ragged", op="attend", B=64, n_lo=5, n_hi=17, len_lo=200, len_hi=4100, q=32, kv=8, d=128,
             page=16, dtype="bf16", heads_first=False),
        # windows of 64 drafts, 7 query heads to a key head, long contexts
        dict(name="attend_b8_k64_long", op="attend", B=8, n_lo=65, n_hi=65, len_lo=9001, len_hi=20001, q=28, kv=4, d=128,
             page=32, dtype="bf16", heads_first=False),
        # two prompt chunks of 2048 tokens on top of a cached prefix: bound by the tensor cores
        dict(name="attend_chunk_2k", op="attend", B=2, n_lo=2048, n_hi=2048, len_lo=6000, len_hi=8192, q=32, kv=8, d=128,
             page=64, dtype="bf16", heads_first=False),
        # one request, K = 8, the drafter's whole distribution uploaded in 32 bits
        dict(name="residual_b1_k8", op="residual", B=1, k_lo=8, k_hi=8, V=128256, dtype="fp32", draft="dense", top=0),
        # 64 requests, 16-bit distributions
        dict(name="residual_b64_k8", op="residual", B=64, k_lo=8, k_hi=8, V=128256, dtype="bf16", draft="dense", top=0),
        # the largest batch; the drafters upload only their 64 likeliest tokens over the wireless link
        dict(name="residual_b512_top64", op="residual", B=512, k_lo=4, k_hi=16, V=152064, dtype="bf16", draft="top", top=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["pages", "append", "attend", "attend", "residual"])
    if op == "pages":
        page = rng.choice([16, 32, 64, 128])
        hi = _log_int(rng, 20, 8000)
        n_hi = _log_int(rng, 1, 17)
        B = _log_int(rng, 1, 512)
        return dict(op=op, B=B, n_lo=rng.randint(1, n_hi), n_hi=n_hi, len_lo=rng.randint(0, hi), len_hi=hi, page=page,
                    width=(hi + n_hi + page - 1) // page + rng.randint(0, 9), spare=B * (n_hi // page + 1) + rng.randint(0, 99))
    if op == "append":
        kv = rng.choice([2, 4, 8])
        page = rng.choice([16, 32, 64, 128])
        T = _log_int(rng, 1, 8192)
        return dict(op=op, T=T, kv=kv, q=kv * rng.choice([1, 4, 7]), d=rng.choice([64, 128]),
                    dtype=rng.choice(["bf16", "fp16"]), page=page, pages=T // page + rng.randint(1, 99),
                    fused=rng.random() < 0.5)
    if op == "attend":
        kv = rng.choice([2, 4, 8])
        chunk = rng.random() < 0.25
        B = _log_int(rng, 1, 3) if chunk else _log_int(rng, 1, 64)
        hi = _log_int(rng, 40, min(20000, 250000 // B))
        n_hi = min(hi, _log_int(rng, 100, max(101, min(2048, 28000000 // (B * hi)))) if chunk else _log_int(rng, 1, 65))
        return dict(op=op, B=B, n_lo=rng.randint(max(1, n_hi // 4), n_hi), n_hi=n_hi, len_lo=rng.randint(0, hi), len_hi=hi,
                    q=kv * rng.choice([1, 4, 7] if kv < 8 else [1, 4]), kv=kv, d=rng.choice([64, 128, 128]),
                    page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "fp16"]),
                    heads_first=rng.random() < 0.5)
    draft = rng.choice(["dense", "top", "none"])
    k_hi = _log_int(rng, 1, 17)
    V = rng.choice([128256, 152064, 32000 + rng.randint(0, 999), 100000 + rng.randint(0, 9999)])
    return dict(op=op, B=_log_int(rng, 1, 64 if draft == "dense" else 200), k_lo=rng.randint(1, k_hi), k_hi=k_hi, V=V,
                dtype=rng.choice(["fp32", "bf16", "fp16"]), draft=draft, top=_log_int(rng, 4, 128) if draft == "top" else 0)


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
    """A block table for requests of these lengths over shuffled pages, and the pages left over."""
    perm = np.random.default_rng(seed + 1).permutation(n_pages).astype(np.int32)
    need = (lens.astype(np.int64) + page - 1) // page
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, c in enumerate(need):
        table[b, :c] = perm[at:at + c]
        at += c
    return table, need.astype(np.int32), perm[at:]


def prepare(case, seed):
    return {"pages": _prepare_pages, "append": _prepare_append, "attend": _prepare_attend,
            "residual": _prepare_residual}[case["op"]](case, seed)


def _cache(**kw):
    import paper_2604_17701_b200 as wisv
    names = {"bf16": wisv.DT_BF16, "fp16": wisv.DT_F16}
    return wisv.PagedCache(**{**kw, "dtype": names[kw["dtype"]], "device": DEV})


def _prepare_pages(c, seed):
    lens, n_new = _spread(c["len_lo"], c["len_hi"], c["B"], seed), _spread(c["n_lo"], c["n_hi"], c["B"], seed + 7)
    held = int(((lens.astype(np.int64) + c["page"] - 1) // c["page"]).sum())
    n_pages = held + c["spare"]
    width = max(c["width"], -(-(int(lens.max()) + int(n_new.max())) // c["page"]))
    table, n_blocks, free = _tables(lens, c["page"], width, n_pages, seed)
    free_list = np.full(n_pages, -1, np.int32)
    free_list[:len(free)] = free
    s = dict(case=c, T=int(n_new.sum()), n_new=_dev(n_new), block_table=_dev(table), n_blocks=_dev(n_blocks),
             free_list=_dev(free_list), n_free=_dev(np.array([len(free)])), seq_len=_dev(lens), keep=_dev(lens))
    if own:
        s["cache"] = cache = _cache(n_heads=8, n_kv_heads=8, head_dim=128, page_size=c["page"], n_pages=n_pages,
                                    max_requests=c["B"], max_blocks=width, dtype="bf16")
        for k in ("block_table", "n_blocks", "free_list", "n_free", "seq_len"):
            getattr(cache, k).copy_(s[k])
    return s


def _prepare_append(c, seed):
    g, T, dt = _gen(seed), c["T"], DTYPES[c["dtype"]]
    rows = torch.randn((T, c["q"] + 2 * c["kv"], c["d"]), generator=g, device=DEV, dtype=torch.float32).to(dt)
    k, v = rows[:, c["q"]:c["q"] + c["kv"]], rows[:, c["q"] + c["kv"]:]
    if not c["fused"]:
        k, v = k.contiguous(), v.contiguous()
    shape = (c["pages"], c["page"], c["kv"], c["d"])
    # runs of up to a page, as requests have them, on shuffled pages
    order = np.random.default_rng(seed).permutation(c["pages"])
    slots = (order[:, None].astype(np.int64) * c["page"] + np.arange(c["page"])).reshape(-1)[:T]
    s = dict(case=c, k=k, v=v, k_pages=torch.zeros(shape, dtype=dt, device=DEV),
             v_pages=torch.zeros(shape, dtype=dt, device=DEV), slot_map=_dev(slots, torch.int64))
    if own:
        s["cache"] = _cache(n_heads=c["q"], n_kv_heads=c["kv"], head_dim=c["d"], page_size=c["page"], n_pages=c["pages"],
                            max_requests=1, max_blocks=c["pages"], dtype=c["dtype"])
    return s


def _attend_lengths(c, seed):
    n_new = _spread(c["n_lo"], c["n_hi"], c["B"], seed + 7)
    return n_new, _spread(c["len_lo"], c["len_hi"], c["B"], seed) + n_new


def _prepare_attend(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    n_new, kv_len = _attend_lengths(c, seed)
    width = -(-int(kv_len.max()) // c["page"])
    n_pages = int(((kv_len.astype(np.int64) + c["page"] - 1) // c["page"]).sum()) + 3
    table, _, _ = _tables(kv_len, c["page"], width, n_pages, seed)
    shape = (n_pages, c["kv"], c["page"], c["d"]) if c["heads_first"] else (n_pages, c["page"], c["kv"], c["d"])

    def pool():
        x = torch.empty(shape, dtype=dt, device=DEV).normal_(generator=g)
        return x.transpose(1, 2) if c["heads_first"] else x

    q_off = np.concatenate([[0], np.cumsum(n_new)])
    T = int(q_off[-1])
    # queries as the projection leaves them: the first heads of a fused q/k/v row
    qkv = torch.empty((T, c["q"] + 2 * c["kv"], c["d"]), dtype=dt, device=DEV).normal_(generator=g)
    s = dict(case=c, T=T, max_new=int(n_new.max()), max_len=int(kv_len.max()), q=qkv[:, :c["q"]], k_pages=pool(),
             v_pages=pool(), block_table=_dev(table), kv_len=_dev(kv_len), q_off=_dev(q_off))
    if own:
        s["cache"] = cache = _cache(n_heads=c["q"], n_kv_heads=c["kv"], head_dim=c["d"], page_size=c["page"],
                                    n_pages=n_pages, max_requests=c["B"], max_blocks=width, dtype=c["dtype"])
        cache.block_table.copy_(s["block_table"])
    return s


def _prepare_residual(c, seed):
    g, dt, V = _gen(seed), DTYPES[c["dtype"]], c["V"]
    K = _spread(c["k_lo"], c["k_hi"], c["B"], seed + 3)
    k_off = np.concatenate([[0], np.cumsum(K)])
    T, B = int(k_off[-1]), c["B"]
    target = torch.empty((T + B, V), dtype=dt, device=DEV)
    dense = torch.empty((T, V), dtype=dt, device=DEV) if c["draft"] == "dense" else None
    top = c["top"]
    ids = torch.empty((T, top), dtype=torch.int32, device=DEV) if top else None
    probs = torch.empty((T, top), dtype=torch.float32, device=DEV) if top else None
    tokens = torch.empty(T, dtype=torch.int32, device=DEV)
    row_of = np.arange(T) + np.repeat(np.arange(B), K)                     # the window row that scores draft t
    draft_of = np.full(T + B, -1, np.int64)
    draft_of[row_of] = np.arange(T)
    for lo in range(0, T + B, 512):                                        # target and drafter logits agree in the main
        hi = min(lo + 512, T + B)
        logits = torch.empty((hi - lo, V), device=DEV).normal_(generator=g).mul_(2.6)
        target[lo:hi] = torch.softmax(logits, 1).to(dt)
        at = torch.from_numpy(np.flatnonzero(draft_of[lo:hi] >= 0)).to(DEV)
        to = torch.from_numpy(draft_of[lo:hi][draft_of[lo:hi] >= 0]).to(DEV)
        if not len(to):
            continue
        q = torch.softmax(logits[at] + 0.6 * torch.empty((len(at), V), device=DEV).normal_(generator=g), 1)
        if c["draft"] == "dense":
            dense[to] = q.to(dt)
            tokens[to] = torch.multinomial(q, 1, generator=g)[:, 0].int()
        elif top:
            best = torch.topk(q, top, dim=1)
            p = best.values / best.values.sum(1, keepdim=True)             # truncated and renormalised on the device
            order = torch.rand(p.shape, generator=g, device=DEV).argsort(1)
            ids[to], probs[to] = best.indices.gather(1, order).int(), p.gather(1, order)
            pick = torch.multinomial(p, 1, generator=g)
            tokens[to] = best.indices.gather(1, pick)[:, 0].int()
        else:
            tokens[to] = q.argmax(1).int()
    s = dict(case=c, T=T, target=target, dense=dense, ids=ids, probs=probs, tokens=tokens, k_off=_dev(k_off),
             u=torch.rand(T, generator=g, device=DEV), u_draw=torch.rand(B, generator=g, device=DEV))
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"pages": _run_pages, "append": _run_append, "attend": _run_attend, "residual": _run_residual}[s["case"]["op"]](s)


def _run_pages(s):
    """A round's layout for every window, then the return of its pages (each window rejected and withdrawn, so that a
    pass leaves the pool as it found it)."""
    c = s["case"]
    if own:
        cache = s["cache"]
        lay = cache.extend(B=c["B"], n_new=s["n_new"], T=s["T"])
        st = cache.commit(s["keep"], B=c["B"])
        return dict(q_off=lay.q_off, kv_len=lay.kv_len, slot_map=lay.slot_map, positions=lay.positions, status=lay.status,
                    status2=st, n_free=cache.n_free, free_list=cache.free_list, block_table=cache.block_table,
                    n_blocks=cache.n_blocks, seq_len=cache.seq_len)
    page, B, T, width = c["page"], c["B"], s["T"], s["block_table"].shape[1]
    n_new, seq, n_blocks, table, free, n_free = (s[k] for k in ("n_new", "seq_len", "n_blocks", "block_table", "free_list",
                                                                "n_free"))
    zero = torch.zeros(1, dtype=torch.int64, device=DEV)
    q_off = torch.cat([zero, torch.cumsum(n_new.long(), 0)])
    want = (seq.long() + n_new + page - 1) // page
    fits = want <= width
    need = torch.where(fits, torch.clamp(want - n_blocks, min=0), zero)
    upto = torch.cumsum(need, 0)
    good = fits & ((need == 0) | (upto <= n_free))
    need = torch.where(good, need, zero)
    start = n_free - need.sum() + torch.cumsum(need, 0) - need
    col = torch.arange(width, device=DEV)
    k = col[None] - n_blocks[:, None]
    new = (k >= 0) & (k < need[:, None])
    table.copy_(torch.where(new, free[(start[:, None] + k).clamp(0, len(free) - 1)], table))
    n_blocks.add_(need)
    n_free.sub_(need.sum())
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(q_off, t, right=True) - 1
    pos = seq[b] + t - q_off[b]
    slot = table[b, (pos // page).clamp(max=width - 1)].long() * page + pos % page
    slot = torch.where(good[b], slot, -torch.ones_like(slot))
    kv_len = torch.where(good, seq + n_new, torch.zeros_like(seq))
    status = torch.where(good, 0, NO_PAGES).int()
    # the return: pages past the kept length go back in request order
    keep = torch.minimum(s["keep"].clamp(min=0), n_blocks * page)
    left = (keep.long() + page - 1) // page
    gone = n_blocks - left
    at = n_free + torch.cumsum(gone, 0) - gone
    k = col[None] - left[:, None]
    out = (k >= 0) & (k < gone[:, None])
    place = torch.where(out, at[:, None] + k, len(free))
    grown = torch.cat([free, zero.int()])
    grown.scatter_(0, place.reshape(-1), table.reshape(-1))
    free.copy_(grown[:-1])
    table.copy_(torch.where(out, -1, table))
    n_blocks.copy_(left)
    n_free.add_(gone.sum())
    seq.copy_(keep)
    return dict(q_off=q_off.int(), kv_len=kv_len, slot_map=slot, positions=pos.int(), status=status,
                status2=torch.zeros_like(status), n_free=n_free, free_list=free, block_table=table, n_blocks=n_blocks,
                seq_len=seq)


def _run_append(s):
    if own:
        s["cache"].append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["slot_map"])
    else:
        page, slot = s["case"]["page"], s["slot_map"]
        at, off = slot // page, slot % page
        s["k_pages"][at, off] = s["k"]
        s["v_pages"][at, off] = s["v"]
    return s["k_pages"], s["v_pages"]


def _run_attend(s):
    c = s["case"]
    if own:
        return s["cache"].attend(s["q"], s["k_pages"], s["v_pages"], s["kv_len"], B=c["B"], max_new=s["max_new"],
                                 q_off=s["q_off"])
    B, n, L, kv, G, d, page = c["B"], s["max_new"], s["max_len"], c["kv"], c["q"] // c["kv"], c["d"], c["page"]
    pages = s["block_table"].clamp(min=0).long()
    length = s["kv_len"][:, None]
    key = torch.arange(pages.shape[1] * page, device=DEV)
    here = (key[None] < length)[:, :, None, None]
    k = s["k_pages"][pages].reshape(B, -1, kv, d)[:, :L].float()
    v = torch.where(here[:, :L], s["v_pages"][pages].reshape(B, -1, kv, d)[:, :L].float(), 0.0)
    off = s["q_off"].long()
    new = off[1:] - off[:-1]
    i = torch.arange(n, device=DEV)
    at = (off[:-1, None] + i).clamp(max=s["T"] - 1)
    q = s["q"][at].float().reshape(B, n, kv, G, d).permute(0, 2, 3, 1, 4).reshape(B, kv, G * n, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(d ** -0.5).reshape(B, kv, G, n, L)
    last = length - new[:, None] + i                                       # the last key that row i sees
    score.masked_fill_((key[None, None, :L] > last[:, :, None])[:, None, None], float("-inf"))
    score.sub_(score.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.reshape(B, kv, G * n, L), v.permute(0, 2, 1, 3)).reshape(B, kv, G, n, d)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, n, kv * G, d)
    return out[(i[None] < new[:, None])].to(DTYPES[c["dtype"]])


def _run_residual(s):
    c = s["case"]
    B, T, V = c["B"], s["T"], c["V"]
    if own:
        import paper_2604_17701_b200 as wisv
        r = wisv.verify_residual(s["target"], s["tokens"], s["u"], s["u_draw"], B=B, k_off=s["k_off"], T=T,
                                 draft_probs=s["dense"] if s["probs"] is None else s["probs"], draft_ids=s["ids"])
        return r.accept_len, r.token, r.status, r.mass
    off = s["k_off"].long()
    K = off[1:] - off[:-1]
    req = torch.searchsorted(off, torch.arange(T, device=DEV), right=True) - 1
    y = s["tokens"].long()
    p = s["target"][torch.arange(T, device=DEV) + req, y].float().clamp(0, 1)
    if s["dense"] is not None:
        q = s["dense"][torch.arange(T, device=DEV), y].float().clamp(0, 1)
    elif s["probs"] is not None:
        q = torch.where(s["ids"] == s["tokens"][:, None], s["probs"], 0.0).sum(1).clamp(0, 1)
    else:
        q = torch.ones_like(p)
    ok = s["u"] < torch.where(q > 0, (p / q).clamp(max=1), (p > 0).float())
    i = torch.arange(T, device=DEV) - off[req]
    first = torch.where(ok, K[req], i)
    A = K.scatter_reduce(0, req, first, "amin")
    full = s["target"][off[:-1] + torch.arange(B, device=DEV) + A].float().clamp(0, 1)
    t = (off[:-1] + A).clamp(max=T - 1)
    if s["dense"] is not None:
        d = s["dense"][t].float().clamp(0, 1)
    elif s["probs"] is not None:
        d = torch.zeros_like(full).scatter_add_(1, s["ids"][t].long(), s["probs"][t]).clamp(0, 1)
    else:
        d = torch.zeros_like(full).scatter_(1, y[t][:, None], 1.0)
    rest = torch.where((A < K)[:, None], (full - d).clamp(min=0), full)
    weight = (rest * FIX).long()
    weight = torch.where((weight.sum(1) > 0)[:, None], weight, (full * FIX).long())
    upto = torch.cumsum(weight, 1)
    W = upto[:, -1]
    m = (s["u_draw"] * float(1 << 31)).long().clamp(0, (1 << 31) - 1)
    goal = (W >> 31) * m + (((W & ((1 << 31) - 1)) * m) >> 31)
    token = torch.searchsorted(upto, goal[:, None], right=True)[:, 0]
    token = torch.where(W > 0, token, -1)
    return A.int(), token.int(), torch.where(W > 0, 0, NO_MASS).int(), W.float() / FIX


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(c):
    if c["op"] == "pages":
        lens, n_new = _spread(c["len_lo"], c["len_hi"], c["B"], 0).astype(np.int64), _spread(c["n_lo"], c["n_hi"], c["B"], 7)
        # what a request's length and window ask for on the average, whatever their pairing
        pages = float(n_new.sum()) / c["page"]
        T = float(n_new.sum())
        # lengths, page counts and windows in; table entries and free list both ways; offsets, slots, positions out
        return {"bytes": c["B"] * 4 * 12 + pages * 4 * 4 + T * 12, "flops": 0}
    if c["op"] == "append":
        return {"bytes": c["T"] * (c["kv"] * c["d"] * 2 * 2 * 2 + 8), "flops": 0}
    if c["op"] == "attend":
        n_new = _spread(c["n_lo"], c["n_hi"], c["B"], 7).astype(np.int64)
        lens = _spread(c["len_lo"], c["len_hi"], c["B"], 0).astype(np.int64)
        new, kept, B = float(n_new.sum()), float(lens.sum()), c["B"]
        seen = new / B * kept + float((n_new * (n_new + 1) // 2).sum())    # keys that the query rows of one head see
        return {"bytes": (kept + new) * c["kv"] * c["d"] * 4 + new * c["q"] * c["d"] * 4,
                "flops": 4.0 * seen * c["q"] * c["d"]}
    size = 4 if c["dtype"] == "fp32" else 2
    K = _spread(c["k_lo"], c["k_hi"], c["B"], 3)
    rows = c["B"] * c["V"] * size
    return {"bytes": rows * (2 if c["draft"] == "dense" else 1) + c["B"] * c["top"] * 8 + float(K.sum()) * 16, "flops": 0}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    if case["op"] == "append":
        s = _prepare_append(case, seed)
        k, v = s["k_pages"].double(), s["v_pages"].double()
        width = case["kv"] * case["d"]
        k.view(-1, width)[s["slot_map"]] = s["k"].double().reshape(-1, width)
        v.view(-1, width)[s["slot_map"]] = s["v"].double().reshape(-1, width)
        return k, v
    if case["op"] == "pages":
        return None                                                        # whole numbers alone
    if case["op"] == "residual":
        return _exact_residual(case, seed)
    s = _prepare_attend(case, seed)
    n_new, kv_len = _attend_lengths(case, seed)
    table = s["block_table"].cpu().numpy()
    page, kv, d = case["page"], case["kv"], case["d"]
    out, at = [], 0
    for b in range(case["B"]):
        n, L = int(n_new[b]), int(kv_len[b])
        slots = torch.from_numpy((table[b].astype(np.int64)[:, None] * page + np.arange(page)).reshape(-1)[:L]).to(DEV)
        heads = []
        hide = torch.arange(L, device=DEV)[None] > (L - n + torch.arange(n, device=DEV))[:, None]
        for h in range(case["q"]):
            g = h // (case["q"] // kv)
            k = s["k_pages"][slots // page, slots % page, g].double()
            v = s["v_pages"][slots // page, slots % page, g].double()
            x = s["q"][at:at + n, h].double() @ k.T / float(d) ** 0.5
            heads.append(torch.softmax(x.masked_fill(hide, float("-inf")), 1) @ v)
        out.append(torch.stack(heads, 1))
        at += n
    return torch.cat(out)


def _exact_residual(case, seed):
    """The mass that each request's token is drawn from; the whole numbers beside it are the fixed-point draw's own."""
    s = _prepare_residual(case, seed)
    k_off, mass = s["k_off"].tolist(), []
    y, u = s["tokens"].tolist(), s["u"].double().tolist()

    def drafter(t):
        if s["dense"] is not None:
            return s["dense"][t].double()
        d = torch.zeros(case["V"], dtype=torch.float64, device=DEV)
        if s["probs"] is not None:
            d.index_add_(0, s["ids"][t].long(), s["probs"][t].double())
        else:
            d[y[t]] = 1.0
        return d

    for b in range(case["B"]):
        for i in range(k_off[b + 1] - k_off[b] + 1):
            t = k_off[b] + i
            p = s["target"][t + b].double()
            if t == k_off[b + 1]:
                mass.append(p.sum())                                       # every draft accepted: the bonus token
                break
            d = drafter(t)
            a, q = float(p[y[t]]), float(d[y[t]])
            if not u[t] < (min(1.0, a / q) if q > 0 else float(a > 0)):
                mass.append((p - d).clamp(min=0).sum())
                break
    return None, None, None, torch.stack(mass)
