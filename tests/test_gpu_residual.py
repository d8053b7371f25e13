"""wisv_verify_residual against a plain model: whole-number arithmetic in Python, so accepted lengths and tokens are equal."""
import numpy as np
import pytest
import torch

import paper_2604_17701_b200 as wisv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BAD_TOKEN, BAD_WINDOW, NO_MASS = 2, 16, 64


def unit(x):
    return np.clip(np.nan_to_num(x.astype(np.float32), nan=0.0, posinf=1.0, neginf=0.0), 0, 1).astype(np.float32)


def model(P, tokens, u, u_draw, k_off, Q=None, ids=None, accept_in=None):
    """(accept_len, token, mass, status) of each request; P [R, V], Q [T, V] or [T, n_top] with ids, fp32 numpy."""
    V = P.shape[1]
    out = []
    for b in range(len(k_off) - 1):
        K, status = k_off[b + 1] - k_off[b], 0

        def drafter(t):
            d = np.zeros(V, np.float32)
            if ids is not None:
                for v, q in zip(ids[t], Q[t]):
                    if 0 <= v < V:
                        d[v] += q
            elif Q is not None:
                d[:] = Q[t]
            else:
                d[min(max(tokens[t], 0), V - 1)] = 1.0
            return unit(d)

        if accept_in is not None:
            A = min(max(int(accept_in[b]), 0), K)
            checked = [A] if A < K else []
        else:
            A, checked = K, range(K)
            for i in range(K):
                t = k_off[b] + i
                y = min(max(int(tokens[t]), 0), V - 1)
                p, q = unit(P[t + b, y:y + 1])[0], drafter(t)[y]
                bound = min(np.float32(p / q), np.float32(1)) if q > 0 else np.float32(p > 0)
                if not u[t] < bound:
                    A = i
                    break
        for i in checked:
            if not 0 <= tokens[k_off[b] + i] < V:
                status |= BAD_TOKEN
        p = unit(P[k_off[b] + b + A])
        w = p
        if A < K:
            w = np.maximum(p - drafter(k_off[b] + A), np.float32(0))
        w = np.floor(w.astype(np.float64) * 2.0 ** 44).astype(np.int64)
        if w.sum() == 0:
            w = np.floor(p.astype(np.float64) * 2.0 ** 44).astype(np.int64)
        W = int(w.sum())
        if W == 0:
            out.append((A, -1, 0.0, status | NO_MASS))
            continue
        goal = W * int(np.float64(u_draw[b]) * 2 ** 31) >> 31
        out.append((A, int(np.searchsorted(np.cumsum(w), goal, side="right")), W / 2 ** 44, status))
    return [np.array(x) for x in zip(*out)]


def make(K, V, dtype, form, n_top=0, seed=0, sharp=2.0, q_dtype=None, pad=0):
    rng = np.random.default_rng(seed)
    k_off = np.concatenate([[0], np.cumsum(K)]).astype(np.int64)
    T, R = int(k_off[-1]), int(k_off[-1]) + len(K)
    logits = rng.standard_normal((R, V)) * sharp
    row = np.arange(T) + np.repeat(np.arange(len(K)), K)
    soft = lambda x: np.exp(x - x.max(1, keepdims=True)) / np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)  # noqa: E731

    def on_device(a, dt):
        t = torch.empty((max(len(a), 1), a.shape[1] + pad), dtype=dt, device=DEV)[:len(a), :a.shape[1]]
        t.copy_(torch.from_numpy(a))
        return t

    P = on_device(soft(logits), TYPES[dtype])
    q = soft(logits[row] + 0.5 * rng.standard_normal((T, V))) if T else np.zeros((0, V))
    tokens = np.array([rng.choice(V, p=x / x.sum()) for x in q], np.int32).reshape(T)
    case = dict(K=K, k_off=k_off, P=P, tokens=tokens, u=rng.random(T, np.float32), u_draw=rng.random(len(K), np.float32),
                Q=None, ids=None)
    if form == "dense":
        case["Q"] = on_device(q, TYPES[q_dtype or dtype])
    elif form == "top":
        n = min(n_top, V)
        best = np.argsort(-q, 1)[:, :n].astype(np.int32)
        for t in range(T):
            rng.shuffle(best[t])
        case["ids"] = torch.from_numpy(best).to(DEV)
        case["Q"] = torch.from_numpy(np.take_along_axis(q, best, 1).astype(np.float32)).to(DEV)
    return case


def call(c, accept_in=None, **kw):
    B = len(c["K"])
    d = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device=DEV)  # noqa: E731
    return wisv.verify_residual(c["P"], d(c["tokens"], torch.int32), d(c["u"], torch.float32), d(c["u_draw"], torch.float32),
                                B=B, k_off=d(c["k_off"], torch.int32), draft_probs=c["Q"], draft_ids=c["ids"],
                                accept_len=None if accept_in is None else d(accept_in, torch.int32), **kw)


def check(c, r, accept_in=None):
    num = lambda t: None if t is None else t.float().cpu().numpy()  # noqa: E731
    want = model(num(c["P"]), c["tokens"], c["u"], c["u_draw"], c["k_off"], num(c["Q"]),
                 None if c["ids"] is None else c["ids"].cpu().numpy(), accept_in)
    assert r.accept_len.tolist() == want[0].tolist()
    assert r.token.tolist() == want[1].tolist()
    assert r.status.tolist() == want[3].tolist()
    # an integer rounded to fp32 once
    assert np.allclose(r.mass.cpu().numpy(), want[2], rtol=2.0 ** -23, atol=0)
    return want


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("form, n_top", [("dense", 0), ("top", 20), ("none", 0)])
@pytest.mark.parametrize("V, pad", [(1000, 0), (1003, 0), (4100, 12), (50000, 0)])
def test_tokens_equal_the_model(dtype, form, n_top, V, pad):
    rng = np.random.default_rng(V)
    c = make(list(rng.integers(0, 9, 24)), V, dtype, form, n_top, seed=V, pad=pad)
    want = check(c, call(c))
    assert len(set(want[0].tolist())) > 2 or form == "none"


@pytest.mark.parametrize("dtype, q_dtype", [("fp32", "bf16"), ("bf16", "fp32"), ("fp16", "bf16"), ("bf16", "fp16"),
                                            ("fp32", "fp16"), ("fp16", "fp32")])
@pytest.mark.parametrize("V", [2048, 777])
def test_mixed_types(dtype, q_dtype, V):
    c = make([4] * 16, V, dtype, "dense", seed=1, q_dtype=q_dtype)
    check(c, call(c))


@pytest.mark.parametrize("V", [1, 2, 7, 31, 33, 127, 128256, 262144])
def test_vocabulary_sizes(V):
    c = make([2, 0, 3, 1], V, "bf16", "dense", seed=V, sharp=1.0)
    check(c, call(c))
    c = make([2, 0, 3, 1], V, "fp32", "top", 256, seed=V, sharp=1.0)
    check(c, call(c))


@pytest.mark.parametrize("B", [1, 3, 150, 700])
def test_batches_and_windows_of_64(B):
    rng = np.random.default_rng(B)
    c = make(list(rng.choice([0, 1, 31, 32, 33, 64], B)) if B < 200 else [3] * B, 600, "bf16", "dense", seed=B)
    # drafts that pass with certainty, so that long windows are walked to their end
    hi = rng.random(len(c["u"])) < 0.97
    c["u"][hi] *= 0.02
    check(c, call(c))
    d = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device=DEV)  # noqa: E731
    if len(set(c["K"])) == 1:                                   # the uniform form
        r = wisv.verify_residual(c["P"], d(c["tokens"], torch.int32), d(c["u"], torch.float32),
                                 d(c["u_draw"], torch.float32), B=B, K=int(c["K"][0]), draft_probs=c["Q"])
        check(c, r)


def test_verdicts_of_the_decision_head_are_taken():
    c = make([5, 5, 0, 7, 2], 3001, "fp32", "dense", seed=9)
    for accept in ([0, 3, 0, 7, 2], [5, 1, 0, 6, 0], [9, -4, 3, 2, 1]):
        check(c, call(c, accept), accept)
    c["ids"], c["Q"] = None, None
    check(c, call(c, [0, 3, 0, 7, 1]), [0, 3, 0, 7, 1])


def test_ends_of_the_draw():
    """u at 0 and just below 1; single tokens that hold all the mass, at the first and the last place."""
    V = 5000
    c = make([0] * 6, V, "fp32", "none", seed=2)
    c["u_draw"][:] = [0.0, np.nextafter(np.float32(1), np.float32(0)), 0.0, 0.999999, 0.5, 0.25]
    c["P"][2:] = 0.0
    c["P"][2, V - 1] = c["P"][3, 0] = 1.0
    c["P"][4, 17], c["P"][4, 4000] = 0.5, 0.5
    c["P"][5, 4999] = 1e-12
    want = check(c, call(c))
    assert want[1].tolist()[2:] == [V - 1, 0, 4000, 4999]


def test_residual_without_mass_falls_back_to_the_target():
    c = make([2] * 4, 900, "fp32", "dense", seed=4)
    c["Q"][:] = 1.0                                             # nothing of P is left
    c["u"][:] = 0.9999
    c["P"][0:3, 5] = 0.7
    c["P"][6:9] = 0.0                                           # request 2: no mass at all
    c["P"][9:12] = float("nan")
    want = check(c, call(c))
    assert want[3].tolist() == [0, 0, NO_MASS, NO_MASS] and want[1].tolist()[2:] == [-1, -1]
    c["Q"] = None
    c["P"][3:6] = 0.0
    c["P"][3, c["tokens"][2]] = 1.0                             # a deterministic drafter that the target agrees with
    c["u"][2:4] = 0.5
    want = check(c, call(c))
    assert want[0][1] == 1 and want[3][1] == NO_MASS


def test_odd_probabilities_and_tokens():
    """NaN, infinite, negative and too large entries; ids out of range, listed twice, never drafted."""
    c = make([3] * 5, 2000, "fp32", "dense", seed=6)
    c["P"][:, 11], c["P"][:, 12], c["P"][:, 13], c["P"][:, 14] = float("nan"), -0.5, float("inf"), 1e-20
    c["Q"][:, 21], c["Q"][:, 22] = float("nan"), float("-inf")
    c["tokens"][0], c["tokens"][4], c["tokens"][7] = -1, 2000, 11
    c["u"][12] = float("nan")
    want = check(c, call(c))
    assert want[3].tolist()[:2] == [BAD_TOKEN, BAD_TOKEN]
    c = make([3] * 40, 2000, "bf16", "top", 33, seed=7)
    c["ids"][:, 4], c["Q"][:, 4] = c["ids"][:, 9], 0.125        # a token named twice
    c["ids"][:, 6], c["ids"][::2, 7] = 2000, -3
    c["tokens"][5] = int(c["ids"][5, 9])
    check(c, call(c))


def test_windows_that_the_device_reports_wrong():
    c = make([2, 2], 300, "fp32", "none", seed=8)
    d = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device=DEV)  # noqa: E731
    r = wisv.verify_residual(c["P"], d(c["tokens"], torch.int32), d(c["u"], torch.float32), d(c["u_draw"], torch.float32),
                             B=2, k_off=d([3, 1, 4], torch.int32), T=4)
    assert r.status.tolist()[0] & BAD_WINDOW and r.accept_len.tolist()[0] == 0


def test_frequencies_follow_the_residual():
    """4096 evenly spaced draws from one row: each token comes up as often as its weight says, to within 1."""
    V, B = 64, 4096
    rng = np.random.default_rng(0)
    p, q = rng.random(V), rng.random(V)
    p, q = p / p.sum(), q / q.sum()
    P = torch.tensor(np.repeat(p[None], 2 * B, 0), dtype=torch.float32, device=DEV)
    Q = torch.tensor(np.repeat(q[None], B, 0), dtype=torch.float32, device=DEV)
    y = torch.full((B,), int(np.argmin(p / q)), dtype=torch.int32, device=DEV)
    r = wisv.verify_residual(P, y, torch.full((B,), 0.99999, device=DEV), (torch.arange(B, device=DEV) + 0.5) / B, B=B, K=1,
                             draft_probs=Q)
    rest = np.maximum(p - q, 0) / np.maximum(p - q, 0).sum()
    assert (r.accept_len == 0).all()
    assert np.abs(np.bincount(r.token.cpu().numpy(), minlength=V) - rest * B).max() <= 1.01


def test_streams_graphs_and_outputs():
    c = make([3, 5, 1], 20000, "bf16", "top", 16, seed=3)
    d = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device=DEV)  # noqa: E731
    args = (c["P"], d(c["tokens"], torch.int32), d(c["u"], torch.float32), d(c["u_draw"], torch.float32))
    kw = dict(B=3, k_off=d(c["k_off"], torch.int32), draft_probs=c["Q"], draft_ids=c["ids"])
    first = wisv.verify_residual(*args, **kw)
    check(c, first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = wisv.verify_residual(*args, **kw, stream=side)
    side.synchronize()
    assert torch.equal(other.token, first.token)
    out = wisv.ResidualOutput(torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wisv.verify_residual(*args, **kw, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.token, first.token) and torch.equal(out.accept_len, first.accept_len)


def test_refusals():
    c = make([2, 2], 100, "fp32", "dense", seed=1)
    d = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device=DEV)  # noqa: E731
    good = dict(target_probs=c["P"], draft_tokens=d(c["tokens"], torch.int32), uniforms=d(c["u"], torch.float32),
                u_draw=d(c["u_draw"], torch.float32), B=2, K=2, draft_probs=c["Q"])
    wisv.verify_residual(**good)
    ids = torch.zeros(4, 100, dtype=torch.int32, device=DEV)
    for bad in (dict(target_probs=c["P"].double()), dict(target_probs=c["P"][:5]), dict(draft_probs=c["Q"][:, :50]),
                dict(draft_probs=c["Q"][:3]), dict(draft_tokens=good["draft_tokens"].long()), dict(uniforms=good["uniforms"][:3]),
                dict(u_draw=good["u_draw"].cpu()), dict(draft_probs=None, draft_ids=ids), dict(draft_ids=ids[:, :4]),
                dict(draft_probs=c["Q"].half(), draft_ids=ids), dict(target_probs=c["P"].t())):
        with pytest.raises(ValueError):
            wisv.verify_residual(**{**good, **bad})
    for bad, code in ((dict(uniforms=None), -1), (dict(K=3, T=4), -2), (dict(B=0), -2),
                      (dict(draft_probs=torch.zeros(4, 300, device=DEV), draft_ids=torch.zeros(4, 300, dtype=torch.int32, device=DEV)), -2)):
        with pytest.raises(wisv.WisvError) as e:
            wisv.verify_residual(**{**good, **bad})
        assert e.value.code == code


@pytest.mark.parametrize("dtype, accept", [("fp32", None), ("bf16", None), ("fp16", [1, 0, 2, 3])])
def test_an_empty_list_names_no_token(dtype, accept):
    """Lists of no entries: Q is 0 everywhere, so a draft is accepted iff P(y) > 0 and the token is drawn from P."""
    c = make([2, 0, 5, 3], 700, dtype, "top", 4, seed=12)
    c["Q"], c["ids"] = c["Q"][:, :0], c["ids"][:, :0]
    c["P"][1, c["tokens"][1]] = 0.0                             # request 0 stops at its second draft
    want = check(c, call(c, accept), accept)
    assert accept is not None or want[0].tolist() == [1, 0, 5, 3]
    for side in (torch.cuda.Stream(),):
        side.wait_stream(torch.cuda.current_stream())
        r = call(c, accept, stream=side)
        side.synchronize()
        check(c, r, accept)
