"""Sampling against a plain float64 definition.

A weight is off by at most 2^-23 (the hardware's exp2), 2^-25 of its argument's fraction and 2^-43 of the largest weight,
so a sum of weights is off by less than 2^-22 of itself and V * 2^-43: DELTA bounds both for V <= 2^20 where a row's
kept weight is at least the largest one.  The cumulative sums that decide (top-p's, and u's) may fall on either
side of a border that is that near; the reference is taken with both and the token has to be one of theirs."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DELTA = 2.0 ** -21


def _all(x, T, k, p, m, u):
    """The (token, prob) that one row of float64 logits can give, with the borders of top-p and u moved by DELTA."""
    ok = x > -math.inf                                   # (False for NaN)
    if not ok.any():
        return {(-1, 0.0)}
    ids = np.flatnonzero(ok)
    order = ids[np.argsort(-x[ids], kind="stable")]
    if not T > 0:
        return {(int(order[0]), 1.0)}
    top = x[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(x[order] == top, 1.0, np.exp((x[order] - top) / T))
    if k > 0:
        order, w = order[:k], w[:k]
    u = 0.0 if not u > 0 else min(u, 1 - 2.0 ** -24)
    sizes = {len(order)}
    if p < 1:
        before, whole = np.concatenate([[0.0], np.cumsum(w)[:-1]]), w.sum()
        sizes = {max(1, int((before < (p + dp) * whole).sum())) for dp in (0.0, -DELTA, DELTA)}
    if m > 0:
        sizes = {min(n, max(1, int((w >= m).sum()))) for n in sizes}
    out = set()
    for n in sizes:
        by_id = np.argsort(order[:n])
        ids, wi = order[:n][by_id], w[:n][by_id]
        cum = np.cumsum(wi)
        for du in (0.0, -DELTA, DELTA):
            at = min(int((cum <= (u + du) * cum[-1]).sum()), n - 1)
            out.add((int(ids[at]), float(wi[at] / cum[-1])))
    return out


def _check(catq, logits, u, T=None, k=None, p=None, m=None, ld=None, repeat=True):
    n, V = logits.shape
    if ld is None:
        dev = logits.cuda()
    else:
        wide = torch.full((n, ld), 1e4, dtype=logits.dtype, device="cuda")     # (what lies between the rows is large)
        wide[:, :V] = logits.cuda()
        dev = wide[:, :V]
    f = lambda v, dt=torch.float32: None if v is None else torch.tensor(v, dtype=dt, device="cuda")  # noqa: E731
    args = dict(temperature=f(T), top_k=f(k, torch.int32), top_p=f(p), min_p=f(m))
    token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((n,), -7.0, device="cuda")
    ws = torch.empty(max(16, catq.catq_aux_sample_workspace_bytes(n, V)), dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    catq.catq_aux_sample(dev, f(u), token, ws, prob=prob, **args)
    x = logits.double().numpy()
    u32 = np.asarray(u, dtype=np.float32).astype(float)
    for r in range(n):
        row = [np.float32(v[r]).astype(float) if v is not None else d for v, d in ((T, 1.0), (p, 1.0), (m, 0.0))]
        kk = 0 if k is None else k[r]
        want = _all(x[r], row[0], kk, row[1], row[2], u32[r])
        got = int(token[r]), float(prob[r])
        near = [q for t, q in want if t == got[0]]
        assert near, (r, got, want, [None if v is None else v[r] for v in (T, k, p, m)], u[r])
        assert min(abs(got[1] - q) for q in near) <= DELTA * got[1] + 1e-30, (r, got, want)
    if repeat:
        again = torch.empty_like(token)
        catq.catq_aux_sample(dev, f(u), again, ws, **args)
        assert torch.equal(again, token)
    return token, prob


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


SIZES = [(1, 1, None), (3, 2, None), (5, 7, 9), (4, 100, None), (6, 1000, 1003), (3, 4097, None),
         (3, 16384, 16389), (3, 16385, None), (8, 32000, None), (5, 50257, 50261), (4, 150000, None), (1, 262147, None), (70, 300, 301), (2, 1 << 20, None)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,ld", SIZES)
def test_sample(catq, rows, V, ld, dtype):
    g = _gen(V + rows)
    x = (torch.randn((rows, V), generator=g) * 2.5).to(dtype)
    x[:, ::max(1, V // 9)] += 5
    r = np.random.RandomState(V)
    for settings in range(7):
        on = [[0, 0, 0], [1, 0, 0], [0, 1, 0], [0, 0, 1], [1, 1, 0], [0, 1, 1], [1, 1, 1]][settings]
        _check(catq, x, r.rand(rows), T=r.uniform(0.3, 1.5, rows),
               k=[int(v) for v in r.choice([1, 2, 40, 400, 5000, 2 ** 31 - 1], rows)] if on[0] else None,
               p=r.uniform(0.05, 0.999, rows) if on[1] else None, m=r.uniform(0.001, 0.3, rows) if on[2] else None,
               ld=ld, repeat=settings == 6)


def test_sample_many_rows(catq):
    """As many rows as the chip has units, each read by one workgroup."""
    g = _gen(6)
    n, V = 257, 40001
    x = torch.randn((n, V), generator=g) * 2.5
    x[:, 17] += 7
    x[100:, V // 2:] = -math.inf
    r = np.random.RandomState(1)
    _check(catq, x, r.rand(n), ld=V + 1, repeat=False)
    _check(catq, x.bfloat16(), r.rand(n), T=r.uniform(0.5, 1.2, n), k=[int(v) for v in r.choice([0, 30, 9000], n)],
           p=r.uniform(0.3, 1.1, n), repeat=False)


def test_sample_ties(catq):
    """Equal logits by the hundred thousand: the filters end inside them, by index; and in every place of the row."""
    V = 100003
    g = _gen(1)
    x = torch.zeros((9, V))
    x[1] = torch.randint(0, 3, (V,), generator=g).float()
    x[2] = -3.0
    x[2, V - 1] = 4.0
    x[3, :50000] = 1.0
    x[4] = torch.randint(0, 2, (V,), generator=g).float() * 1e-30        # different keys, one bin
    x[5] = 1.0 + torch.randint(0, 100000, (V,), generator=g).float() * 2.0 ** -23
    x[6] = torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0)        # the same logit
    x[7, ::2] = -math.inf
    x[8, 1:] = -40.0                                                       # the others weigh nothing
    for dtype in (torch.float32, torch.bfloat16):
        for k, p in ((None, None), (30000, None), (None, 0.37), (70001, 0.61), (7, 0.5), (2049, 0.999), (1, 0.3)):
            _check(catq, x.to(dtype), [0.0, 0.3, 0.5, 0.9, 0.123, 0.77, 0.999, 0.2, 0.4], T=[1.0, 0.7, 2.0] * 3,
                   k=None if k is None else [k] * 9, p=None if p is None else [p] * 9)


def test_sample_kept_sets(catq):
    """Over all u, exactly the kept tokens come out."""
    V, n = 50, 4000
    g = _gen(2)
    row = torch.randn(V, generator=g) * 2
    u = (np.arange(n) + 0.5) / n
    order = torch.argsort(row, descending=True, stable=True).tolist()
    w = torch.softmax(row.double(), 0)
    for k, p, m in ((3, 1.0, 0.0), (0, 0.8, 0.0), (0, 1.0, 0.1), (10, 0.9, 0.05), (0, 1e-9, 0.0), (0, 1.0, 1.0)):
        token, _ = _check(catq, row.expand(n, V).contiguous(), u, T=[1.0] * n, k=[k] * n, p=[p] * n, m=[m] * n,
                          repeat=False)
        ws = w[order[:k or V]]
        before = ws.cumsum(0) - ws
        keep = [t for j, t in enumerate(order[:k or V])
                if j == 0 or (before[j] < np.float32(p) * ws.sum() and w[t] >= np.float32(m) * w[order[0]])]
        share = {t: float(w[t] / w[keep].sum()) for t in keep}
        counts = torch.bincount(token.cpu(), minlength=V)
        for t in range(V):
            assert abs(int(counts[t]) - share.get(t, 0.0) * n) <= 2, (t, k, p, m)


def test_sample_odd_rows(catq):
    V = 3001
    inf, nan = math.inf, math.nan
    g = _gen(3)
    x = torch.randn((14, V), generator=g)
    x[0] = -inf
    x[1] = nan
    x[2] = -inf
    x[2, 77] = -3e38                          # one token is left
    x[3, 5], x[3, 2000], x[3, 2999] = inf, inf, inf
    x[4, 9] = nan
    x[5, ::3] = nan
    x[6] = -inf
    x[6, 3000], x[6, 0] = 1.0, 1.0
    x[7] = x[7] * 1e38
    x[8] = 3.0e38
    x[8, 4] = -3.0e38
    for u in (0.0, 0.34, 0.67, 0.9999999):
        token, prob = _check(catq, x, [u] * 14)
        assert token[:2].tolist() == [-1, -1] and prob[:2].tolist() == [0.0, 0.0] and int(token[2]) == 77
        assert int(token[3]) in (5, 2000, 2999)
        _check(catq, x, [u] * 14, k=[5] * 14, p=[0.9] * 14, m=[0.01] * 14)
        # settings at and past their ends
        one = [0.0, -1.0, nan, inf, 1e-30, 1e30, 1e-45, 3e38, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0]
        _check(catq, x[9:10].expand(14, V).contiguous(), [u] * 14, T=one, k=[50] * 14, p=[0.95] * 14)
        _check(catq, x[9:10].expand(14, V).contiguous(), [u] * 14, k=[-1, 0, 1, V, V + 1, 2 ** 31 - 1, -2 ** 31] * 2,
               p=[1.0, 2.0, inf, nan, -inf, 0.0, -1.0] + [0.5] * 7, m=[0.0, -1.0, nan, 1.0, 2.0, inf, 0.2] * 2)
    bad = [nan, -1.0, inf, 1.0, 1.5, -inf, 1 - 2.0 ** -24] * 2
    token, _ = _check(catq, x[9:10].expand(14, V).contiguous(), bad, repeat=False)
    assert int(token[0]) == int(token[1]) == int(token[5]) and int(token[2]) == int(token[3]) == int(token[4])


def test_sample_captured_and_on_another_stream(catq):
    g = _gen(4)
    V = 120000
    x = (torch.randn((3, 5, V), generator=g) * 2).cuda()
    u = torch.rand((3, 5), generator=g).cuda()
    logits, uu = torch.empty((5, V), device="cuda"), torch.empty(5, device="cuda")
    token, prob = torch.empty(5, dtype=torch.int32, device="cuda"), torch.empty(5, device="cuda")
    ws = torch.empty(max(16, catq.catq_aux_sample_workspace_bytes(5, V)), dtype=torch.uint8, device="cuda")
    top_k = torch.tensor([0, 50, 0, 5000, 0], dtype=torch.int32, device="cuda")
    top_p = torch.tensor([0.9, 1.0, 1.0, 0.99, 0.5], device="cuda")

    def step(stream=None):
        catq.catq_aux_sample(logits, uu, token, ws, top_k=top_k, top_p=top_p, prob=prob, stream=stream)

    want = []
    for i in range(3):
        logits.copy_(x[i])
        uu.copy_(u[i])
        step()
        want.append((token.clone(), prob.clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 2, 1):
        logits.copy_(x[i])
        uu.copy_(u[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token, want[i][0]) and torch.equal(prob, want[i][1])
    side = torch.cuda.Stream()
    logits.copy_(x[0])
    uu.copy_(u[0])
    side.wait_stream(torch.cuda.current_stream())
    step(side.cuda_stream)
    side.synchronize()
    assert torch.equal(token, want[0][0]) and torch.equal(prob, want[0][1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,ld", [(4, 1000, 1003), (5, 40000, 40001), (3, 150000, None), (256, 40000, 40001)])
def test_sample_min_p_and_tied_logits(catq, rows, V, ld, dtype):
    """No weight is above 1: a min_p of 1 keeps all tokens that tie with the largest logit, one above it the first of them
    alone, with every filter beside it."""
    x = (torch.randn((rows, V), generator=_gen(V)) * 2).to(dtype)
    x[:, [5, V // 2, V - 1]] = 20.0
    x[1, [17, V // 3, V - 2]] = math.inf
    x[2] = 1.0
    first = torch.full((rows,), 5, dtype=torch.int32)
    first[1], first[2] = 17, 0
    T = [(0.5, 1.0, 2.0)[r % 3] for r in range(rows)]
    above = [(1.5, 1 + 2.0 ** -23, 3e38, math.inf)[r % 4] for r in range(rows)]
    dev = torch.full((rows, ld or V), 1e4, dtype=dtype, device="cuda")[:, :V]
    dev.copy_(x)
    f = lambda v, dt=torch.float32: None if v is None else torch.tensor([v] * rows, dtype=dt, device="cuda")  # noqa: E731
    ws = torch.empty(max(16, catq.catq_aux_sample_workspace_bytes(rows, V)), dtype=torch.uint8, device="cuda")
    for k, p in ((None, None), (50, None), (None, 0.7), (50, 0.7), (2, 0.9), (5000, 0.99)):
        for u in (0.0, 0.5, 0.9, 0.999):
            token = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
            prob = torch.full((rows,), -7.0, device="cuda")
            catq.catq_aux_sample(dev, f(u), token, ws, temperature=torch.tensor(T, device="cuda"), top_k=f(k, torch.int32),
                                 top_p=f(p), min_p=torch.tensor(above, device="cuda"), prob=prob)
            assert torch.equal(token.cpu(), first) and (prob == 1.0).all(), (k, p, u)
    for k, p in ((None, None), (2, None), (None, 0.7), (50, 0.7)):
        _check(catq, x[:3], [0.4, 0.6, 0.9], T=T[:3], k=None if k is None else [k] * 3, p=None if p is None else [p] * 3,
               m=[1.0, 1.0, 1.0], ld=ld, repeat=False)


@pytest.mark.parametrize("V", [20000, 65536, 66000])
def test_sample_one_workspace_for_fewer_rows(catq, V):
    """The workspace of the largest batch serves every smaller one; rows that a workgroup reads alone need none."""
    most = 300
    x = (torch.randn((most, V), generator=_gen(V)) * 2.5).bfloat16().cuda()
    u = torch.rand(most, generator=_gen(1)).cuda()
    top_p = torch.full((most,), 0.8, device="cuda")
    ws = torch.empty(catq.catq_aux_sample_workspace_bytes(most, V), dtype=torch.uint8, device="cuda")
    for n in (most, 256, 255, 9, 1):
        own = torch.empty(max(16, catq.catq_aux_sample_workspace_bytes(n, V)), dtype=torch.uint8, device="cuda")
        spaces = [ws, own] + ([None] if n >= 256 and V <= 65536 else [])
        got = []
        for w in spaces:
            token, prob = torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), -7.0, device="cuda")
            catq.catq_aux_sample(x[:n], u[:n], token, w, top_p=top_p[:n], prob=prob)
            assert (token >= 0).all() and (prob > 0).all()
            got.append((token, prob))
        for token, prob in got[1:]:
            assert torch.equal(token, got[0][0]) and torch.equal(prob, got[0][1])
