"""The routed experts' layer on packed weights and 8-bit activations against plain float64.

Tolerances.  A gate or up value is a sum over groups of exact integers times scales: (groups + 8) roundings of 2^-24 of
the sum of magnitudes.  a = silu(gate) up takes these through its derivatives (|silu'| <= 1.1) and adds 2^-20 of itself
(exponential, division, products).  A code of a may be the next one where a / s is that near to a half, which moves the
output by s |W| at that place; the scale carries the largest a's relative error; weights of the softmax are good to 2^-20;
the last sum has groups + experts + 16 roundings; bf16 adds half a step."""
import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu

F64 = torch.float64
EPS24 = 2.0 ** -24


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _inputs(T, E, k, h, F, gs, seed=0, scale=1.0):
    g = _gen(seed + T * 7 + E + h)
    r = lambda *s: torch.rand(s, generator=g)  # noqa: E731
    return dict(
        logits=torch.randn((T, E), generator=g), q=torch.randint(-127, 128, (T, h), generator=g).to(torch.int8),
        x_scale=(r(T) + 0.2) / 60 * scale,
        gu_packed=torch.randint(0, 256, (E, 2 * F, h // 4), generator=g).to(torch.uint8),     # (the invalid code too)
        gu_alpha=(r(E, 2 * F, h // gs) + 0.2) * 0.05,
        down_packed=torch.randint(0, 256, (E, h, F // 4), generator=g).to(torch.uint8),
        down_alpha=(r(E, h, F // gs) + 0.2) * 0.05)


def _routing(logits, k):
    """ids and weights as the routing call defines them (lowest id among equals, NaN last)."""
    T, E = logits.shape
    ids, w = [], []
    for t in range(T):
        row = logits[t].tolist()
        order = sorted(range(E), key=lambda e: (row[e] != row[e], -row[e] if row[e] == row[e] else 0.0, e))[:k]
        sel = torch.tensor([row[e] for e in order], dtype=F64)
        ids.append(order)
        w.append(torch.exp(sel - sel[0]) / torch.exp(sel - sel[0]).sum())
    return ids, torch.stack(w)


def _reference(d, k, gs, res):
    """y and how far a kernel may be from it, [T][h] each."""
    T, h = d["q"].shape
    E, F = d["logits"].shape[1], d["down_packed"].shape[2] * 4
    x = d["q"].to(F64) * d["x_scale"].to(F64)[:, None]
    ids, w = _routing(d["logits"], k)
    y = torch.zeros((T, h), dtype=F64)
    tol = torch.zeros((T, h), dtype=F64)
    mag = torch.zeros((T, h), dtype=F64)
    cache = {}
    for t in range(T):
        for j, e in enumerate(ids[t]):
            if e not in cache:
                cache[e] = (ref.ternary(d["gu_packed"][e], d["gu_alpha"][e], gs),
                            ref.ternary(d["down_packed"][e], d["down_alpha"][e], gs))
            W1, W2 = cache[e]
            z, zm = W1 @ x[t], W1.abs() @ x[t].abs()
            dz = (h // 128 + 8) * EPS24 * zm
            g, u = z[:F], z[F:]
            silu = g * torch.sigmoid(g)
            a = silu * u
            da = 1.1 * dz[:F] * u.abs() + dz[F:] * silu.abs() + 1.1 * dz[:F] * dz[F:] + 2.0 ** -20 * a.abs()
            s = a.abs().max() / 127
            if s == 0:
                continue
            ds = da[a.abs() >= a.abs().max() - da].max() / (127 * s)      # relative
            t_ = a / s
            qa = torch.round(t_)
            near = ((t_ - t_.floor() - 0.5).abs() <= da / s + 127 * (ds + 2.0 ** -22)).to(F64)
            out = W2 @ (qa * s)
            m = W2.abs() @ (qa * s).abs()
            y[t] += w[t, j] * out
            mag[t] += w[t, j] * m
            tol[t] += w[t, j] * (s * (W2.abs() @ near) + (ds + 2.0 ** -20) * m)
    tol += (F // 128 + k + 16) * EPS24 * mag
    if res is not None:
        y += res.to(F64)
        tol += EPS24 * (mag + res.to(F64).abs())
    return y, tol


def _run(catq, d, k, gs, res, dtype, stream=None, pad=0):
    T, h = d["q"].shape
    E, F = d["logits"].shape[1], d["down_packed"].shape[2] * 4
    desc = catq.moe_desc(E, k, h, F, gs)
    dev = {n: t.cuda() for n, t in d.items()}
    if pad:
        wide = torch.full((T, h + pad), 99, dtype=torch.int8, device="cuda")
        wide[:, :h] = dev["q"]
        dev["q"] = wide[:, :h]
    y = torch.full((T, h), 7.0, dtype=dtype, device="cuda")
    ws = torch.full((catq.catq_ternary_moe_a8_workspace_bytes(desc, T),), 255, dtype=torch.uint8, device="cuda")
    catq.catq_ternary_moe_a8(desc, y=y, workspace=ws, res=None if res is None else res.to(dtype).cuda(), stream=stream,
                             **dev)
    return y


CASES = [
    # T, E, k, hidden, ffn, g
    (1, 1, 1, 128, 128, 128), (1, 8, 2, 256, 128, 128), (1, 128, 8, 512, 384, 128), (2, 4, 4, 384, 640, 128),
    (3, 16, 3, 1152, 256, 128), (5, 60, 6, 256, 1408, 128), (7, 8, 1, 512, 512, 256), (16, 8, 2, 256, 256, 128),
    (17, 6, 5, 384, 128, 128), (33, 128, 8, 256, 256, 128), (40, 3, 2, 1024, 1024, 512), (64, 5, 1, 128, 384, 128),
    (130, 12, 4, 256, 128, 128), (1, 1024, 16, 128, 128, 128), (20, 300, 16, 128, 256, 128), (4, 2, 2, 2304, 128, 128),
    (2, 3, 2, 4096, 2176, 128), (9, 4, 2, 2048, 1024, 1024), (1, 4, 4, 256, 8192, 128), (8, 6, 4, 256, 256, 128),
    (1, 6, 2, 1024, 512, 256), (300, 20, 16, 128, 128, 128), (1024, 4, 1, 128, 128, 128), (1, 1, 1, 32768, 128, 128),
    (2, 2, 1, 128, 32768, 128), (32, 40, 2, 384, 1664, 128),
]


@pytest.mark.parametrize("T,E,k,h,F,gs", CASES)
def test_moe_layer(catq, T, E, k, h, F, gs):
    d = _inputs(T, E, k, h, F, gs)
    res = torch.randn((T, h), generator=_gen(5))
    for dtype, r in ((torch.float32, res), (torch.bfloat16, res.bfloat16().float()), (torch.float32, None)):
        y = _run(catq, d, k, gs, r, dtype, pad=16 if r is None else 0)
        want, tol = _reference(d, k, gs, r)
        if dtype is torch.bfloat16:
            tol = tol + 2.0 ** -8 * (want.abs() + tol)
        err = (y.cpu().to(F64) - want).abs()
        assert (err <= tol).all(), float((err - tol).max())
        assert torch.equal(y, _run(catq, d, k, gs, r, dtype))


def test_moe_routing_is_the_calls(catq):
    """The experts and weights are those of catq_aux_moe_route: with one-hot experts the output tells them apart."""
    T, E, k = 6, 70, 4
    g = _gen(9)
    logits = torch.randint(-2, 3, (T, E), generator=g).float()          # ties everywhere
    logits[1] = float("-inf")
    logits[2, 5:] = float("-inf")
    logits[3, 2:] = float("nan")
    logits[3, :2] = 1.0
    logits[4] = 0.0
    logits[5] = torch.randn(E, generator=g)
    d = _inputs(T, E, k, 128, 128, 128)
    d["logits"] = logits
    ids = torch.empty((T, k), dtype=torch.int32, device="cuda")
    w = torch.empty((T, k), device="cuda")
    perm, off = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty(E + 1, dtype=torch.int64, device="cuda")
    ws = torch.empty(catq.catq_aux_moe_route_workspace_bytes(T, E, k), dtype=torch.uint8, device="cuda")
    catq.catq_aux_moe_route(logits.cuda(), k, ids, w, perm, off, ws)
    y = _run(catq, d, k, 128, None, torch.float32).cpu()
    for t in range(T):
        if not torch.isfinite(w[t]).all():
            assert torch.isnan(y[t]).all()
            continue
        only = dict(d, logits=torch.full((T, E), -1e9))
        only["logits"][:, ids[t].long().cpu()] = torch.log(w[t].cpu().clamp(min=1e-30))
        again = _run(catq, only, k, 128, None, torch.float32).cpu()
        assert torch.allclose(again[t], y[t], rtol=1e-4, atol=1e-4 * float(y[t].abs().max()))


def test_moe_what_a_token_does_not_hit(catq):
    """NaN and infinite scales of other experts, other tokens' values and what the workspace held do not reach a token."""
    T, E, k, h, F = 20, 12, 3, 256, 256
    d = _inputs(T, E, k, h, F, 128)
    ids, _ = _routing(d["logits"], k)
    clean = _run(catq, d, k, 128, None, torch.float32)
    bad = {n: t.clone() for n, t in d.items()}
    bad["gu_alpha"][3] = float("nan")
    bad["down_alpha"][7] = float("inf")
    bad["down_alpha"][8, :, 1] = float("nan")
    bad["x_scale"][2] = float("nan")
    bad["x_scale"][4] = float("inf")
    y = _run(catq, bad, k, 128, None, torch.float32)
    hit = [t for t in range(T) if t in (2, 4) or set(ids[t]) & {3, 7, 8}]
    rest = [t for t in range(T) if t not in hit]
    assert rest and torch.equal(y[rest], clean[rest])
    assert not torch.isfinite(y[hit]).all(1).any()
    # tokens of zeros: the residual comes back
    d["q"][5] = 0
    res = torch.randn((T, h), generator=_gen(1))
    assert torch.equal(_run(catq, d, k, 128, res, torch.float32)[5].cpu(), res[5])


def test_moe_in_place_captured_and_on_another_stream(catq):
    T, E, k, h, F = 5, 16, 4, 512, 256
    desc = catq.moe_desc(E, k, h, F, 128)
    sets = [_inputs(T, E, k, h, F, 128, seed=s) for s in range(3)]
    weights = {n: sets[0][n].cuda() for n in ("gu_packed", "gu_alpha", "down_packed", "down_alpha")}
    logits, q = torch.empty((T, E), device="cuda"), torch.empty((T, h), dtype=torch.int8, device="cuda")
    xs, y = torch.empty(T, device="cuda"), torch.empty((T, h), device="cuda")
    ws = torch.empty(catq.catq_ternary_moe_a8_workspace_bytes(desc, T), dtype=torch.uint8, device="cuda")

    def load(i):
        logits.copy_(sets[i]["logits"])
        q.copy_(sets[i]["q"])
        xs.copy_(sets[i]["x_scale"])
        y.fill_(i + 1.0)

    def step(stream=None):     # (the residual is y itself)
        catq.catq_ternary_moe_a8(desc, logits, q, xs, y=y, workspace=ws, res=y, stream=stream, **weights)

    want = []
    for i in range(3):
        load(i)
        step()
        want.append(y.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 2, 0):
        load(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])
    side = torch.cuda.Stream()
    load(1)
    side.wait_stream(torch.cuda.current_stream())
    step(side.cuda_stream)
    side.synchronize()
    assert torch.equal(y, want[1])
    y.zero_()
    catq.catq_ternary_moe_a8(desc, logits[:0], q[:0], xs[:0], y=y[:0], workspace=ws, **weights)    # no tokens
    assert (y == 0).all()
