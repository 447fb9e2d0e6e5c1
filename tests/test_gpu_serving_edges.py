"""Calls of the serving operators at the ends of their ranges."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from test_gpu_serving import BF, F64, Serving, _attention_check, _linear_inputs, _rand

pytestmark = pytest.mark.gpu

# 1 / (2 pi) to 2^-230
_INV_2PI = Fraction(0xA2F9836E4E441529FC2757D1F534DDC0DB6295993C439041FE5163ABDE, 1 << 234)


def _turn(pos, f):
    """The fraction of a turn, within a half, that pos * f radians come to."""
    t = pos * Fraction(float(f)) * _INV_2PI
    return float(t - round(t))


@pytest.mark.parametrize("fmax", [1.0, 64.0, 2.0 ** 19])
@pytest.mark.parametrize("pos", [1, 40_000, 999_999, 2 ** 24 - 1, 2 ** 24 + 1, 2 ** 28 + 77, 2 ** 31 - 300])
def test_angles_at_any_position(catq, pos, fmax):
    """A pair turns by position * frequency to 2^-25 of a turn, the last positions of 32 bits among them.
    The pairs nearly cancel in one of their two results, so a wrong angle is not lost in the rounding to
    bf16: of R = |pair|, an angle off by 2 pi 2^-25 moves a result by as much, sine and cosine off by two
    steps (2^-23) each and the products and their sum off by half a step by as much of |a| + |b|; then
    half a bf16 step of what is left."""
    c, d, ps, pages = catq, 64, 256, 4
    width = pos // ps + 2
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, pos // ps], table[0, pos // ps + 1] = 2, 1
    desc = c.kv_desc(1, 1, d, ps, 16, pages, width)
    cache = c.kv_cache(desc, torch.zeros((pages, 1, ps, d), dtype=torch.int8, device="cuda"),
                       torch.zeros((pages, 1, ps // 4, d, 4), dtype=torch.int8, device="cuda"),
                       *(torch.zeros((pages, 1, ps // 16), device="cuda") for _ in range(2)))
    rng = np.random.default_rng(pos % 1000)
    inv = (rng.random(32) * fmax * rng.choice([-1.0, 1.0], 32)).astype(np.float32)
    x = torch.zeros((2, 3, d), dtype=torch.bfloat16)
    want = np.zeros((2, d))
    tol = np.zeros((2, d))
    for t in range(2):
        for i in range(32):
            a = 2 * math.pi * _turn(pos + t, inv[i])
            cs, sn = math.cos(a), math.sin(a)
            big = torch.arange(128, 256, dtype=F64) / 128             # every bf16 of [1, 2)
            if abs(cs) >= abs(sn):
                p, q = (big * sn / cs).bfloat16().to(F64), big
            else:
                p, q = big, (big * cs / sn).bfloat16().to(F64)
            j = int((p * cs - q * sn).abs().argmin())
            p, q = float(p[j]), float(q[j])
            x[t, 0, i], x[t, 0, 32 + i] = p, q
            for k, w in ((i, p * cs - q * sn), (32 + i, q * cs + p * sn)):
                want[t, k] = w
                tol[t, k] = (2 * math.pi * 2.0 ** -25 * math.hypot(p, q) + (2.0 ** -23 + 2.0 ** -23) * (abs(p) + abs(q))
                             + BF * abs(w))
    batch = c.kv_batch(desc, table, torch.tensor([0, 2], dtype=torch.int32).cuda(),
                       torch.tensor([pos], dtype=torch.int32).cuda(), 2, 2, pos + 2)
    q_out = torch.empty((2, d), dtype=torch.bfloat16, device="cuda")
    prep = c.kv_prep(desc, torch.from_numpy(inv).cuda(), rot_dim=d)
    c.catq_aux_kv_append(desc, cache, batch, prep, x.view(2, -1).cuda(), q_out)
    err = np.abs(q_out.cpu().to(F64).numpy() - want)
    assert (err <= tol).all(), float((err / tol).max())


def test_non_finite_frequencies(catq):
    """A pair whose frequency is NaN or infinite turns into NaN, and only that pair."""
    c, d, ps = catq, 64, 16
    sv = Serving(c, [(3, 4)], 1, 1, d, ps, 16).upload()
    inv = torch.ones(32)
    inv[5], inv[9] = float("nan"), float("-inf")
    x = _rand(sv.g, 4, 3 * d)
    q = torch.empty((4, d), dtype=torch.bfloat16, device="cuda")
    c.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, c.kv_prep(sv.desc, inv.cuda(), rot_dim=d), x.cuda(), q)
    bad = torch.zeros(d, dtype=torch.bool)
    bad[[5, 9, 37, 41]] = True
    assert torch.equal(torch.isnan(q.cpu()), bad.expand(4, d))


# ------------------------------------------------------------------ rows and tokens that are not seen

def _attend(catq, sv, q, scale=None):
    ws = torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)), dtype=torch.uint8,
                     device="cuda")
    o = torch.full((sv.tokens, sv.n_q * sv.d), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((sv.tokens, sv.n_q), 3.0, device="cuda")
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q, o, ws, lse=lse, scale=scale)
    return o, lse


@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38])
@pytest.mark.parametrize("ctx,new,ps,d", [(40, 1, 16, 64), (40, 12, 64, 128), (700, 12, 64, 64), (40, 40, 16, 128),
                                          (40, 40, 64, 64), (3000, 40, 128, 128), (40, 200, 32, 64), (40, 200, 64, 128),
                                          (40, 40, 64, 256)])
def test_a_row_that_sees_nothing_is_zero(catq, ctx, new, ps, d, value):
    """Also where its query is not finite, or so large that its scores are not."""
    sv = Serving(catq, [(ctx, new), (33, new)], 2, 1, d, ps, 16)
    sv.table[0] = -1
    sv.upload()
    q = _rand(sv.g, sv.tokens, 2 * d)
    clean = q.clone()
    q[:new] = value
    o, lse = _attend(catq, sv, q.cuda(), scale=200.0 if value == 3e38 else None)
    assert (o[:new] == 0).all() and torch.isneginf(lse[:new]).all()
    if value != 3e38:
        _attention_check(o, lse, sv, clean, sv.oracle())


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("new,d", [(1, 64), (1, 128), (12, 256), (40, 64), (40, 128), (200, 128)])
def test_a_query_that_is_not_finite_gives_nan(catq, new, d, value):
    """One such value is enough, also where every score it makes is -infinite, and in no other row."""
    sv = Serving(catq, [(0, new), (600, new)], 2, 1, d, 64, 16)
    sv.k[:] = -sv.k.abs() - (sv.k == 0).to(torch.int8)          # (no code is 0)
    sv.upload()
    q = _rand(sv.g, sv.tokens, 2 * d)
    bad = torch.zeros((sv.tokens, 2), dtype=torch.bool)
    bad[[0, sv.tokens - 1], [1, 0]] = True
    p = q.clone()
    p[0, d + 3] = p[-1, d - 1] = value
    (o, lse), (clean, cl) = _attend(catq, sv, p.cuda()), _attend(catq, sv, q.cuda())
    rows = o.view(-1, 2, d)
    assert torch.isnan(rows[bad.cuda()]).all() and torch.equal(torch.isnan(lse.cpu()), bad)
    rows[bad.cuda()] = clean.view(-1, 2, d)[bad.cuda()]
    lse[bad.cuda()] = cl[bad.cuda()]
    _attention_check(o, lse, sv, q, sv.oracle())


@pytest.mark.parametrize("bt", [1, 16])
@pytest.mark.parametrize("new", [1, 12, 40, 300])
def test_attention_scales_at_the_border(catq, new, bt):
    """A v scale of 2^-60, or one step above, counts, beside others that are below and do not."""
    sv = Serving(catq, [(90, new), (33, new)], 2, 1, 128, 64, bt)
    low = torch.rand(sv.vs.shape, generator=sv.g)
    sv.vs[:] = 2.0 ** -60
    sv.vs[low < 0.6] = 2.0 ** -60 * (1 + 2.0 ** -23)
    sv.vs[low < 0.3] = 2.0 ** -60 * (1 - 2.0 ** -24)
    sv.upload()
    q = _rand(sv.g, sv.tokens, 256)
    o, lse = _attend(catq, sv, q.cuda())
    oracle = sv.oracle()
    oracle.scales[1][oracle.scales[1] < 2.0 ** -60] = 0
    _attention_check(o, lse, sv, q, oracle)


# ------------------------------------------------------------------ arguments in another order

def test_scales_in_another_order_are_refused(catq):
    """alpha and scales laid out group by group are not read as rows of groups; nothing is written."""
    q, packed, alpha, xs = [t.cuda() for t in _linear_inputs(5, 24, 512, 128, 0)]
    Y = torch.full((5, 24), 5.0, device="cuda")
    with pytest.raises(ValueError, match="alpha"):
        catq.catq_ternary_linear_a8(q, xs, packed, alpha.T.contiguous(), Y)
    x = torch.ones((5, 512), dtype=torch.bfloat16, device="cuda")
    s = torch.full((4, 5), 5.0, device="cuda")
    with pytest.raises(ValueError, match="scale"):
        catq.catq_aux_act_quant8(x, q, s, group=128)
    with pytest.raises(ValueError, match="scale"):
        catq.catq_aux_rmsnorm_quant(x, q, s, group=128)
    assert (Y == 5.0).all() and (s == 5.0).all()
