"""Calls of the serving operators at the ends of their ranges: far positions and large frequencies,
pages that are missing, contents behind the mask, scales at the border of what counts, rows that
see nothing, storage at its least alignment."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import serving_ref as ref
from test_gpu_serving import BF, F64, Serving, _attention_check, _linear_check, _linear_inputs, _rand

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


MASKED = [(20, 1), (20, 10), (35, 30), (20, 200), (1500, 1), (1500, 10), (1500, 40)]   # ctx, new: one span and several


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("bt", [1, 16])
@pytest.mark.parametrize("ctx,new", MASKED)
def test_attention_contents_behind_the_mask(catq, ctx, new, bt, d):
    """NaN and infinite scales at positions that a row does not see, in its own pages and in others', change
    nothing in it; the rows that see one are NaN."""
    sv = Serving(catq, [(ctx, new)], 2, 1, d, 64, bt, extra_pages=2)
    total, q = ctx + new, _rand(sv.g, new, 2 * d)
    oracle = sv.oracle()
    pages = sv.table[0, :-(-total // 64)]
    other = [p for p in range(sv.desc.n_pages) if p not in pages.tolist()]
    tail = -(-(total % 64) // bt)                 # first block of the last page that no row sees
    assert other and total % 64 and tail < 64 // bt
    for s, a, b in ((sv.ks, math.nan, math.inf), (sv.vs, math.inf, math.nan)):
        s[other] = a
        s[pages[-1], :, tail:] = b
    sv.upload()
    o, lse = _attend(catq, sv, q.cuda())
    _attention_check(o, lse, sv, q, oracle)
    # a block that the later rows see, in k and then in v
    start = -(-(ctx + new // 2) // bt) * bt
    if start >= total:
        return
    first = max(0, start - ctx)
    for w in (2, 3):
        held = sv.dev[w].clone()
        sv.dev[w][pages[start // 64], :, start % 64 // bt] = math.nan
        got, gl = _attend(catq, sv, q.cuda())
        sv.dev[w].copy_(held)
        assert torch.isnan(got[first:]).all() and torch.isnan(gl[first:]).all()
        got[first:], gl[first:] = o[first:], lse[first:]
        _attention_check(got, gl, sv, q, oracle)


@pytest.mark.parametrize("ctx,new,d", [(100, 1, 64), (100, 14, 128), (100, 40, 64), (100, 200, 128), (1500, 1, 128),
                                       (1500, 14, 64), (1500, 40, 128), (1500, 300, 64), (900, 30, 256)])
@pytest.mark.parametrize("ps,bt", [(16, 16), (16, 1), (32, 16), (64, 64), (128, 1)])
def test_attention_over_missing_pages(catq, ctx, new, d, ps, bt):
    """Page ids that are none, first, last, single and several in a row between the others: their tokens are
    unseen, whatever page 0 holds."""
    sv = Serving(catq, [(ctx, new), (37, 2)], 2, 1, d, ps, bt)
    n = -(-(ctx + new) // ps)
    gone = torch.rand(n, generator=sv.g) < 0.3
    gone[n // 2] = True
    gone[n // 3] = False
    sv.table[0, :n][gone] = torch.tensor([-1, -2 ** 31, sv.desc.n_pages, 2 ** 31 - 1], dtype=torch.int32)[
        torch.randint(0, 4, (int(gone.sum()),), generator=sv.g)]
    if 0 not in sv.table.tolist()[0] + sv.table.tolist()[1]:
        sv.ks[0], sv.vs[0] = math.nan, math.nan
    sv.upload()
    q = _rand(sv.g, sv.tokens, 2 * d)
    o, lse = _attend(catq, sv, q.cuda())
    _attention_check(o, lse, sv, q, sv.oracle())


@pytest.mark.parametrize("bt", [1, 16, 64])
@pytest.mark.parametrize("new", [1, 40])
def test_attention_beside_scales_past_the_range(catq, bt, new):
    """V scales from 1e-20 to 1e12: where a row sees none above 2^30 it is as the reference has it, with the
    scales below 2^-60 counted as 0."""
    sv = Serving(catq, [(200, new), (70, new)], 4, 2, 128, 64, bt)
    g = sv.g
    sv.vs *= 10.0 ** (torch.rand(sv.vs.shape, generator=g) * 26 - 20)
    held = sv.table[1, :-(-(70 + new) // 64)].long()
    sv.vs[held, 0] = sv.vs[held, 0].clamp(max=2.0 ** 30)         # one sequence's one head sees none
    sv.vs[sv.table[0, 0], 0, 0] = 2.0 ** 31                      # another sequence's first block is
    sv.upload()
    q = _rand(g, sv.tokens, 4 * 128)
    o, lse = _attend(catq, sv, q.cuda())
    oracle = sv.oracle()
    oracle.scales[1][oracle.scales[1] < 2.0 ** -60] = 0
    seen = torch.zeros((sv.tokens, 2), dtype=F64)      # the largest scale that each row's heads see
    for i, (ctx, n) in enumerate(sv.seqs):
        for r in range(n):
            top = torch.stack([oracle.scales[1][(at := oracle.place(sv.table[i], p))[0], :, at[1] // bt]
                               for p in range(ctx + r + 1)]).amax(0)
            seen[int(sv.cu[i]) + r] = top
    bad = (seen > 2.0 ** 30).repeat_interleave(2, 1)
    assert bad.any() and (~bad).any()
    assert torch.equal(torch.isnan(lse.cpu()), bad)
    rows = o.view(-1, 4, 128)
    assert torch.isnan(rows[bad.cuda()]).all() and torch.isfinite(rows[~bad.cuda()].float()).all()
    # the rows that are not NaN, against the reference (its own values in the others' place)
    for i, (ctx, n) in enumerate(sv.seqs):
        r0 = int(sv.cu[i])
        w, wl = ref.attention(q[r0:r0 + n].to(F64).view(n, 4, 128), oracle, sv.table[i], ctx, 128 ** -0.5, 2)[:2]
        b = bad[r0:r0 + n].cuda()
        rows[r0:r0 + n][b] = w.bfloat16().cuda()[b]
        lse[r0:r0 + n][b] = wl.float().cuda()[b]
    _attention_check(o, lse, sv, q, oracle)


# ------------------------------------------------------------------ the product's storage

@pytest.mark.parametrize("M,d_out,d_in,g", [(1, 100, 640, 128), (4, 4111, 2176, 128), (16, 333, 1024, 512),
                                            (33, 34001, 896, 128), (45, 16421, 2176, 128), (48, 5120, 1152, 128),
                                            (130, 515, 1280, 128), (1000, 16421, 128, 128), (257, 300, 896, 128)])
def test_linear_a8_storage_at_its_least_alignment(catq, M, d_out, d_in, g):
    """packed 8 bytes past a multiple of 16, x_scale and a bf16 Y 4 bytes past one."""
    q, packed, alpha, xs = _linear_inputs(M, d_out, d_in, g, M + d_in)
    held = torch.full((packed.numel() + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    dp = held[8:8 + packed.numel()].view(packed.shape)
    dp.copy_(packed)
    dx = torch.full((M + 2,), float("nan"), device="cuda")[1:M + 1]
    dx.copy_(xs)
    room = torch.full((M * d_out + 4,), 5.0, dtype=torch.bfloat16, device="cuda")
    Y = room[2:2 + M * d_out].view(M, d_out)
    assert dp.data_ptr() % 16 == 8 and dx.data_ptr() % 16 == 4 and Y.data_ptr() % 16 == 4
    catq.catq_ternary_linear_a8(q.cuda(), dx, dp, alpha.cuda(), Y, g=g)
    _linear_check(Y, q, packed, alpha, xs, g, True)
    assert (room[:2] == 5.0).all() and (room[2 + M * d_out:] == 5.0).all()
