"""The serving operators of the 8-bit-activation setting against plain float64:
residual RMSNorm with 8-bit output, the packed-ternary product on codes, the append to
the paged cache with rotation, its read-back, and attention over it.

Tolerances.  A value that the kernels form in fp32 and the reference in float64
differs by a few units of 2^-24 relative; FP below is that bound for the longest sums
here (32 terms per thread, 22 levels of a tree, halved by the square root, and 10
elementary steps: under 40 roundings).  A code is right if it is the nearest integer to
the reference's quotient up to that error.  bf16 results add half a step, 2^-8."""
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu

FP = 40 * 2.0 ** -24
BF = 2.0 ** -8
F64 = torch.float64


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _rand(g, *shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(dtype)


def _codes_ok(q, xhat, s, tol=FP):
    """|xhat / s - q| <= 1/2 up to the relative error of the quotient."""
    t = xhat / torch.where(s > 0, s, torch.ones_like(s))
    assert q.abs().max() <= 127
    assert ((q - t).abs() <= 0.5 + 127 * 2 * tol).all(), float((q - t).abs().max())


# ------------------------------------------------------------ norm and quantizer

NORM = [
    # rows, n, group, x, res, weight
    (1, 8, 8, "b", None, False), (1, 256, 256, "b", "f", True), (3, 2048, 128, "b", "b", False),
    (5, 5120, 5120, "b", "f", True), (7, 4104, 24, "f", "f", True), (2, 8200, 8200, "b", "b", True),
    (2, 17408, 128, "f", None, True), (3, 32768, 32768, "b", "f", False), (65, 768, 192, "b", "b", True),
    (4, 1024, 512, "f", "b", False), (2, 4096, 1024, "b", "f", True), (33, 264, 8, "b", None, True),
]


@pytest.mark.parametrize("rows,n,group,xt,rt,weighted", NORM)
def test_norm_quant(catq, rows, n, group, xt, rt, weighted):
    T = {"b": torch.bfloat16, "f": torch.float32}
    g = _gen(rows * n + group)
    x = _rand(g, rows, n, dtype=T[xt])
    x[:, ::61] *= 8
    res = None if rt is None else _rand(g, rows, n, dtype=T[rt], std=2.0)
    w = _rand(g, n, std=0.5) if weighted else None
    h, xhat = ref.norm_xhat(x, res, w, 1e-6, None if rt is None else T[rt])
    dx, dr = x.cuda(), None if res is None else res.cuda()
    dw = None if w is None else w.cuda()
    q = torch.full((rows, n), 99, dtype=torch.int8, device="cuda")
    sc = torch.full((rows, n // group), -1.0, device="cuda")
    y = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    total = None if res is None else torch.empty_like(dr)
    catq.catq_aux_rmsnorm_quant(dx, q, sc, res=dr, weight=dw, sum=total, y=y, group=group)
    if res is not None:
        assert torch.equal(total.cpu().to(F64), h)
    s64 = (xhat.view(rows, -1, group).abs().amax(-1) / 127)
    s = sc.cpu().to(F64)
    assert ((s - s64).abs() <= FP * s64).all()
    se = s.repeat_interleave(group, 1)
    _codes_ok(q.cpu().to(F64), xhat, se)
    assert torch.equal(y, (q.float() * sc.repeat_interleave(group, 1)).bfloat16())
    # in place, and each output alone
    if res is not None:
        q2, sc2 = torch.empty_like(q), torch.empty_like(sc)
        r2 = dr.clone()
        catq.catq_aux_rmsnorm_quant(dx, q2, sc2, res=r2, weight=dw, sum=r2, group=group)
        assert torch.equal(q2, q) and torch.equal(sc2, sc) and torch.equal(r2, total)
        if xt == rt:
            x2 = dx.clone()
            catq.catq_aux_rmsnorm_quant(x2, q2, sc2, res=dr, weight=dw, sum=x2, group=group)
            assert torch.equal(q2, q) and torch.equal(x2, total)
    y2 = torch.empty_like(y)
    catq.catq_aux_rmsnorm_quant(dx, res=dr, weight=dw, y=y2, group=group)
    assert torch.equal(y2, y)


@pytest.mark.parametrize("n,group,dtype", [(64, 64, torch.bfloat16), (5120, 5120, torch.bfloat16),
                                           (1280, 40, torch.float32), (2048, 128, torch.bfloat16),
                                           (17408, 17408, torch.bfloat16), (32768, 4096, torch.float32)])
def test_act_quant8_is_act_quant(catq, n, group, dtype):
    """Codes times scale are the values of the fake quantizer, bit for bit, ties
    and subnormal groups among them."""
    g = _gen(n + group)
    x = _rand(g, 9, n, dtype=dtype)
    x[1] = 0
    x[2, :group] = torch.arange(group).to(dtype) % 9 - 4           # many equal magnitudes
    x[3] = (torch.randint(-254, 255, (n,), generator=g) * 0.5).to(dtype)
    x[3, ::group] = 127.0                                          # scale 1: halves are ties
    x[4] = (torch.randint(-300, 301, (n,), generator=g).double() * 2.0 ** -149).to(dtype)
    x[5] = x[5] * 1e30
    x = x.cuda()
    q = torch.empty(x.shape, dtype=torch.int8, device="cuda")
    s = torch.empty((9, n // group), device="cuda")
    y = torch.empty(x.shape, dtype=torch.bfloat16, device="cuda")
    catq.catq_aux_act_quant8(x, q, s, group=group)
    catq.catq_aux_act_quant(x, y, group=group)
    assert torch.equal((q.float() * s.repeat_interleave(group, 1)).bfloat16().view(torch.int16) & 0x7fff,
                       y.view(torch.int16) & 0x7fff)               # (a zero code has no sign)
    assert torch.equal(q.sign().float() * (y != 0), y.sign().float())


def test_norm_quant_special_rows(catq):
    x = _rand(_gen(1), 6, 512).cuda()
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    x[4, 100] = float("-inf")
    q = torch.empty((6, 512), dtype=torch.int8, device="cuda")
    s = torch.empty((6, 4), device="cuda")
    y = torch.empty_like(x)
    catq.catq_aux_rmsnorm_quant(x, q, s, y=y, group=128)
    assert (q[1] == 0).all() and (s[1] == 0).all() and (y[1] == 0).all()
    for r in (2, 3, 4):   # the norm carries it to the whole row: NaN, or 0 / inf and inf / inf
        bad = torch.isnan(s[r])
        assert bad.any() and (q[r].view(4, 128)[bad] == 0).all()
        assert torch.isnan(y[r].view(4, 128)[bad]).all()
    assert torch.isfinite(y[[0, 5]].float()).all()
    catq.catq_aux_act_quant8(x, q, s, group=128)
    assert torch.isnan(s[2]).tolist() == [True, False, False, False]
    assert torch.isnan(s[3]).tolist() == [True, False, False, False]
    assert (q[4, :128] == 0).all() and torch.isfinite(s[4, 1:]).all()
    # no rows
    e = x[:0]
    catq.catq_aux_act_quant8(e, q[:0], s[:0], group=128)
    catq.catq_aux_rmsnorm_quant(e, q[:0], s[:0], group=128)


# ------------------------------------------------------- ternary product on codes

LINEAR = [
    # M, d_out, d_in, g
    (1, 1, 128, 128), (1, 17, 256, 256), (2, 100, 512, 128), (4, 333, 1024, 512), (5, 64, 5120, 128),
    (16, 48, 384, 128), (17, 129, 640, 128), (33, 250, 2048, 1024), (64, 128, 17408, 128),
    (65, 300, 896, 128), (130, 515, 1280, 128), (257, 96, 8320, 128), (3, 31, 65536, 128),
    (40, 1000, 256, 128), (200, 40, 65536, 65536),
]


def _linear_inputs(M, d_out, d_in, g, seed):
    r = _gen(seed)
    q = torch.randint(-127, 128, (M, d_in), generator=r).to(torch.int8)
    packed = torch.randint(0, 256, (d_out, d_in // 4), generator=r).to(torch.uint8)   # every code, 3 too
    alpha = torch.rand((d_out, d_in // g), generator=r) * 0.05
    xs = torch.rand(M, generator=r) * 0.1
    return q, packed, alpha, xs


def _linear_check(Y, q, packed, alpha, xs, g, bf):
    """fp32 sums over the groups: each of at most n_groups + 3 roundings of a partial sum
    no larger than the sum of magnitudes."""
    W = ref.ternary(packed, alpha, g)
    x = q.to(F64) * xs.to(F64)[:, None]
    want, mag = x @ W.T, x.abs() @ W.abs().T
    ng = W.shape[1] // 128
    tol = (ng + 8) * 2.0 ** -24 * mag + (BF if bf else 0) * want.abs()
    err = (Y.cpu().to(F64) - want).abs()
    assert (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("M,d_out,d_in,g", LINEAR)
def test_linear_a8(catq, M, d_out, d_in, g):
    q, packed, alpha, xs = _linear_inputs(M, d_out, d_in, g, M + d_out)
    dq, dp, da, dxs = q.cuda(), packed.cuda(), alpha.cuda(), xs.cuda()
    for dt in (torch.float32, torch.bfloat16):
        Y = torch.full((M, d_out), 7.0, dtype=dt, device="cuda")
        catq.catq_ternary_linear_a8(dq, dxs, dp, da, Y, g=g)
        _linear_check(Y, q, packed, alpha, xs, g, dt == torch.bfloat16)
        Z = torch.empty_like(Y)
        catq.catq_ternary_linear_a8(dq, dxs, dp, da, Z, g=g)
        assert torch.equal(Y, Z)


@pytest.mark.parametrize("M,d_out,d_in,g", [
    (3, 4111, 2176, 128), (3, 8203, 5248, 128), (13, 8203, 5248, 128), (21, 4111, 2176, 128), (33, 34001, 896, 128),
    (45, 16421, 2176, 128), (45, 16421, 2304, 256), (1000, 16421, 128, 128), (257, 16421, 896, 128),
    (500, 8203, 2176, 128), (1000, 4111, 2304, 256), (4090, 4111, 896, 128), (8200, 2049, 768, 256)])
def test_linear_a8_many_rows(catq, M, d_out, d_in, g):
    """The launch shapes for many rows, the last tile of rows and of tokens cut off, strided; the rows
    behind as they were."""
    q, packed, alpha, xs = _linear_inputs(M, d_out, d_in, g, M + d_out)
    wide = torch.full((M, d_in + 16), 77, dtype=torch.int8, device="cuda")
    wide[:, :d_in] = q.cuda()
    out = torch.full((M + 1, d_out + 3), 5.0, device="cuda")
    catq.catq_ternary_linear_a8(wide[:, :d_in], xs.cuda(), packed.cuda(), alpha.cuda(), out[:M, :d_out],
                              g=g)
    _linear_check(out[:M, :d_out], q, packed, alpha, xs, g, False)
    assert (out[:, d_out:] == 5.0).all() and (out[M] == 5.0).all()


@pytest.mark.parametrize("M", [3, 20, 150])
def test_linear_a8_strided_rows(catq, M):
    d_out, d_in = 70, 512
    q, packed, alpha, xs = _linear_inputs(M, d_out, d_in, 128, M)
    wide = torch.full((M, d_in + 48), 77, dtype=torch.int8, device="cuda")
    wide[:, :d_in] = q.cuda()
    out = torch.full((M, d_out + 9), 5.0, device="cuda")
    catq.catq_ternary_linear_a8(wide[:, :d_in], xs.cuda(), packed.cuda(), alpha.cuda(), out[:, :d_out])
    _linear_check(out[:, :d_out], q, packed, alpha, xs, 128, False)
    assert (out[:, d_out:] == 5.0).all()


@pytest.mark.parametrize("M,d_out,d_in", [(3, 100, 640), (33, 34001, 896), (70, 200, 640)])
def test_linear_a8_far_rows(catq, M, d_out, d_in):
    """Rows of activations 2^24 apart, the largest stride: offsets past 2^29."""
    q, packed, alpha, xs = _linear_inputs(M, d_out, d_in, 128, M + d_in)
    far = torch.empty((M, 1 << 24), dtype=torch.int8, device="cuda")[:, :d_in]
    far.copy_(q)
    out = torch.empty((M, d_out), device="cuda")
    catq.catq_ternary_linear_a8(far, xs.cuda(), packed.cuda(), alpha.cuda(), out)
    _linear_check(out, q, packed, alpha, xs, 128, False)


def test_linear_a8_extremes(catq):
    """Every code at its largest: the integer sums of a group do not overflow, and one
    group of 65536 is exact."""
    d_in = 65536
    q = torch.full((2, d_in), 127, dtype=torch.int8)
    q[1] = -127
    packed = torch.full((20, d_in // 4), 0xAA, dtype=torch.uint8)     # every T = +1
    alpha, xs = torch.ones((20, 1)), torch.ones(2)
    Y = torch.empty((2, 20), device="cuda")
    catq.catq_ternary_linear_a8(q.cuda(), xs.cuda(), packed.cuda(), alpha.cuda(), Y, g=d_in)
    assert (Y[0] == 127.0 * d_in).all() and (Y[1] == -127.0 * d_in).all()


# ------------------------------------------------------------------- the cache

class Serving:
    """A pool with stale contents, and sequences of (ctx, new) tokens on scattered pages."""

    def __init__(self, catq, seqs, n_q, n_kv, d, ps, bt, seed=0, spare=2, extra_rows=0, extra_pages=1):
        g = self.g = _gen(seed + ps * bt + d)
        self.catq, self.seqs, self.ps, self.bt = catq, seqs, ps, bt
        self.n_q, self.n_kv, self.d = n_q, n_kv, d
        need = [max(0, -(-(c + n) // ps)) for c, n in seqs]
        pages = sum(need) + spare
        width = max(need) + extra_pages
        perm = torch.randperm(pages, generator=g).to(torch.int32)
        self.table = torch.full((len(seqs), width), -1, dtype=torch.int32)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = perm[at:at + n]
            at += n
        self.cu = torch.tensor([0] + list(np.cumsum([n for _, n in seqs])), dtype=torch.int32)
        self.ctx = torch.tensor([c for c, _ in seqs], dtype=torch.int32)
        self.tokens = int(self.cu[-1]) + extra_rows
        self.max_new = max(n for _, n in seqs)
        self.max_len = max(max(c + n for c, n in seqs), 0)
        self.k = torch.randint(-127, 128, (pages, n_kv, ps, d), generator=g).to(torch.int8)
        self.v = torch.randint(-127, 128, (pages, n_kv, ps // 4, d, 4), generator=g).to(torch.int8)
        self.ks = (torch.rand((pages, n_kv, ps // bt), generator=g) + 0.5) / 60
        self.vs = (torch.rand((pages, n_kv, ps // bt), generator=g) + 0.5) / 60
        self.desc = catq.kv_desc(n_q, n_kv, d, ps, bt, pages, width)

    def upload(self):
        c = self.catq
        self.dev = [t.cuda() for t in (self.k, self.v, self.ks, self.vs)]
        self.cache = c.kv_cache(self.desc, *self.dev)
        self.batch = c.kv_batch(self.desc, self.table.cuda(), self.cu.cuda(), self.ctx.cuda(), self.tokens,
                                self.max_new, self.max_len)
        return self

    def oracle(self):
        return ref.Cache(self.k, self.v, self.ks, self.vs, self.ps, self.bt)

    def download(self):
        return ref.Cache(*[t.cpu() for t in self.dev], self.ps, self.bt)


def _prep64(sv, x, ctx, inv, rot, inter, norm, qw, kw, rs):
    """[new][heads][d] float64 -> q, k, v as the append has them before rounding."""
    n_q, n_kv = sv.n_q, sv.n_kv
    x = x.to(F64)
    q, k, v = x.split([n_q, n_kv, n_kv], 1)
    if norm:
        q = q / (q.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
        k = k / (k.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
        q = q if qw is None else q * qw.to(F64)
        k = k if kw is None else k * kw.to(F64)
    q = torch.stack([ref.rotate(t, ctx + i, inv, rot, inter, rs) for i, t in enumerate(q)]) if len(q) else q
    k = torch.stack([ref.rotate(t, ctx + i, inv, rot, inter, rs) for i, t in enumerate(k)]) if len(k) else k
    return q, k, v


def _close_codes(now, oracle):
    """Codes: the nearest integer to the reference's quotient, up to the quotient's error where
    it is at a half (a value of half the largest in magnitude is 63.5 scales: such ties are no
    accident).  Scales: equal up to FP."""
    for w in (0, 1):
        got, want = now.scales[w], oracle.scales[w]
        fin = torch.isfinite(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert ((got - want).abs()[fin] <= FP * want[fin]).all()
        worst = float((now.codes[w] - oracle.quot[w]).abs().max())
        assert worst <= 0.5 + 127 * 2 * FP, worst


CACHE = [
    # seqs (ctx, new), n_q, n_kv, d, page, block, rot, interleaved, norm, a8, rope_scale
    ([(0, 1)], 2, 1, 64, 16, 16, 64, False, False, False, 1.0),
    ([(0, 16), (5, 3), (17, 1)], 4, 2, 64, 32, 16, 64, False, True, True, 1.0),
    ([(3, 1), (0, 40), (0, 0), (31, 2)], 4, 2, 128, 32, 32, 128, False, True, False, 1.0),
    ([(60, 9), (64, 64), (1, 1)], 5, 1, 128, 64, 64, 64, True, False, True, 1.0),
    ([(100, 60), (7, 130)], 8, 8, 128, 128, 128, 16, True, True, False, 1.25),
    ([(10, 7), (0, 1), (33, 30)], 6, 2, 64, 16, 1, 32, False, False, False, 1.0),
    ([(10, 7), (16, 17)], 4, 4, 256, 64, 1, 256, False, True, True, 1.0),
    ([(130, 40), (0, 5)], 4, 2, 256, 256, 128, 128, False, True, False, 0.5),
    ([(15, 2), (14, 4)], 16, 1, 64, 16, 16, 0, False, False, False, 1.0),
    ([(250, 20)], 40, 8, 128, 256, 64, 128, False, True, True, 1.0),
]


@pytest.mark.parametrize("case", CACHE, ids=[str(i) for i in range(len(CACHE))])
def test_append_and_read(catq, case):
    seqs, n_q, n_kv, d, ps, bt, rot, inter, norm, a8, rs = case
    sv = Serving(catq, seqs, n_q, n_kv, d, ps, bt, extra_rows=3)
    g = sv.g
    x = _rand(g, sv.tokens, n_q + 2 * n_kv, d)
    if len(seqs) > 1:       # one sequence's values small: its block's older tokens keep their scale
        x[int(sv.cu[-2]):] *= 0.05
    inv = (1e4 ** (-torch.arange(rot // 2) / max(rot // 2, 1))).float()
    qw, kw = (_rand(g, d), _rand(g, d)) if norm and d != 128 else (None, None)
    sv.upload()
    prep = catq.kv_prep(sv.desc, inv.cuda() if rot else None, rot_dim=rot, interleaved=inter, qk_norm=norm,
                        q_weight=None if qw is None else qw.cuda(),
                        k_weight=None if kw is None else kw.cuda(), act_quant=a8, rope_scale=rs)
    qkv = x.reshape(sv.tokens, -1).cuda()
    q_out = torch.full((sv.tokens, n_q * d), 3.0, dtype=torch.bfloat16, device="cuda")
    oracle = sv.oracle()
    catq.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, prep, qkv, q_out)
    first = [t.clone() for t in sv.dev]
    rows = int(sv.cu[-1])
    q_got = q_out.cpu()
    assert (q_got[rows:] == 3.0).all()            # rows of no sequence
    for i, (ctx, new) in enumerate(seqs):
        if new == 0:
            continue
        r0 = int(sv.cu[i])
        q, k, v = _prep64(sv, x[r0:r0 + new], ctx, inv, rot, inter, norm, qw, kw, rs)
        got = q_got[r0:r0 + new].to(F64).view(new, n_q, d)
        if a8:     # the nearest code to the value, as in _close_codes, and its bf16 rounding
            s = q.abs().amax(-1, keepdim=True) / 127
            worst = float(((got - q).abs() - (0.5 + 127 * 2 * FP) * s - BF * got.abs()).max())
            assert worst <= 0, worst
        else:
            big = q.abs().amax(-1, keepdim=True)
            assert ((got - q).abs() <= BF * q.abs() + 4 * FP * big).all()
        oracle.append(0, sv.table[i], ctx, k)
        oracle.append(1, sv.table[i], ctx, v)
    now = sv.download()
    _close_codes(now, oracle)
    # the same tokens again: nothing changes
    catq.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, prep, qkv, q_out)
    for a, b in zip(first, sv.dev):
        assert torch.equal(a, b)
    # read back everything that the cache holds of each sequence
    spans = [(0, max(0, c + n)) for c, n in seqs]
    cu = torch.tensor([0] + list(np.cumsum([n for _, n in spans])), dtype=torch.int32).cuda()
    zero = torch.zeros(len(seqs), dtype=torch.int32, device="cuda")
    total = int(cu[-1])
    rb = catq.kv_batch(sv.desc, sv.batch.tensors[0], cu, zero, total, max(n for _, n in spans), sv.max_len)
    ko, vo = (torch.full((total, n_kv * d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    catq.catq_aux_kv_read(sv.desc, sv.cache, rb, ko, vo)
    for w, out in ((0, ko), (1, vo)):
        out = out.cpu().view(total, n_kv, d)
        r = 0
        for i, (_, n) in enumerate(spans):
            for p in range(n):
                val = now.value(w, sv.table[i], p)
                assert torch.equal(out[r], val.float().bfloat16())
                r += 1
    only = torch.empty_like(ko)
    catq.catq_aux_kv_read(sv.desc, sv.cache, rb, k_out=only)
    assert torch.equal(only, ko)
    catq.catq_aux_kv_read(sv.desc, sv.cache, rb, v_out=only)
    assert torch.equal(only, vo)


def test_append_token_by_token(catq):
    """A block filled one token at a time, its scale growing on the way: every step as
    the reference has it, starting from what the cache held before that step."""
    n_q, n_kv, d, ps, bt = 2, 2, 64, 32, 32
    sv = Serving(catq, [(0, 40)], n_q, n_kv, d, ps, bt).upload()
    prep = catq.kv_prep(sv.desc)
    x = _rand(sv.g, 40, n_q + 2 * n_kv, d)
    x *= torch.linspace(0.2, 3, 40)[torch.randperm(40, generator=sv.g)][:, None, None].bfloat16()
    cu = torch.tensor([0, 1], dtype=torch.int32).cuda()
    q_out = torch.empty((1, n_q * d), dtype=torch.bfloat16, device="cuda")
    for t in range(40):
        before = sv.download()
        ctx = torch.tensor([t], dtype=torch.int32).cuda()
        b = catq.kv_batch(sv.desc, sv.batch.tensors[0], cu, ctx, 1, 1, 64)
        catq.catq_aux_kv_append(sv.desc, sv.cache, b, prep, x[t].reshape(1, -1).cuda(), q_out)
        assert torch.equal(q_out.cpu().view(n_q, d), x[t, :n_q])
        for w, part in ((0, x[t:t + 1, n_q:n_q + n_kv]), (1, x[t:t + 1, n_q + n_kv:])):
            before.append(w, sv.table[0], t, part.to(F64))
        _close_codes(sv.download(), before)


def test_append_far_positions(catq):
    """Angles at position 10^6: formed in float64, so as exact as at 0."""
    d, ps = 64, 256
    c = catq
    pages = 4
    pos = 999_999
    width = pos // ps + 2
    table = torch.full((1, width), -1, dtype=torch.int32)
    table[0, pos // ps] = 2
    table[0, pos // ps + 1] = 1
    desc = c.kv_desc(2, 1, d, ps, 16, pages, width)
    k = torch.zeros((pages, 1, ps, d), dtype=torch.int8, device="cuda")
    v = torch.zeros((pages, 1, ps // 4, d, 4), dtype=torch.int8, device="cuda")
    ks, vs = (torch.zeros((pages, 1, ps // 16), device="cuda") for _ in range(2))
    cache = c.kv_cache(desc, k, v, ks, vs)
    inv = (1e6 ** (-torch.arange(32) / 32)).float()
    batch = c.kv_batch(desc, table.cuda(), torch.tensor([0, 2], dtype=torch.int32).cuda(),
                       torch.tensor([pos], dtype=torch.int32).cuda(), 2, 2, pos + 2)
    x = _rand(_gen(4), 2, 4, d)
    q = torch.empty((2, 2 * d), dtype=torch.bfloat16, device="cuda")
    c.catq_aux_kv_append(desc, cache, batch, c.kv_prep(desc, inv.cuda(), rot_dim=d), x.view(2, -1).cuda(), q)
    for t in range(2):
        want = ref.rotate(x[t, :2].to(F64), pos + t, inv, d, False)
        err = (q[t].cpu().to(F64).view(2, d) - want).abs()
        assert (err <= BF * want.abs() + 4 * FP * want.abs().max()).all()


def test_pool_past_32_bits(catq):
    """Pages more than 2^32 bytes into the pool: the same as in a small one."""
    c, n_q, n_kv, d, ps, bt, width = catq, 16, 8, 128, 256, 16, 3
    i32 = dict(dtype=torch.int32, device="cuda")
    g = _gen(11)
    seqs = [(250, 200), (511, 1), (0, 40)]
    n = sum(s[1] for s in seqs)
    x = _rand(g, n, (n_q + 2 * n_kv) * d).cuda()
    old = _rand(g, 761, (n_q + 2 * n_kv) * d).cuda()
    inv = (1e4 ** (-torch.arange(64) / 64)).float().cuda()
    got = []
    for pages in (9, 20480):                             # 2^18 bytes each: 5 GB
        k = torch.empty((pages, n_kv, ps, d), dtype=torch.int8, device="cuda")
        v = torch.empty((pages, n_kv, ps // 4, d, 4), dtype=torch.int8, device="cuda")
        ks, vs = (torch.zeros((pages, n_kv, ps // bt), device="cuda") for _ in range(2))
        desc = c.kv_desc(n_q, n_kv, d, ps, bt, pages, width)
        cache, prep = c.kv_cache(desc, k, v, ks, vs), c.kv_prep(desc, inv, rot_dim=d, qk_norm=True)
        table = torch.arange(pages - 1, pages - 10, -1, **i32).view(3, width)
        first = c.kv_batch(desc, table, torch.tensor([0, 250, 761, 761], **i32), torch.zeros(3, **i32), 761, 511, 511)
        q = torch.empty((761, n_q * d), dtype=torch.bfloat16, device="cuda")
        c.catq_aux_kv_append(desc, cache, first, prep, old, q)
        out = [q]
        for part in ([0, 200, 201, 241], [0, 1, 2, 3]):      # tiles of many rows, single tokens
            b = c.kv_batch(desc, table, torch.tensor(part, **i32), torch.tensor([s[0] for s in seqs], **i32), part[-1],
                           max(part[i + 1] - part[i] for i in range(3)), 512)
            q, o = (torch.zeros((part[-1], n_q * d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            kv = [torch.zeros((part[-1], n_kv * d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            ws = torch.empty(max(1, c.catq_paged_attention_workspace_bytes(desc, b)), dtype=torch.uint8, device="cuda")
            c.catq_aux_kv_append(desc, cache, b, prep, x[:part[-1]].contiguous(), q)
            c.catq_aux_kv_read(desc, cache, b, *kv)
            c.catq_aux_paged_attention(desc, cache, b, q, o, ws)
            out += [q, o, *kv]
        got.append(out)
    assert pages * n_kv * ps * d > 2 ** 32
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)


def test_append_refuses_another_heads_preparation(catq):
    """Gains for heads of 64 values are not read as gains of 128."""
    sv = Serving(catq, [(0, 2)], 2, 1, 128, 16, 16).upload()
    small = catq.kv_desc(2, 1, 64, 16, 16, sv.desc.n_pages, sv.desc.max_pages)
    prep = catq.kv_prep(small, torch.ones(32, device="cuda"), rot_dim=64, qk_norm=True,
                        q_weight=torch.ones(64, dtype=torch.bfloat16, device="cuda"))
    x = torch.zeros((sv.tokens, 4 * 128), dtype=torch.bfloat16, device="cuda")
    q = torch.full((sv.tokens, 2 * 128), 3.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="heads of 64"):
        catq.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, prep, x, q)
    assert (q == 3.0).all()


def test_append_leaves_the_rest(catq):
    """Codes and scales that no new token touches keep their bits: older blocks, later
    tokens of the page, other pages, blocks of other heads."""
    sv = Serving(catq, [(21, 5), (64, 1)], 2, 2, 128, 64, 16).upload()
    before = [t.clone() for t in sv.dev]
    x = _rand(sv.g, 6, 6, 128, std=0.001)       # smaller than what the blocks hold: no scale grows
    q = torch.empty((6, 256), dtype=torch.bfloat16, device="cuda")
    catq.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, catq.kv_prep(sv.desc), x.view(6, -1).cuda(), q)
    k, v, ks, vs = [t.clone() for t in sv.dev]
    p0, p1 = int(sv.table[0, 0]), int(sv.table[1, 1])
    k[p0, :, 21:26] = before[0][p0, :, 21:26]
    k[p1, :, 0] = before[0][p1, :, 0]
    vt, bt = v.transpose(-1, -2).reshape(-1, 2, 64, 128).clone(), before[1].transpose(-1, -2).reshape(-1, 2, 64, 128)
    vt[p0, :, 21:26] = bt[p0, :, 21:26]
    vt[p1, :, 0] = bt[p1, :, 0]
    assert torch.equal(k, before[0]) and torch.equal(vt, bt)
    for s, b in ((ks, before[2]), (vs, before[3])):
        s[p1, :, 0] = b[p1, :, 0]               # a block of new tokens alone has a scale of its own
        assert torch.equal(s, b)


def test_append_non_finite(catq):
    """A NaN or an infinity makes its block NaN, and nothing else."""
    sv = Serving(catq, [(0, 40)], 1, 1, 64, 64, 16).upload()
    x = _rand(sv.g, 40, 3, 64)
    x[3, 2, 5] = float("nan")
    x[20, 1, 0] = float("inf")
    q = torch.empty((40, 64), dtype=torch.bfloat16, device="cuda")
    catq.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, catq.kv_prep(sv.desc), x.view(40, -1).cuda(), q)
    ko, vo = (torch.empty((40, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    catq.catq_aux_kv_read(sv.desc, sv.cache, sv.batch, ko, vo)
    assert torch.isnan(vo[:16]).all() and torch.isfinite(vo[16:].float()).all()
    assert torch.isnan(ko[16:32]).all() and torch.isfinite(torch.cat([ko[:16], ko[32:]]).float()).all()


def test_bad_device_values(catq):
    """Page ids, lengths and offsets that make no sense on the device: nothing out of
    bounds is touched, and what makes sense is done."""
    sv = Serving(catq, [(5, 4), (0, 6), (30, 3), (2, 2)], 4, 2, 64, 16, 16)
    sv.table[0, 0] = -7                       # positions 5..8 on no page
    sv.table[1, 0] = 10 ** 9
    sv.upload()
    before = [t.clone() for t in sv.dev]
    x = _rand(sv.g, 15, 8, 64)
    q = torch.full((15, 256), 3.0, dtype=torch.bfloat16, device="cuda")
    prep = catq.kv_prep(sv.desc)
    catq.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, prep, x.view(15, -1).cuda(), q)
    assert torch.equal(q.cpu().view(15, 4, 64), x[:, :4])
    o = torch.full_like(q, 3.0)
    lse = torch.zeros((15, 4), device="cuda")
    ws = torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)), dtype=torch.uint8,
                     device="cuda")
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q, o, ws, lse=lse)
    assert (o[:10] == 0).all() and torch.isneginf(lse[:10]).all()
    assert torch.isfinite(lse[10:]).all()
    ko = torch.full((15, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    catq.catq_aux_kv_read(sv.desc, sv.cache, sv.batch, k_out=ko)
    assert (ko[:10] == 0).all() and (ko[10:] != 0).any()
    # offsets past the rows, decreasing and negative ones; a negative and a huge length
    t, i32 = sv.batch.tensors[0], dict(dtype=torch.int32, device="cuda")
    for cu, ctx in (([0, 9, 4, 400, 12], [0, 0, 0, 0]), ([-5, 3, 3, 2 ** 31 - 1, -1], [0, 1, 2, 3]),
                    ([0, 4, 8, 12, 15], [-2 ** 31, -2, 2 ** 31 - 1, 2 ** 30])):
        b = catq.kv_batch(sv.desc, t, torch.tensor(cu, **i32), torch.tensor(ctx, **i32), 15, 6, 33)
        catq.catq_aux_kv_append(sv.desc, sv.cache, b, prep, x.view(15, -1).cuda(), q)
        catq.catq_aux_paged_attention(sv.desc, sv.cache, b, q, o, ws, lse=lse)
        catq.catq_aux_kv_read(sv.desc, sv.cache, b, k_out=ko)
    torch.cuda.synchronize()
    # pages of no sequence are as they were
    held = set(sv.table[sv.table >= 0].tolist()) & set(range(sv.desc.n_pages))
    for p in set(range(sv.desc.n_pages)) - held:
        for a, b in zip(sv.dev, before):
            assert torch.equal(a[p], b[p])


# -------------------------------------------------------------------- attention

ATTN = [
    # seqs (ctx, new), n_q, n_kv, d, page, block
    ([(0, 1)], 1, 1, 64, 16, 16), ([(0, 1), (15, 1), (16, 1), (31, 1)], 4, 2, 64, 16, 16),
    ([(300, 1), (7, 1), (1500, 1)], 5, 1, 128, 64, 32), ([(1000, 1)], 40, 8, 128, 32, 1),
    ([(700, 1), (1, 1)], 16, 4, 256, 128, 128), ([(90, 3), (0, 2), (513, 4)], 8, 2, 128, 16, 16),
    ([(60, 7), (0, 9), (0, 0), (255, 1)], 4, 2, 64, 64, 1), ([(0, 100), (37, 50)], 6, 2, 64, 32, 32),
    ([(0, 33), (200, 70)], 5, 1, 128, 64, 64), ([(20, 60)], 8, 1, 256, 256, 16),
    ([(1030, 130)], 2, 2, 128, 128, 16), ([(2500, 2), (31, 1)], 64, 1, 64, 16, 16),
    ([(100, 17), (3, 16)], 3, 3, 128, 16, 1),
]


def _attention_check(o, lse, sv, q, oracle, scale=None):
    """Scores: d products and 16 more roundings of fp32 (scaling, the sum with log2 of the v
    scale of up to 128 in magnitude, exponentials), so they are off by at most e.  o: each
    probability off by e and its rounding to fp16, 2^-11, or 2^-25 of the largest term where
    it is subnormal there (times a code of up to 127); the sum of them by e; half a bf16 step."""
    scale = sv.d ** -0.5 if scale is None else scale
    for i, (ctx, new) in enumerate(sv.seqs):
        if new == 0:
            continue
        r0 = int(sv.cu[i])
        qi = q[r0:r0 + new].to(F64).view(new, sv.n_q, sv.d)
        want, wl, mag, big, top = ref.attention(qi, oracle, sv.table[i], ctx, scale, sv.n_kv)
        got = o[r0:r0 + new].cpu().to(F64).view(want.shape)
        e = ((sv.d + 16) * big + 144) * 2.0 ** -24
        tol = BF * want.abs() + (2.0 ** -11 + 2 * e[..., None]) * mag + 127 * 2.0 ** -25 * top[..., None]
        assert ((got - want).abs() <= tol).all(), (i, float(((got - want).abs() - tol).max()))
        if lse is not None:
            gl = lse[r0:r0 + new].cpu().to(F64)
            none = torch.isneginf(wl)
            assert torch.equal(torch.isneginf(gl), none)
            assert ((gl - wl).abs() <= e + 2.0 ** -22 * wl.abs())[~none].all()


@pytest.mark.parametrize("case", ATTN, ids=[str(i) for i in range(len(ATTN))])
def test_attention(catq, case):
    seqs, n_q, n_kv, d, ps, bt = case
    sv = Serving(catq, seqs, n_q, n_kv, d, ps, bt, extra_rows=2).upload()
    q = _rand(sv.g, sv.tokens, n_q * d, std=2.0)
    rows = int(sv.cu[-1])
    ws = torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)), dtype=torch.uint8,
                     device="cuda")
    o = torch.full((sv.tokens, n_q * d), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((sv.tokens, n_q), 3.0, device="cuda")
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q.cuda(), o, ws, lse=lse)
    assert (o[rows:] == 3.0).all() and (lse[rows:] == 3.0).all()
    _attention_check(o, lse, sv, q, sv.oracle())
    again = torch.empty_like(o)
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q.cuda(), again, ws)
    assert torch.equal(again[:rows], o[:rows])


def _far_scales(catq, bt, new, lo, hi):
    sv = Serving(catq, [(500, new), (70, new)], 4, 2, 128, 64, bt)
    g = sv.g
    sv.vs *= 10.0 ** (torch.rand(sv.vs.shape, generator=g) * (hi - lo) + lo)
    sv.vs[torch.rand(sv.vs.shape, generator=g) < 0.2] = 0
    sv.ks[torch.rand(sv.ks.shape, generator=g) < 0.2] = 0
    sv.upload()
    q = _rand(g, sv.tokens, 4 * 128)
    q[0] *= 20
    q[-1] = 0
    ws = torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)), dtype=torch.uint8,
                     device="cuda")
    o = torch.empty((sv.tokens, 512), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((sv.tokens, 4), device="cuda")
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q.cuda(), o, ws, lse=lse, scale=0.05)
    return sv, q, o, lse


@pytest.mark.parametrize("bt", [1, 16, 64])
@pytest.mark.parametrize("new", [1, 40])
def test_attention_scales_far_apart(catq, bt, new):
    """V scales from below 2^-60 (they count as 0) to 1e9, zero ones, K scales of 0; sharp
    and flat rows."""
    sv, q, o, lse = _far_scales(catq, bt, new, -18, 10)
    oracle = sv.oracle()
    assert (oracle.scales[1] <= 2.0 ** 30).all()
    oracle.scales[1][oracle.scales[1] < 2.0 ** -60] = 0
    _attention_check(o, lse, sv, q, oracle, scale=0.05)


@pytest.mark.parametrize("bt", [1, 16, 64])
@pytest.mark.parametrize("new", [1, 40])
def test_attention_scales_past_the_range(catq, bt, new):
    """V scales from 1e-20 to 1e20: a row that sees one above 2^30 is NaN, the others are
    as the reference has them."""
    sv, q, o, lse = _far_scales(catq, bt, new, -20, 20)
    oracle = sv.oracle()
    oracle.scales[1][oracle.scales[1] < 2.0 ** -60] = 0
    for i, (ctx, n) in enumerate(sv.seqs):
        r0 = int(sv.cu[i])
        huge = torch.zeros(2, dtype=torch.bool)
        seen = []
        for p in range(ctx + n):
            page, tok = oracle.place(sv.table[i], p)
            huge |= oracle.scales[1][page, :, tok // bt] > 2.0 ** 30
            seen.append(huge.clone())
        bad = torch.stack(seen)[ctx:].repeat_interleave(2, 1)          # [new][n_q]
        got = o[r0:r0 + n].cpu().view(n, 4, 128)
        assert torch.isnan(got[bad]).all() and torch.isfinite(got[~bad].float()).all()
        assert torch.equal(torch.isnan(lse[r0:r0 + n].cpu()), bad)


@pytest.mark.parametrize("bt", [1, 32])
@pytest.mark.parametrize("new", [1, 20, 300])
def test_attention_tiny_scales_count_as_zero(catq, bt, new):
    """Below 2^-60 a v scale is 0, whatever its codes are: the output is exactly 0, and so is it
    where the others' tokens are far below it."""
    sv = Serving(catq, [(40, new)], 2, 1, 128, 64, bt)
    sv.vs[:] = 2.0 ** -61
    sv.upload()
    q = _rand(sv.g, new, 256)
    ws = torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)), dtype=torch.uint8,
                     device="cuda")
    o = torch.empty((new, 256), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((new, 2), device="cuda")
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q.cuda(), o, ws, lse=lse)
    assert (o == 0).all() and torch.isfinite(lse).all()


def test_attention_masked_contents_do_not_count(catq):
    """NaN and infinite scales at positions that a row does not see, and on a page that is
    not the sequence's, change nothing; one that a row sees reaches that row."""
    for bt in (1, 16):
        sv = Serving(catq, [(20, 30)], 2, 1, 64, 64, bt, extra_pages=2)
        q = _rand(sv.g, 30, 128)
        oracle = sv.oracle()
        page = int(sv.table[0, 0])
        other = [p for p in range(sv.desc.n_pages) if p != page]
        for s in (sv.ks, sv.vs):
            s[other] = float("nan")
            s[page, :, 50 // bt + (50 % bt > 0):] = float("inf")
        sv.upload()
        ws = torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)),
                         dtype=torch.uint8, device="cuda")
        o = torch.empty((30, 128), dtype=torch.bfloat16, device="cuda")
        catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q.cuda(), o, ws)
        if bt == 1:
            _attention_check(o, None, sv, q, oracle)
            sv.dev[3][page, 0, 40] = float("nan")       # rows from 20 on see position 40
            catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q.cuda(), o, ws)
            assert torch.isfinite(o[:20].float()).all() and torch.isnan(o[20:]).all()
        else:
            assert torch.isfinite(o[:28].float()).all()


@pytest.mark.parametrize("new,heads,d", [(1, 2, 64), (9, 2, 128), (30, 2, 128), (90, 2, 64), (200, 2, 128)])
def test_attention_non_finite_queries(catq, new, heads, d):
    """A query row of NaN or infinities changes no other row, in no form of the kernel."""
    sv = Serving(catq, [(700, new), (33, new)], heads, 1, d, 32, 16).upload()
    q = _rand(sv.g, sv.tokens, heads * d).cuda()
    ws = torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)), dtype=torch.uint8,
                     device="cuda")
    o, o2 = (torch.empty((sv.tokens, heads * d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q, o, ws)
    q2 = q.clone()
    q2[new // 2, :d] = float("nan")
    q2[new, d:] = float("inf")
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q2, o2, ws)
    touched = torch.zeros((sv.tokens, heads), dtype=torch.bool, device="cuda")
    touched[new // 2, 0] = touched[new, 1] = True
    rows, rows2 = o.view(-1, heads, d), o2.view(-1, heads, d)
    assert torch.isnan(rows2[new // 2, 0]).all()
    assert torch.equal(rows2[~touched], rows[~touched])


def test_workspace_and_streams(catq):
    """A workspace that is too small is refused; a call on another stream than the
    tensors' gives the same."""
    sv = Serving(catq, [(3000, 1)], 8, 2, 128, 64, 64).upload()
    q = _rand(sv.g, 1, 1024).cuda()
    need = catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)
    assert need > 0
    o, p = torch.empty_like(q), torch.empty_like(q)
    for ws in (None, torch.empty(need - 1, dtype=torch.uint8, device="cuda")):
        with pytest.raises(catq.CatqError) as e:
            catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q, o, ws)
        assert e.value.status == 6
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q, o, ws)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    catq.catq_aux_paged_attention(sv.desc, sv.cache, sv.batch, q, p, ws, stream=st.cuda_stream)
    st.synchronize()
    assert torch.equal(o, p)


# --------------------------------------------------------------- all of them together

def test_a_block_served(catq):
    """A W1.58A8 decoder block's attention half as it is served: norm and codes, the q|k|v
    product on the 2-bit storage, the append, the attention, the output's codes and the o
    product; a prompt in two chunks and then single tokens, against the same block in float64
    whose codes are the kernels' own at every step; and the single-token step captured into
    a graph whose lengths are moved on the device between replays."""
    g = _gen(11)
    h, n_q, n_kv, d, ps, bt, total = 256, 4, 2, 64, 16, 16, 60
    N = (n_q + 2 * n_kv) * d
    pk = lambda o, i: torch.randint(0, 256, (o, i // 4), generator=g).to(torch.uint8)   # noqa: E731
    al = lambda o, i: torch.rand((o, i // 128), generator=g) * 0.1                      # noqa: E731
    wq, aq, wo, ao = pk(N, h), al(N, h), pk(h, n_q * d), al(h, n_q * d)
    Wq, Wo = ref.ternary(wq, aq, 128), ref.ternary(wo, ao, 128)
    x = _rand(g, total, h, dtype=torch.float32)
    inv = (1e4 ** (-torch.arange(d // 2) / (d // 2))).float()
    width = 5
    table = torch.tensor([[3, 0, 6, 1, 5]], dtype=torch.int32)
    desc = catq.kv_desc(n_q, n_kv, d, ps, bt, 7, width)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = [torch.zeros((7, n_kv, ps, d), dtype=torch.int8, device="cuda"),
            torch.zeros((7, n_kv, ps // 4, d, 4), dtype=torch.int8, device="cuda"),
            torch.zeros((7, n_kv, 1), device="cuda"), torch.zeros((7, n_kv, 1), device="cuda")]
    cache = catq.kv_cache(desc, *pool)
    prep = catq.kv_prep(desc, inv.cuda(), rot_dim=d, qk_norm=True, act_quant=True)
    dev = [t.cuda() for t in (wq, aq, wo, ao)]

    class Step:
        def __init__(self, n):
            e = lambda *s, **k: torch.empty(s, device="cuda", **k)   # noqa: E731
            self.n, b = n, torch.bfloat16
            self.x, self.qx, self.sx = e(n, h), e(n, h, dtype=torch.int8), e(n, 1)
            self.res, self.qkv, self.q = e(n, h), e(n, N, dtype=b), e(n, n_q * d, dtype=b)
            self.o, self.qo, self.so = e(n, n_q * d, dtype=b), e(n, n_q * d, dtype=torch.int8), e(n, 1)
            self.y = e(n, h)
            self.ctx = torch.zeros(1, **i32)
            self.batch = catq.kv_batch(desc, table.cuda(), torch.tensor([0, n], **i32), self.ctx, n, n, 80)
            self.ws = torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(desc, self.batch)),
                                  dtype=torch.uint8, device="cuda")

        def run(self):
            catq.catq_aux_rmsnorm_quant(self.x, self.qx, self.sx)
            catq.catq_ternary_linear_a8(self.qx, self.sx, dev[0], dev[1], self.qkv)
            catq.catq_aux_kv_append(desc, cache, self.batch, prep, self.qkv, self.q)
            catq.catq_aux_paged_attention(desc, cache, self.batch, self.q, self.o, self.ws)
            catq.catq_aux_act_quant8(self.o, self.qo, self.so)
            catq.catq_ternary_linear_a8(self.qo, self.so, dev[2], dev[3], self.y)

        def check(self, ctx):
            n = self.n
            xs = x[ctx:ctx + n]
            _, xhat = ref.norm_xhat(xs, None, None, 1e-6, None)
            _codes_ok(self.qx.cpu().to(F64), xhat, self.sx.cpu().to(F64))
            _linear_check(self.qkv, self.qx.cpu(), wq, aq, self.sx.cpu().view(-1), 128, True)
            held = ref.Cache(*[t.cpu() for t in pool], ps, bt)
            seq = SimpleNamespace(seqs=[(ctx, n)], cu=[0], d=d, n_q=n_q, n_kv=n_kv, table=table)
            _attention_check(self.o, None, seq, self.q.cpu(), held)
            _codes_ok(self.qo.cpu().to(F64), self.o.cpu().to(F64), self.so.cpu().to(F64))
            _linear_check(self.y, self.qo.cpu(), wo, ao, self.so.cpu().view(-1), 128, False)

    at = 0
    for n in (33, 7):
        s = Step(n)
        s.x.copy_(x[at:at + n])
        s.ctx.fill_(at)
        s.run()
        s.check(at)
        at += n
    one = Step(1)
    eager = []
    start = [t.clone() for t in pool]
    for t in range(at, total):
        one.x.copy_(x[t:t + 1])
        one.ctx.fill_(t)
        one.run()
        one.check(t)
        eager.append(one.y.clone())
    for a, b in zip(pool, start):
        a.copy_(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.run()
    for t in range(at, total):
        one.x.copy_(x[t:t + 1])
        one.ctx.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(one.y, eager[t - at])
    # what the whole comes to: the block in float64 without any quantization is near
    held = ref.Cache(*[t.cpu() for t in pool], ps, bt)
    _, xh = ref.norm_xhat(x, None, None, 1e-6, None)
    qkv = (xh @ Wq.T).view(total, -1, d)
    sv = SimpleNamespace(n_q=n_q, n_kv=n_kv)
    q, k, v = _prep64(sv, qkv, 0, inv, d, False, True, None, None, 1.0)
    for p in range(total):
        kk = held.value(0, table[0], p)
        assert (kk - k[p]).norm() <= 0.03 * k[p].norm()
        vv = held.value(1, table[0], p)
        assert (vv - v[p]).norm() <= 0.05 * v[p].norm()
