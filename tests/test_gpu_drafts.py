"""Drafted tokens over the paged 8-bit cache against plain float64: the append of a tree, attention of a tree, pages
copied, accepted tokens moved to the front, and a run of them together.  Tolerances are those of the append and the
attention (the same sums); moved codes are right if they are the nearest integer to code * scale / new scale, a
quotient and a product of two roundings: within 127 * 2^-23 of a half either neighbour is."""
import math

import numpy as np
import pytest
import torch

import serving_ref as ref
from test_gpu_serving import BF, F64, FP, Serving, _close_codes, _gen, _prep64, _rand

pytestmark = pytest.mark.gpu


def _words(rows, max_new, words=None):
    """Truth values, one list per token, as int64 words [n][words]."""
    words = words or -(-max_new // 64) or 1
    out = torch.zeros((len(rows), words), dtype=torch.int64)
    for r, row in enumerate(rows):
        for j, b in enumerate(row):
            if b:
                w = int(out[r, j // 64]) & (1 << 64) - 1 | 1 << j % 64
                out[r, j // 64] = w - (1 << 64) if w >> 63 else w
    return out


def _trees(g, seqs, extra=0):
    """Random trees: parents, depths and masks (truth values) of all tokens."""
    depths, rows = [], []
    for _, n in seqs:
        d, m = [], []
        for j in range(n):
            p = int(torch.randint(-1, j, (1,), generator=g)) if j else -1
            if j and torch.rand((), generator=g) < 0.6:
                p = j - 1
            d.append(0 if p < 0 else d[p] + 1)
            m.append(([False] * n if p < 0 else list(m[p])))
            m[-1][j] = True
        depths += d
        rows += m
    return depths + [0] * extra, rows + [[] for _ in range(extra)]


def _tree_reference(q, oracle, table, ctx, rows, scale, n_kv):
    """As serving_ref.attention, row i seeing what is before ctx and its mask's new tokens."""
    new, n_q, d = q.shape
    o, ab = torch.zeros_like(q), torch.zeros_like(q)
    big, top = torch.zeros((new, n_q), dtype=F64), torch.zeros((new, n_q), dtype=F64)
    lse = torch.full((new, n_q), -math.inf, dtype=F64)
    ks, vs, sv, where = [], [], [], []
    for pos in range(max(0, ctx + new)):
        k = oracle.value(0, table, pos)
        if k is not None:
            ks.append(k)
            vs.append(oracle.value(1, table, pos))
            page, tok = oracle.place(table, pos)
            sv.append(oracle.scales[1][page, :, tok // oracle.bt])
            where.append(pos)
    if not ks:
        return o, lse, ab, big, top
    k, v, sv = torch.stack(ks), torch.stack(vs), torch.stack(sv)
    for i in range(new):
        seen = torch.tensor([p < ctx or rows[i][p - ctx] for p in where])
        if not seen.any():
            continue
        for h in range(n_q):
            kk, vv, ss = (t[seen, h // (n_q // n_kv)] for t in (k, v, sv))
            s = kk @ q[i, h] * scale
            lse[i, h] = torch.logsumexp(s, 0)
            p = (s - lse[i, h]).exp()
            o[i, h], ab[i, h] = p @ vv, p @ vv.abs()
            big[i, h] = (kk.abs() @ q[i, h].abs()).max() * scale
            top[i, h] = len(p) * (p * ss).max()
    return o, lse, ab, big, top


def _tree_check(o, lse, sv, q, oracle, rows, scale=None):
    scale = sv.d ** -0.5 if scale is None else scale
    for i, (ctx, new) in enumerate(sv.seqs):
        if new == 0:
            continue
        r0 = int(sv.cu[i])
        qi = q[r0:r0 + new].to(F64).view(new, sv.n_q, sv.d)
        want, wl, mag, big, top = _tree_reference(qi, oracle, sv.table[i], ctx, rows[r0:r0 + new], scale, sv.n_kv)
        got = o[r0:r0 + new].cpu().to(F64).view(want.shape)
        e = ((sv.d + 16) * big + 144) * 2.0 ** -24
        tol = BF * want.abs() + (2.0 ** -11 + 2 * e[..., None]) * mag + 127 * 2.0 ** -25 * top[..., None]
        assert ((got - want).abs() <= tol).all(), (i, float(((got - want).abs() - tol).max()))
        gl = lse[r0:r0 + new].cpu().to(F64)
        none = torch.isneginf(wl)
        assert torch.equal(torch.isneginf(gl), none)
        assert ((gl - wl).abs() <= e + 2.0 ** -22 * wl.abs())[~none].all()


def _workspace(catq, sv):
    return torch.empty(max(1, catq.catq_paged_attention_workspace_bytes(sv.desc, sv.batch)), dtype=torch.uint8,
                       device="cuda")


TREE = [
    # seqs (ctx, new), n_q, n_kv, d, page, block, random mask
    ([(0, 1)], 1, 1, 64, 16, 16, False), ([(0, 5), (15, 1), (16, 3), (31, 2)], 4, 2, 64, 16, 16, True),
    ([(300, 7), (7, 1), (1500, 4)], 5, 1, 128, 64, 32, False), ([(1000, 6)], 40, 8, 128, 32, 1, True),
    ([(700, 9), (1, 12)], 16, 4, 256, 128, 128, True), ([(0, 70), (61, 65), (0, 0), (63, 64)], 4, 2, 64, 64, 1, True),
    ([(62, 60), (200, 33)], 10, 2, 128, 64, 64, False), ([(0, 130), (129, 90)], 6, 2, 64, 32, 32, True),
    ([(1030, 130)], 2, 2, 128, 128, 16, False), ([(50, 200), (3, 1)], 8, 1, 128, 16, 1, True),
    ([(2500, 8), (31, 40)], 8, 1, 64, 16, 16, False), ([(20, 60)], 8, 1, 256, 256, 16, True),
]


@pytest.mark.parametrize("case", TREE, ids=[str(i) for i in range(len(TREE))])
def test_tree_attention(catq, case):
    seqs, n_q, n_kv, d, ps, bt, scattered = case
    sv = Serving(catq, seqs, n_q, n_kv, d, ps, bt, extra_rows=2).upload()
    _, rows = _trees(sv.g, seqs, extra=2)
    if scattered:       # any set of tokens, none among them
        rows = [[bool(torch.rand((), generator=sv.g) < 0.4) for _ in r] for r in rows]
        rows[0] = [False] * len(rows[0])
    words = 1 + -(-sv.max_new // 64)                     # more than needed, with bits set past the new tokens
    mask = _words([r + [True] * (64 * words - len(r)) for r in rows], sv.max_new, words)
    tree = catq.kv_tree(sv.batch, mask.cuda())
    q = _rand(sv.g, sv.tokens, n_q * d, std=2.0)
    n = int(sv.cu[-1])
    ws = _workspace(catq, sv)
    o = torch.full((sv.tokens, n_q * d), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((sv.tokens, n_q), 3.0, device="cuda")
    catq.catq_aux_tree_attention(sv.desc, sv.cache, sv.batch, tree, q.cuda(), o, ws, lse=lse)
    assert (o[n:] == 3.0).all() and (lse[n:] == 3.0).all()
    _tree_check(o, lse, sv, q, sv.oracle(), rows)
    again = torch.empty_like(o)
    catq.catq_aux_tree_attention(sv.desc, sv.cache, sv.batch, tree, q.cuda(), again, ws)
    assert torch.equal(again[:n], o[:n])


@pytest.mark.parametrize("bt,new,n_q", [(1, 6, 2), (1, 50, 4), (16, 6, 2), (16, 90, 4)])
def test_tree_unseen_contents(catq, bt, new, n_q):
    """What a row does not see may be anything: NaN and infinite scales, missing pages, the type's largest codes."""
    seqs = [(45, new), (0, new)]
    sv = Serving(catq, seqs, n_q, 1, 64, 16, bt)
    g = sv.g
    rows = [[j == i or (j < i and (i + j) % 3 == 0) for j in range(new)] for _ in seqs for i in range(new)]
    # of every sequence, tokens new/2 .. are seen by nobody; their pages are missing or poisoned
    half = -(-new // 2)
    rows = [[b and j < half for j, b in enumerate(r)] for r in rows]
    clean = Serving(catq, seqs, n_q, 1, 64, 16, bt)
    for i, (ctx, n) in enumerate(seqs):
        for pos in range(ctx + half, ctx + n):
            page, tok = int(sv.table[i, pos // 16]), pos % 16
            if (ctx + half) // 16 == pos // 16 and bt != 1:
                continue                                 # (its scale is a seen token's too)
            sv.ks[page, :, tok // bt] = (math.nan, math.inf, -math.inf)[pos % 3]
            sv.vs[page, :, tok // bt] = (math.inf, math.nan, math.nan)[pos % 3]
        last = (ctx + n - 1) // 16
        if last > (ctx + half) // 16:
            sv.table[i, last] = (-1, 10 ** 9)[i]
    q = _rand(g, sv.tokens, n_q * 64)
    out = []
    for s in (sv, clean):
        s.upload()
        o = torch.empty((s.tokens, n_q * 64), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((s.tokens, n_q), device="cuda")
        tree = catq.kv_tree(s.batch, _words(rows, new).cuda())
        catq.catq_aux_tree_attention(s.desc, s.cache, s.batch, tree, q.cuda(), o, _workspace(catq, s), lse=lse)
        out.append((o, lse))
    assert torch.isfinite(out[0][0].float()).all()
    _tree_check(*out[0], clean, q, clean.oracle(), rows)
    _tree_check(*out[1], clean, q, clean.oracle(), rows)
    # the rows from half on of the sequence without cached tokens see only what is before half
    empty = [i for i, r in enumerate(rows) if not any(r) and i >= new]
    assert (out[0][0][empty] == 0).all() and torch.isneginf(out[0][1][empty]).all()


def test_tree_odd_queries(catq):
    """A query with a NaN or an infinity is NaN where it sees a token, 0 where it sees none; the others are as ever."""
    sv = Serving(catq, [(0, 40)], 2, 1, 64, 16, 16).upload()
    rows = [[j <= i and i % 4 != 1 for j in range(40)] for i in range(40)]
    q = _rand(sv.g, 40, 128)
    bad = q.clone()
    bad[4, 3], bad[5, 70], bad[6, 0] = math.nan, math.inf, -math.inf
    tree = catq.kv_tree(sv.batch, _words(rows, 40).cuda())
    out = []
    for x in (q, bad):
        o, lse = torch.empty((40, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((40, 2), device="cuda")
        catq.catq_aux_tree_attention(sv.desc, sv.cache, sv.batch, tree, x.cuda(), o, _workspace(catq, sv), lse=lse)
        out.append(o.view(40, 2, 64).clone())
    a, b = out
    assert torch.isnan(b[4, 0]).all() and torch.isnan(b[6, 0]).all() and (b[5] == 0).all()
    b[4, 0], b[6, 0] = a[4, 0], a[6, 0]
    assert torch.equal(a, b)


DRAFT = [
    # seqs, n_q, n_kv, d, page, block, rot, interleaved, norm, a8
    ([(0, 1)], 2, 1, 64, 16, 16, 64, False, False, False),
    ([(0, 16), (5, 9), (17, 3)], 4, 2, 64, 32, 16, 64, False, True, True),
    ([(60, 70), (64, 33), (1, 0)], 5, 1, 128, 64, 64, 64, True, False, False),
    ([(100, 60), (7, 130)], 8, 8, 128, 128, 128, 16, True, True, False),
    ([(10, 7), (16, 17)], 4, 4, 256, 64, 1, 256, False, True, True),
    ([(15, 20)], 16, 1, 64, 16, 16, 0, False, False, False),
]


@pytest.mark.parametrize("case", DRAFT, ids=[str(i) for i in range(len(DRAFT))])
def test_append_tree(catq, case):
    seqs, n_q, n_kv, d, ps, bt, rot, inter, norm, a8 = case
    sv = Serving(catq, seqs, n_q, n_kv, d, ps, bt, extra_rows=2).upload()
    depths, _ = _trees(sv.g, seqs, extra=2)
    x = _rand(sv.g, sv.tokens, n_q + 2 * n_kv, d)
    inv = (1e4 ** (-torch.arange(rot // 2) / max(rot // 2, 1))).float()
    prep = catq.kv_prep(sv.desc, inv.cuda() if rot else None, rot_dim=rot, interleaved=inter, qk_norm=norm, act_quant=a8)
    qkv = x.reshape(sv.tokens, -1).cuda()
    q_out = torch.full((sv.tokens, n_q * d), 3.0, dtype=torch.bfloat16, device="cuda")
    oracle = sv.oracle()
    tree = catq.kv_tree(sv.batch, depth=torch.tensor(depths, dtype=torch.int32).cuda())
    catq.catq_aux_kv_append_tree(sv.desc, sv.cache, sv.batch, tree, prep, qkv, q_out)
    q_got = q_out.cpu()
    assert (q_got[int(sv.cu[-1]):] == 3.0).all()
    for i, (ctx, new) in enumerate(seqs):
        if new == 0:
            continue
        r0 = int(sv.cu[i])
        parts = [_prep64(sv, x[r0 + j:r0 + j + 1], ctx + depths[r0 + j], inv, rot, inter, norm, None, None, 1.0)
                 for j in range(new)]
        q, k, v = (torch.cat(t) for t in zip(*parts))
        got = q_got[r0:r0 + new].to(F64).view(new, n_q, d)
        if a8:
            s = q.abs().amax(-1, keepdim=True) / 127
            assert ((got - q).abs() <= (0.5 + 127 * 2 * FP) * s + BF * got.abs()).all()
        else:
            assert ((got - q).abs() <= BF * q.abs() + 4 * FP * q.abs().amax(-1, keepdim=True)).all()
        oracle.append(0, sv.table[i], ctx, k)
        oracle.append(1, sv.table[i], ctx, v)
    _close_codes(sv.download(), oracle)


def test_append_tree_of_a_chain(catq):
    """A chain, by its depths or without any, is the plain append bit for bit; so are far, equal and negative positions."""
    out = []
    for kind in range(3):
        sv = Serving(catq, [(21, 5), (130, 40)], 4, 2, 128, 64, 16).upload()
        x = _rand(sv.g, 45, 8 * 128).cuda()
        prep = catq.kv_prep(sv.desc, (1e4 ** (-torch.arange(64) / 64)).float().cuda(), rot_dim=128, qk_norm=True)
        q = torch.empty((45, 512), dtype=torch.bfloat16, device="cuda")
        depth = torch.tensor(list(range(5)) + list(range(40)), dtype=torch.int32).cuda()
        if kind == 0:
            catq.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, prep, x, q)
        else:
            tree = catq.kv_tree(sv.batch, depth=depth if kind == 1 else None)
            catq.catq_aux_kv_append_tree(sv.desc, sv.cache, sv.batch, tree, prep, x, q)
        out.append([q] + sv.dev)
    for a, b, c in zip(*out):
        assert torch.equal(a, b) and torch.equal(a, c)
    # one token at depth D behind c cached ones turns as one behind c + D
    got = []
    for ctx, depth in ((30, 2 ** 30), (2 ** 30 + 30 - 7, 7), (40, -10 + 2 ** 30)):
        sv = Serving(catq, [(30, 1)], 2, 1, 64, 16, 16).upload()
        x = _rand(sv.g, 1, 4 * 64).cuda()
        prep = catq.kv_prep(sv.desc, (1e4 ** (-torch.arange(32) / 32)).float().cuda(), rot_dim=64)
        b = catq.kv_batch(sv.desc, sv.batch.tensors[0], sv.batch.tensors[1],
                          torch.tensor([ctx], dtype=torch.int32).cuda(), 1, 1, sv.max_len)
        q = torch.empty((1, 128), dtype=torch.bfloat16, device="cuda")
        tree = catq.kv_tree(b, depth=torch.tensor([depth], dtype=torch.int32).cuda())
        catq.catq_aux_kv_append_tree(sv.desc, sv.cache, b, tree, prep, x, q)
        got.append(q)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_append_tree_of_a_long_chain(catq):
    """More new tokens than a mask has bits for: by their depths alone the append takes what the plain one takes."""
    n, out = 70001, []
    for kind in range(3):
        sv = Serving(catq, [(9, n)], 1, 1, 64, 256, 16).upload()
        x = _rand(_gen(2), n, 3 * 64).cuda()
        prep = catq.kv_prep(sv.desc, (1e4 ** (-torch.arange(32) / 32)).float().cuda(), rot_dim=64)
        q = torch.full((n, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        if kind == 0:
            catq.catq_aux_kv_append(sv.desc, sv.cache, sv.batch, prep, x, q)
        else:
            tree = catq.kv_tree(sv.batch, depth=torch.arange(n, dtype=torch.int32, device="cuda") if kind == 1 else None)
            catq.catq_aux_kv_append_tree(sv.desc, sv.cache, sv.batch, tree, prep, x, q)
        out.append([q] + sv.dev)
    for a, b, c in zip(*out):
        assert torch.equal(a, b) and torch.equal(a, c)


# ------------------------------------------------------------------------ pages

@pytest.mark.parametrize("n_kv,d,ps,bt", [(1, 64, 16, 16), (3, 64, 16, 1), (8, 128, 64, 16), (2, 256, 256, 128),
                                          (5, 128, 32, 1)])
def test_copy_pages(catq, n_kv, d, ps, bt):
    sv = Serving(catq, [(5, 1)], n_kv, n_kv, d, ps, bt, spare=12).upload()
    n = sv.desc.n_pages
    src = [0, 1, 0, 3, -1, n, 4, 2 ** 31 - 1, 5, 6]
    dst = [7, 8, 9, 3, 10, 11, -5, 11, n, 10]
    src, dst = src[:10], dst[:10]
    want = [t.clone() for t in sv.dev]
    for a, b in zip(src, dst):
        if 0 <= a < n and 0 <= b < n:
            for t, w in zip(sv.dev, want):
                w[b] = t[a]
    i32 = dict(dtype=torch.int32, device="cuda")
    catq.catq_aux_kv_copy_pages(sv.desc, sv.cache, torch.tensor(src, **i32), torch.tensor(dst, **i32))
    for t, w in zip(sv.dev, want):
        assert torch.equal(t, w)
    catq.catq_aux_kv_copy_pages(sv.desc, sv.cache, torch.empty(0, **i32), torch.empty(0, **i32))


def test_copy_pages_past_32_bits(catq):
    n_kv, ps, d, pages = 8, 256, 128, 20480
    k = torch.empty((pages, n_kv, ps, d), dtype=torch.int8, device="cuda")
    v = torch.empty((pages, n_kv, ps // 4, d, 4), dtype=torch.int8, device="cuda")
    ks, vs = (torch.zeros((pages, n_kv, ps // 16), device="cuda") for _ in range(2))
    for i, t in enumerate((k, v, ks, vs)):
        t[20000], t[3] = i + 1, i + 11
    desc = catq.kv_desc(8, n_kv, d, ps, 16, pages, 1)
    i32 = dict(dtype=torch.int32, device="cuda")
    catq.catq_aux_kv_copy_pages(desc, catq.kv_cache(desc, k, v, ks, vs), torch.tensor([20000, 3], **i32),
                                torch.tensor([5, 20479], **i32))
    for i, t in enumerate((k, v, ks, vs)):
        assert (t[5] == i + 1).all() and (t[20479] == i + 11).all() and (t[20000] == i + 1).all() and (t[3] == i + 11).all()


def _compact_reference(oracle, table, ctx, new, keep):
    """Moves in the plain cache, block by block from a copy; codes are left as quotients in ``quot``."""
    n = 0
    while n < len(keep) and 0 <= keep[n] < new and (n == 0 or keep[n] > keep[n - 1]):
        n += 1
    bt = oracle.bt
    for w in (0, 1):
        codes, scales = oracle.codes[w].clone(), oracle.scales[w].clone()
        i = max(0, -ctx)
        while i < n:
            pos = ctx + i
            m = min(bt - pos % bt, n - i)
            at = oracle.place(table, pos)
            if at is not None:
                page, tok = at
                b, t0 = tok // bt, tok // bt * bt
                src = [(page, t) for t in range(t0, tok)] if i == max(0, -ctx) else []
                src += [oracle.place(table, ctx + keep[i + j]) for j in range(m)]
                zero = torch.zeros(codes.shape[1], dtype=F64)
                sc = torch.stack([zero if s is None else scales[s[0], :, s[1] // bt] for s in src])
                cd = torch.stack([torch.zeros_like(codes[0, :, 0]) if s is None else codes[s[0], :, s[1]] for s in src])
                now = sc.amax(0)                          # (a NaN where there is one)
                r = torch.where(now > sc, (sc / now), torch.ones_like(sc))[..., None]
                first = tok + m - len(src)
                oracle.quot[w][page, :, first:tok + m] = (cd * r).movedim(0, 1)
                oracle.codes[w][page, :, first:tok + m] = torch.round(cd * r).movedim(0, 1)
                oracle.scales[w][page, :, b] = now
            i += m


def _moved_ok(now, oracle):
    for w in (0, 1):
        a, b = now.scales[w], oracle.scales[w]
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(), b.nan_to_num())
        err = (now.codes[w] - oracle.quot[w]).abs()
        assert (err <= 0.5 + 127 * 2.0 ** -23).all(), float(err.max())
        whole = oracle.quot[w] == oracle.quot[w].round()
        assert torch.equal(now.codes[w][whole], oracle.quot[w][whole])


COMPACT = [
    # seqs, n_kv, d, page, block, keep of each
    ([(0, 1)], 1, 64, 16, 16, [[0]]),
    ([(5, 9), (17, 3), (3, 4)], 2, 64, 32, 16, [[0, 3, 8], [2], []]),
    ([(60, 70), (64, 33), (1, 0)], 1, 128, 64, 64, [[0, 1, 2, 3, 4, 66, 69], list(range(33)), []]),
    ([(100, 60), (7, 130)], 3, 128, 128, 128, [[59], list(range(0, 130, 3))]),
    ([(10, 7), (16, 17)], 2, 256, 64, 1, [[1, 2, 6], [16]]),
    ([(0, 300), (33, 200)], 2, 64, 16, 16, [list(range(1, 300, 2)), list(range(100, 200))]),
    ([(0, 300)], 2, 128, 64, 1, [[i for i in range(300) if i % 7 != 3]]),
    ([(20, 100)], 1, 256, 256, 128, [[i for i in range(100) if i % 3]]),
    # many windows, pages and passes
    ([(77, 900), (0, 513)], 2, 128, 128, 32, [[i for i in range(900) if i % 5 != 1], list(range(513))]),
    ([(130, 700)], 1, 64, 256, 16, [list(range(350, 700))]),
    ([(3, 600)], 1, 256, 64, 1, [[i for i in range(600) if i % 2]]),
    ([(200, 600)], 1, 256, 128, 128, [[i for i in range(600) if i % 4 != 2]]),
    # lists that end early: repeated, falling, out of range
    ([(5, 9), (17, 8), (3, 4), (2, 6)], 2, 64, 32, 16, [[0, 3, 3, 8], [4, 2, 7], [-1, 2], [1, 6]]),
]


@pytest.mark.parametrize("case", COMPACT, ids=[str(i) for i in range(len(COMPACT))])
def test_compact(catq, case):
    seqs, n_kv, d, ps, bt, keeps = case
    sv = Serving(catq, seqs, n_kv, n_kv, d, ps, bt, extra_rows=1).upload()
    oracle = sv.oracle()
    keep = torch.full((sv.tokens,), 77, dtype=torch.int32)
    for i, kk in enumerate(keeps):
        r0 = int(sv.cu[i])
        keep[r0:r0 + len(kk)] = torch.tensor(kk, dtype=torch.int32)
        _compact_reference(oracle, sv.table[i], *seqs[i], kk)
    n_keep = torch.tensor([len(kk) for kk in keeps], dtype=torch.int32)
    catq.catq_aux_kv_compact(sv.desc, sv.cache, sv.batch, keep.cuda(), n_keep.cuda())
    _moved_ok(sv.download(), oracle)


def test_compact_odd_scales_and_pages(catq):
    """Scales of 0, NaN and infinity go with their tokens; tokens from missing pages come as zeros, to missing pages
    nothing is written; lengths and counts out of range do what they can."""
    seqs, bt, ps = [(10, 40), (0, 64), (5, 40), (14, 40)], 16, 16
    sv = Serving(catq, seqs, 2, 2, 64, ps, bt)
    g = sv.g
    for s in (sv.ks, sv.vs):
        s[torch.rand(s.shape, generator=g) < 0.3] = 0
        s[torch.rand(s.shape, generator=g) < 0.1] = math.inf
        s[torch.rand(s.shape, generator=g) < 0.1] = math.nan
    sv.table[2, 1] = -1                        # a source page that is not there
    sv.table[3, 1] = 10 ** 8                   # nor is a destination
    sv.upload()
    oracle = sv.oracle()
    keeps = [list(range(0, 40, 2)), list(range(3, 60, 5)), list(range(12, 40, 4)), list(range(4, 34))]
    keep = torch.zeros(sv.tokens, dtype=torch.int32)
    for i, kk in enumerate(keeps):
        keep[int(sv.cu[i]):int(sv.cu[i]) + len(kk)] = torch.tensor(kk, dtype=torch.int32)
        _compact_reference(oracle, sv.table[i], *seqs[i], kk)
    n_keep = torch.tensor([len(kk) for kk in keeps], dtype=torch.int32).cuda()
    catq.catq_aux_kv_compact(sv.desc, sv.cache, sv.batch, keep.cuda(), n_keep)
    _moved_ok(sv.download(), oracle)
    i32 = dict(dtype=torch.int32, device="cuda")
    held = set(sv.table[(sv.table >= 0) & (sv.table < sv.desc.n_pages)].tolist())
    before = [t.clone() for t in sv.dev]
    for cu, ctx, nk in (([0, 9, 4, 400, 12], [0, 0, 0, 0], [99, -3, 2 ** 31 - 1, 5]),
                        ([-5, 3, 3, 2 ** 31 - 1, -1], [0, 1, 2, 3], [5, 5, 5, 5]),
                        ([0, 40, 104, 144, 184], [-2 ** 31, -20, 2 ** 31 - 1, 2 ** 30], [40, 40, 40, 40])):
        b = catq.kv_batch(sv.desc, sv.batch.tensors[0], torch.tensor(cu, **i32), torch.tensor(ctx, **i32), sv.tokens,
                          64, 64)
        catq.catq_aux_kv_compact(sv.desc, sv.cache, b, keep.cuda(), torch.tensor(nk, **i32))
    torch.cuda.synchronize()
    for p in set(range(sv.desc.n_pages)) - held:
        for a, b in zip(sv.dev, before):
            assert torch.equal(a[p].nan_to_num(), b[p].nan_to_num())


# --------------------------------------------------------------------- together

def test_a_verified_draft_is_the_plain_sequence(catq):
    """Drafted trees appended, attended, forked and compacted to their accepted paths hold, with a scale per token,
    exactly what a plain append of the paths holds, and their rows' attention is that of the path alone."""
    n_q, n_kv, d, ps = 4, 2, 128, 16
    seqs = [(37, 24), (0, 9), (16, 31)]
    sv = Serving(catq, seqs, n_q, n_kv, d, ps, 1, spare=24, extra_pages=2).upload()
    depths, rows = _trees(sv.g, seqs)
    x = _rand(sv.g, sv.tokens, (n_q + 2 * n_kv) * d)
    prep = catq.kv_prep(sv.desc, (1e4 ** (-torch.arange(64) / 64)).float().cuda(), rot_dim=d, qk_norm=True)
    tree = catq.kv_tree(sv.batch, _words(rows, sv.max_new).cuda(), torch.tensor(depths, dtype=torch.int32).cuda())
    q = torch.empty((sv.tokens, n_q * d), dtype=torch.bfloat16, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((sv.tokens, n_q), device="cuda")
    catq.catq_aux_kv_append_tree(sv.desc, sv.cache, sv.batch, tree, prep, x.cuda(), q)
    catq.catq_aux_tree_attention(sv.desc, sv.cache, sv.batch, tree, q, o, _workspace(catq, sv), lse=lse)
    # the deepest token's path of every sequence
    keep, n_keep, paths = torch.zeros(sv.tokens, dtype=torch.int32), [], []
    for i, (_, n) in enumerate(seqs):
        r0 = int(sv.cu[i])
        leaf = max(range(n), key=lambda j: depths[r0 + j])
        path = [j for j in range(n) if rows[r0 + leaf][j]]
        keep[r0:r0 + len(path)] = torch.tensor(path, dtype=torch.int32)
        n_keep.append(len(path))
        paths.append([r0 + j for j in path])
    # forks: the pages from ctx on are copied to free ones first
    fork, free = sv.table.clone(), sorted(set(range(sv.desc.n_pages)) - set(sv.table.flatten().tolist()))
    src, dst = [], []
    for i, (ctx, n) in enumerate(seqs):
        for p in range(ctx // ps, -(-(ctx + n) // ps)):
            src.append(int(fork[i, p]))
            dst.append(free.pop())
            fork[i, p] = dst[-1]
    i32 = dict(dtype=torch.int32, device="cuda")
    untouched = [t.clone() for t in sv.dev]
    catq.catq_aux_kv_copy_pages(sv.desc, sv.cache, torch.tensor(src, **i32), torch.tensor(dst, **i32))
    fb = catq.kv_batch(sv.desc, fork.cuda(), sv.batch.tensors[1], sv.batch.tensors[2], sv.tokens, sv.max_new, sv.max_len)
    catq.catq_aux_kv_compact(sv.desc, sv.cache, fb, keep.cuda(), torch.tensor(n_keep, **i32))
    for a, b in zip(sv.dev, untouched):
        for p in set(sv.table[sv.table >= 0].tolist()):
            assert torch.equal(a[p], b[p])
    # the plain sequence: the paths alone
    chain = Serving(catq, [(c, m) for (c, _), m in zip(seqs, n_keep)], n_q, n_kv, d, ps, 1)
    for i, (ctx, _) in enumerate(seqs):                  # (the same cached tokens before)
        for p in range(-(-ctx // ps)):
            for a, b in zip((chain.k, chain.v, chain.ks, chain.vs), (sv.k, sv.v, sv.ks, sv.vs)):
                a[int(chain.table[i, p])] = b[int(sv.table[i, p])]
    chain.upload()
    order = [r for p in paths for r in p]
    qc = torch.empty((len(order), n_q * d), dtype=torch.bfloat16, device="cuda")
    oc, lc = torch.empty_like(qc), torch.empty((len(order), n_q), device="cuda")
    catq.catq_aux_kv_append(chain.desc, chain.cache, chain.batch, prep, x[order].cuda(), qc)
    catq.catq_aux_paged_attention(chain.desc, chain.cache, chain.batch, qc, oc, _workspace(catq, chain), lse=lc)
    assert torch.equal(qc, q[order])
    back = []
    for s, table in ((sv, fork), (chain, chain.table)):
        cu = torch.tensor([0] + list(np.cumsum([c + m for (c, _), m in zip(seqs, n_keep)])), **i32)
        b = catq.kv_batch(s.desc, table.cuda(), cu, torch.zeros(3, **i32), int(cu[-1]), 64, 64)
        kv = [torch.empty((int(cu[-1]), n_kv * d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        catq.catq_aux_kv_read(s.desc, s.cache, b, *kv)
        back.append(kv)
    for a, b in zip(*back):
        assert torch.equal(a, b)
    # (both within the attention's error of the same numbers)
    _tree_check(o, lse, sv, q.cpu(), _held_before(sv, untouched), rows)
    assert (o[order].float() - oc.float()).abs().max() <= 2 * (2 * BF) * o.float().abs().max()
    assert (lse[order] - lc).abs().max() <= 1e-3


def _held_before(sv, dev):
    return ref.Cache(*[t.cpu() for t in dev], sv.ps, sv.bt)


def test_drafts_captured_and_on_another_stream(catq):
    """A captured step replayed with new contents between the replays is the eager step every time."""
    n_q, n_kv, d, ps, bt = 8, 2, 64, 16, 16
    seqs = [(900, 12), (3, 5)]
    sv = Serving(catq, seqs, n_q, n_kv, d, ps, bt, spare=8).upload()
    depths, rows = _trees(sv.g, seqs)
    mask, depth = _words(rows, sv.max_new).cuda(), torch.tensor(depths, dtype=torch.int32).cuda()
    tree = catq.kv_tree(sv.batch, mask, depth)
    prep = catq.kv_prep(sv.desc, (1e4 ** (-torch.arange(32) / 32)).float().cuda(), rot_dim=d, act_quant=True)
    qkv = torch.empty((sv.tokens, (n_q + 2 * n_kv) * d), dtype=torch.bfloat16, device="cuda")
    q = torch.empty((sv.tokens, n_q * d), dtype=torch.bfloat16, device="cuda")
    o, lse, ws = torch.empty_like(q), torch.empty((sv.tokens, n_q), device="cuda"), _workspace(catq, sv)
    i32 = dict(dtype=torch.int32, device="cuda")
    free = sorted(set(range(sv.desc.n_pages)) - set(sv.table.flatten().tolist()))[:2]
    src, dst = torch.tensor([int(sv.table[0, 56]), int(sv.table[1, 0])], **i32), torch.tensor(free, **i32)
    keep = torch.zeros(sv.tokens, **i32)
    keep[:3] = torch.tensor([1, 5, 11], **i32)
    n_keep = torch.tensor([3, 1], **i32)

    def step(stream=None):
        catq.catq_aux_kv_append_tree(sv.desc, sv.cache, sv.batch, tree, prep, qkv, q, stream=stream)
        catq.catq_aux_tree_attention(sv.desc, sv.cache, sv.batch, tree, q, o, ws, lse=lse, stream=stream)
        catq.catq_aux_kv_copy_pages(sv.desc, sv.cache, src, dst, stream=stream)
        catq.catq_aux_kv_compact(sv.desc, sv.cache, sv.batch, keep, n_keep, stream=stream)

    first = [t.clone() for t in sv.dev]
    inputs = [_rand(sv.g, *qkv.shape).cuda() for _ in range(3)]
    want = []
    for x in inputs:
        for a, b in zip(sv.dev, first):
            a.copy_(b)
        qkv.copy_(x)
        step()
        want.append([t.clone() for t in (q, o, lse, *sv.dev)])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in (0, 1, 2, 0):
        for a, b in zip(sv.dev, first):
            a.copy_(b)
        qkv.copy_(inputs[n])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((q, o, lse, *sv.dev), want[n]):
            assert torch.equal(a, b)
    side = torch.cuda.Stream()
    for a, b in zip(sv.dev, first):
        a.copy_(b)
    qkv.copy_(inputs[1])
    side.wait_stream(torch.cuda.current_stream())
    step(side.cuda_stream)
    side.synchronize()
    for a, b in zip((q, o, lse, *sv.dev), want[1]):
        assert torch.equal(a, b)
