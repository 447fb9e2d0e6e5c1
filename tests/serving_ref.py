"""Plain float64 versions of the serving operators (CPU tensors, one value at a
time where that is the clearest), used by the tests only."""
import math

import torch

F64 = torch.float64


def quant8(x, s):
    """rne(x / s) within +-127, 0 where s is 0."""
    q = torch.round(x / torch.where(s > 0, s, torch.ones_like(s))).clamp(-127, 127)
    return torch.where(s > 0, q, torch.zeros_like(q))


def norm_xhat(x, res, weight, eps, r_dtype):
    h = x.to(F64)
    if res is not None:
        h = (x.float() + res.float()).to(r_dtype).to(F64)
    n = h / (h.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    return h, n if weight is None else n * weight.to(F64)


def unpack(packed):
    c = torch.stack([(packed >> (2 * j)) & 3 for j in range(4)], -1).flatten(-2)
    return torch.tensor([-1, 0, 1, 0], dtype=F64)[c.long()]


def ternary(packed, alpha, g):
    return unpack(packed) * alpha.to(F64).reshape(packed.shape[0], -1).repeat_interleave(g, 1)


def rotate(x, pos, inv_freq, rot, inter, scale=1.0):
    """One head vector (or a stack of them) at position ``pos``."""
    if rot == 0:
        return x.clone()
    y = x.clone()
    a = pos * inv_freq.to(F64)
    c, s = a.cos() * scale, a.sin() * scale
    i = torch.arange(rot // 2)
    i0, i1 = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
    y[..., i0] = x[..., i0] * c - x[..., i1] * s
    y[..., i1] = x[..., i1] * c + x[..., i0] * s
    return y


class Cache:
    """The pool in a plain layout: codes float64 [2][page][head][token][d], scales
    [2][page][head][block]; ``quot`` holds what each code was rounded from."""

    def __init__(self, k, v, ks, vs, ps, bt):
        self.ps, self.bt = ps, bt
        p, h, _, d = k.shape
        self.codes = [k.to(F64).clone(), v.to(F64).transpose(-1, -2).reshape(p, h, ps, d).clone()]
        self.quot = [c.clone() for c in self.codes]
        self.scales = [ks.to(F64).clone(), vs.to(F64).clone()]

    def place(self, table, pos):
        if pos < 0 or pos >= len(table) * self.ps:
            return None
        page = int(table[pos // self.ps])
        return (page, pos % self.ps) if 0 <= page < self.codes[0].shape[0] else None

    def append(self, which, table, ctx, x):
        """x [new][head][d] (float64) at positions ctx ..: block by block."""
        bt, new = self.bt, x.shape[0]
        i = max(0, -ctx)
        while i < new:
            pos = ctx + i
            n = min(bt - pos % bt, new - i)
            at = self.place(table, pos)
            if at is not None:
                page, tok = at
                for h in range(x.shape[1]):
                    vals = x[i:i + n, h]
                    s = (vals.abs().max() / 127).float().to(F64)
                    if not torch.isfinite(vals).all():
                        s = torch.tensor(math.nan, dtype=F64)
                    b, t0 = tok // bt, tok // bt * bt
                    if tok % bt:
                        was = self.scales[which][page, h, b]
                        if s > was:
                            r = (was.float() / s.float()).to(F64)
                            c = self.codes[which][page, h, t0:tok]
                            self.quot[which][page, h, t0:tok] = c * r
                            self.codes[which][page, h, t0:tok] = torch.round(c * r)
                        elif not torch.isnan(s):
                            s = was.clone()
                    self.scales[which][page, h, b] = s
                    q = torch.zeros_like(vals) if torch.isnan(s) else quant8(vals, s)
                    self.codes[which][page, h, tok:tok + n] = q
                    self.quot[which][page, h, tok:tok + n] = vals / s if s > 0 else q
            i += n

    def value(self, which, table, pos):
        """[head][d] of a position, or None where its page does not exist."""
        at = self.place(table, pos)
        if at is None:
            return None
        page, tok = at
        return self.codes[which][page, :, tok] * self.scales[which][page, :, tok // self.bt, None]


def attention(q, cache, table, ctx, scale, n_kv):
    """q [new][n_q][d] of one sequence -> o, lse and, for tolerances, sum_j p_j |v_j|, the
    largest sum of magnitudes behind a score, and n * max_j p_j * v_scale_j."""
    new, n_q, d = q.shape
    o = torch.zeros_like(q)
    ab = torch.zeros_like(q)
    big = torch.zeros((new, n_q), dtype=F64)
    top = torch.zeros((new, n_q), dtype=F64)
    lse = torch.full((new, n_q), -math.inf, dtype=F64)
    ks, vs, sv, where = [], [], [], []
    for pos in range(max(0, ctx + new)):
        k = cache.value(0, table, pos)
        if k is not None:
            ks.append(k)
            vs.append(cache.value(1, table, pos))
            page, tok = cache.place(table, pos)
            sv.append(cache.scales[1][page, :, tok // cache.bt])
            where.append(pos)
    if not ks:
        return o, lse, ab, big, top
    k, v, sv, where = torch.stack(ks), torch.stack(vs), torch.stack(sv), torch.tensor(where)
    G = n_q // n_kv
    for i in range(new):
        seen = where <= ctx + i
        if not seen.any():
            continue
        for h in range(n_q):
            s = k[seen, h // G] @ q[i, h] * scale
            lse[i, h] = torch.logsumexp(s, 0)
            p = (s - lse[i, h]).exp()
            o[i, h] = p @ v[seen, h // G]
            ab[i, h] = p @ v[seen, h // G].abs()
            big[i, h] = (k[seen, h // G].abs() @ q[i, h].abs()).max() * scale
            top[i, h] = len(p) * (p * sv[seen, h // G]).max()
    return o, lse, ab, big, top
