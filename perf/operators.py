"""The serving operators of the 8-bit-activation setting, as measurable cases.

A case is a dict of plain values; its "kind" says which operator one pass
takes:

  norm     residual addition, RMSNorm and the 8-bit output with its scales
  linear   the packed-ternary product on 8-bit activations
  append   new tokens' q, k, v: head norms, rotation, and the append to a paged
           8-bit cache, whose changed blocks are then read back
  attn     attention of new tokens over that cache, ragged sequences

With ``own`` false a pass computes the operator in elementary torch operations
in 32 bits (the plain form); with ``own`` true it makes the package's calls.
``exact`` is the same definition in 64 bits, written apart.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 1e6


# ------------------------------------------------------------------- cases

def listed():
    return [
        # generating one token: the residual stream (fp32) of a Qwen3-14B-shaped block
        dict(name="norm-token", kind="norm", rows=1, n=5120, group=5120, x="bf16", res="f32", weight=True),
        # a ragged prompt with a bf16 residual stream, one scale per 128 values
        dict(name="norm-ragged", kind="norm", rows=1000, n=2048, group=128, x="bf16", res="bf16", weight=False),
        # reading two samples of 4096 tokens
        dict(name="norm-prompt", kind="norm", rows=8192, n=5120, group=5120, x="bf16", res="f32", weight=True),
        # generating one token: the gate|up layer of a Qwen3-14B-shaped block
        dict(name="linear-token", kind="linear", M=1, d_out=34816, d_in=5120, g=128, out="bf16"),
        # 48 sequences generating together: the down layer
        dict(name="linear-batch", kind="linear", M=48, d_out=5120, d_in=17408, g=128, out="f32"),
        # a prompt of 1000 tokens through gate|up
        dict(name="linear-prompt", kind="linear", M=1000, d_out=34816, d_in=5120, g=128, out="bf16"),
        # 64 sequences of different lengths, one new token each (Qwen3-14B-shaped heads)
        dict(name="append-tokens", kind="append", seqs=64, ctx=4000, new=1, n_q=40, n_kv=8, d=128, page=64,
             block=16, rot=128, inter=False, norm=True, a8=True),
        # five prompts, the first long, into empty or half-filled blocks (Llama-3-8B-shaped heads)
        dict(name="append-prompts", kind="append", seqs=5, ctx=90, new=2500, n_q=32, n_kv=8, d=128, page=128,
             block=64, rot=128, inter=False, norm=False, a8=False),
        # one short conversation (Qwen3-1.7B-shaped heads): latency is what counts
        dict(name="attn-token", kind="attn", seqs=1, ctx=300, new=1, n_q=16, n_kv=8, d=128, page=16, block=16),
        # 64 sequences of up to 8192 tokens, one new token each
        dict(name="attn-batch", kind="attn", seqs=64, ctx=8191, new=1, n_q=40, n_kv=8, d=128, page=64, block=64),
        # one far conversation, one scale per token and head
        dict(name="attn-long", kind="attn", seqs=1, ctx=131071, new=1, n_q=32, n_kv=8, d=128, page=128, block=1),
        # chunks of three prompts behind what is cached of them
        dict(name="attn-prompts", kind="attn", seqs=3, ctx=4000, new=2000, n_q=40, n_kv=8, d=128, page=64, block=32),
    ]


def _log(rng, lo, hi, step=1):
    """An integer multiple of ``step`` from lo to hi, even over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["norm", "linear", "append", "attn", "attn"])
    if kind == "norm":
        n = _log(rng, 256, 17408, 8)
        rows = _log(rng, 1, max(1, min(8192, 40_000_000 // n)))
        return dict(kind=kind, rows=rows, n=n, group=128 if n % 128 == 0 and rng.random() < 0.5 else n,
                    x=rng.choice(["bf16", "bf16", "f32"]), res=rng.choice(["f32", "bf16", "none"]),
                    weight=rng.random() < 0.5)
    if kind == "linear":
        g = rng.choice([128, 128, 256, 512])
        d_in, d_out = _log(rng, max(256, g), 17408, g), _log(rng, 64, 34816)
        return dict(kind=kind, M=_log(rng, 1, max(1, min(1500, 170_000_000_000 // (d_in * d_out)))), d_out=d_out,
                    d_in=d_in, g=g, out=rng.choice(["bf16", "f32"]))
    n_kv = rng.choice([1, 2, 4, 8])
    heads = dict(n_q=n_kv * rng.choice([1, 2, 4, 5, 8]), n_kv=n_kv, d=rng.choice([64, 128, 128]),
                 page=rng.choice([16, 32, 64, 128]))
    heads["block"] = rng.choice([b for b in (1, 16, 32, 64, 128) if b <= heads["page"]])
    seqs = _log(rng, 1, 64)
    if kind == "append":
        return dict(kind=kind, seqs=seqs, ctx=_log(rng, 1, 4000), new=_log(rng, 1, max(2, 2500 // seqs)), **heads,
                    rot=rng.choice([heads["d"], heads["d"], heads["d"] // 2]), inter=rng.random() < 0.3,
                    norm=rng.random() < 0.5, a8=rng.random() < 0.3)
    if rng.random() < 0.6:   # one or a few new tokens
        new = rng.choice([1, 1, 1, 2, 4, 7])
        return dict(kind=kind, seqs=seqs, ctx=_log(rng, 16, min(100_000, 400_000 // seqs)), new=new, **heads)
    seqs, ctx = rng.randint(1, 6), _log(rng, 16, 4000)
    pairs = 300_000_000_000 // (4 * heads["n_q"] * heads["d"] * seqs)   # new tokens so that no case is the largest
    return dict(kind=kind, seqs=seqs, ctx=ctx, **heads,
                new=_log(rng, 16, max(32, min(5000 // seqs, int(math.sqrt(ctx * ctx + 2 * pairs)) - ctx))))


def _lens(case):
    """(cached, new) tokens of every sequence: the first has the most, the others spread below it."""
    out = []
    for i in range(case["seqs"]):
        a, b = (0.6180339887 * i) % 1.0, (0.7548776662 * i) % 1.0
        out.append((round(case["ctx"] * (1 - 0.9 * a)), max(1, round(case["new"] * (1 - 0.8 * b)))))
    return out


def work(case):
    if case["kind"] == "norm":
        rs = {"f32": 4, "bf16": 2, "none": 0}[case["res"]]
        e = case["rows"] * case["n"]
        by = e * ((4 if case["x"] == "f32" else 2) + 2 * rs + 1 + 2) + 4 * e // case["group"]
        return {"bytes": by + (2 * case["n"] if case["weight"] else 0), "flops": 8 * e}
    if case["kind"] == "linear":
        M, N, K = case["M"], case["d_out"], case["d_in"]
        by = N * K // 4 + 4 * N * K // case["g"] + M * (K + 4) + M * N * (2 if case["out"] == "bf16" else 4)
        return {"bytes": by, "flops": 2 * M * N * K}
    lens, n_q, n_kv, d = _lens(case), case["n_q"], case["n_kv"], case["d"]
    new = sum(b for _, b in lens)
    if case["kind"] == "append":
        back = sum(c % case["block"] + b for c, b in lens)
        by = new * d * ((n_q + 2 * n_kv) * 2 + n_q * 2 + 2 * n_kv) + back * n_kv * d * 2 * 3
        return {"bytes": by + 8 * n_kv * back // case["block"], "flops": new * d * (n_q + 2 * n_kv) * 8}
    held = sum(c + b for c, b in lens)
    pairs = sum(b * c + b * (b + 1) // 2 for c, b in lens)
    by = held * n_kv * (2 * d + 8 / case["block"]) + new * n_q * (4 * d + 4)
    return {"bytes": by, "flops": 4 * pairs * n_q * d}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _codes(g, shape):
    return (torch.randn(shape, generator=g, device=DEV) * 40).round_().clamp_(-127, 127).to(torch.int8)


def _paged(case, g):
    """A pool of pages in no order, and the sequences that hold some of them; pages past a sequence's end are -1."""
    lens, ps = _lens(case), case["page"]
    need = [-(-(c + b) // ps) for c, b in lens]
    pages, most, n_kv, d, nb = sum(need) + 3, max(need) + 1, case["n_kv"], case["d"], ps // case["block"]
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), most), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    i32 = dict(dtype=torch.int32, device=DEV)
    cu = [0]
    for _, b in lens:
        cu.append(cu[-1] + b)
    scales = [(torch.rand((pages, n_kv, nb), generator=g, device=DEV) + 0.5) / 40 for _ in range(2)]
    return SimpleNamespace(
        k=_codes(g, (pages, n_kv, ps, d)), v=_codes(g, (pages, n_kv, ps // 4, d, 4)),   # v: tokens by four
        k_scale=scales[0], v_scale=scales[1], table=table, cu=torch.tensor(cu, **i32),
        ctx=torch.tensor([c for c, _ in lens], **i32), pages=pages, most=most, n_tokens=cu[-1],
        max_new=max(b for _, b in lens), max_len=max(c + b for c, b in lens), kept=None)


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    if kind == "norm":
        rows, n = case["rows"], case["n"]
        x = _normal(g, (rows, n), 1.0, _type(case["x"]))
        x[:, ::97] *= 4      # some channels stand out
        res = None if case["res"] == "none" else _normal(g, (rows, n), 2.0, _type(case["res"]))
        w = 1 + _normal(g, (n,), 0.1, torch.float32) if case["weight"] else None
        return SimpleNamespace(
            case=case, x=x, res=res, w=None if w is None else w.to(torch.bfloat16),
            sum=None if res is None else torch.empty_like(res),
            q=torch.empty((rows, n), dtype=torch.int8, device=DEV),
            scale=torch.empty((rows, n // case["group"]), device=DEV),
            y=torch.empty((rows, n), dtype=torch.bfloat16, device=DEV))
    if kind == "linear":
        M, N, K, gs = case["M"], case["d_out"], case["d_in"], case["g"]
        packed = torch.zeros((N, K // 4), dtype=torch.uint8, device=DEV)
        for j in range(4):
            packed |= torch.randint(0, 3, (N, K // 4), generator=g, device=DEV, dtype=torch.uint8) << 2 * j
        return SimpleNamespace(
            case=case, q=_codes(g, (M, K)), x_scale=(torch.rand(M, generator=g, device=DEV) + 0.5) / 40,
            packed=packed, alpha=(torch.rand((N, K // gs), generator=g, device=DEV) + 0.5) * 0.02,
            Y=torch.empty((M, N), dtype=_type(case["out"]), device=DEV))
    s = _paged(case, g)
    s.case = case
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d"]
    if kind == "append":
        s.qkv = _normal(g, (s.n_tokens, (n_q + 2 * n_kv) * d))
        half = case["rot"] // 2
        s.inv_freq = (THETA ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
        ws = [(1 + _normal(g, (d,), 0.1, torch.float32)).to(torch.bfloat16) for _ in range(2)]
        s.q_w, s.k_w = ws if case["norm"] else (None, None)
        s.q = torch.empty((s.n_tokens, n_q * d), dtype=torch.bfloat16, device=DEV)
        # what is read back: from the first changed block's first token on
        lens, bt = _lens(case), case["block"]
        cu = [0]
        for c, b in lens:
            cu.append(cu[-1] + c % bt + b)
        s.back_cu = torch.tensor(cu, dtype=torch.int32, device=DEV)
        s.back_ctx = s.ctx // bt * bt
        s.back_n, s.back_max = cu[-1], max(c % bt + b for c, b in lens)
        s.k_out, s.v_out = (torch.empty((s.back_n, n_kv * d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return s
    s.q = _normal(g, (s.n_tokens, n_q * d), 2.0)
    s.o = torch.empty_like(s.q)
    s.lse = torch.empty((s.n_tokens, n_q), device=DEV)
    return s


# --------------------------------------------------------------- one pass

def run(s):
    kind = s.case["kind"]
    if own:
        return _OWN[kind](s)
    return _PLAIN[kind](s)


def _own_norm(s):
    import paper_2606_26650_amd as lib
    lib.catq_aux_rmsnorm_quant(s.x, s.q, s.scale, res=s.res, weight=s.w, sum=s.sum, y=s.y,
                               group=s.case["group"], eps=EPS)
    return dict(sum=s.sum, y=s.y, scale=s.scale)


def _own_linear(s):
    import paper_2606_26650_amd as lib
    lib.catq_ternary_linear_a8(s.q, s.x_scale, s.packed, s.alpha, s.Y, g=s.case["g"])
    return s.Y


def _own_cache(s):
    """The descriptors that a program makes once for its pool, its batch and its model."""
    import paper_2606_26650_amd as lib
    c = s.case
    s.kept = SimpleNamespace(desc=lib.kv_desc(c["n_q"], c["n_kv"], c["d"], c["page"], c["block"], s.pages, s.most))
    s.kept.cache = lib.kv_cache(s.kept.desc, s.k, s.v, s.k_scale, s.v_scale)
    s.kept.batch = lib.kv_batch(s.kept.desc, s.table, s.cu, s.ctx, s.n_tokens, s.max_new, s.max_len)
    if c["kind"] == "append":
        s.kept.prep = lib.kv_prep(s.kept.desc, s.inv_freq, rot_dim=c["rot"], interleaved=c["inter"],
                                  qk_norm=c["norm"], q_weight=s.q_w, k_weight=s.k_w, eps=EPS, act_quant=c["a8"])
        s.kept.back = lib.kv_batch(s.kept.desc, s.table, s.back_cu, s.back_ctx, s.back_n, s.back_max, s.max_len)
    else:
        s.kept.ws = torch.empty(lib.catq_paged_attention_workspace_bytes(s.kept.desc, s.kept.batch),
                                dtype=torch.uint8, device=DEV)
    return s.kept


def _own_append(s):
    import paper_2606_26650_amd as lib
    t = s.kept or _own_cache(s)
    lib.catq_aux_kv_append(t.desc, t.cache, t.batch, t.prep, s.qkv, s.q)
    lib.catq_aux_kv_read(t.desc, t.cache, t.back, s.k_out, s.v_out)
    return dict(q=s.q, k=s.k_out, v=s.v_out, k_scale=s.k_scale, v_scale=s.v_scale)


def _own_attn(s):
    import paper_2606_26650_amd as lib
    t = s.kept or _own_cache(s)
    lib.catq_aux_paged_attention(t.desc, t.cache, t.batch, s.q, s.o, t.ws, lse=s.lse)
    return dict(o=s.o, lse=s.lse)


def _quant(x, s):
    """rint(x / s) within +-127; 0 where s is 0."""
    return torch.where(s > 0, (x / s).round().clamp(-127, 127), torch.zeros((), device=x.device))


def _norm(s):
    c = s.case
    h = s.x.float()
    if s.res is not None:
        s.sum.copy_(h + s.res.float())
        h = s.sum.float()
    h = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    if s.w is not None:
        h = h * s.w.float()
    h = h.view(c["rows"], -1, c["group"])
    sc = h.abs().amax(-1, keepdim=True) / 127.0
    s.y.copy_((_quant(h, sc) * sc).view(c["rows"], c["n"]))
    s.scale.copy_(sc.view(c["rows"], -1))
    return dict(sum=s.sum, y=s.y, scale=s.scale)


def _linear(s):
    c = s.case
    shifts = torch.tensor([0, 2, 4, 6], dtype=torch.uint8, device=DEV)
    code = (s.packed[..., None] >> shifts) & 3
    t = torch.where(code == 3, 0.0, code.float() - 1.0).view(c["d_out"], -1, c["g"])
    w = (t * s.alpha[..., None]).view(c["d_out"], c["d_in"])
    s.Y.copy_((s.q.float() @ w.T) * s.x_scale[:, None])
    return s.Y


def _of_token(cu, n):
    """(sequence, place in it) of each of n rows laid out by cu."""
    i = torch.arange(n, device=DEV)
    seq = torch.searchsorted(cu[1:].long(), i, right=True)
    return seq, i - cu.long()[seq]


def _rotate(x, pos, inv_freq, rot, inter):
    """x [tokens][heads][d] rotated in its first ``rot`` values by angles taken in 64 bits."""
    turn = pos.double()[:, None] * inv_freq.double()
    cs, sn = turn.cos().float()[:, None], turn.sin().float()[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    p, q = a * cs - b * sn, b * cs + a * sn
    y = torch.stack([p, q], -1).flatten(-2) if inter else torch.cat([p, q], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _append_one(new, codes, at, scale, page, block, fresh, old):
    """New values [blocks][bt][n_kv][d] into codes[at], of blocks that may hold older tokens."""
    new = torch.where(fresh[..., None, None], new, torch.zeros((), device=DEV))
    sc = new.abs().amax((1, 3)) / 127.0
    was = torch.where(old.any(1)[:, None], scale[page, :, block], torch.zeros((), device=DEV))
    now = torch.maximum(sc, was)
    had = codes[at].float()
    ratio = torch.where(now > was, was / now, torch.ones((), device=DEV))
    kept = (had * ratio[:, None, :, None]).round()
    out = torch.where(fresh[..., None, None], _quant(new, now[:, None, :, None]), kept)
    out = torch.where((fresh | old)[..., None, None], out, had).to(torch.int8)
    codes[at] = out
    scale[page, :, block] = now


_ALL = slice(None)


def _k_at(page, tok):
    return page, _ALL, tok


def _v_at(page, tok):
    return page, _ALL, tok // 4, _ALL, tok % 4


def _append(s):
    c = s.case
    n_q, n_kv, d, bt, ps = c["n_q"], c["n_kv"], c["d"], c["block"], c["page"]
    seq, i = _of_token(s.cu, s.n_tokens)
    pos = s.ctx.long()[seq] + i
    x = s.qkv.float().view(s.n_tokens, n_q + 2 * n_kv, d)
    qk, v = x[:, :n_q + n_kv], x[:, n_q + n_kv:]
    if c["norm"]:
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + EPS)
        qk = torch.cat([qk[:, :n_q] * s.q_w.float(), qk[:, n_q:] * s.k_w.float()], 1)
    qk = _rotate(qk, pos, s.inv_freq, c["rot"], c["inter"])
    q, k = qk[:, :n_q], qk[:, n_q:]
    if c["a8"]:
        sc = q.abs().amax(-1, keepdim=True) / 127.0
        q = _quant(q, sc) * sc
    s.q.copy_(q.reshape(s.n_tokens, -1))
    # the blocks that new tokens reach, as many for every sequence as the most (the last again for the others)
    ctx, new = s.ctx.long(), (s.cu[1:] - s.cu[:-1]).long()
    most = (s.max_new + bt - 2) // bt + 1
    b0 = ctx // bt
    b = torch.minimum(b0[:, None] + torch.arange(most, device=DEV), ((ctx + new - 1) // bt)[:, None])
    at = (b[..., None] * bt + torch.arange(bt, device=DEV)).view(-1, bt)           # positions [blocks][bt]
    of = torch.arange(c["seqs"], device=DEV)[:, None].expand(-1, most).reshape(-1)
    end = (ctx + new)[of, None]
    fresh, old = (at >= ctx[of, None]) & (at < end), at < ctx[of, None]
    row = (s.cu.long()[of, None] + at - ctx[of, None]).clamp(0, s.n_tokens - 1)
    page, block, tok = s.table.long()[of, at[:, 0] // ps], at[:, 0] % ps // bt, at % ps
    _append_one(k[row], s.k, _k_at(page[:, None], tok), s.k_scale, page, block, fresh, old)
    _append_one(v[row], s.v, _v_at(page[:, None], tok), s.v_scale, page, block, fresh, old)
    seq, i = _of_token(s.back_cu, s.back_n)
    p = s.back_ctx.long()[seq] + i
    page, tok = s.table.long()[seq, p // ps], p % ps
    s.k_out.copy_((s.k[_k_at(page, tok)].float() * s.k_scale[page, :, tok // bt][..., None]).view(s.back_n, -1))
    s.v_out.copy_((s.v[_v_at(page, tok)].float() * s.v_scale[page, :, tok // bt][..., None]).view(s.back_n, -1))
    return dict(q=s.q, k=s.k_out, v=s.v_out, k_scale=s.k_scale, v_scale=s.v_scale)


def _attn(s):
    c = s.case
    S, n_q, n_kv, d, ps, bt = c["seqs"], c["n_q"], c["n_kv"], c["d"], c["page"], c["block"]
    G, L, N = n_q // n_kv, s.most * ps, s.max_new
    ids = s.table.clamp(min=0).long()
    ks = s.k_scale[ids].repeat_interleave(bt, -1)[..., None]
    vs = s.v_scale[ids].repeat_interleave(bt, -1)[..., None]
    k = (s.k[ids].float() * ks).transpose(1, 2).reshape(S, n_kv, L, d)
    v = s.v[ids].float().transpose(-1, -2).reshape(S, s.most, n_kv, ps, d)
    v = (v * vs).transpose(1, 2).reshape(S, n_kv, L, d)
    row = (s.cu[:-1, None].long() + torch.arange(N, device=DEV)).clamp(max=s.n_tokens - 1)
    q = s.q.float().view(-1, n_kv, G, d)[row].permute(0, 2, 3, 1, 4).reshape(S, n_kv, G * N, d)
    p = (q @ k.transpose(-1, -2).contiguous()).view(S, n_kv, G, N, L) * d ** -0.5
    last = s.ctx[:, None].long() + torch.arange(N, device=DEV)                     # [S][N]
    seen = torch.arange(L, device=DEV) <= last[..., None]
    p = p.masked_fill_(~seen[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(m).exp_()
    t = p.sum(-1, keepdim=True)
    o = ((p.view(S, n_kv, G * N, L) @ v).view(S, n_kv, G, N, d) / t).permute(0, 3, 1, 2, 4)
    lse = (m + t.log()).squeeze(-1).permute(0, 3, 1, 2)
    seq, i = _of_token(s.cu, s.n_tokens)
    s.o.copy_(o[seq, i].reshape(s.n_tokens, -1))
    s.lse.copy_(lse[seq, i].reshape(s.n_tokens, -1))
    return dict(o=s.o, lse=s.lse)


_OWN = dict(norm=_own_norm, linear=_own_linear, append=_own_append, attn=_own_attn)
_PLAIN = dict(norm=_norm, linear=_linear, append=_append, attn=_attn)


# ------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["kind"]](case, s)


def _code64(x, s):
    q = torch.round(x / s.clamp(min=1e-300)).clamp(-127, 127)
    return q * (s > 0)


def _norm64(c, s):
    h = s.x.double()
    if s.res is not None:
        h = (h + s.res.double()).to(s.res.dtype).double()
    n = h / (h.pow(2).sum(1, keepdim=True) / c["n"] + EPS).sqrt()
    n = n if s.w is None else n * s.w.double()
    g = n.reshape(-1, c["group"])
    sc = g.abs().max(1, keepdim=True).values / 127
    return dict(sum=None if s.res is None else h, y=(_code64(g, sc) * sc).reshape(n.shape),
                scale=sc.reshape(c["rows"], -1))


def _linear64(c, s):
    w = torch.empty((c["d_out"], c["d_in"]), dtype=torch.float64, device=DEV)
    for j in range(4):
        w[:, j::4] = ((s.packed >> (2 * j)) & 3).double() - 1
    w *= s.alpha.double().repeat_interleave(c["g"], 1)
    return (s.q.double() * s.x_scale.double()[:, None]) @ w.T


def _held64(c, s, i, n):
    """K and V values [n][n_kv][d] of sequence i's first n positions, with their codes and scales by token."""
    ps, n_kv, d = c["page"], c["n_kv"], c["d"]
    ids = s.table[i, :-(-n // ps)].long()
    out = []
    for codes, scale in ((s.k, s.k_scale), (s.v, s.v_scale)):
        x = codes[ids]
        x = x if x.dim() == 4 else x.movedim(-1, 3).reshape(len(ids), n_kv, ps, d)
        x = x.movedim(1, 0).reshape(n_kv, -1, d)[:, :n].double()
        t = scale[ids].movedim(1, 0).reshape(n_kv, -1).double()
        out.append((x, t, t.repeat_interleave(c["block"], 1)[:, :n, None]))
    return out


def _turned64(x, pos, s, c):
    rot = c["rot"]
    z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV).expand(len(pos), rot // 2).contiguous(),
                    pos.double()[:, None] * s.inv_freq.double())[:, None]
    y = x.clone()
    if c["inter"]:
        y[..., :rot] = torch.view_as_real(torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * z).flatten(-2)
    else:
        w = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * z
        y[..., :rot // 2], y[..., rot // 2:rot] = w.real, w.imag
    return y


def _append64(c, s):
    n_q, n_kv, d, bt, ps = c["n_q"], c["n_kv"], c["d"], c["block"], c["page"]
    x = s.qkv.double().view(-1, n_q + 2 * n_kv, d)
    scales = [s.k_scale.double(), s.v_scale.double()]
    qs, back = [], ([], [])
    at = 0
    for i, (ctx, new) in enumerate(_lens(c)):
        t = x[at:at + new]
        at += new
        pos = torch.arange(ctx, ctx + new, device=DEV)
        q, k, v = t.split([n_q, n_kv, n_kv], 1)
        if c["norm"]:
            q = q / (q.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * s.q_w.double()
            k = k / (k.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * s.k_w.double()
        q, k = _turned64(q, pos, s, c), _turned64(k, pos, s, c)
        if c["a8"]:
            sc = q.abs().max(-1, keepdim=True).values / 127
            q = _code64(q, sc) * sc
        qs.append(q.reshape(new, -1))
        first, end = ctx // bt * bt, ctx + new
        held = _held64(c, s, i, end)
        pad = -end % bt
        for j, val in enumerate((k, v)):
            codes, old, _ = held[j]
            codes = torch.nn.functional.pad(codes[:, first:], (0, 0, 0, pad)).unflatten(1, (-1, bt))
            was = old[:, first // bt:first // bt + codes.shape[1]].clone()
            was[:, (1 if ctx % bt else 0):] = 0
            val = torch.nn.functional.pad(val.movedim(1, 0), (0, 0, ctx - first, pad)).unflatten(1, (-1, bt))
            now = torch.maximum(val.abs().amax((2, 3)) / 127, was)
            mine = torch.arange(first, end + pad, device=DEV).view(-1, bt) >= ctx
            r = (was / now.clamp(min=1e-300))[..., None, None]
            q8 = torch.where(mine[None, ..., None], _code64(val, now[..., None, None]),
                             torch.where(r < 1, torch.round(codes * r), codes))
            y = (q8 * now[..., None, None]).flatten(1, 2)[:, :end - first]
            back[j].append(y.movedim(0, 1).reshape(end - first, -1))
            b = torch.arange(first // bt, -(-end // bt), device=DEV)
            scales[j][s.table[i].long()[b * bt // ps], :, b % (ps // bt)] = now.movedim(0, 1)
    return dict(q=torch.cat(qs), k=torch.cat(back[0]), v=torch.cat(back[1]), k_scale=scales[0], v_scale=scales[1])


def _attn64(c, s):
    n_q, n_kv, d = c["n_q"], c["n_kv"], c["d"]
    q = s.q.double().view(-1, n_kv, n_q // n_kv, d)
    outs, lses, at = [], [], 0
    for i, (ctx, new) in enumerate(_lens(c)):
        (kc, _, ks), (vc, _, vs) = _held64(c, s, i, ctx + new)
        hidden = torch.arange(ctx + new, device=DEV) > torch.arange(ctx, ctx + new, device=DEV)[:, None]
        o = torch.empty((new, n_q, d), dtype=torch.float64, device=DEV)
        lse = torch.empty((new, n_q), dtype=torch.float64, device=DEV)
        for h in range(n_kv):
            k, v = kc[h] * ks[h], vc[h] * vs[h]
            for g in range(n_q // n_kv):
                sc = (q[at:at + new, h, g] @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                l = torch.logsumexp(sc, -1)
                o[:, h * (n_q // n_kv) + g] = (sc - l[:, None]).exp() @ v
                lse[:, h * (n_q // n_kv) + g] = l
        outs.append(o.view(new, -1))
        lses.append(lse)
        at += new
    return dict(o=torch.cat(outs), lse=torch.cat(lses))


_EXACT = dict(norm=_norm64, linear=_linear64, append=_append64, attn=_attn64)
