"""The operators of a decode step with drafted tokens, as measurable cases.

A case is a dict of plain values; its "kind" says which operator one pass
takes:

  moe      routed experts on packed-ternary weights and 8-bit activations, from
           the router's logits to the combined output, for few tokens
  draft    a tree of drafted tokens' q, k, v: head norms, rotation at the tokens'
           depths, and the append to a paged 8-bit cache, whose changed blocks are
           then read back
  tree     attention of such a tree over that cache
  sample   a token per row of logits: temperature, top-k, top-p, min-p and a given
           uniform number
  copy     pages of the cache copied to others
  accept   forks of drafted sequences: the pages that hold the drafted tokens are
           copied to the fork's own, the accepted path moves to the front there, and what
           changed is read back

With ``own`` false a pass computes the operator in elementary torch operations
in 32 bits (the plain form; the sampler in 64); with ``own`` true it makes the package's
calls.  ``exact`` is the same definition in 64 bits, written apart.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 1e6


# ------------------------------------------------------------------- cases

def listed():
    return [
        # generating one token: the experts of a 128-expert block, latency and the 8 experts' bytes
        dict(name="moe-token", kind="moe", T=1, E=128, k=8, hidden=4096, ffn=1536, g=128),
        # 32 sequences generating together: nearly every expert is hit, by a token or two
        dict(name="moe-batch", kind="moe", T=32, E=128, k=8, hidden=4096, ffn=1536, g=128),
        # one short conversation with a handful of drafted tokens: latency
        dict(name="draft-one", kind="draft", seqs=1, ctx=300, new=7, n_q=16, n_kv=8, d=128, page=16, block=1,
             rot=128, inter=False, norm=True, a8=False),
        # 48 sequences that draft up to 60 tokens each
        dict(name="draft-batch", kind="draft", seqs=48, ctx=4000, new=60, n_q=40, n_kv=8, d=128, page=64, block=16,
             rot=128, inter=False, norm=True, a8=True),
        # the attention of that handful of drafted tokens
        dict(name="tree-one", kind="tree", seqs=1, ctx=300, new=7, n_q=16, n_kv=8, d=128, page=16, block=1),
        # up to 60 drafted tokens in each of 32 sequences of up to 8000
        dict(name="tree-batch", kind="tree", seqs=32, ctx=8000, new=60, n_q=40, n_kv=8, d=128, page=64, block=64),
        # one sequence's next token
        dict(name="sample-one", kind="sample", rows=1, vocab=32000, dtype="bf16"),
        # the next tokens of 64 sequences with settings of their own, a large vocabulary
        dict(name="sample-batch", kind="sample", rows=64, vocab=150000, dtype="f32"),
        # four sequences forked: the last page of each
        dict(name="copy-fork", kind="copy", pages=4, n_kv=8, d=128, page=64, block=16),
        # sequences of 40000 tokens together moved to other places of the pool
        dict(name="copy-move", kind="copy", pages=625, n_kv=8, d=128, page=64, block=1),
        # one sequence keeps a path of its drafted tokens
        dict(name="accept-one", kind="accept", seqs=1, ctx=300, new=7, keep=3, n_kv=8, d=128, page=16, block=1),
        # 64 sequences keep up to 8 of 60
        dict(name="accept-batch", kind="accept", seqs=64, ctx=4000, new=60, keep=8, n_kv=8, d=128, page=64, block=16),
    ]


def _log(rng, lo, hi, step=1):
    """An integer multiple of ``step`` from lo to hi, even over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["moe", "moe", "draft", "tree", "tree", "sample", "sample", "copy", "accept"])
    if kind == "moe":
        E, g = _log(rng, 4, 128), rng.choice([128, 128, 256])
        return dict(kind=kind, T=_log(rng, 1, 32), E=E, k=rng.randint(1, min(8, E)), hidden=_log(rng, 256, 4096, g),
                    ffn=_log(rng, 256, 1536, g), g=g)
    if kind == "sample":
        return dict(kind=kind, rows=_log(rng, 1, 64), vocab=_log(rng, 100, 150000), dtype=rng.choice(["f32", "bf16"]))
    n_kv = rng.choice([1, 2, 4, 8])
    heads = dict(n_q=n_kv * rng.choice([1, 2, 4, 5, 8]), n_kv=n_kv, d=rng.choice([64, 128, 128]),
                 page=rng.choice([16, 32, 64, 128]))
    heads["block"] = rng.choice([b for b in (1, 16, 32, 64, 128) if b <= heads["page"]])
    if kind == "copy":
        del heads["n_q"]
        return dict(kind=kind, pages=_log(rng, 1, max(1, 40000 // heads["page"])), **heads)
    seqs = _log(rng, 1, 48 if kind == "draft" else 32)
    new = _log(rng, 1, 60)
    if kind == "draft":
        return dict(kind=kind, seqs=seqs, ctx=_log(rng, 1, 4000), new=new, **heads,
                    rot=rng.choice([heads["d"], heads["d"], heads["d"] // 2]), inter=rng.random() < 0.3,
                    norm=rng.random() < 0.5, a8=rng.random() < 0.3)
    if kind == "tree":
        return dict(kind=kind, seqs=seqs, ctx=_log(rng, 1, min(100_000, 256_000 // seqs)), new=new, **heads)
    del heads["n_q"]
    return dict(kind=kind, seqs=seqs, ctx=_log(rng, 1, 4000), new=new, keep=rng.randint(1, min(new, 12)), **heads)


def _lens(case):
    """(cached, new) tokens of every sequence: the first has the most, the others spread below it."""
    out = []
    for i in range(case["seqs"]):
        a, b = (0.6180339887 * i) % 1.0, (0.7548776662 * i) % 1.0
        out.append((round(case["ctx"] * (1 - 0.9 * a)), max(1, round(case["new"] * (1 - 0.8 * b)))))
    return out


def _kept(case):
    """How many drafted tokens every sequence keeps."""
    return [min(b, max(0, round(case["keep"] * (1 - 0.57 * i % 1.0)))) for i, (_, b) in enumerate(_lens(case))]


def _tail(case):
    """The page indexes [first, end) of every sequence that hold its drafted tokens."""
    return [(c // case["page"], -(-(c + b) // case["page"])) for c, b in _lens(case)]


def work(case):
    if case["kind"] == "moe":
        T, E, k, h, F, g = (case[x] for x in ("T", "E", "k", "hidden", "ffn", "g"))
        hit = E * (1 - (1 - k / E) ** T)       # experts hit, expected
        by = hit * 3 * h * F * (1 / 4 + 4 / g) + T * (h + 4 + 4 * E + 4 * h)
        return {"bytes": by, "flops": 6 * T * k * h * F}
    if case["kind"] == "sample":
        e = case["rows"] * case["vocab"]
        return {"bytes": e * (4 if case["dtype"] == "f32" else 2) + 28 * case["rows"], "flops": 8 * e}
    n_kv, d, ps, bt = case["n_kv"], case["d"], case["page"], case["block"]
    page = 2 * n_kv * ps * (d + 4 / bt)
    if case["kind"] == "copy":
        return {"bytes": 2 * case["pages"] * page, "flops": 0}
    lens = _lens(case)
    new = sum(b for _, b in lens)
    if case["kind"] == "accept":
        kept = sum(_kept(case))
        back = sum(c % bt for c, _ in lens) + kept
        by = 2 * page * sum(b - a for a, b in _tail(case)) + (kept * 4 + back * 6) * n_kv * d
        return {"bytes": by, "flops": 0}
    n_q = case["n_q"]
    if case["kind"] == "draft":
        back = sum(c % bt + b for c, b in lens)
        by = new * d * ((n_q + 2 * n_kv) * 2 + n_q * 2 + 2 * n_kv) + back * n_kv * d * 2 * 3
        return {"bytes": by + 8 * n_kv * back / bt, "flops": new * d * (n_q + 2 * n_kv) * 8}
    held = sum(c + b for c, b in lens)
    pairs = sum(b * c + 4 * b for c, b in lens)          # (a token has a few drafted ones before it)
    by = held * n_kv * (2 * d + 8 / bt) + new * n_q * (4 * d + 4)
    return {"bytes": by, "flops": 4 * pairs * n_q * d}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _codes(g, shape):
    return (torch.randn(shape, generator=g, device=DEV) * 40).round_().clamp_(-127, 127).to(torch.int8)


def _ternary(g, shape, group):
    """Packed codes [..., n / 4] of ternary weights [..., n] and their group scales."""
    four = [sum((v // 3 ** j % 3) << 2 * j for j in range(4)) for v in range(81)]
    table = torch.tensor(four, dtype=torch.uint8, device=DEV)
    lead = shape[:-1]
    at = torch.randint(0, 81, lead + (shape[-1] // 4,), generator=g, device=DEV, dtype=torch.uint8)
    alpha = (torch.rand(lead + (shape[-1] // group,), generator=g, device=DEV) + 0.5) * 0.02
    return table[at.int()], alpha


def _tree(rng, n):
    """Parents (-1: the last cached token) of n drafted tokens, each after its parent, and their depths."""
    parent = [-1] + [max(-1, j - 1 - int(rng.expovariate(0.25))) for j in range(1, n)]
    depth = []
    for p in parent:
        depth.append(0 if p < 0 else depth[p] + 1)
    return parent, depth


def _paged(case, g, extra=3):
    """A pool of pages in no order, and the sequences that hold some of them; pages past a sequence's end are -1."""
    lens, ps = _lens(case), case["page"]
    need = [-(-(c + b) // ps) for c, b in lens]
    pages, most, n_kv, d, nb = sum(need) + extra, max(need) + 1, case["n_kv"], case["d"], ps // case["block"]
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
        k_scale=scales[0], v_scale=scales[1], table=table, free=order[at:], cu=torch.tensor(cu, **i32),
        ctx=torch.tensor([c for c, _ in lens], **i32), pages=pages, most=most, n_tokens=cu[-1],
        max_new=max(b for _, b in lens), max_len=max(c + b for c, b in lens), kept=None)


def _drafted(case, s, seed):
    """The trees of a batch: depths [n_tokens] and, per token, the bits of the drafted tokens that it sees."""
    rng = random.Random(seed)
    words = -(-s.max_new // 64)
    depths, masks = [], []
    for _, n in _lens(case):
        parent, depth = _tree(rng, n)
        rows = []
        for j, p in enumerate(parent):
            rows.append((rows[p] if p >= 0 else 0) | 1 << j)
        depths += depth
        masks += [[(r >> 64 * w & (1 << 64) - 1) - ((r >> 64 * w + 63 & 1) << 64) for w in range(words)] for r in rows]
    s.depth = torch.tensor(depths, dtype=torch.int32, device=DEV)
    s.mask = torch.tensor(masks, dtype=torch.int64, device=DEV)


def _read_back(case, s, counts):
    """The positions that a pass changes: from the first changed block's first token on."""
    bt, cu, most = case["block"], [0], 0
    for (c, _), n in zip(_lens(case), counts):
        cu.append(cu[-1] + c % bt + n)
        most = max(most, c % bt + n)
    s.back_cu = torch.tensor(cu, dtype=torch.int32, device=DEV)
    s.back_ctx = s.ctx // bt * bt
    s.back_n, s.back_max = cu[-1], most
    s.k_out, s.v_out = (torch.empty((s.back_n, case["n_kv"] * case["d"]), dtype=torch.bfloat16, device=DEV)
                        for _ in range(2))


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    if kind == "moe":
        T, E, h, F = case["T"], case["E"], case["hidden"], case["ffn"]
        gu, gu_alpha = _ternary(g, (E, 2 * F, h), case["g"])
        down, down_alpha = _ternary(g, (E, h, F), case["g"])
        return SimpleNamespace(
            case=case, logits=torch.randn((T, E), generator=g, device=DEV), q=_codes(g, (T, h)),
            x_scale=(torch.rand(T, generator=g, device=DEV) + 0.5) / 40, gu=gu, gu_alpha=gu_alpha, down=down,
            down_alpha=down_alpha, res=_normal(g, (T, h)), kept=None,
            y=torch.empty((T, h), dtype=torch.bfloat16, device=DEV))
    if kind == "sample":
        rows, V = case["rows"], case["vocab"]
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        rng = random.Random(seed)
        logits = (torch.randn((rows, V), generator=g, device=DEV) * 2.5)
        at = torch.randint(0, V, (rows, 12), generator=g, device=DEV)      # a few tokens stand out
        logits.scatter_add_(1, at, 4 + 6 * torch.rand((rows, 12), generator=g, device=DEV))
        # each row has settings of its own: some greedy, some with one filter, some with all, some with none
        f32, i32 = dict(dtype=torch.float32, device=DEV), dict(dtype=torch.int32, device=DEV)
        pick = [rng.choice(["greedy", "k", "p", "m", "all", "all", "kp", "none"]) for _ in range(rows)]
        return SimpleNamespace(
            case=case, logits=logits.to(dt), kept=None,
            temperature=torch.tensor([0.0 if x == "greedy" else rng.uniform(0.4, 1.3) for x in pick], **f32),
            top_k=torch.tensor([rng.choice([1, 20, 50, 400]) if x in ("k", "kp", "all") else 0 for x in pick], **i32),
            top_p=torch.tensor([rng.uniform(0.5, 0.98) if x in ("p", "kp", "all") else 1.0 for x in pick], **f32),
            min_p=torch.tensor([rng.uniform(0.01, 0.2) if x in ("m", "all") else 0.0 for x in pick], **f32),
            u=torch.rand(rows, generator=g, device=DEV), token=torch.empty(rows, **i32), prob=torch.empty(rows, **f32))
    if kind == "copy":
        n, ps = case["pages"], case["page"]
        pool, nb = 2 * n + 3, ps // case["block"]
        order = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
        return SimpleNamespace(
            case=case, k=_codes(g, (pool, case["n_kv"], ps, case["d"])),
            v=_codes(g, (pool, case["n_kv"], ps // 4, case["d"], 4)), pages=pool, most=n, src=order[:n].clone(),
            dst=order[n:2 * n].clone(), kept=None,
            **{x: torch.rand((pool, case["n_kv"], nb), generator=g, device=DEV) + 0.5 for x in ("k_scale", "v_scale")})
    tails = _tail(case) if kind == "accept" else []
    s = _paged(case, g, extra=3 + sum(b - a for a, b in tails))
    s.case = case
    if kind == "accept":
        # the fork shares the pages before its drafted tokens and has the others for itself
        s.fork, src, at = s.table.clone(), [], 0
        for i, (a, b) in enumerate(tails):
            src.append(s.table[i, a:b])
            s.fork[i, a:b] = s.free[at:at + b - a]
            at += b - a
        s.src, s.dst = torch.cat(src), s.free[:at].clone()
        rng, keep = random.Random(seed), []
        counts = _kept(case)
        for (_, b), n in zip(_lens(case), counts):
            path = sorted(rng.sample(range(b), n))
            keep += path + [0] * (b - n)
        s.keep = torch.tensor(keep, dtype=torch.int32, device=DEV)
        s.n_keep = torch.tensor(counts, dtype=torch.int32, device=DEV)
        _read_back(case, s, counts)
        return s
    _drafted(case, s, seed)
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d"]
    if kind == "draft":
        s.qkv = _normal(g, (s.n_tokens, (n_q + 2 * n_kv) * d))
        half = case["rot"] // 2
        s.inv_freq = (THETA ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
        ws = [(1 + _normal(g, (d,), 0.1, torch.float32)).to(torch.bfloat16) for _ in range(2)]
        s.q_w, s.k_w = ws if case["norm"] else (None, None)
        s.q = torch.empty((s.n_tokens, n_q * d), dtype=torch.bfloat16, device=DEV)
        _read_back(case, s, [b for _, b in _lens(case)])
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


def _own_moe(s):
    import paper_2606_26650_amd as lib
    c = s.case
    if s.kept is None:     # what a program makes once for its model
        s.kept = SimpleNamespace(desc=lib.moe_desc(c["E"], c["k"], c["hidden"], c["ffn"], c["g"]))
        s.kept.ws = torch.empty(lib.catq_ternary_moe_a8_workspace_bytes(s.kept.desc, c["T"]), dtype=torch.uint8,
                                device=DEV)
    lib.catq_ternary_moe_a8(s.kept.desc, s.logits, s.q, s.x_scale, s.gu, s.gu_alpha, s.down, s.down_alpha, s.y,
                            s.kept.ws, res=s.res)
    return s.y


def _own_sample(s):
    import paper_2606_26650_amd as lib
    c = s.case
    if s.kept is None:
        s.kept = torch.empty(lib.catq_aux_sample_workspace_bytes(c["rows"], c["vocab"]), dtype=torch.uint8, device=DEV)
    lib.catq_aux_sample(s.logits, s.u, s.token, s.kept, temperature=s.temperature, top_k=s.top_k, top_p=s.top_p,
                        min_p=s.min_p, prob=s.prob)
    return dict(token=s.token, prob=s.prob)


def _own_cache(s):
    """The descriptors that a program makes once for its pool, its batch and its model."""
    import paper_2606_26650_amd as lib
    c = s.case
    s.kept = SimpleNamespace(desc=lib.kv_desc(c.get("n_q", c["n_kv"]), c["n_kv"], c["d"], c["page"], c["block"],
                                              s.pages, s.most))
    s.kept.cache = lib.kv_cache(s.kept.desc, s.k, s.v, s.k_scale, s.v_scale)
    if c["kind"] == "copy":
        return s.kept
    table = s.fork if c["kind"] == "accept" else s.table
    s.kept.batch = lib.kv_batch(s.kept.desc, table, s.cu, s.ctx, s.n_tokens, s.max_new, s.max_len)
    if c["kind"] != "tree":
        s.kept.back = lib.kv_batch(s.kept.desc, table, s.back_cu, s.back_ctx, s.back_n, s.back_max, s.max_len)
    if c["kind"] in ("draft", "tree"):
        s.kept.tree = lib.kv_tree(s.kept.batch, s.mask, s.depth)
    if c["kind"] == "draft":
        s.kept.prep = lib.kv_prep(s.kept.desc, s.inv_freq, rot_dim=c["rot"], interleaved=c["inter"],
                                  qk_norm=c["norm"], q_weight=s.q_w, k_weight=s.k_w, eps=EPS, act_quant=c["a8"])
    if c["kind"] == "tree":
        s.kept.ws = torch.empty(lib.catq_paged_attention_workspace_bytes(s.kept.desc, s.kept.batch),
                                dtype=torch.uint8, device=DEV)
    return s.kept


def _own_draft(s):
    import paper_2606_26650_amd as lib
    t = s.kept or _own_cache(s)
    lib.catq_aux_kv_append_tree(t.desc, t.cache, t.batch, t.tree, t.prep, s.qkv, s.q)
    lib.catq_aux_kv_read(t.desc, t.cache, t.back, s.k_out, s.v_out)
    return dict(q=s.q, k=s.k_out, v=s.v_out, k_scale=s.k_scale, v_scale=s.v_scale)


def _own_tree(s):
    import paper_2606_26650_amd as lib
    t = s.kept or _own_cache(s)
    lib.catq_aux_tree_attention(t.desc, t.cache, t.batch, t.tree, s.q, s.o, t.ws, lse=s.lse)
    return dict(o=s.o, lse=s.lse)


def _own_copy(s):
    import paper_2606_26650_amd as lib
    t = s.kept or _own_cache(s)
    lib.catq_aux_kv_copy_pages(t.desc, t.cache, s.src, s.dst)
    return dict(k=s.k, v=s.v, k_scale=s.k_scale, v_scale=s.v_scale)


def _own_accept(s):
    import paper_2606_26650_amd as lib
    t = s.kept or _own_cache(s)
    lib.catq_aux_kv_copy_pages(t.desc, t.cache, s.src, s.dst)
    lib.catq_aux_kv_compact(t.desc, t.cache, t.batch, s.keep, s.n_keep)
    lib.catq_aux_kv_read(t.desc, t.cache, t.back, s.k_out, s.v_out)
    return dict(k=s.k_out, v=s.v_out, k_scale=s.k_scale, v_scale=s.v_scale)


def _quant(x, s):
    """rint(x / s) within +-127; 0 where s is 0."""
    return torch.where(s > 0, (x / s).round().clamp(-127, 127), torch.zeros((), device=x.device))


def _unpacked(packed, alpha, g):
    """Packed codes [..., n / 4] and group scales as fp32 weights [..., n]."""
    shifts = torch.tensor([0, 2, 4, 6], dtype=torch.uint8, device=DEV)
    code = (packed[..., None] >> shifts) & 3
    t = torch.where(code == 3, 0.0, code.float() - 1.0).flatten(-2)
    return (t.unflatten(-1, (-1, g)) * alpha[..., None]).flatten(-2)


def _expert(x, gu, down, F):
    """Values x [..., rows][h] through experts with weights gu [...][2F][h], down [...][h][F]."""
    z = x @ gu.transpose(-1, -2).contiguous()
    a = z[..., :F] * torch.sigmoid(z[..., :F]) * z[..., F:]
    sc = a.abs().amax(-1, keepdim=True) / 127.0
    return (_quant(a, sc) * sc) @ down.transpose(-1, -2).contiguous()


def _moe(s):
    c = s.case
    T, E, k, F, g = c["T"], c["E"], c["k"], c["ffn"], c["g"]
    x = s.q.float() * s.x_scale[:, None]
    top, ids = torch.sort(s.logits, dim=-1, descending=True, stable=True)
    w = torch.exp(top[:, :k] - top[:, :1])
    w = w / w.sum(-1, keepdim=True)
    ids = ids[:, :k]
    if T * k <= 64:       # the experts of every slot
        at = ids.reshape(-1)
        z = _expert(x.repeat_interleave(k, 0)[:, None], _unpacked(s.gu[at], s.gu_alpha[at], g),
                    _unpacked(s.down[at], s.down_alpha[at], g), F)
        y = (z.view(T, k, -1) * w[..., None]).sum(1)
    else:                 # every expert for all tokens, with weight 0 where it is not theirs
        y = torch.zeros_like(x)
        each = torch.zeros_like(s.logits).scatter_(1, ids, w)
        for e in range(E):
            y += each[:, e, None] * _expert(x, _unpacked(s.gu[e], s.gu_alpha[e], g),
                                            _unpacked(s.down[e], s.down_alpha[e], g), F)
    s.y.copy_(y + s.res.float())
    return s.y


def _sample(s):
    x = s.logits.double()
    t = s.temperature.double()[:, None]
    w = torch.exp((x - x.amax(-1, keepdim=True)) / torch.where(t > 0, t, 1.0))
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    rank = torch.arange(x.shape[1], device=DEV)
    top = torch.where(t > 0, torch.where(s.top_k[:, None] > 0, s.top_k[:, None], x.shape[1]), 1)
    kept = rank < top
    ws = ws * kept
    cum = ws.cumsum(-1)
    before = cum - ws
    p = s.top_p.double()[:, None]
    kept &= (before < p * cum[:, -1:]) | (p >= 1) | (rank == 0)
    kept &= (ws >= s.min_p.double()[:, None]) | (rank == 0)
    kept = torch.zeros_like(kept).scatter_(1, order, kept)
    w = w * kept
    cum = w.cumsum(-1)
    token = (cum > s.u.double()[:, None] * cum[:, -1:]).int().argmax(-1)
    s.token.copy_(token)
    s.prob.copy_(w.gather(1, token[:, None]).squeeze(1) / cum[:, -1])
    return dict(token=s.token, prob=s.prob)


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


def _blocks_of(s, table, counts):
    """The blocks that positions ctx .. ctx + count - 1 reach, as many for every sequence as the most (the
    last again for the others): positions [blocks][bt], sequence, page, block of the page, token of the page,
    new ones, older ones."""
    c = s.case
    bt, ps, S = c["block"], c["page"], c["seqs"]
    ctx = s.ctx.long()
    most = (s.max_new + bt - 2) // bt + 1
    last = torch.maximum((ctx + counts - 1) // bt, ctx // bt)
    b = torch.minimum((ctx // bt)[:, None] + torch.arange(most, device=DEV), last[:, None])
    at = (b[..., None] * bt + torch.arange(bt, device=DEV)).view(-1, bt)
    of = torch.arange(S, device=DEV)[:, None].expand(-1, most).reshape(-1)
    fresh, old = (at >= ctx[of, None]) & (at < (ctx + counts)[of, None]), at < ctx[of, None]
    page = table.long()[of, (at[:, 0] // ps).clamp(max=table.shape[1] - 1)].clamp(min=0)
    return at, of, page, at[:, 0] % ps // bt, at % ps, fresh, old


def _values_back(s, table):
    c = s.case
    ps, bt = c["page"], c["block"]
    seq, i = _of_token(s.back_cu, s.back_n)
    p = s.back_ctx.long()[seq] + i
    page, tok = table.long()[seq, p // ps], p % ps
    s.k_out.copy_((s.k[_k_at(page, tok)].float() * s.k_scale[page, :, tok // bt][..., None]).view(s.back_n, -1))
    s.v_out.copy_((s.v[_v_at(page, tok)].float() * s.v_scale[page, :, tok // bt][..., None]).view(s.back_n, -1))


def _draft(s):
    c = s.case
    n_q, n_kv, d = c["n_q"], c["n_kv"], c["d"]
    seq, i = _of_token(s.cu, s.n_tokens)
    x = s.qkv.float().view(s.n_tokens, n_q + 2 * n_kv, d)
    qk, v = x[:, :n_q + n_kv], x[:, n_q + n_kv:]
    if c["norm"]:
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + EPS)
        qk = torch.cat([qk[:, :n_q] * s.q_w.float(), qk[:, n_q:] * s.k_w.float()], 1)
    qk = _rotate(qk, s.ctx.long()[seq] + s.depth, s.inv_freq, c["rot"], c["inter"])
    q, k = qk[:, :n_q], qk[:, n_q:]
    if c["a8"]:
        sc = q.abs().amax(-1, keepdim=True) / 127.0
        q = _quant(q, sc) * sc
    s.q.copy_(q.reshape(s.n_tokens, -1))
    at, of, page, block, tok, fresh, old = _blocks_of(s, s.table, (s.cu[1:] - s.cu[:-1]).long())
    row = (s.cu.long()[of, None] + at - s.ctx.long()[of, None]).clamp(0, s.n_tokens - 1)
    _append_one(k[row], s.k, _k_at(page[:, None], tok), s.k_scale, page, block, fresh, old)
    _append_one(v[row], s.v, _v_at(page[:, None], tok), s.v_scale, page, block, fresh, old)
    _values_back(s, s.table)
    return dict(q=s.q, k=s.k_out, v=s.v_out, k_scale=s.k_scale, v_scale=s.v_scale)


def _seen_drafted(s):
    """[n_tokens][64 words] truth values of the mask's bits."""
    bits = torch.arange(64, device=DEV)
    return ((s.mask[..., None] >> bits) & 1).flatten(1).bool()


def _tree_attn(s):
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
    j = torch.arange(L, device=DEV) - s.ctx.long()[:, None]                      # [S][L]: which drafted token
    bits = _seen_drafted(s)
    seen = bits[row].gather(2, j[:, None].clamp(0, bits.shape[1] - 1).expand(S, N, L))
    n = (s.cu[1:] - s.cu[:-1]).long()
    seen = ((j < 0)[:, None] | seen) & (j < n[:, None])[:, None]
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


def _copy(s):
    for t in (s.k, s.v, s.k_scale, s.v_scale):
        t[s.dst.long()] = t[s.src.long()]
    return dict(k=s.k, v=s.v, k_scale=s.k_scale, v_scale=s.v_scale)


def _accept_one(codes, scale, place, s, moved):
    """The accepted tokens of one of the cache's arrays to the front of their sequences' drafted ones."""
    c = s.case
    bt, ps = c["block"], c["page"]
    at, of, page, block, tok, fresh, old = moved
    i = (at - s.ctx.long()[of, None]).clamp(min=0)
    src = s.ctx.long()[of, None] + s.keep.long()[(s.cu.long()[of, None] + i).clamp(max=s.n_tokens - 1)]
    src = torch.where(fresh, src, at)                                       # positions that tokens come from
    from_page = s.fork.long()[of[:, None], (src // ps).clamp(max=s.most - 1)].clamp(min=0)
    have = codes[place(from_page, src % ps)].float()                        # [blocks][bt][n_kv][d]
    sc = scale[from_page, :, src % ps // bt]                                # [blocks][bt][n_kv]
    now = torch.where((fresh | old)[..., None], sc, torch.zeros((), device=DEV)).amax(1)
    some = fresh.any(1)
    now = torch.where(some[:, None], now, scale[page, :, block])
    out = (have * (sc / now[:, None])[..., None]).round()
    write = ((fresh | old) & some[:, None])[..., None, None]
    codes[place(page[:, None], tok)] = torch.where(write, out, codes[place(page[:, None], tok)].float()).to(torch.int8)
    scale[page, :, block] = now


def _accept(s):
    for t in (s.k, s.v, s.k_scale, s.v_scale):
        t[s.dst.long()] = t[s.src.long()]
    moved = _blocks_of(s, s.fork, s.n_keep.long())
    _accept_one(s.k, s.k_scale, _k_at, s, moved)
    _accept_one(s.v, s.v_scale, _v_at, s, moved)
    _values_back(s, s.fork)
    return dict(k=s.k_out, v=s.v_out, k_scale=s.k_scale, v_scale=s.v_scale)


_OWN = dict(moe=_own_moe, draft=_own_draft, tree=_own_tree, sample=_own_sample, copy=_own_copy, accept=_own_accept)
_PLAIN = dict(moe=_moe, draft=_draft, tree=_tree_attn, sample=_sample, copy=_copy, accept=_accept)


# ------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["kind"]](case, s)


def _code64(x, s):
    q = torch.round(x / s.clamp(min=1e-300)).clamp(-127, 127)
    return q * (s > 0)


def _weights64(packed, alpha, g):
    w = torch.empty(packed.shape[:-1] + (packed.shape[-1] * 4,), dtype=torch.float64, device=DEV)
    for j in range(4):
        w[..., j::4] = ((packed >> (2 * j)) & 3).double() - 1
    return w * alpha.double().repeat_interleave(g, -1)


def _moe64(c, s):
    F, k = c["ffn"], c["k"]
    logits = s.logits.double().cpu().numpy()
    x = s.q.double() * s.x_scale.double()[:, None]
    y = s.res.double()
    users = {}
    for t in range(c["T"]):
        ids = sorted(range(c["E"]), key=lambda e: (-logits[t, e], e))[:k]
        w = np.exp(logits[t, ids] - logits[t, ids].max())
        for e, v in zip(ids, w / w.sum()):
            users.setdefault(e, []).append((t, float(v)))
    for e, us in sorted(users.items()):
        at = torch.tensor([t for t, _ in us], device=DEV)
        w = torch.tensor([v for _, v in us], dtype=torch.float64, device=DEV)
        z = x[at] @ _weights64(s.gu[e], s.gu_alpha[e], c["g"]).T
        a = z[:, :F] / (1 + torch.exp(-z[:, :F])) * z[:, F:]
        sc = a.abs().max(1, keepdim=True).values / 127
        y[at] += w[:, None] * ((_code64(a, sc) * sc) @ _weights64(s.down[e], s.down_alpha[e], c["g"]).T)
    return y


def _sample64(c, s):
    x = s.logits.double().cpu().numpy()
    T, K, P, M, U = (getattr(s, n).double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p", "u"))
    tokens, probs = [], []
    for r in range(c["rows"]):
        order = np.argsort(-x[r], kind="stable")
        n = 1 if T[r] <= 0 else len(order) if K[r] <= 0 else min(len(order), int(K[r]))
        order = order[:n]
        e = np.exp((x[r, order] - x[r, order[0]]) / (T[r] if T[r] > 0 else 1.0))
        if P[r] < 1:
            ahead = np.concatenate([[0.0], np.cumsum(e)])
            n = max(1, int((ahead[:-1] < P[r] * ahead[-1]).sum()))
        n = min(n, max(1, int((e >= M[r]).sum())))
        ids = np.sort(order[:n])
        w = np.exp((x[r, ids] - x[r, order[0]]) / (T[r] if T[r] > 0 else 1.0))
        cum = np.cumsum(w)
        at = min(int(np.searchsorted(cum, U[r] * cum[-1], side="right")), n - 1)
        tokens.append(int(ids[at]))
        probs.append(w[at] / cum[-1])
    return dict(token=torch.tensor(tokens, dtype=torch.int32, device=DEV),
                prob=torch.tensor(probs, dtype=torch.float64, device=DEV))


def _held64(c, s, table, i, n):
    """K and V codes [n_kv][n][d] of sequence i's first n positions, with their scales by token."""
    ps, n_kv, d = c["page"], c["n_kv"], c["d"]
    ids = table[i, :-(-n // ps)].long()
    out = []
    for codes, scale in ((s.k, s.k_scale), (s.v, s.v_scale)):
        x = codes[ids]
        x = x if x.dim() == 4 else x.movedim(-1, 3).reshape(len(ids), n_kv, ps, d)
        x = x.movedim(1, 0).reshape(n_kv, -1, d)[:, :n].double()
        t = scale[ids].movedim(1, 0).reshape(n_kv, -1).double()
        out.append((x, t.repeat_interleave(c["block"], 1)[:, :n]))
    return out


def _turned64(x, pos, s, c):
    rot = c["rot"]
    z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV).expand(len(pos), rot // 2).contiguous(),
                    pos.double()[:, None] * s.inv_freq.double())[:, None]
    y = x.clone()
    if c["inter"]:
        pairs = torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous())
        y[..., :rot] = torch.view_as_real(pairs * z).flatten(-2)
    else:
        w = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * z
        y[..., :rot // 2], y[..., rot // 2:rot] = w.real, w.imag
    return y


def _put64(c, table, i, scales, which, first, now):
    """Block scales [n_kv][blocks] from position ``first`` on into a copy of the pool's."""
    bt, ps = c["block"], c["page"]
    b = torch.arange(first // bt, first // bt + now.shape[1], device=DEV)
    scales[which][table[i].long()[b * bt // ps], :, b % (ps // bt)] = now.movedim(0, 1)


def _draft64(c, s):
    n_q, n_kv, d, bt = c["n_q"], c["n_kv"], c["d"], c["block"]
    x = s.qkv.double().view(-1, n_q + 2 * n_kv, d)
    scales = [s.k_scale.double(), s.v_scale.double()]
    qs, back, at = [], ([], []), 0
    for i, (ctx, new) in enumerate(_lens(c)):
        q, k, v = x[at:at + new].split([n_q, n_kv, n_kv], 1)
        pos = ctx + s.depth[at:at + new]
        at += new
        if c["norm"]:
            q = q / (q.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * s.q_w.double()
            k = k / (k.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * s.k_w.double()
        q, k = _turned64(q, pos, s, c), _turned64(k, pos, s, c)
        if c["a8"]:
            sc = q.abs().max(-1, keepdim=True).values / 127
            q = _code64(q, sc) * sc
        qs.append(q.reshape(new, -1))
        first, end = ctx // bt * bt, ctx + new
        held = _held64(c, s, s.table, i, end)
        pad = -end % bt
        for j, val in enumerate((k, v)):
            codes, old = held[j]
            codes = torch.nn.functional.pad(codes[:, first:], (0, 0, 0, pad)).unflatten(1, (-1, bt))
            was = torch.zeros(codes.shape[:2], dtype=torch.float64, device=DEV)
            if ctx % bt:
                was[:, 0] = old[:, first]
            val = torch.nn.functional.pad(val.movedim(1, 0), (0, 0, ctx - first, pad)).unflatten(1, (-1, bt))
            now = torch.maximum(val.abs().amax((2, 3)) / 127, was)
            mine = torch.arange(first, end + pad, device=DEV).view(-1, bt) >= ctx
            r = (was / now.clamp(min=1e-300))[..., None, None]
            q8 = torch.where(mine[None, ..., None], _code64(val, now[..., None, None]),
                             torch.where(r < 1, torch.round(codes * r), codes))
            y = (q8 * now[..., None, None]).flatten(1, 2)[:, :end - first]
            back[j].append(y.movedim(0, 1).reshape(end - first, -1))
            _put64(c, s.table, i, scales, j, first, now)
    return dict(q=torch.cat(qs), k=torch.cat(back[0]), v=torch.cat(back[1]), k_scale=scales[0], v_scale=scales[1])


def _tree64(c, s):
    n_q, n_kv, d = c["n_q"], c["n_kv"], c["d"]
    G = n_q // n_kv
    q = s.q.double().view(-1, n_kv, G, d)
    outs, lses, at = [], [], 0
    words = s.mask.tolist()
    for i, (ctx, new) in enumerate(_lens(c)):
        (kc, ks), (vc, vs) = _held64(c, s, s.table, i, ctx + new)
        hidden = torch.zeros((new, ctx + new), dtype=torch.bool)
        for r in range(new):
            for j in range(new):
                hidden[r, ctx + j] = not words[at + r][j // 64] >> j % 64 & 1
        hidden = hidden.to(DEV)
        o = torch.empty((new, n_q, d), dtype=torch.float64, device=DEV)
        lse = torch.empty((new, n_q), dtype=torch.float64, device=DEV)
        for h in range(n_kv):
            k, v = kc[h] * ks[h, :, None], vc[h] * vs[h, :, None]
            for g in range(G):
                sc = (q[at:at + new, h, g] @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                l = torch.logsumexp(sc, -1)
                o[:, h * G + g] = (sc - l[:, None]).exp() @ v
                lse[:, h * G + g] = l
        outs.append(o.view(new, -1))
        lses.append(lse)
        at += new
    return dict(o=torch.cat(outs), lse=torch.cat(lses))


def _copy64(c, s):
    out = {}
    for n in ("k", "v", "k_scale", "v_scale"):
        t = getattr(s, n).clone()
        for a, b in zip(s.src.tolist(), s.dst.tolist()):
            t[b] = t[a]
        out[n] = t.double() if n.endswith("scale") else None
    return out


def _accept64(c, s):
    n_kv, bt = c["n_kv"], c["block"]
    scales = [s.k_scale.double(), s.v_scale.double()]
    for t in scales:
        t[s.dst.long()] = t[s.src.long()]
    keep, back, at = s.keep.tolist(), ([], []), 0
    for i, ((ctx, new), n) in enumerate(zip(_lens(c), _kept(c))):
        first, end = ctx // bt * bt, ctx + n
        src = list(range(first, ctx)) + [ctx + keep[at + j] for j in range(n)]
        at += new
        held = _held64(c, s, s.table, i, ctx + new)      # (the fork's pages start as the sequence's)
        for j, (codes, scale) in enumerate(held):
            x, sc = codes[:, src], scale[:, src]
            if n:
                pad = -len(src) % bt
                now = torch.nn.functional.pad(sc, (0, pad)).unflatten(1, (-1, bt)).amax(2)
                _put64(c, s.fork, i, scales, j, first, now)
                by = now.repeat_interleave(bt, 1)[:, :len(src)]
                x, sc = torch.round(x * (sc / by)[..., None]), by
            back[j].append((x * sc[..., None]).movedim(0, 1).reshape(len(src), n_kv * c["d"]))
    return dict(k=torch.cat(back[0]), v=torch.cat(back[1]), k_scale=scales[0], v_scale=scales[1])


_EXACT = dict(moe=_moe64, draft=_draft64, tree=_tree64, sample=_sample64, copy=_copy64, accept=_accept64)
