"""A decode step with drafted tokens, all its calls together: a layer of attention over the cache and routed experts on packed
weights, its logits and the sampled tokens, for a tree of drafted tokens at once and for the same tokens one after the
other.  Both run the same codes through the same products; only the attention takes another way (tiles, order of sums,
probabilities rounded to fp16 there and here), so its bf16 output may differ by a rounding or two, and with it a code of the
8-bit quantizer: 1/127 of a row's largest value.  Over the few layers' sums that stays below a few percent of the largest
logit; tokens are compared where the largest logit leads by more."""
import pytest
import torch

pytestmark = pytest.mark.gpu

N_Q, N_KV, D, H, F, E, K, VOCAB, PS = 8, 2, 64, 512, 256, 12, 3, 9000, 16


class Model:
    """One layer with random packed weights, and what a program keeps for it."""

    def __init__(self, catq, pages, width, bt):
        self.c = catq
        g = torch.Generator(device="cuda")
        g.manual_seed(7)
        r = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731

        def packed(*shape):
            w = torch.zeros(shape[:-1] + (shape[-1] // 4,), dtype=torch.uint8, device="cuda")
            for j in range(4):
                w |= torch.randint(0, 3, w.shape, generator=g, device="cuda", dtype=torch.uint8) << 2 * j
            return w, (r(*shape[:-1], shape[-1] // 128) + 0.5) * 1.2 / shape[-1] ** 0.5
        self.qkv, self.o = packed((N_Q + 2 * N_KV) * D, H), packed(H, N_Q * D)
        self.gu, self.down = packed(E, 2 * F, H), packed(E, H, F)
        self.router = torch.randn((H, E), generator=g, device="cuda") / H ** 0.5
        self.embed = torch.randn((VOCAB, H), generator=g, device="cuda")
        self.moe = catq.moe_desc(E, K, H, F)
        self.desc = catq.kv_desc(N_Q, N_KV, D, PS, bt, pages, width)
        i8 = dict(dtype=torch.int8, device="cuda")
        self.pool = (torch.zeros((pages, N_KV, PS, D), **i8), torch.zeros((pages, N_KV, PS // 4, D, 4), **i8),
                     torch.zeros((pages, N_KV, PS // bt), device="cuda"), torch.zeros((pages, N_KV, PS // bt), device="cuda"))
        self.cache = catq.kv_cache(self.desc, *self.pool)
        self.prep = catq.kv_prep(self.desc, (1e4 ** (-torch.arange(D // 2) / (D // 2))).float().cuda(), rot_dim=D, qk_norm=True)

    def step(self, tokens, batch, tree=None):
        """fp32 logits of the batch's tokens."""
        c, n = self.c, len(tokens)
        bf = dict(dtype=torch.bfloat16, device="cuda")

        def quant(x, **kw):
            q, s = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
            c.catq_aux_rmsnorm_quant(x, q, s, **kw)
            return q, s
        x = self.embed[tokens]
        q8, s8 = quant(x)
        qkv, q, o, y = (torch.empty((n, w), **bf) for w in ((N_Q + 2 * N_KV) * D, N_Q * D, N_Q * D, H))
        c.catq_ternary_linear_a8(q8, s8, *self.qkv, qkv)
        ws = torch.empty(max(1, c.catq_paged_attention_workspace_bytes(self.desc, batch)), dtype=torch.uint8, device="cuda")
        if tree is None:
            c.catq_aux_kv_append(self.desc, self.cache, batch, self.prep, qkv, q)
            c.catq_aux_paged_attention(self.desc, self.cache, batch, q, o, ws)
        else:
            c.catq_aux_kv_append_tree(self.desc, self.cache, batch, tree, self.prep, qkv, q)
            c.catq_aux_tree_attention(self.desc, self.cache, batch, tree, q, o, ws)
        oq, os = torch.empty(o.shape, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        c.catq_aux_act_quant8(o, oq, os)
        c.catq_ternary_linear_a8(oq, os, *self.o, y)
        h = torch.empty_like(x)
        q8, s8 = quant(y, res=x, sum=h)
        logits = (q8.float() * s8[:, None]) @ self.router
        out = torch.empty((n, H), device="cuda")
        mws = torch.empty(c.catq_ternary_moe_a8_workspace_bytes(self.moe, n), dtype=torch.uint8, device="cuda")
        c.catq_ternary_moe_a8(self.moe, logits, q8, s8, *self.gu, *self.down, out, mws, res=h)
        return out @ self.embed.T / H ** 0.5

    def sample(self, logits, u, **kw):
        n = len(logits)
        token, prob = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
        ws = torch.empty(max(16, self.c.catq_aux_sample_workspace_bytes(n, VOCAB)), dtype=torch.uint8, device="cuda")
        self.c.catq_aux_sample(logits, u, token, ws, prob=prob, **kw)
        return token


@pytest.mark.parametrize("bt", [1, 16])
def test_a_step_with_drafted_tokens(catq, bt):
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator()
    g.manual_seed(3)
    prompts = [37, 5]
    parents = [[-1, 0, 0, 1, 2, 3, 3, -1], [-1, 0, 1, 1]]
    paths = [[0, 1, 3, 6], [0, 1, 3]]
    table = torch.full((2, 5), -1, dtype=torch.int32)
    table[0, :4] = torch.tensor([8, 2, 5, 0])
    table[1, :2] = torch.tensor([3, 7])
    ids = [torch.randint(0, VOCAB, (p + len(t),), generator=g).cuda() for p, t in zip(prompts, parents)]
    got = []
    for drafted in (True, False):
        m = Model(catq, 9, 5, bt)
        t = table.cuda()
        cu = torch.tensor([0, prompts[0], sum(prompts)], **i32)
        first = catq.kv_batch(m.desc, t, cu, torch.zeros(2, **i32), sum(prompts), max(prompts), max(prompts))
        m.step(torch.cat([x[:p] for x, p in zip(ids, prompts)]), first)
        ctx = torch.tensor(prompts, **i32)
        if drafted:
            n = [len(p) for p in parents]
            depth, masks = [], []
            for tree in parents:
                d, rows = [], []
                for j, p in enumerate(tree):
                    d.append(0 if p < 0 else d[p] + 1)
                    rows.append((rows[p] if p >= 0 else 0) | 1 << j)
                depth += d
                masks += rows
            b = catq.kv_batch(m.desc, t, torch.tensor([0, n[0], sum(n)], **i32), ctx, sum(n), max(n), 64)
            tree = catq.kv_tree(b, torch.tensor(masks, dtype=torch.int64).view(-1, 1).cuda(), torch.tensor(depth, **i32))
            logits = m.step(torch.cat([x[p:] for x, p in zip(ids, prompts)]), b, tree)
            rows = [j for j in paths[0]] + [n[0] + j for j in paths[1]]
            keep = torch.zeros(sum(n), **i32)
            keep[:4], keep[n[0]:n[0] + 3] = torch.tensor(paths[0]), torch.tensor(paths[1])
            catq.catq_aux_kv_compact(m.desc, m.cache, b, keep, torch.tensor([4, 3], **i32))
            logits = logits[rows]
        else:
            out = [[], []]
            for i in range(4):       # the paths, a token of each sequence at a time
                live = [s for s in range(2) if i < len(paths[s])]
                tok = torch.stack([ids[s][prompts[s] + paths[s][i]] for s in live])
                b = catq.kv_batch(m.desc, t[live].contiguous(), torch.arange(len(live) + 1, **i32),
                                  (ctx + i)[live].contiguous(), len(live), 1, 64)
                for s, row in zip(live, m.step(tok, b)):
                    out[s].append(row)
            logits = torch.stack(out[0] + out[1])
        # what follows: one more token of each sequence, behind its path
        tok = torch.tensor([11, 12], device="cuda")
        b = catq.kv_batch(m.desc, t, torch.tensor([0, 1, 2], **i32), ctx + torch.tensor([4, 3], **i32), 2, 1, 64)
        logits = torch.cat([logits, m.step(tok, b)])
        n = len(logits)
        u = torch.linspace(0.01, 0.99, n).cuda()
        greedy = m.sample(logits, u, temperature=torch.zeros(n, device="cuda"))
        top = m.sample(logits, u, top_k=torch.full((n,), 1, **i32))
        assert torch.equal(greedy, logits.argmax(-1).int()) and torch.equal(greedy, top)
        some = m.sample(logits, u, top_k=torch.full((n,), 5, **i32), top_p=torch.full((n,), 0.9, device="cuda"))
        assert (logits.gather(1, some[:, None].long()) >= logits.topk(5).values[:, 4:]).all()
        got.append((logits, greedy))
    (a, ta), (b, tb) = got
    assert torch.isfinite(a).all()
    bound = 0.05 * b.abs().max()
    assert (a - b).abs().max() <= bound, float((a - b).abs().max() / b.abs().max())
    lead = b.topk(2).values
    clear = lead[:, 0] - lead[:, 1] > 2 * bound
    assert torch.equal(ta[clear], tb[clear])
