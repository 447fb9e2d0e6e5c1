"""Refusals of the calls for drafted tokens, pages, sampling and the experts' layer, without a GPU: everything below fails
a check before any launch (the fake device addresses are never dereferenced), or is a no-op."""
import ctypes as C
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_26650_amd", "libcatq.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libcatq.so not built")

FAKE = 0x100000
NULL, SHAPE, DTYPE, VALUE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5, 6
R = C.byref


@pytest.fixture(scope="module")
def cq():
    import paper_2606_26650_amd as pkg
    return pkg


def _structs(cq, **kw):
    def pick(base):
        return dict(base, **{k: v for k, v in kw.items() if k in base})
    d = cq.KvDesc(**pick(dict(n_q=8, n_kv=2, head_dim=128, page_size=64, scale_block=16, n_pages=10, max_pages=4)))
    b = cq.KvBatch(**pick(dict(page_table=FAKE, cu_new=FAKE, ctx_len=FAKE, n_tokens=5, n_seqs=2, max_new=3, max_len=100)))
    c = cq.KvCache(**pick(dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE)))
    p = cq.KvPrep(**pick(dict(inv_freq=FAKE, q_weight=None, k_weight=None, rot_dim=128, interleaved=0, qk_norm=1,
                              act_quant=0, rope_scale=1.0, eps=1e-6)))
    t = cq.KvTree(**pick(dict(mask=FAKE, depth=FAKE, words=1)))
    return d, c, b, p, t


def test_tree_refusals(cq):
    L = cq.lib

    def both(qkv=FAKE, q=FAKE, o=FAKE, lse=FAKE, ws=FAKE, n=1 << 40, scale=0.1, **kw):
        d, c, b, p, t = _structs(cq, **kw)
        return (L.catq_aux_kv_append_tree(R(d), R(c), R(b), R(t), R(p), qkv, q, None),
                L.catq_aux_tree_attention(R(d), R(c), R(b), R(t), q, scale, o, lse, ws, n, None))

    for k in ("k", "v", "k_scale", "v_scale", "page_table", "cu_new", "ctx_len"):
        assert both(**{k: None}) == (NULL, NULL), k
    for kw in (dict(n_q=7), dict(head_dim=96), dict(page_size=48), dict(scale_block=24), dict(max_len=257),
               dict(n_tokens=-1), dict(words=0), dict(words=-1), dict(words=1025), dict(max_new=65),
               dict(max_new=129, words=2)):
        assert both(**kw) == (SHAPE, SHAPE), kw
    assert both(mask=FAKE + 4) == (ALIGN, ALIGN) and both(depth=FAKE + 2) == (ALIGN, ALIGN)
    assert both(q=FAKE + 8) == (ALIGN, ALIGN) and both(q=None) == (NULL, NULL)
    for kw in (dict(n_seqs=0, page_table=None), dict(n_tokens=0), dict(max_new=0)):
        assert both(qkv=None, q=None, o=None, **kw) == (0, 0), kw
    assert both(mask=None)[1] == NULL                      # (the append does not read it: no call here)
    d, c, b, p, t = _structs(cq)
    assert L.catq_aux_kv_append_tree(R(d), R(c), R(b), None, R(p), FAKE, FAKE, None) == NULL
    assert L.catq_aux_kv_append_tree(R(d), R(c), R(b), R(t), None, FAKE, FAKE, None) == NULL
    assert L.catq_aux_tree_attention(R(d), R(c), R(b), None, FAKE, 0.1, FAKE, None, None, 0, None) == NULL
    assert both(scale=-1.0)[1] == VALUE and both(scale=float("nan"))[1] == VALUE
    assert both(o=None)[1] == NULL and both(lse=FAKE + 2)[1] == ALIGN
    long = dict(page_size=256, max_pages=64, n_pages=64, max_len=16384)
    d, c, b, _, _ = _structs(cq, **long)
    need = L.catq_paged_attention_workspace_bytes(R(d), R(b))
    assert need > 0
    assert both(n=need - 1, **long)[1] == WORKSPACE and both(ws=None, **long)[1] == WORKSPACE


def test_append_by_depth_alone_has_no_mask_limits(cq):
    """The append of a tree does not read the mask: without one its words are not looked at, and as many new tokens are
    taken as by the plain append (no tokens here, so nothing is launched)."""
    L = cq.lib
    big = dict(n_tokens=0, max_new=70000, max_pages=2000, n_pages=2000, max_len=100000)

    def append(qkv=FAKE, **kw):
        d, c, b, p, t = _structs(cq, **dict(big, **kw))
        return L.catq_aux_kv_append_tree(R(d), R(c), R(b), R(t), R(p), qkv, FAKE, None)

    for words in (1094, 1024, 1, 0, -1):
        assert append(mask=None, words=words) == 0, words
        assert append(mask=None, depth=None, words=words) == 0, words
    assert append(mask=None, max_new=1 << 24) == 0 and append(mask=None, max_new=(1 << 24) + 1) == SHAPE
    assert append(mask=None, depth=FAKE + 2) == ALIGN
    assert append(words=1024) == SHAPE and append(words=1094) == SHAPE       # (a mask, too long for the attention)
    d, c, b, p, t = _structs(cq, **big, mask=None, words=1)
    assert L.catq_aux_tree_attention(R(d), R(c), R(b), R(t), FAKE, 0.1, FAKE, None, None, 0, None) == SHAPE
    b.device = -1
    assert cq.kv_tree(b).words == 1094


def test_page_refusals(cq):
    L = cq.lib

    def copy(src=FAKE, dst=FAKE, n=3, **kw):
        d, c = _structs(cq, **kw)[:2]
        return L.catq_aux_kv_copy_pages(R(d), R(c), src, dst, n, None)

    assert copy(n=0, src=None, dst=None) == 0
    assert copy(src=None) == NULL and copy(dst=None) == NULL and copy(k=None) == NULL and copy(v_scale=None) == NULL
    assert copy(n=-1) == SHAPE and copy(n=1 << 24) == SHAPE and copy(n=1 << 40) == SHAPE
    assert copy(head_dim=32) == SHAPE and copy(n_pages=0) == SHAPE
    assert copy(src=FAKE + 2) == ALIGN and copy(dst=FAKE + 1) == ALIGN and copy(v=FAKE + 8) == ALIGN
    d, c, b = _structs(cq)[:3]
    assert L.catq_aux_kv_copy_pages(None, R(c), FAKE, FAKE, 1, None) == NULL
    assert L.catq_aux_kv_copy_pages(R(d), None, FAKE, FAKE, 1, None) == NULL

    def compact(keep=FAKE, n_keep=FAKE, **kw):
        d, c, b = _structs(cq, **kw)[:3]
        return L.catq_aux_kv_compact(R(d), R(c), R(b), keep, n_keep, None)

    for kw in (dict(n_seqs=0, page_table=None), dict(n_tokens=0), dict(max_new=0)):
        assert compact(keep=None, n_keep=None, **kw) == 0
    assert compact(keep=None) == NULL and compact(n_keep=None) == NULL and compact(cu_new=None) == NULL
    assert compact(keep=FAKE + 2) == ALIGN and compact(n_keep=FAKE + 1) == ALIGN
    assert compact(scale_block=2) == SHAPE and compact(n_seqs=65536) == SHAPE
    assert L.catq_aux_kv_compact(R(d), R(c), None, FAKE, FAKE, None) == NULL


def test_sample_refusals(cq):
    ok = dict(x=FAKE, dt=0, rows=4, V=100, ld=100, T=FAKE, k=FAKE, p=FAKE, m=FAKE, u=FAKE, tok=FAKE, prob=FAKE, ws=FAKE,
              n=1 << 40)

    def call(**kw):
        a = dict(ok, **kw)
        return cq.lib.catq_aux_sample(a["x"], a["dt"], a["rows"], a["V"], a["ld"], a["T"], a["k"], a["p"], a["m"], a["u"],
                                      a["tok"], a["prob"], a["ws"], a["n"], None)

    assert call(rows=0, x=None, u=None, tok=None, ws=None) == 0
    assert call(rows=-1) == SHAPE and call(rows=65536) == SHAPE
    assert call(x=None) == NULL and call(u=None) == NULL and call(tok=None) == NULL
    assert call(dt=2) == DTYPE
    assert call(V=0) == SHAPE and call(V=(1 << 20) + 1, ld=1 << 21) == SHAPE and call(ld=99) == SHAPE
    assert call(rows=60000, ld=1 << 23) == SHAPE
    for k in ("x", "ws"):
        assert call(**{k: FAKE + 8}) == ALIGN, k
    for k in ("T", "k", "p", "m", "u", "tok", "prob"):
        assert call(**{k: FAKE + 2}) == ALIGN, k
    need = cq.catq_aux_sample_workspace_bytes(64, 150000)
    if need:
        assert call(rows=64, V=150000, ld=150000, n=need - 1) == WORKSPACE
        assert call(rows=64, V=150000, ld=150000, ws=None) == WORKSPACE
    assert cq.catq_aux_sample_workspace_bytes(0, 5) == 0 and cq.catq_aux_sample_workspace_bytes(-1, -1) == 0


def test_sample_workspace_serves_fewer_rows(cq):
    """A program sizes its workspace once, for its largest batch: the size never falls as rows (or the vocabulary) rise."""
    need = cq.catq_aux_sample_workspace_bytes
    rows = [1, 2, 64, 254, 255, 256, 257, 300, 1024, 1025, 65535]
    for V in (1, 16384, 16385, 32000, 65536, 65537, 150000, 1 << 20):
        sizes = [need(r, V) for r in rows]
        assert sizes == sorted(sizes), V
    for r in rows:
        sizes = [need(r, V) for V in (1, 16384, 16385, 65536, 65537, 1 << 20)]
        assert sizes == sorted(sizes), r
    assert need(65536, 32000) == 0 and need(5, (1 << 20) + 1) == 0 and need(5, 0) == 0


def test_moe_refusals(cq):
    ok = dict(E=8, k=2, h=256, F=128, g=128, x=FAKE, q=FAKE, T=4, ld=256, xs=FAKE, P1=FAKE, A1=FAKE, P2=FAKE, A2=FAKE,
              res=FAKE, y=FAKE, dt=1, ws=FAKE, n=1 << 40)

    def call(**kw):
        a = dict(ok, **kw)
        d = cq.MoeDesc(a["E"], a["k"], a["h"], a["F"], a["g"])
        return cq.lib.catq_ternary_moe_a8(R(d), a["x"], a["q"], a["T"], a["ld"], a["xs"], a["P1"], a["A1"], a["P2"],
                                          a["A2"], a["res"], a["y"], a["dt"], a["ws"], a["n"], None)

    assert call(T=0, x=None, q=None, y=None, ws=None) == 0
    for k in ("x", "q", "xs", "P1", "A1", "P2", "A2", "y"):
        assert call(**{k: None}) == NULL, k
    assert cq.lib.catq_ternary_moe_a8(None, *[FAKE] * 2, 1, 256, *[FAKE] * 7, 1, FAKE, 1 << 40, None) == NULL
    for kw in (dict(E=0), dict(E=1025), dict(k=0), dict(k=9), dict(k=17, E=32), dict(h=192, ld=192), dict(F=100),
               dict(h=0), dict(F=-128), dict(h=32768 + 128, ld=1 << 16), dict(F=32768 + 128), dict(T=-1), dict(T=1025),
               dict(ld=240), dict(ld=264), dict(ld=(1 << 24) + 16)):
        assert call(**kw) == SHAPE, kw
    for g in (0, 64, 384, -128):
        assert call(g=g, h=768, ld=768, F=768) == VALUE, g
    assert call(g=256) == SHAPE                              # (ffn 128)
    assert call(dt=3) == DTYPE
    for k in ("q", "P1", "A1", "P2", "A2", "res", "y", "ws"):
        assert call(**{k: FAKE + 8}) == ALIGN, k
    for k in ("x", "xs"):
        assert call(**{k: FAKE + 2}) == ALIGN, k
    need = cq.catq_ternary_moe_a8_workspace_bytes(cq.moe_desc(8, 2, 256, 128), 4)
    assert need >= 4 * 2 * 128 * 5
    assert call(n=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE
    assert cq.catq_ternary_moe_a8_workspace_bytes(cq.moe_desc(8, 2, 256, 128), 0) == 0
    assert cq.catq_ternary_moe_a8_workspace_bytes(cq.moe_desc(8, 9, 256, 128), 4) == 0


def test_wrappers_refuse_other_tensors(cq):
    """What the Python face checks before the library sees a pointer."""
    with pytest.raises(ValueError):
        cq.moe_desc(2 ** 31, 1, 128, 128)
    d = cq.moe_desc(4, 2, 256, 128)
    t = dict(logits=torch.zeros(3, 4), q=torch.zeros((3, 256), dtype=torch.int8), x_scale=torch.zeros(3),
             gu_packed=torch.zeros((4, 256, 64), dtype=torch.uint8), gu_alpha=torch.zeros((4, 256, 2)),
             down_packed=torch.zeros((4, 256, 32), dtype=torch.uint8), down_alpha=torch.zeros((4, 256, 1)),
             y=torch.zeros((3, 256)), workspace=torch.zeros(64, dtype=torch.uint8))
    for name, bad, err in (
            ("logits", torch.zeros(3, 5), ValueError), ("logits", torch.zeros(3, 4).double(), TypeError),
            ("q", torch.zeros((3, 256)), TypeError), ("q", torch.zeros((2, 256), dtype=torch.int8), ValueError),
            ("q", torch.zeros((256, 3), dtype=torch.int8).T, ValueError), ("x_scale", torch.zeros(4), ValueError),
            ("gu_packed", torch.zeros((4, 128, 64), dtype=torch.uint8), ValueError),
            ("gu_alpha", torch.zeros((4, 256, 1)), ValueError),
            ("down_packed", torch.zeros((4, 256, 32), dtype=torch.int8), TypeError),
            ("down_alpha", torch.zeros((4, 1, 256)).transpose(1, 2)[:, ::2], ValueError),
            ("y", torch.zeros((3, 256), dtype=torch.float16), TypeError), ("res", torch.zeros((3, 256)).bfloat16(), TypeError)):
        with pytest.raises(err):
            cq.catq_ternary_moe_a8(d, **dict(t, **{name: bad}))
    with pytest.raises(ValueError, match="on a GPU"):
        cq.catq_ternary_moe_a8(d, **t)
    s = dict(logits=torch.zeros(3, 50), u=torch.zeros(3), token=torch.zeros(3, dtype=torch.int32))
    for name, bad, err in (
            ("logits", torch.zeros(3, 50).half(), TypeError), ("logits", torch.zeros(50), ValueError),
            ("logits", torch.zeros(50, 3).T, ValueError), ("u", torch.zeros(4), ValueError),
            ("token", torch.zeros(3, dtype=torch.int64), TypeError), ("top_k", torch.zeros(3), TypeError),
            ("temperature", torch.zeros(3, 1), ValueError), ("prob", torch.zeros(6)[::2], ValueError)):
        with pytest.raises(err):
            cq.catq_aux_sample(**dict(s, **{name: bad}))
    with pytest.raises(ValueError, match="on a GPU"):
        cq.catq_aux_sample(**s)


def test_tree_wrappers(cq):
    b = cq.KvBatch(None, None, None, 5, 2, 70, 100)
    b.device = -1
    for mask, depth, err in ((torch.zeros(5, 2), None, TypeError), (torch.zeros((4, 2), dtype=torch.int64), None, ValueError),
                             (torch.zeros(5, dtype=torch.int64), None, ValueError),
                             (None, torch.zeros(4, dtype=torch.int32), ValueError),
                             (None, torch.zeros(5, dtype=torch.int64), TypeError),
                             (torch.zeros((5, 4), dtype=torch.int64)[:, ::2], None, ValueError)):
        with pytest.raises(err):
            cq.kv_tree(b, mask, depth)
    assert cq.kv_tree(b).words == 2 and cq.kv_tree(b, torch.zeros((5, 3), dtype=torch.int64)).words == 3
    other = cq.KvBatch(None, None, None, 6, 2, 70, 100)
    other.device = -1
    with pytest.raises(ValueError, match="made for 5"):
        cq._tree_same(cq.kv_tree(b), other)
