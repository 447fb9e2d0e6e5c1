"""Refusals of the serving entry points, without a GPU: everything below fails a check
before any launch (the fake device addresses are never dereferenced), or is a no-op."""
import ctypes as C
import os

import pytest
import torch

import serving_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_26650_amd", "libcatq.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libcatq.so not built")

FAKE = 0x100000
NULL, SHAPE, DTYPE, VALUE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def cq():
    import paper_2606_26650_amd as pkg
    return pkg


def test_norm_quant_refusals(cq):
    ok = dict(x=FAKE, xd=1, res=FAKE, rd=0, w=FAKE, rows=4, n=256, group=64, eps=1e-6, sum=FAKE + 4096, y=FAKE,
              q=FAKE, s=FAKE)

    def call(**kw):
        a = dict(ok, **kw)
        return cq.lib.catq_aux_rmsnorm_quant(a["x"], a["xd"], a["res"], a["rd"], a["w"], a["rows"], a["n"],
                                             a["group"], a["eps"], a["sum"], a["y"], a["q"], a["s"], None)

    assert call(rows=0, x=None, q=None) == 0                 # no rows: nothing is read
    assert call(rows=-1) == SHAPE
    assert call(x=None) == NULL
    assert call(q=None) == NULL and call(s=None) == NULL     # q and scale go together
    assert call(q=None, s=None, y=None) == NULL
    assert call(res=None) == NULL                            # sum without res
    assert call(xd=2) == DTYPE and call(rd=7) == DTYPE
    assert call(group=24) == SHAPE and call(n=252, group=252) == SHAPE and call(group=0) == SHAPE
    assert call(n=32776, group=32776) == SHAPE
    assert call(rows=1 << 40) == SHAPE
    assert call(eps=-1.0) == VALUE and call(eps=float("nan")) == VALUE
    assert call(sum=FAKE) == VALUE                           # an fp32 sum over a bf16 x
    for k in ("x", "res", "w", "sum", "y"):
        assert call(**{k: FAKE + 8}) == ALIGN, k
    assert call(q=FAKE + 4) == ALIGN and call(s=FAKE + 2) == ALIGN
    f = cq.lib.catq_aux_act_quant8
    assert f(None, 1, 0, 64, 64, None, None, None) == 0
    assert f(FAKE, 1, 4, 64, 24, FAKE, FAKE, None) == SHAPE
    assert f(FAKE, 1, 4, 64, 64, None, FAKE, None) == NULL and f(FAKE, 1, 4, 64, 64, FAKE, None, None) == NULL
    assert f(FAKE, 5, 4, 64, 64, FAKE, FAKE, None) == DTYPE
    assert f(FAKE + 2, 1, 4, 64, 64, FAKE, FAKE, None) == ALIGN


def test_linear_a8_refusals(cq):
    ok = dict(q=FAKE, M=4, ldq=256, xs=FAKE, P=FAKE, A=FAKE, d_out=32, d_in=256, g=128, Y=FAKE, dt=0, ldy=32)

    def call(**kw):
        a = dict(ok, **kw)
        return cq.lib.catq_ternary_linear_a8(a["q"], a["M"], a["ldq"], a["xs"], a["P"], a["A"], a["d_out"],
                                             a["d_in"], a["g"], a["Y"], a["dt"], a["ldy"], None)

    assert call(M=0, q=None, P=None) == 0
    assert call(M=-1) == SHAPE
    for k in ("q", "xs", "P", "A", "Y"):
        assert call(**{k: None}) == NULL
    assert call(d_in=192) == SHAPE and call(d_out=0) == SHAPE
    assert call(g=64) == VALUE and call(g=0) == VALUE and call(g=384, d_in=768, ldq=768) == VALUE
    assert call(d_in=65536 + 128, ldq=65536 + 128) == SHAPE
    assert call(ldq=240) == SHAPE and call(ldq=264) == SHAPE and call(ldq=(1 << 24) + 16) == SHAPE
    assert call(ldy=31) == SHAPE
    assert call(dt=3) == DTYPE
    assert call(M=16 * 65536) == SHAPE
    assert call(q=FAKE + 8) == ALIGN and call(A=FAKE + 4) == ALIGN and call(P=FAKE + 4) == ALIGN
    assert call(Y=FAKE + 2) == ALIGN and call(xs=FAKE + 2) == ALIGN


def _structs(cq, **kw):
    d = dict(n_q=8, n_kv=2, head_dim=128, page_size=64, scale_block=16, n_pages=10, max_pages=4)
    d.update({k: v for k, v in kw.items() if k in d})
    b = dict(page_table=FAKE, cu_new=FAKE, ctx_len=FAKE, n_tokens=5, n_seqs=2, max_new=3, max_len=100)
    b.update({k: v for k, v in kw.items() if k in b})
    c = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE)
    c.update({k: v for k, v in kw.items() if k in c})
    p = dict(inv_freq=FAKE, q_weight=None, k_weight=None, rot_dim=128, interleaved=0, qk_norm=1, act_quant=0,
             rope_scale=1.0, eps=1e-6)
    p.update({k: v for k, v in kw.items() if k in p})
    return cq.KvDesc(**d), cq.KvCache(**c), cq.KvBatch(**b), cq.KvPrep(**p)


def test_cache_refusals(cq):
    L, R = cq.lib, C.byref

    def all_of(qkv=FAKE, q=FAKE, ko=FAKE, o=FAKE, lse=FAKE, ws=FAKE, scale=0.1, **kw):
        d, c, b, p = _structs(cq, **kw)
        return (L.catq_aux_kv_append(R(d), R(c), R(b), R(p), qkv, q, None),
                L.catq_aux_kv_read(R(d), R(c), R(b), ko, None, None),
                L.catq_aux_paged_attention(R(d), R(c), R(b), q, scale, o, lse, ws, 1 << 40, None))

    for k in ("k", "v", "k_scale", "v_scale", "page_table", "cu_new", "ctx_len"):
        assert all_of(**{k: None}) == (NULL,) * 3, k
    for k in ("k", "v", "k_scale", "v_scale"):
        assert all_of(**{k: FAKE + 8}) == (ALIGN,) * 3, k
    assert all_of(cu_new=FAKE + 2) == (ALIGN,) * 3
    for kw in (dict(n_q=7), dict(n_q=0), dict(n_q=2048, n_kv=2), dict(head_dim=96), dict(page_size=8), dict(page_size=48),
               dict(page_size=512, max_pages=1), dict(scale_block=2), dict(scale_block=24), dict(scale_block=128),
               dict(page_size=256, scale_block=256), dict(n_pages=0), dict(max_pages=0), dict(max_len=257),
               dict(n_seqs=-1), dict(n_tokens=-1), dict(max_new=-1), dict(max_len=-1), dict(n_seqs=65536),
               dict(n_tokens=1 << 31), dict(max_new=(1 << 24) + 1), dict(n_pages=2 ** 31 - 1, n_kv=8)):
        assert all_of(**kw) == (SHAPE,) * 3, kw
    # nothing to do: nothing is read
    for kw in (dict(n_seqs=0, page_table=None), dict(n_tokens=0), dict(max_new=0)):
        assert all_of(qkv=None, q=None, o=None, ko=None, **kw) == (0, 0, 0), kw

    def append(qkv=FAKE, q=FAKE, **kw):
        d, c, b, p = _structs(cq, **kw)
        return L.catq_aux_kv_append(R(d), R(c), R(b), R(p), qkv, q, None)

    d, c, b, p = _structs(cq)
    assert L.catq_aux_kv_append(None, R(c), R(b), R(p), FAKE, FAKE, None) == NULL
    assert L.catq_aux_kv_append(R(d), None, R(b), R(p), FAKE, FAKE, None) == NULL
    assert L.catq_aux_kv_append(R(d), R(c), None, R(p), FAKE, FAKE, None) == NULL
    assert L.catq_aux_kv_append(R(d), R(c), R(b), None, FAKE, FAKE, None) == NULL
    assert append(qkv=None) == NULL and append(q=None) == NULL and append(inv_freq=None) == NULL
    assert append(qkv=FAKE + 8) == ALIGN and append(q=FAKE + 8) == ALIGN and append(k_weight=FAKE + 2) == ALIGN
    assert append(rot_dim=24) == SHAPE and append(rot_dim=144) == SHAPE and append(rot_dim=-16) == SHAPE
    assert append(interleaved=2) == VALUE and append(qk_norm=-1) == VALUE and append(eps=-1.0) == VALUE
    assert L.catq_aux_kv_read(R(d), R(c), R(b), None, None, None) == NULL
    assert L.catq_aux_kv_read(R(d), R(c), R(b), FAKE + 8, None, None) == ALIGN

    def attend(q=FAKE, scale=0.1, o=FAKE, lse=None, ws=FAKE, n=1 << 40, **kw):
        d, c, b, _ = _structs(cq, **kw)
        return L.catq_aux_paged_attention(R(d), R(c), R(b), q, scale, o, lse, ws, n, None)

    assert attend(q=None) == NULL and attend(o=None) == NULL
    assert attend(scale=-0.1) == VALUE and attend(scale=float("nan")) == VALUE and attend(scale=float("inf")) == VALUE
    assert attend(q=FAKE + 8) == ALIGN and attend(o=FAKE + 2) == ALIGN and attend(lse=FAKE + 2) == ALIGN
    assert attend(ws=FAKE + 8) == ALIGN
    assert attend(max_pages=4000, max_len=200000, ws=None, n=0) == WORKSPACE
    assert attend(max_pages=4000, max_len=200000, n=64) == WORKSPACE


def test_launch_limits(cq):
    """A call whose launch would have 2^32 threads or more along one axis is refused."""
    L, R = cq.lib, C.byref
    norm = lambda rows, n: L.catq_aux_rmsnorm_quant(FAKE, 1, None, 1, None, rows, n, n, 1e-6, None, FAKE, None,
                                                    None, None)
    assert norm(1 << 24, 8192) == SHAPE and norm(1 << 22, 16384) == SHAPE
    assert L.catq_aux_act_quant8(FAKE, 1, 1 << 24, 64, 64, FAKE, FAKE, None) == SHAPE
    assert L.catq_ternary_linear_a8(FAKE, 4, 256, FAKE, FAKE, FAKE, 1 << 27, 256, 128, FAKE, 0, 1 << 27,
                                    None) == SHAPE
    for kw in (dict(n_tokens=(1 << 24) // 8, n_seqs=1, max_pages=100, max_len=6000),      # the spans' join
               dict(n_q=1024, n_kv=1024, max_new=1 << 22, max_len=1 << 20, max_pages=1 << 14, n_pages=1)):
        d, c, b, _ = _structs(cq, **kw)
        assert L.catq_aux_paged_attention(R(d), R(c), R(b), FAKE, 0.1, FAKE, None, FAKE, 1 << 62, None) == SHAPE, kw
    d, c, b, p = _structs(cq, n_q=1024, n_kv=1024, n_tokens=1 << 20, max_new=1 << 20, max_pages=1 << 16, n_pages=1)
    assert L.catq_aux_kv_append(R(d), R(c), R(b), R(p), FAKE, FAKE, None) == SHAPE
    assert L.catq_aux_kv_read(R(d), R(c), R(b), FAKE, None, None) == SHAPE


def test_workspace_bytes(cq):
    """None for what needs none or is refused; as many partial results as spans otherwise."""
    def need(**kw):
        d, _, b, _ = _structs(cq, **kw)
        return cq.catq_paged_attention_workspace_bytes(d, b)

    assert need(n_seqs=0) == 0 and need(head_dim=96) == 0 and need(max_len=64) == 0
    one = need(max_pages=4000, max_len=100000, n_tokens=1, n_seqs=1, max_new=1)
    assert one >= 8 * (128 + 2) * 4 and one % 256 == 0
    assert need(max_pages=4000, max_len=100000, n_tokens=2, n_seqs=2, max_new=1) <= 2 * one


def test_python_checks(cq):
    """The wrappers refuse host tensors, types, shapes and layouts before the library."""
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    q, s = torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2, 1)
    with pytest.raises(ValueError, match="GPU"):
        cq.catq_aux_rmsnorm_quant(x, q, s)
    with pytest.raises(TypeError, match="dtype"):
        cq.catq_aux_rmsnorm_quant(x.half(), q, s)
    with pytest.raises(ValueError, match="contiguous"):
        cq.catq_aux_act_quant8(torch.zeros(64, 2, dtype=torch.bfloat16).T, q, s)
    with pytest.raises(TypeError, match="packed"):
        cq.catq_ternary_linear_a8(q, s, q, s, x)
    d = cq.kv_desc(4, 2, 64, 16, 16, 3, 2)
    with pytest.raises(ValueError, match="shape"):
        cq.kv_cache(d, torch.zeros(3, 2, 16, 32, dtype=torch.int8), q, s, s)
    with pytest.raises(ValueError, match="GPU"):
        cq.kv_batch(d, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                    torch.zeros(1, dtype=torch.int32), 1, 1, 1)
    with pytest.raises(TypeError, match="dtype"):
        cq.kv_prep(d, torch.zeros(32, dtype=torch.float64), rot_dim=64)


def test_scales_in_another_order_are_refused(cq):
    """Scales and alpha laid out group by group have the right count; flat ones, and rows in several
    dimensions, are taken (up to the refusal of host tensors)."""
    z = torch.zeros
    x, q = z(6, 512, dtype=torch.bfloat16), z(6, 512, dtype=torch.int8)
    packed, Y = z(24, 128, dtype=torch.uint8), z(6, 24)
    norm = lambda s, **kw: cq.catq_aux_rmsnorm_quant(x, q, s, **kw)                     # noqa: E731
    quant = lambda s, **kw: cq.catq_aux_act_quant8(x, q, s, **kw)                       # noqa: E731
    linear = lambda a, **kw: cq.catq_ternary_linear_a8(q, z(6), packed, a, Y, **kw)     # noqa: E731
    for call in (lambda: norm(z(4, 6), group=128), lambda: quant(z(4, 6), group=128), lambda: linear(z(4, 24)),
                 lambda: linear(z(24, 2, 2)), lambda: linear(z(2, 24), g=256), lambda: norm(z(6, 3), group=128),
                 lambda: norm(z(4, 6).T, group=128), lambda: linear(z(24, 8)[:, ::2])):
        with pytest.raises(ValueError, match="scale|alpha"):
            call()
    for call in (lambda: norm(z(6, 4), group=128), lambda: norm(z(24), group=128), lambda: norm(z(2, 3, 4), group=128),
                 lambda: norm(z(6)), lambda: norm(z(6, 1)), lambda: norm(z(1, 6)), lambda: quant(z(6, 4), group=128),
                 lambda: linear(z(24, 4)), lambda: linear(z(96)), lambda: linear(z(1, 24), g=512),
                 lambda: linear(z(24, 4), g=128)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="GPU"):
        cq.catq_ternary_linear_a8(q[:0], z(0), packed, z(24, 4), Y[:0])


def test_sizes_past_32_bits_are_refused(cq):
    """Not cut to their lower 32 bits, which would be another size."""
    ok = dict(n_q=4, n_kv=2, head_dim=64, page_size=16, scale_block=16, n_pages=3, max_pages=2)
    for name in ok:
        for far in (2 ** 32, -2 ** 32, 2 ** 31):
            with pytest.raises(ValueError, match=name):
                cq.kv_desc(**dict(ok, **{name: ok[name] + far}))
    d = cq.kv_desc(**ok)
    arrays = [torch.zeros(s, dtype=torch.int32) for s in ((1, 2), (2,), (1,))]
    with pytest.raises(ValueError, match="max_new"):
        cq.kv_batch(d, *arrays, 5, 2 ** 32 + 1, 20)
    with pytest.raises(ValueError, match="max_len"):
        cq.kv_batch(d, *arrays, 5, 1, 2 ** 32 + 20)
    with pytest.raises(ValueError, match="rot_dim"):
        cq.kv_prep(d, rot_dim=2 ** 32)
    assert cq.kv_desc(**dict(ok, n_pages=2 ** 31 - 1)).n_pages == 2 ** 31 - 1


# ---------------------------------------------------------------- the reference itself

def test_reference_rotation():
    """Rotation keeps lengths, composes, and a pair turns by position * frequency."""
    g = torch.Generator()
    g.manual_seed(0)
    inv = torch.tensor([1.0, 0.1, 0.01, 0.001, 0.5, 0.25, 0.3, 0.7])
    for inter in (False, True):
        x = torch.randn(32, generator=g, dtype=torch.float64)
        y = ref.rotate(x, 5, inv, 16, inter)
        assert torch.equal(y[16:], x[16:])
        assert abs(float(y.norm() - x.norm())) < 1e-12
        assert torch.allclose(ref.rotate(y, 7, inv, 16, inter), ref.rotate(x, 12, inv, 16, inter))
    x = torch.zeros(32, dtype=torch.float64)
    x[0] = 1
    assert torch.allclose(ref.rotate(x, 1, inv, 16, True)[:2], torch.tensor([0.5403023, 0.8414710], dtype=torch.float64))
    assert abs(float(ref.rotate(x, 1, inv, 16, False)[8]) - 0.8414710) < 1e-6


def test_reference_cache_grows_a_scale():
    """A block's second token ten times the first: the first's codes shrink with the scale."""
    z = torch.zeros
    c = ref.Cache(z(1, 1, 16, 16, dtype=torch.int8), z(1, 1, 4, 16, 4, dtype=torch.int8), z(1, 1, 1), z(1, 1, 1), 16, 16)
    table = torch.tensor([0])
    c.append(0, table, 0, torch.full((1, 1, 16), 1.27, dtype=torch.float64))
    assert (c.codes[0][0, 0, 0] == 127).all()
    c.append(0, table, 1, torch.full((1, 1, 16), -12.7, dtype=torch.float64))
    assert (c.codes[0][0, 0, 0] == 13).all() and (c.codes[0][0, 0, 1] == -127).all()
    c.append(0, table, 2, torch.full((1, 1, 16), 0.1, dtype=torch.float64))
    assert (c.codes[0][0, 0, 2] == 1).all() and abs(float(c.value(0, table, 1)[0, 0]) + 12.7) < 1e-5
    assert c.value(0, torch.tensor([3]), 0) is None and c.value(0, table, 16) is None


def test_reference_ternary_codes():
    p = torch.tensor([[0b11100100]], dtype=torch.uint8)
    assert ref.unpack(p).tolist() == [[-1.0, 0.0, 1.0, 0.0]]
