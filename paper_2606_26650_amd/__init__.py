"""CAT-Q calibration hot path on AMD Instinct MI355X (gfx950).

Python face of libcatq.so: the functions below carry the C ABI's names and do
argument marshalling only (torch tensors supply device memory and the current
HIP stream); every step of the path runs in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import _lib
from ._lib import (BF16, F32, HARD, IDENTITY, SOFT, WS_LINEAR_BWD, WS_LOSS, AttnDesc, CatqError,
                   KvBatch, KvCache, KvDesc, KvPrep, LmstParams)

__all__ = [
    "catq_modulate_ternarize", "catq_fakeq_linear_fwd", "catq_fakeq_linear_bwd",
    "catq_block_recon_loss", "catq_block_recon_loss_noalloc", "catq_pack_ternary", "catq_ternarize_pack",
    "catq_fakeq_gateup_swiglu_fwd",
    "catq_fakeq_down_swiglu_bwd", "catq_ternary_linear", "catq_workspace_size",
    "catq_aux_act_quant", "catq_aux_rmsnorm_fwd", "catq_aux_rmsnorm_bwd", "catq_aux_attention_fwd",
    "catq_aux_attention_bwd", "catq_attn_saved_bytes", "catq_attn_bwd_workspace_bytes",
    "catq_aux_swiglu_fwd", "catq_aux_swiglu_bwd", "catq_aux_moe_route",
    "catq_aux_moe_route_workspace_bytes", "catq_aux_moe_gather", "catq_aux_moe_combine",
    "catq_aux_moe_combine_bwd", "catq_aux_moe_scatter_add", "catq_aux_adamw", "catq_aux_add",
    "catq_ternary_linear_a8", "catq_aux_rmsnorm_quant", "catq_aux_act_quant8", "catq_aux_kv_append",
    "catq_aux_kv_read", "catq_aux_paged_attention", "catq_paged_attention_workspace_bytes",
    "kv_desc", "kv_cache", "kv_batch", "kv_prep", "KvDesc", "KvCache", "KvBatch", "KvPrep",
    "lmst_params", "attn_desc", "IDENTITY", "SOFT", "HARD", "F32", "BF16", "CatqError",
    "LmstParams", "AttnDesc", "lib", "catq_trace_enable", "catq_trace_pause",
    "catq_trace_reset", "catq_trace_count", "catq_trace_get", "catq_trace_disable",
    "trace_records",
]

lib = _lib.load()


def _ptr(t):
    if t is None or isinstance(t, int):
        return t
    return t.data_ptr()


_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}


def _dt(t):
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return dt


# the handle of a device's current stream, without the torch.cuda.Stream object
# that torch.cuda.current_stream() builds around it on every call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is not None:
        return stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def lmst_params(group_size=128, mode=SOFT, delta0=0.5, s=15.0, s_bwd=30.0, strides=(1, 1, 1)):
    p = LmstParams()
    p.group_size = group_size
    p.mode = mode
    p.delta0 = delta0
    p.s = s
    p.s_bwd = s_bwd
    for i in range(3):
        p.factor_stride[i] = strides[i]
    return p


def attn_desc(batch, seq, n_q, n_kv, head_dim, qk_norm, rope_theta, eps=1e-6, act_quant=False):
    a = AttnDesc()
    a.batch, a.seq, a.n_q, a.n_kv, a.head_dim = batch, seq, n_q, n_kv, head_dim
    a.qk_norm = int(bool(qk_norm))
    a.rope_theta = rope_theta
    a.eps = eps
    a.act_quant = int(bool(act_quant))
    return a


def catq_modulate_ternarize(W, d_mu, d_alpha, d_delta, params, stats, stats_mode, W_fake=None,
                            codes=None, alpha_out=None, stream=None):
    d_out, d_in = W.shape[-2], W.shape[-1]
    rows = W.numel() // d_in
    wf_dt = _dt(W_fake) if W_fake is not None else BF16
    st = lib.catq_modulate_ternarize(_ptr(W), _dt(W), rows, d_in, _ptr(d_mu), _ptr(d_alpha),
                                     _ptr(d_delta), C.byref(params), _ptr(stats), stats_mode,
                                     _ptr(W_fake), wf_dt, _ptr(codes), _ptr(alpha_out),
                                     _stream(stream))
    _lib.check("catq_modulate_ternarize", st)


def catq_fakeq_linear_fwd(X, W_fake, Y, M, N, K, n_experts=1, row_offsets=None, residual=None,
                          stream=None):
    r_dt = _dt(residual) if residual is not None else _dt(Y)
    st = lib.catq_fakeq_linear_fwd(_ptr(X), _ptr(W_fake), _dt(X), _ptr(Y), _dt(Y), M, N, K,
                                   n_experts, _ptr(row_offsets), _ptr(residual), r_dt,
                                   _stream(stream))
    _lib.check("catq_fakeq_linear_fwd", st)


def catq_fakeq_linear_bwd(dY, X, W_fake, M, N, K, W, stats, d_mu, d_alpha, d_delta, params,
                          g_d_mu, g_d_alpha, g_d_delta, workspace, dX=None, dW_fake=None,
                          n_experts=1, row_offsets=None, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = lib.catq_fakeq_linear_bwd(_ptr(dY), _ptr(X), _ptr(W_fake), _dt(X), M, N, K, n_experts,
                                   _ptr(row_offsets), _ptr(W), _dt(W), _ptr(stats), _ptr(d_mu),
                                   _ptr(d_alpha), _ptr(d_delta), C.byref(params), _ptr(dX),
                                   _ptr(g_d_mu), _ptr(g_d_alpha), _ptr(g_d_delta), _ptr(dW_fake),
                                   _ptr(workspace), ws_bytes, _stream(stream))
    _lib.check("catq_fakeq_linear_bwd", st)


def catq_block_recon_loss(Y_q, Y_fp, loss, dY_q, workspace, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size()
    dy_dt = _dt(dY_q) if dY_q is not None else BF16
    st = lib.catq_block_recon_loss(_ptr(Y_q), _ptr(Y_fp), _dt(Y_q), Y_q.numel(), _ptr(loss),
                                   _ptr(dY_q), dy_dt, _ptr(workspace), ws_bytes, _stream(stream))
    _lib.check("catq_block_recon_loss", st)


def catq_block_recon_loss_noalloc(Y_q, Y_fp, loss, dY_q, stream=None):
    """catq_block_recon_loss with the library's own scratch (no workspace,
    no allocation); calls that overlap on one GPU race on that scratch."""
    dy_dt = _dt(dY_q) if dY_q is not None else BF16
    st = lib.catq_block_recon_loss_noalloc(_ptr(Y_q), _ptr(Y_fp), _dt(Y_q), Y_q.numel(),
                                           _ptr(loss), _ptr(dY_q), dy_dt, _stream(stream))
    _lib.check("catq_block_recon_loss_noalloc", st)


def catq_ternarize_pack(W, d_mu, d_alpha, d_delta, params, stats, stats_mode, packed,
                        alpha_out=None, stream=None):
    d_in = W.shape[-1]
    rows = W.numel() // d_in
    st = lib.catq_ternarize_pack(_ptr(W), _dt(W), rows, d_in, _ptr(d_mu), _ptr(d_alpha),
                                 _ptr(d_delta), C.byref(params), _ptr(stats), stats_mode,
                                 _ptr(packed), _ptr(alpha_out), _stream(stream))
    _lib.check("catq_ternarize_pack", st)


def catq_pack_ternary(codes, packed, stream=None):
    d_in = codes.shape[-1]
    rows = codes.numel() // d_in
    st = lib.catq_pack_ternary(_ptr(codes), rows, d_in, _ptr(packed), _stream(stream))
    _lib.check("catq_pack_ternary", st)


def catq_ternary_linear(X, packed, alpha, Y, g=128, stream=None):
    """Y = X (alpha * T)^T from the 2-bit storage: X bf16 [M][d_in] (rows may
    be strided), packed uint8 [d_out][d_in/4], alpha fp32 [d_out][d_in/g],
    Y fp32 or bf16 [M][d_out] (rows may be strided)."""
    d_out, d_in = packed.shape[0], packed.shape[1] * 4
    M = X.shape[0]
    st = lib.catq_ternary_linear(_ptr(X), M, X.stride(0) if M else d_in, _ptr(packed),
                                 _ptr(alpha), d_out, d_in, g, _ptr(Y), _dt(Y),
                                 Y.stride(0) if M else d_out, _stream(stream))
    _lib.check("catq_ternary_linear", st)


def catq_fakeq_gateup_swiglu_fwd(X, W_fake, gu, a, M, F, K, stream=None):
    st = lib.catq_fakeq_gateup_swiglu_fwd(_ptr(X), _ptr(W_fake), M, F, K, _ptr(gu), _ptr(a),
                                          _stream(stream))
    _lib.check("catq_fakeq_gateup_swiglu_fwd", st)


def catq_fakeq_down_swiglu_bwd(dY, W_fake, gu, dgu, M, N, F, da=None, stream=None):
    st = lib.catq_fakeq_down_swiglu_bwd(_ptr(dY), _ptr(W_fake), M, N, F, _ptr(gu), _ptr(dgu),
                                        _ptr(da), _stream(stream))
    _lib.check("catq_fakeq_down_swiglu_bwd", st)


def catq_workspace_size(which, M, N, K, n_experts=1):
    return int(lib.catq_workspace_size(which, M, N, K, n_experts))


def catq_aux_act_quant(x, y, group=None, stream=None):
    """8-bit absmax fake quantization of each group of `group` consecutive
    values of every row of x (default: the whole row) into bf16 y (may be x)."""
    n = x.shape[-1]
    st = lib.catq_aux_act_quant(_ptr(x), _dt(x), x.numel() // n if n else 0, n,
                                group or n, _ptr(y), _stream(stream))
    _lib.check("catq_aux_act_quant", st)


def catq_aux_rmsnorm_fwd(x, y, rstd, eps=1e-6, stream=None):
    n = x.shape[-1]
    st = lib.catq_aux_rmsnorm_fwd(_ptr(x), _dt(x), x.numel() // n, n, eps, _ptr(y), _ptr(rstd),
                                  _stream(stream))
    _lib.check("catq_aux_rmsnorm_fwd", st)


def catq_aux_rmsnorm_bwd(x, rstd, dy, dx, dres=None, stream=None):
    n = x.shape[-1]
    st = lib.catq_aux_rmsnorm_bwd(_ptr(x), _dt(x), _ptr(rstd), _ptr(dy), _ptr(dres),
                                  x.numel() // n, n, _ptr(dx), _stream(stream))
    _lib.check("catq_aux_rmsnorm_bwd", st)


def catq_attn_saved_bytes(desc):
    return int(lib.catq_attn_saved_bytes(C.byref(desc)))


def catq_attn_bwd_workspace_bytes(desc):
    return int(lib.catq_attn_bwd_workspace_bytes(C.byref(desc)))


def catq_aux_attention_fwd(desc, qkv, o, saved, stream=None):
    st = lib.catq_aux_attention_fwd(C.byref(desc), _ptr(qkv), _ptr(o), _ptr(saved),
                                    saved.numel() * saved.element_size(), _stream(stream))
    _lib.check("catq_aux_attention_fwd", st)


def catq_aux_attention_bwd(desc, qkv, o, saved, d_o, dqkv, workspace, stream=None):
    st = lib.catq_aux_attention_bwd(C.byref(desc), _ptr(qkv), _ptr(o), _ptr(saved), _ptr(d_o),
                                    _ptr(dqkv), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream(stream))
    _lib.check("catq_aux_attention_bwd", st)


def catq_aux_swiglu_fwd(gu, a, stream=None):
    F = a.shape[-1]
    st = lib.catq_aux_swiglu_fwd(_ptr(gu), a.numel() // F, F, _ptr(a), _stream(stream))
    _lib.check("catq_aux_swiglu_fwd", st)


def catq_aux_swiglu_bwd(gu, da, dgu, stream=None):
    F = da.shape[-1]
    st = lib.catq_aux_swiglu_bwd(_ptr(gu), _ptr(da), da.numel() // F, F, _ptr(dgu),
                                 _stream(stream))
    _lib.check("catq_aux_swiglu_bwd", st)


def catq_aux_moe_route_workspace_bytes(T, E, k):
    return int(lib.catq_aux_moe_route_workspace_bytes(T, E, k))


def catq_aux_moe_route(logits, k, expert_ids, weights, perm_row, row_offsets, workspace,
                       stream=None):
    T, E = logits.shape
    st = lib.catq_aux_moe_route(_ptr(logits), T, E, k, _ptr(expert_ids), _ptr(weights),
                                _ptr(perm_row), _ptr(row_offsets), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream))
    _lib.check("catq_aux_moe_route", st)


def catq_aux_moe_gather(x, perm_row, k, xg, stream=None):
    T, h = x.shape
    st = lib.catq_aux_moe_gather(_ptr(x), _ptr(perm_row), T, k, h, _ptr(xg), _stream(stream))
    _lib.check("catq_aux_moe_gather", st)


def catq_aux_moe_combine(yg, perm_row, weights, res, y, k, stream=None):
    T, h = y.shape
    st = lib.catq_aux_moe_combine(_ptr(yg), _ptr(perm_row), _ptr(weights), _ptr(res), T, k, h,
                                  _ptr(y), _dt(y), _stream(stream))
    _lib.check("catq_aux_moe_combine", st)


def catq_aux_moe_combine_bwd(dy, perm_row, weights, dyg, k, stream=None):
    T, h = dy.shape
    st = lib.catq_aux_moe_combine_bwd(_ptr(dy), _ptr(perm_row), _ptr(weights), T, k, h,
                                      _ptr(dyg), _stream(stream))
    _lib.check("catq_aux_moe_combine_bwd", st)


def catq_aux_moe_scatter_add(dxg, perm_row, dx, k, stream=None):
    T, h = dx.shape
    st = lib.catq_aux_moe_scatter_add(_ptr(dxg), _ptr(perm_row), T, k, h, _ptr(dx),
                                      _stream(stream))
    _lib.check("catq_aux_moe_scatter_add", st)


def catq_aux_adamw(p, grad, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, lo=-1e30, hi=1e30,
                   stream=None):
    st = lib.catq_aux_adamw(_ptr(p), _ptr(grad), _ptr(m), _ptr(v), p.numel(), step, lr, beta1,
                            beta2, eps, lo, hi, _stream(stream))
    _lib.check("catq_aux_adamw", st)


def catq_aux_add(a, b, y, stream=None):
    st = lib.catq_aux_add(_ptr(a), _ptr(b), _ptr(y), _dt(a), a.numel(), _stream(stream))
    _lib.check("catq_aux_add", st)


# ------------------------------------------------------------------ serving
#
# The calls below take tensors as they are: a tensor of another dtype, shape or
# layout than the call documents, or one on another device than the first, is a
# TypeError or ValueError here, before the library sees a pointer.  They run on the
# device of their tensors and, without ``stream``, on that device's current stream.

def _want(t, name, dtype, shape=None, device=None):
    """t, a contiguous tensor of the dtype, shape and device (an index) asked for."""
    if t.dtype is not dtype:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if t.get_device() != device:
        if device is None:
            if t.is_cuda:
                return t
            raise ValueError(f"{name}: must be on a GPU")
        raise ValueError(f"{name}: on {t.device}, expected GPU {device}")
    return t


def _act(t, name):
    """The catq dtype of an activation tensor (bf16 or fp32)."""
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name}: dtype {t.dtype}, expected bfloat16 or float32")
    return dt


def _per_group(t, name, rows, n, group, device):
    """t, fp32 [rows][n/group] (the rows in any number of dimensions, or all of it flat)."""
    _want(t, name, torch.float32, None, device)
    if group > 0:     # (the library refuses the others)
        each = n // group
        if t.numel() != rows * each or (each > 1 and t.dim() != 1 and t.shape[-1] != each):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {(rows, each)}")


def _rows(t, name, shape, device):
    """The row stride of a 2-d tensor whose rows are contiguous."""
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    if t.stride(1) != 1 and shape[1] > 1:
        raise ValueError(f"{name}: rows must be contiguous")
    if t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, expected GPU {device}")
    return t.stride(0) if shape[0] > 1 else shape[1]


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _run_on(device, stream, fn, name, *args):
    if device < 0:
        raise ValueError(f"{name}: the tensors must be on a GPU")
    if device == _current_device():
        st = fn(*args, _stream(stream) if _raw_stream is None or stream is not None else _raw_stream(device))
    else:
        with torch.cuda.device(device):
            st = fn(*args, _stream(stream))
    if st:
        _lib.check(name, st)


def _bytes(ws):
    return 0 if ws is None else ws.numel() * ws.element_size()


def catq_aux_rmsnorm_quant(x, q=None, scale=None, res=None, weight=None, sum=None, y=None, group=None,
                           eps=1e-6, stream=None):
    """h = x + res (into ``sum``), RMSNorm with gain ``weight``, and its 8-bit codes q
    with their scales [rows][n/group] (default: one per row), or their values y in
    bf16, or both."""
    xd = _act(x, "x")
    shape, dev = x.shape, x.get_device()
    _want(x, "x", x.dtype, None, dev)
    n = shape[-1]
    rows = x.numel() // n if n else 0
    if group is None:
        group = n
    rd = BF16
    if res is not None:
        rd = _act(res, "res")
        _want(res, "res", res.dtype, shape, dev)
        if sum is not None:
            _want(sum, "sum", res.dtype, shape, dev)
    elif sum is not None:
        raise ValueError("sum: needs res")
    if weight is not None:
        _want(weight, "weight", torch.bfloat16, (n,), dev)
    if y is not None:
        _want(y, "y", torch.bfloat16, shape, dev)
    if q is not None:
        _want(q, "q", torch.int8, shape, dev)
    if scale is not None:
        _per_group(scale, "scale", rows, n, group, dev)
    _run_on(dev, stream, lib.catq_aux_rmsnorm_quant, "catq_aux_rmsnorm_quant", x.data_ptr(), xd, _ptr(res), rd,
            _ptr(weight), rows, n, group, eps, _ptr(sum), _ptr(y), _ptr(q), _ptr(scale))


def catq_aux_act_quant8(x, q, scale, group=None, stream=None):
    """The 8-bit codes of every group of ``group`` consecutive values of x's rows
    (default: the whole row) and their scales."""
    xd = _act(x, "x")
    n, dev = x.shape[-1], x.get_device()
    _want(x, "x", x.dtype, None, dev)
    rows = x.numel() // n if n else 0
    if group is None:
        group = n
    _want(q, "q", torch.int8, x.shape, dev)
    _per_group(scale, "scale", rows, n, group, dev)
    _run_on(dev, stream, lib.catq_aux_act_quant8, "catq_aux_act_quant8", x.data_ptr(), xd, rows, n, group,
            q.data_ptr(), scale.data_ptr())


def catq_ternary_linear_a8(q, x_scale, packed, alpha, Y, g=128, stream=None):
    """Y = x_scale * q (alpha * T)^T from the 2-bit storage: codes q int8 [M][d_in]
    (rows may be strided), x_scale fp32 [M], packed uint8 [d_out][d_in/4], alpha
    fp32 [d_out][d_in/g], Y fp32 or bf16 [M][d_out] (rows may be strided)."""
    dev = packed.get_device()
    _want(packed, "packed", torch.uint8, None, dev)
    d_out, d_in = packed.shape[0], packed.shape[1] * 4
    M = q.shape[0]
    if q.dtype is not torch.int8:
        raise TypeError(f"q: dtype {q.dtype}, expected torch.int8")
    yd = _act(Y, "Y")
    ldq, ldy = _rows(q, "q", (M, d_in), dev), _rows(Y, "Y", (M, d_out), dev)
    _want(x_scale, "x_scale", torch.float32, None, dev)
    if x_scale.numel() != M:
        raise ValueError(f"x_scale: {x_scale.numel()} values, expected {M}")
    _per_group(alpha, "alpha", d_out, d_in, g, dev)
    _run_on(dev, stream, lib.catq_ternary_linear_a8, "catq_ternary_linear_a8", q.data_ptr(), M, ldq,
            x_scale.data_ptr(), packed.data_ptr(), alpha.data_ptr(), d_out, d_in, g, Y.data_ptr(), yd, ldy)


def _int32(**sizes):
    """Sizes that a descriptor holds in 32 bits (a ctypes field would drop the upper ones)."""
    for name, v in sizes.items():
        if not -2 ** 31 <= v < 2 ** 31:
            raise ValueError(f"{name}: {v} does not fit 32 bits")


def kv_desc(n_q, n_kv, head_dim, page_size, scale_block, n_pages, max_pages):
    """Geometry of a paged 8-bit cache (see catq_kv_desc in the header)."""
    _int32(n_q=n_q, n_kv=n_kv, head_dim=head_dim, page_size=page_size, scale_block=scale_block, n_pages=n_pages,
           max_pages=max_pages)
    return KvDesc(n_q, n_kv, head_dim, page_size, scale_block, n_pages, max_pages)


def kv_cache(desc, k, v, k_scale, v_scale):
    """The pool's arrays: k int8 [n_pages][n_kv][page_size][head_dim], v int8
    [n_pages][n_kv][page_size/4][head_dim][4], scales fp32
    [n_pages][n_kv][page_size/scale_block].  The returned struct keeps them."""
    d = desc
    _want(k, "k", torch.int8, (d.n_pages, d.n_kv, d.page_size, d.head_dim))
    dev = k.get_device()
    _want(v, "v", torch.int8, (d.n_pages, d.n_kv, d.page_size // 4, d.head_dim, 4), dev)
    blocks = (d.n_pages, d.n_kv, d.page_size // d.scale_block if d.scale_block > 0 else 0)
    _want(k_scale, "k_scale", torch.float32, blocks, dev)
    _want(v_scale, "v_scale", torch.float32, blocks, dev)
    c = KvCache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
    c.tensors, c.device, c.geometry = (k, v, k_scale, v_scale), dev, bytes(d)[:24]
    return c


def kv_batch(desc, page_table, cu_new, ctx_len, n_tokens, max_new, max_len):
    """The new tokens of a batch (see catq_kv_batch in the header): page_table int32
    [n_seqs][max_pages], cu_new int32 [n_seqs + 1], ctx_len int32 [n_seqs], on the
    device; their values may change between calls.  The returned struct keeps them."""
    n = ctx_len.shape[0]
    _int32(max_new=max_new, max_len=max_len)
    _want(page_table, "page_table", torch.int32, (n, desc.max_pages))
    dev = page_table.get_device()
    _want(cu_new, "cu_new", torch.int32, (n + 1,), dev)
    _want(ctx_len, "ctx_len", torch.int32, (n,), dev)
    b = KvBatch(page_table.data_ptr(), cu_new.data_ptr(), ctx_len.data_ptr(), n_tokens, n, max_new, max_len)
    b.tensors, b.device, b.width = (page_table, cu_new, ctx_len), dev, desc.max_pages
    return b


def kv_prep(desc, inv_freq=None, rot_dim=0, interleaved=False, qk_norm=False, q_weight=None, k_weight=None,
            eps=1e-6, rope_scale=1.0, act_quant=False):
    """What happens to q and k on the way to the cache (see catq_kv_prep in the
    header).  The returned struct keeps the tensors."""
    _int32(rot_dim=rot_dim)
    first = next((t for t in (inv_freq, q_weight, k_weight) if t is not None), None)
    dev = None if first is None else first.get_device()
    if inv_freq is not None:
        _want(inv_freq, "inv_freq", torch.float32, (rot_dim // 2,))
    for t, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if t is not None:
            _want(t, name, torch.bfloat16, (desc.head_dim,), dev)
    p = KvPrep(_ptr(inv_freq), _ptr(q_weight), _ptr(k_weight), rot_dim, int(bool(interleaved)),
               int(bool(qk_norm)), int(bool(act_quant)), rope_scale, eps)
    p.tensors, p.device, p.width = (inv_freq, q_weight, k_weight), dev, desc.head_dim
    return p


def _kv_same(desc, cache, batch):
    dev = cache.device
    if batch.device != dev:
        raise ValueError(f"batch: on GPU {batch.device}, expected {dev}")
    if bytes(desc)[:24] != cache.geometry:
        raise ValueError("the cache was made for another descriptor")
    if batch.width != desc.max_pages:
        raise ValueError("the batch's page table is not max_pages wide")
    return dev


def catq_aux_kv_append(desc, cache, batch, prep, qkv, q_out, stream=None):
    """New tokens' qkv [n_tokens][(n_q + 2 n_kv) head_dim] (bf16): normed and rotated
    q into q_out [n_tokens][n_q head_dim], k and v into the cache."""
    dev, n, d = _kv_same(desc, cache, batch), batch.n_tokens, desc.head_dim
    if prep.device is not None and prep.device != dev:
        raise ValueError(f"prep: on GPU {prep.device}, expected {dev}")
    if prep.width != d:
        raise ValueError(f"prep: made for heads of {prep.width} values, expected {d}")
    _want(qkv, "qkv", torch.bfloat16, (n, (desc.n_q + 2 * desc.n_kv) * d), dev)
    _want(q_out, "q_out", torch.bfloat16, (n, desc.n_q * d), dev)
    _run_on(dev, stream, lib.catq_aux_kv_append, "catq_aux_kv_append", C.byref(desc), C.byref(cache),
            C.byref(batch), C.byref(prep), _ptr(qkv), _ptr(q_out))


def catq_aux_kv_read(desc, cache, batch, k_out=None, v_out=None, stream=None):
    """The batch's positions back as bf16 values [n_tokens][n_kv head_dim]."""
    dev, shape = _kv_same(desc, cache, batch), (batch.n_tokens, desc.n_kv * desc.head_dim)
    for t, name in ((k_out, "k_out"), (v_out, "v_out")):
        if t is not None:
            _want(t, name, torch.bfloat16, shape, dev)
    _run_on(dev, stream, lib.catq_aux_kv_read, "catq_aux_kv_read", C.byref(desc), C.byref(cache),
            C.byref(batch), _ptr(k_out), _ptr(v_out))


def catq_paged_attention_workspace_bytes(desc, batch):
    return int(lib.catq_paged_attention_workspace_bytes(C.byref(desc), C.byref(batch)))


def catq_aux_paged_attention(desc, cache, batch, q, o, workspace=None, scale=None, lse=None, stream=None):
    """Attention of the new tokens' q over the cache that holds them (scale None:
    1/sqrt(head_dim)); o like q, lse fp32 [n_tokens][n_q] or None."""
    dev, shape = _kv_same(desc, cache, batch), (batch.n_tokens, desc.n_q * desc.head_dim)
    _want(q, "q", torch.bfloat16, shape, dev)
    _want(o, "o", torch.bfloat16, shape, dev)
    if lse is not None:
        _want(lse, "lse", torch.float32, (batch.n_tokens, desc.n_q), dev)
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        raise ValueError(f"workspace: must be contiguous and on GPU {dev}")
    _run_on(dev, stream, lib.catq_aux_paged_attention, "catq_aux_paged_attention", C.byref(desc),
            C.byref(cache), C.byref(batch), _ptr(q), desc.head_dim ** -0.5 if scale is None else scale, _ptr(o),
            _ptr(lse), _ptr(workspace), _bytes(workspace))


def catq_trace_enable(capacity):
    _lib.check("catq_trace_enable", lib.catq_trace_enable(capacity))


def catq_trace_pause(paused=True):
    lib.catq_trace_pause(int(bool(paused)))


def catq_trace_reset():
    lib.catq_trace_reset()


def catq_trace_count():
    return int(lib.catq_trace_count())


def catq_trace_get(i):
    r = _lib.TraceRec()
    _lib.check("catq_trace_get", lib.catq_trace_get(i, C.byref(r)))
    return dict(tag=r.tag.decode(), flops=r.flops, bytes=r.bytes, M=r.M, N=r.N, K=r.K, ms=r.ms)


def catq_trace_disable():
    lib.catq_trace_disable()


def trace_records():
    """Every record since the last reset, with its event-measured duration."""
    return [catq_trace_get(i) for i in range(catq_trace_count())]
