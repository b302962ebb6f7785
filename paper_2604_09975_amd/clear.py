"""Binding of include/ckks_clear.h: the key holder's steps in the clear between two encrypted projections.

Argument marshalling only, as in `binding`: every function has the name of the C entry point it calls, takes torch tensors on
the current HIP device and enqueues on torch's current stream.  Rows may be strided; their last dimension is contiguous.
Types are float32, float16 and bfloat16; pages of 8 bits are float8_e4m3fn or int8.  Workspaces come from torch's allocator, on the stream of the call.

None of the calls is recorded by autograd (a layer norm's gradient is a call of its own): a tensor that requires a gradient is
refused while gradients are recorded.  Tensors that a call writes in place count as modified, so a backward pass that
needs their old values notices.

A call's kernels can take less time than its marshalling (one token: 4 to 7 us), so the argument struct is packed in one go
and each tensor is asked for as little as its check needs.
"""
import struct

import torch
from torch.autograd.graph import increment_version as _written

from .binding import C, _check, _raw_stream, _stream, lib

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_f32, _i32 = torch.float32, torch.int32
_rowwise = torch.contiguous_format
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device

# The argument structs of the header, field by field.
_NORM = struct.Struct("=6Q2q4IfI").pack
_NORM_GRAD = struct.Struct("=10Q3q4I").pack
_PAGES, _BATCH = "2Q6q6I", "3Qq4I"
_APPEND = struct.Struct("=" + _PAGES + _BATCH + "7Q8q4I").pack
_ATTEND = struct.Struct("=" + _PAGES + _BATCH + "5Q4q3If").pack
_LOGITS = struct.Struct("=12Q3q6I").pack
_PACKED = "4Q12q6I"
_PACKED_APPEND = struct.Struct("=" + _PACKED + _BATCH + "9Q8q5If").pack
_PACKED_ATTEND = struct.Struct("=" + _PACKED + _BATCH + "5Q4q3If").pack
_PACKED_READ = struct.Struct("=" + _PACKED + _BATCH + "2Q4q").pack
_SAMPLE = struct.Struct("=8Qq4I").pack

for _n in ("layer_norm", "layer_norm_grad", "cache_append", "attend", "logits", "packed_append", "packed_attend", "packed_read", "sample"):
    getattr(lib, "ckks_clear_" + _n).argtypes = [C.c_char_p, C.c_void_p]
    getattr(lib, "ckks_clear_" + _n).restype = C.c_int
lib.ckks_clear_layer_norm_grad_work_bytes.argtypes = [C.c_uint32] * 3
lib.ckks_clear_layer_norm_grad_work_bytes.restype = C.c_uint64
lib.ckks_clear_attend_work_bytes.argtypes = [C.c_char_p]
lib.ckks_clear_attend_work_bytes.restype = C.c_uint64
lib.ckks_clear_packed_attend_work_bytes.argtypes = [C.c_char_p]
lib.ckks_clear_packed_attend_work_bytes.restype = C.c_uint64
_norm, _norm_grad, _append, _attend, _logits = (
    getattr(lib, "ckks_clear_" + _n) for _n in ("layer_norm", "layer_norm_grad", "cache_append", "attend", "logits"))
_packed_append, _packed_attend, _packed_read, _sample = (
    getattr(lib, "ckks_clear_" + _n) for _n in ("packed_append", "packed_attend", "packed_read", "sample"))
_packed_attend_work = lib.ckks_clear_packed_attend_work_bytes
_norm_grad_work, _attend_work = lib.ckks_clear_layer_norm_grad_work_bytes, lib.ckks_clear_attend_work_bytes


def _on(dev):
    """The raw handle of the current stream of device `dev`."""
    return _raw_stream(dev) if _raw_stream is not None else _stream()


def _refuse(what):
    """For a tensor that requires a gradient: it would be lost without a word."""
    if torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, which this call does not record: detach it, or call under torch.no_grad()")


def _ptr(t, dtype, dev, what):
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != dev:
        raise TypeError(f"{what}: expected a {dtype} tensor on device {dev}")
    if t.requires_grad:
        _refuse(what)
    return t.data_ptr()


def _vec(t, dtype, n, dev, what):
    """Pointer of a contiguous vector of n entries (n None: of any length); 0 for None."""
    if t is None:
        return 0
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != dev:
        raise TypeError(f"{what}: expected a {dtype} tensor on device {dev}")
    if t.requires_grad:
        _refuse(what)
    if t.dim() != 1 or (n is not None and t.numel() != n) or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous vector" + (f" of {n}" if n is not None else ""))
    return t.data_ptr()


def _type(t, what):
    code = _TYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if code is None:
        raise TypeError(f"{what}: expected a float32, float16 or bfloat16 tensor")
    return code


def _rows(t, what):
    """[..., cols] as (rows, cols, row stride); the leading dimensions must be those of evenly spaced rows."""
    if t.dim() != 2:
        if t.dim() == 0:
            raise ValueError(f"{what} must have at least one dimension")
        t = t.view(-1, t.shape[-1]) if t.numel() else t.reshape(0, t.shape[-1])
    rows, cols = t.shape
    st = t.stride()
    if cols > 1 and st[1] != 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    return rows, cols, st[0]


def _param(t, dtype, cols, dev, what):
    """Type code and pointer of a weight or bias: float32 or the rows' type."""
    if t.dtype is not _f32 and t.dtype is not dtype:
        raise TypeError(f"{what} must be float32 or of the rows' type")
    return _TYPES[t.dtype], _vec(t, t.dtype, cols, dev, what)


def ckks_clear_layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stats=True):
    """x [..., C] -> (y, mean, rstd): y of x's type, mean and rstd float32 of the rows (None without `stats`)."""
    dev, code, dtype = _device(), _type(x, "x"), x.dtype
    px = _ptr(x, dtype, dev, "x")
    rows, cols, xs = _rows(x, "x")
    wt = bt = pw = pb = 0
    if weight is not None:
        wt, pw = _param(weight, dtype, cols, dev, "weight")
    if bias is not None:
        bt, pb = _param(bias, dtype, cols, dev, "bias")
        if weight is None:
            wt = bt
        elif wt != bt:
            raise TypeError("weight and bias must be of one type")
    given = out
    if out is None:
        out = torch.empty_like(x, memory_format=_rowwise)
        py, ys = out.data_ptr(), cols
    else:
        py, ys = _ptr(out, dtype, dev, "out"), _rows(out, "out")[2]
        if out.shape != x.shape:
            raise ValueError("out must have the input's shape")
    mean = rstd = None
    pm = pr = 0
    if stats:
        both = x.new_empty((2,) + x.shape[:-1], dtype=_f32)
        mean, rstd = both.unbind(0)
        pm = both.data_ptr()
        pr = pm + 4 * rows
    rc = _norm(_NORM(px, pw, pb, py, pm, pr, xs, ys, rows, cols, code, wt, eps, 0), _on(dev))
    if rc:
        _check(rc)
    if given is not None:
        _written(given)
    return out, mean, rstd


def ckks_clear_layer_norm_grad(dy, x, mean, rstd, weight=None, dx=None, params=True):
    """-> (dx, dweight, dbias) of the call that gave mean and rstd; the parameters' gradients have the weight's type (float32
    without a weight) and are None without `params`."""
    dev, code, dtype = _device(), _type(x, "x"), x.dtype
    px, pdy = _ptr(x, dtype, dev, "x"), _ptr(dy, dtype, dev, "dy")
    rows, cols, xs = _rows(x, "x")
    if dy.shape != x.shape:
        raise ValueError("dy must have x's shape")
    for t, what in ((mean, "mean"), (rstd, "rstd")):
        _ptr(t, _f32, dev, what)
        if t.numel() != rows or not t.is_contiguous():
            raise ValueError(f"{what} must hold one value for each row")
    wt = pw = 0
    if weight is not None:
        wt, pw = _param(weight, dtype, cols, dev, "weight")
    given = dx
    if dx is None:
        dx = torch.empty_like(x, memory_format=_rowwise)
        pdx, dxs = dx.data_ptr(), cols
    else:
        pdx, dxs = _ptr(dx, dtype, dev, "dx"), _rows(dx, "dx")[2]
        if dx.shape != x.shape:
            raise ValueError("dx must have the input's shape")
    dw = db = None
    pgw = pgb = pwork = need = 0
    if params:
        grads = x.new_empty((2, cols), dtype=_f32 if weight is None else weight.dtype)
        dw, db = grads.unbind(0)
        pgw = grads.data_ptr()
        pgb = pgw + cols * grads.element_size()
        need = _norm_grad_work(rows, cols, code)
        work = x.new_empty(max(need, 4), dtype=torch.uint8)
        pwork = work.data_ptr()
    rc = _norm_grad(_NORM_GRAD(pdy, px, pw, mean.data_ptr(), rstd.data_ptr(), pdx, pgw, pgb, pwork, need,
                               _rows(dy, "dy")[2], xs, dxs, rows, cols, code, wt), _on(dev))
    if rc:
        _check(rc)
    if given is not None:
        _written(given)
    return dx, dw, db


def _heads(t, dtype, n, dim, dev, what):
    """Pointer, heads and strides {token, head} of [n][heads][dim]."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != dev:
        raise TypeError(f"{what}: expected a {dtype} tensor on device {dev}")
    if t.requires_grad:
        _refuse(what)
    if t.dim() != 3:
        raise ValueError(f"{what} must be [{n}][heads][{dim}]")
    rows, heads, width = t.shape
    s0, s1, s2 = t.stride()
    if rows != n or width != dim:
        raise ValueError(f"{what} must be [{n}][heads][{dim}]")
    if dim > 1 and s2 != 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    return t.data_ptr(), heads, s0, s1


def _cache(k_pages, v_pages, page_table, q_start, kv_len, n_tokens, dev):
    """Fields of ckks_clear_pages_t and ckks_clear_batch_t."""
    code, dtype = _type(k_pages, "k_pages"), k_pages.dtype
    pk, pv = _ptr(k_pages, dtype, dev, "k_pages"), _ptr(v_pages, dtype, dev, "v_pages")
    shape = k_pages.shape
    if len(shape) != 4 or v_pages.shape != shape:
        raise ValueError("k_pages and v_pages must be [n_pages][kv_heads][page_size][head_dim]")
    n_pages, kv_heads, page_size, dim = shape
    k0, k1, k2, k3 = k_pages.stride()
    v0, v1, v2, v3 = v_pages.stride()
    if dim > 1 and (k3 != 1 or v3 != 1):
        raise ValueError("the last dimension of the pages must be contiguous")
    pt = _ptr(page_table, _i32, dev, "page_table")
    if page_table.dim() != 2:
        raise ValueError("page_table must be [n_seq][pages]")
    n_seq, width = page_table.shape
    t0, t1 = page_table.stride()
    if width > 1 and t1 != 1:
        raise ValueError("the last dimension of page_table must be contiguous")
    return (pk, pv, k0, k1, k2, v0, v1, v2, n_pages, page_size, kv_heads, dim, code, 0,
            _vec(q_start, _i32, n_seq + 1, dev, "q_start"), _vec(kv_len, _i32, n_seq, dev, "kv_len"), pt, t0, n_seq, n_tokens, width, 0)


def ckks_clear_cache_append(k, v, k_pages, v_pages, page_table, q_start, kv_len, cos=None, sin=None, interleaved=False,
                            positions=None, q=None, q_out=None):
    """k, v [T][kv_heads][head_dim] into the pages, rotated by cos / sin [n_pos][rot/2] at their positions; q [T][heads][head_dim]
    rotated alike into q_out -> q_out (None without q)."""
    dev, dtype = _device(), k_pages.dtype
    n = k.shape[0]
    cache = _cache(k_pages, v_pages, page_table, q_start, kv_len, n, dev)
    kv_heads, dim = cache[10], cache[11]
    pk, hk, k0, k1 = _heads(k, dtype, n, dim, dev, "k")
    pv, hv, v0, v1 = _heads(v, dtype, n, dim, dev, "v")
    if hk != kv_heads or hv != kv_heads:
        raise ValueError(f"k and v must have {kv_heads} heads")
    pq = po = q0 = q1 = o0 = o1 = heads = 0
    if q is not None:
        pq, heads, q0, q1 = _heads(q, dtype, n, dim, dev, "q")
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=_rowwise)
        po, ho, o0, o1 = _heads(q_out, dtype, n, dim, dev, "q_out")
        if ho != heads:
            raise ValueError("q_out must have q's heads")
    elif q_out is not None:
        raise ValueError("q_out without q")
    pc = ps = rot = n_pos = 0
    if cos is not None or sin is not None:
        pc, ps = _ptr(cos, _f32, dev, "cos"), _ptr(sin, _f32, dev, "sin")
        if cos.dim() != 2 or cos.shape != sin.shape or not cos.is_contiguous() or not sin.is_contiguous():
            raise ValueError("cos and sin must be contiguous [n_pos][rot/2]")
        n_pos, rot = cos.shape[0], 2 * cos.shape[1]
    rc = _append(_APPEND(*cache, pk, pv, pq, po, pc, ps, _vec(positions, _i32, n, dev, "positions"), k0, k1, v0, v1, q0, q1, o0, o1,
                         heads, rot, n_pos, 1 if interleaved else 0), _on(dev))
    if rc:
        _check(rc)
    _written((k_pages, v_pages) if q is None else (k_pages, v_pages, q_out))
    return q_out


def ckks_clear_attend(q, k_pages, v_pages, page_table, q_start, kv_len, scale=None, causal=True, window=0, out=None, lse=None):
    """q [T][heads][head_dim] over the cache -> out [T][heads][head_dim]; lse: float32 [T][heads] to fill, or None.  scale None:
    1 / sqrt(head_dim)."""
    dev, dtype = _device(), k_pages.dtype
    n, heads, dim = q.shape
    cache = _cache(k_pages, v_pages, page_table, q_start, kv_len, n, dev)
    if dim != cache[11]:
        raise ValueError(f"q must be [{n}][heads][{cache[11]}]")
    pq, heads, q0, q1 = _heads(q, dtype, n, dim, dev, "q")
    given = tuple(t for t in (out, lse) if t is not None)
    if out is None:
        out = torch.empty_like(q, memory_format=_rowwise)
        po, o0, o1 = out.data_ptr(), heads * dim, dim
    else:
        po, ho, o0, o1 = _heads(out, dtype, n, dim, dev, "out")
        if ho != heads:
            raise ValueError("out must have q's heads")
    pl = 0
    if lse is not None:
        pl = _ptr(lse, _f32, dev, "lse")
        if lse.shape != (n, heads) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous [T][heads]")
    if scale is None:
        scale = dim ** -0.5
    causal = 1 if causal else 0
    args = _ATTEND(*cache, pq, po, pl, 0, 0, q0, q1, o0, o1, heads, window, causal, scale)
    need = _attend_work(args)
    if need:
        work = q.new_empty(need, dtype=torch.uint8)
        args = _ATTEND(*cache, pq, po, pl, work.data_ptr(), need, q0, q1, o0, o1, heads, window, causal, scale)
    rc = _attend(args, _on(dev))
    if rc:
        _check(rc)
    if given:
        _written(given)
    return out


def ckks_clear_logits(logits, out=None, tokens=None, token_start=None, n_prompt=None, repetition=None, frequency=None, presence=None,
                      bias_ids=None, bias=None, bias_start=None, mask=None):
    """logits [R][V] (or [V]) under the rules -> out (logits' type or float32; new if None, may be logits itself)."""
    dev, code, dtype = _device(), _type(logits, "logits"), logits.dtype
    pl = _ptr(logits, dtype, dev, "logits")
    rows, vocab, ls = _rows(logits, "logits")
    given = out
    if out is None:
        out = torch.empty_like(logits, memory_format=_rowwise)
        po, os, oc = out.data_ptr(), vocab, code
    else:
        oc = _type(out, "out")
        po, os = _ptr(out, out.dtype, dev, "out"), _rows(out, "out")[2]
        if out.shape != logits.shape:
            raise ValueError("out must have the logits' shape")
    pm = ms = 0
    if mask is not None:
        pm = _ptr(mask, _i32, dev, "mask")
        mr, words, ms = _rows(mask, "mask")
        if mr != rows or words < (vocab + 31) // 32:
            raise ValueError("mask must hold one bit for each logit, 32 to a word")
    n_tokens = tokens.numel() if tokens is not None else 0
    n_biases = bias_ids.numel() if bias_ids is not None else 0
    rc = _logits(
        _LOGITS(pl, po, _vec(tokens, _i32, None, dev, "tokens"), _vec(token_start, _i32, rows + 1, dev, "token_start"),
                _vec(n_prompt, _i32, rows, dev, "n_prompt"), _vec(repetition, _f32, rows, dev, "repetition"),
                _vec(frequency, _f32, rows, dev, "frequency"), _vec(presence, _f32, rows, dev, "presence"),
                _vec(bias_ids, _i32, None, dev, "bias_ids"), _vec(bias_start, _i32, rows + 1, dev, "bias_start"),
                _vec(bias, _f32, n_biases, dev, "bias"), pm, ls, os, ms, rows, vocab, n_tokens, n_biases, code, oc), _on(dev))
    if rc:
        _check(rc)
    if given is not None:
        _written(given)
    return out


_FORMATS = {torch.float8_e4m3fn: 16, torch.int8: 17}
_u8 = torch.uint8


def _packed(k_pages, v_pages, k_power, v_power, page_table, q_start, kv_len, n_tokens, dtype, dev):
    """Fields of ckks_clear_packed_t and ckks_clear_batch_t; the type of the queries and rows is `dtype`."""
    form = _FORMATS.get(k_pages.dtype) if isinstance(k_pages, torch.Tensor) else None
    if form is None:
        raise TypeError("k_pages: expected a float8_e4m3fn or int8 tensor")
    code = _TYPES.get(dtype)
    if code is None:
        raise TypeError(f"packed pages meet float32, float16 or bfloat16, not {dtype}")
    pk, pv = _ptr(k_pages, k_pages.dtype, dev, "k_pages"), _ptr(v_pages, k_pages.dtype, dev, "v_pages")
    zk, zv = _ptr(k_power, _u8, dev, "k_power"), _ptr(v_power, _u8, dev, "v_power")
    shape, blocks = k_pages.shape, k_power.shape
    if len(shape) != 4 or v_pages.shape != shape:
        raise ValueError("k_pages and v_pages must be [n_pages][kv_heads][page_size][head_dim]")
    n_pages, kv_heads, page_size, dim = shape
    if blocks != (n_pages, kv_heads, page_size, (dim + 31) // 32) or v_power.shape != blocks:
        raise ValueError("k_power and v_power must be [n_pages][kv_heads][page_size][ceil(head_dim / 32)]")
    k0, k1, k2, k3 = k_pages.stride()
    v0, v1, v2, v3 = v_pages.stride()
    y0, y1, y2, y3 = k_power.stride()
    z0, z1, z2, z3 = v_power.stride()
    if (dim > 1 and (k3 != 1 or v3 != 1)) or (dim > 32 and (y3 != 1 or z3 != 1)):
        raise ValueError("the last dimension of pages and powers must be contiguous")
    pt = _ptr(page_table, _i32, dev, "page_table")
    if page_table.dim() != 2:
        raise ValueError("page_table must be [n_seq][pages]")
    n_seq, width = page_table.shape
    t0, t1 = page_table.stride()
    if width > 1 and t1 != 1:
        raise ValueError("the last dimension of page_table must be contiguous")
    return (pk, pv, zk, zv, k0, k1, k2, v0, v1, v2, y0, y1, y2, z0, z1, z2, n_pages, page_size, kv_heads, dim, form, code,
            _vec(q_start, _i32, n_seq + 1, dev, "q_start"), _vec(kv_len, _i32, n_seq, dev, "kv_len"), pt, t0, n_seq, n_tokens, width, 0)


def ckks_clear_packed_append(k, v, k_pages, v_pages, k_power, v_power, page_table, q_start, kv_len, cos=None, sin=None, interleaved=False,
                             positions=None, q=None, q_out=None, k_norm=None, q_norm=None, eps=1e-6):
    """k, v [T][kv_heads][head_dim] into pages of 8 bits (float8_e4m3fn or int8, uint8 powers of two), the keys normed by k_norm [head_dim]
    and rotated as in ckks_clear_cache_append; q [T][heads][head_dim] normed by q_norm and rotated alike into q_out -> q_out (None
    without q)."""
    dev, dtype = _device(), k.dtype
    n = k.shape[0]
    cache = _packed(k_pages, v_pages, k_power, v_power, page_table, q_start, kv_len, n, dtype, dev)
    kv_heads, dim = cache[18], cache[19]
    pk, hk, k0, k1 = _heads(k, dtype, n, dim, dev, "k")
    pv, hv, v0, v1 = _heads(v, dtype, n, dim, dev, "v")
    if hk != kv_heads or hv != kv_heads:
        raise ValueError(f"k and v must have {kv_heads} heads")
    pq = po = q0 = q1 = o0 = o1 = heads = 0
    if q is not None:
        pq, heads, q0, q1 = _heads(q, dtype, n, dim, dev, "q")
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=_rowwise)
        po, ho, o0, o1 = _heads(q_out, dtype, n, dim, dev, "q_out")
        if ho != heads:
            raise ValueError("q_out must have q's heads")
    elif q_out is not None or q_norm is not None:
        raise ValueError("q_out or q_norm without q")
    kt = qt = pkn = pqn = 0
    if k_norm is not None:
        kt, pkn = _param(k_norm, dtype, dim, dev, "k_norm")
    if q_norm is not None:
        qt, pqn = _param(q_norm, dtype, dim, dev, "q_norm")
        if k_norm is None:
            kt = qt
        elif kt != qt:
            raise TypeError("k_norm and q_norm must be of one type")
    pc = ps = rot = n_pos = 0
    if cos is not None or sin is not None:
        pc, ps = _ptr(cos, _f32, dev, "cos"), _ptr(sin, _f32, dev, "sin")
        if cos.dim() != 2 or cos.shape != sin.shape or not cos.is_contiguous() or not sin.is_contiguous():
            raise ValueError("cos and sin must be contiguous [n_pos][rot/2]")
        n_pos, rot = cos.shape[0], 2 * cos.shape[1]
    rc = _packed_append(_PACKED_APPEND(*cache, pk, pv, pq, po, pkn, pqn, pc, ps, _vec(positions, _i32, n, dev, "positions"), k0, k1, v0, v1,
                                       q0, q1, o0, o1, heads, rot, n_pos, 1 if interleaved else 0, kt, eps), _on(dev))
    if rc:
        _check(rc)
    _written((k_pages, v_pages, k_power, v_power) if q is None else (k_pages, v_pages, k_power, v_power, q_out))
    return q_out


def ckks_clear_packed_attend(q, k_pages, v_pages, k_power, v_power, page_table, q_start, kv_len, scale=None, causal=True, window=0, out=None,
                             lse=None):
    """ckks_clear_attend over pages of 8 bits: q [T][heads][head_dim] -> out [T][heads][head_dim]."""
    dev, dtype = _device(), q.dtype
    n, heads, dim = q.shape
    cache = _packed(k_pages, v_pages, k_power, v_power, page_table, q_start, kv_len, n, dtype, dev)
    if dim != cache[19]:
        raise ValueError(f"q must be [{n}][heads][{cache[19]}]")
    pq, heads, q0, q1 = _heads(q, dtype, n, dim, dev, "q")
    given = tuple(t for t in (out, lse) if t is not None)
    if out is None:
        out = torch.empty_like(q, memory_format=_rowwise)
        po, o0, o1 = out.data_ptr(), heads * dim, dim
    else:
        po, ho, o0, o1 = _heads(out, dtype, n, dim, dev, "out")
        if ho != heads:
            raise ValueError("out must have q's heads")
    pl = 0
    if lse is not None:
        pl = _ptr(lse, _f32, dev, "lse")
        if lse.shape != (n, heads) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous [T][heads]")
    if scale is None:
        scale = dim ** -0.5
    causal = 1 if causal else 0
    args = _PACKED_ATTEND(*cache, pq, po, pl, 0, 0, q0, q1, o0, o1, heads, window, causal, scale)
    need = _packed_attend_work(args)
    if need:
        work = q.new_empty(need, dtype=_u8)
        args = _PACKED_ATTEND(*cache, pq, po, pl, work.data_ptr(), need, q0, q1, o0, o1, heads, window, causal, scale)
    rc = _packed_attend(args, _on(dev))
    if rc:
        _check(rc)
    if given:
        _written(given)
    return out


def ckks_clear_packed_read(k_pages, v_pages, k_power, v_power, page_table, q_start, kv_len, n_tokens, dtype=torch.float32, k_out=None, v_out=None):
    """Rows out of pages of 8 bits -> (k, v) [n_tokens][kv_heads][head_dim] of `dtype`: of sequence b the last q_start[b+1] - q_start[b] of
    its kv_len[b]."""
    dev = _device()
    cache = _packed(k_pages, v_pages, k_power, v_power, page_table, q_start, kv_len, n_tokens, dtype, dev)
    kv_heads, dim = cache[18], cache[19]
    given = tuple(t for t in (k_out, v_out) if t is not None)
    if k_out is None:
        k_out = k_pages.new_empty((n_tokens, kv_heads, dim), dtype=dtype)
    if v_out is None:
        v_out = k_pages.new_empty((n_tokens, kv_heads, dim), dtype=dtype)
    pk, hk, k0, k1 = _heads(k_out, dtype, n_tokens, dim, dev, "k_out")
    pv, hv, v0, v1 = _heads(v_out, dtype, n_tokens, dim, dev, "v_out")
    if hk != kv_heads or hv != kv_heads:
        raise ValueError(f"k_out and v_out must have {kv_heads} heads")
    rc = _packed_read(_PACKED_READ(*cache, pk, pv, k0, k1, v0, v1), _on(dev))
    if rc:
        _check(rc)
    if given:
        _written(given)
    return k_out, v_out


def ckks_clear_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, out=None, prob=None):
    """Draws a token of each row of logits [R][V] by u [R] of [0, 1) -> out int32 [R] (-1 for a row without a finite logit).
    temperature, top_p, min_p float32 [R], top_k int32 [R]; prob: float32 [R] to fill with the drawn tokens' probabilities, or None."""
    dev, code = _device(), _type(logits, "logits")
    pl = _ptr(logits, logits.dtype, dev, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be [rows][vocab]")
    rows, vocab, ls = _rows(logits, "logits")
    given = tuple(t for t in (out, prob) if t is not None)
    if out is None:
        out = logits.new_empty(rows, dtype=_i32)
    rc = _sample(_SAMPLE(pl, _vec(out, _i32, rows, dev, "out"), _vec(prob, _f32, rows, dev, "prob"), _vec(u, _f32, rows, dev, "u"),
                         _vec(temperature, _f32, rows, dev, "temperature"), _vec(top_p, _f32, rows, dev, "top_p"),
                         _vec(min_p, _f32, rows, dev, "min_p"), _vec(top_k, _i32, rows, dev, "top_k"), ls, rows, vocab, code, 0), _on(dev))
    if rc:
        _check(rc)
    if given:
        _written(given)
    return out
