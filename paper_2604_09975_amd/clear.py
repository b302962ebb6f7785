"""Binding of include/ckks_clear.h: the key holder's steps in the clear between two encrypted projections.

Argument marshalling only, as in `binding`: every function has the name of the C entry point it calls, takes torch tensors on
the current HIP device and enqueues on torch's current stream.  Rows may be strided; their last dimension is contiguous.
Types are float32, float16 and bfloat16.  Workspaces come from torch's allocator, on the stream of the call.
"""
import struct

import torch

from .binding import C, _check, _raw_stream, _stream, lib

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

# The argument structs of the header, field by field.
_NORM = struct.Struct("=6Q2q4IfI")
_NORM_GRAD = struct.Struct("=10Q3q4I")
_PAGES, _BATCH = "2Q6q6I", "3Qq4I"
_APPEND = struct.Struct("=" + _PAGES + _BATCH + "7Q8q4I")
_ATTEND = struct.Struct("=" + _PAGES + _BATCH + "5Q4q3If")
_LOGITS = struct.Struct("=12Q3q6I")

for _n in ("layer_norm", "layer_norm_grad", "cache_append", "attend", "logits"):
    getattr(lib, "ckks_clear_" + _n).argtypes = [C.c_char_p, C.c_void_p]
    getattr(lib, "ckks_clear_" + _n).restype = C.c_int
lib.ckks_clear_layer_norm_grad_work_bytes.argtypes = [C.c_uint32] * 3
lib.ckks_clear_layer_norm_grad_work_bytes.restype = C.c_uint64
lib.ckks_clear_attend_work_bytes.argtypes = [C.c_char_p]
lib.ckks_clear_attend_work_bytes.restype = C.c_uint64


class _Call:
    """The tensors of one call: all on the current device."""
    __slots__ = ("device",)

    def __init__(self):
        self.device = torch.cuda.current_device()

    def ptr(self, t, dtype, what):
        if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != self.device:
            raise TypeError(f"{what}: expected a {dtype} tensor on device {self.device}")
        return t.data_ptr()

    def vec(self, t, dtype, n, what):
        """Pointer of a contiguous vector (n None: of any length); 0 for None."""
        if t is None:
            return 0
        p = self.ptr(t, dtype, what)
        if t.dim() != 1 or (n is not None and t.shape[0] != n) or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous vector of {n}" if n is not None else f"{what} must be a contiguous vector")
        return p

    def stream(self):
        return _raw_stream(self.device) if _raw_stream is not None else _stream()


def _type(t, what):
    code = _TYPES.get(getattr(t, "dtype", None))
    if code is None:
        raise TypeError(f"{what}: expected a float32, float16 or bfloat16 tensor")
    return code


def _rows(t, what):
    """[..., cols] as (rows, cols, row stride); the leading dimensions must be those of evenly spaced rows."""
    if t.dim() == 0:
        raise ValueError(f"{what} must have at least one dimension")
    if t.dim() != 2:
        t = t.view(-1, t.shape[-1]) if t.numel() else t.reshape(0, t.shape[-1])
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    return t.shape[0], t.shape[1], t.stride(0)


def _out(out, like, dtype, what):
    if out is None:
        return torch.empty(like.shape, dtype=dtype, device=like.device)
    if out.shape != like.shape:
        raise ValueError(f"{what} must have the input's shape")
    return out


def _param(call, t, x, cols, what):
    """Type code and pointer of a weight or bias: float32 or the rows' type."""
    if t is None:
        return None, 0
    if t.dtype is not torch.float32 and t.dtype is not x.dtype:
        raise TypeError(f"{what} must be float32 or of the rows' type")
    return _TYPES[t.dtype], call.vec(t, t.dtype, cols, what)


def ckks_clear_layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stats=True):
    """x [..., C] -> (y, mean, rstd): y of x's type, mean and rstd float32 of the rows (None without `stats`)."""
    call, code = _Call(), _type(x, "x")
    px = call.ptr(x, x.dtype, "x")
    rows, cols, xs = _rows(x, "x")
    wt, pw = _param(call, weight, x, cols, "weight")
    bt, pb = _param(call, bias, x, cols, "bias")
    if wt is not None and bt is not None and wt != bt:
        raise TypeError("weight and bias must be of one type")
    y = _out(out, x, x.dtype, "out")
    py = call.ptr(y, x.dtype, "out")
    mean = rstd = None
    if stats:
        mean, rstd = torch.empty((2,) + x.shape[:-1], dtype=torch.float32, device=x.device).unbind(0)
    wt = wt if wt is not None else bt if bt is not None else 0
    _check(lib.ckks_clear_layer_norm(
        _NORM.pack(px, pw, pb, py, mean.data_ptr() if stats else 0, rstd.data_ptr() if stats else 0, xs, _rows(y, "out")[2],
                   rows, cols, code, wt, eps, 0), call.stream()))
    return y, mean, rstd


def ckks_clear_layer_norm_grad(dy, x, mean, rstd, weight=None, dx=None, params=True):
    """-> (dx, dweight, dbias) of the call that gave mean and rstd; the parameters' gradients have the weight's type (float32
    without a weight) and are None without `params`."""
    call, code = _Call(), _type(x, "x")
    px, pdy = call.ptr(x, x.dtype, "x"), call.ptr(dy, x.dtype, "dy")
    rows, cols, xs = _rows(x, "x")
    if dy.shape != x.shape:
        raise ValueError("dy must have x's shape")
    for t, what in ((mean, "mean"), (rstd, "rstd")):
        call.ptr(t, torch.float32, what)
        if t.numel() != rows or not t.is_contiguous():
            raise ValueError(f"{what} must hold one value for each row")
    wt, pw = _param(call, weight, x, cols, "weight")
    gx = _out(dx, x, x.dtype, "dx")
    pgx = call.ptr(gx, x.dtype, "dx")
    dw = db = work = None
    need = 0
    if params:
        dw, db = torch.empty((2, cols), dtype=weight.dtype if weight is not None else torch.float32, device=x.device).unbind(0)
        need = lib.ckks_clear_layer_norm_grad_work_bytes(rows, cols, code)
        work = torch.empty(max(need, 4), dtype=torch.uint8, device=x.device)
    _check(lib.ckks_clear_layer_norm_grad(
        _NORM_GRAD.pack(pdy, px, pw, mean.data_ptr(), rstd.data_ptr(), pgx, dw.data_ptr() if params else 0,
                        db.data_ptr() if params else 0, work.data_ptr() if params else 0, need,
                        _rows(dy, "dy")[2], xs, _rows(gx, "dx")[2], rows, cols, code, wt if wt is not None else 0), call.stream()))
    return gx, dw, db


def _heads(call, t, dtype, n, heads, dim, what):
    """Pointer and strides {token, head} of [n][heads][dim]."""
    p = call.ptr(t, dtype, what)
    if t.dim() != 3 or t.shape[0] != n or (heads is not None and t.shape[1] != heads) or t.shape[2] != dim:
        raise ValueError(f"{what} must be [{n}][{heads if heads is not None else 'heads'}][{dim}]")
    st = t.stride()
    if dim > 1 and st[2] != 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    return p, st[0], st[1]


def _cache(call, k_pages, v_pages, page_table, q_start, kv_len, n_tokens):
    """Fields of ckks_clear_pages_t and ckks_clear_batch_t."""
    code = _type(k_pages, "k_pages")
    pk, pv = call.ptr(k_pages, k_pages.dtype, "k_pages"), call.ptr(v_pages, k_pages.dtype, "v_pages")
    if k_pages.dim() != 4 or v_pages.shape != k_pages.shape:
        raise ValueError("k_pages and v_pages must be [n_pages][kv_heads][page_size][head_dim]")
    ks, vs = k_pages.stride(), v_pages.stride()
    n_pages, kv_heads, page_size, dim = k_pages.shape
    if dim > 1 and (ks[3] != 1 or vs[3] != 1):
        raise ValueError("the last dimension of the pages must be contiguous")
    pt = call.ptr(page_table, torch.int32, "page_table")
    if page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table must be [n_seq][pages], its last dimension contiguous")
    n_seq = page_table.shape[0]
    return (pk, pv, ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], n_pages, page_size, kv_heads, dim, code, 0,
            call.vec(q_start, torch.int32, n_seq + 1, "q_start"), call.vec(kv_len, torch.int32, n_seq, "kv_len"), pt,
            page_table.stride(0), n_seq, n_tokens, page_table.shape[1], 0)


def ckks_clear_cache_append(k, v, k_pages, v_pages, page_table, q_start, kv_len, cos=None, sin=None, interleaved=False,
                            positions=None, q=None, q_out=None):
    """k, v [T][kv_heads][head_dim] into the pages, rotated by cos / sin [n_pos][rot/2] at their positions; q [T][heads][head_dim]
    rotated alike into q_out -> q_out (None without q)."""
    call = _Call()
    dtype, n = k_pages.dtype, k.shape[0]
    cache = _cache(call, k_pages, v_pages, page_table, q_start, kv_len, n)
    kv_heads, dim = k_pages.shape[1], k_pages.shape[3]
    pk, k0, k1 = _heads(call, k, dtype, n, kv_heads, dim, "k")
    pv, v0, v1 = _heads(call, v, dtype, n, kv_heads, dim, "v")
    pq = po = q0 = q1 = o0 = o1 = heads = 0
    if q is not None:
        pq, q0, q1 = _heads(call, q, dtype, n, None, dim, "q")
        heads = q.shape[1]
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=dtype, device=q.device)
        po, o0, o1 = _heads(call, q_out, dtype, n, heads, dim, "q_out")
    elif q_out is not None:
        raise ValueError("q_out without q")
    pc = ps = rot = n_pos = 0
    if cos is not None or sin is not None:
        pc, ps = call.ptr(cos, torch.float32, "cos"), call.ptr(sin, torch.float32, "sin")
        if cos.dim() != 2 or cos.shape != sin.shape or not cos.is_contiguous() or not sin.is_contiguous():
            raise ValueError("cos and sin must be contiguous [n_pos][rot/2]")
        n_pos, rot = cos.shape[0], 2 * cos.shape[1]
    _check(lib.ckks_clear_cache_append(
        _APPEND.pack(*cache, pk, pv, pq, po, pc, ps, call.vec(positions, torch.int32, n, "positions"), k0, k1, v0, v1, q0, q1, o0, o1,
                     heads, rot, n_pos, 1 if interleaved else 0), call.stream()))
    return q_out


def ckks_clear_attend(q, k_pages, v_pages, page_table, q_start, kv_len, scale=None, causal=True, window=0, out=None, lse=None):
    """q [T][heads][head_dim] over the cache -> out [T][heads][head_dim]; lse: float32 [T][heads] to fill, or None.  scale None:
    1 / sqrt(head_dim)."""
    call = _Call()
    dtype, dim = k_pages.dtype, k_pages.shape[-1]
    n = q.shape[0]
    cache = _cache(call, k_pages, v_pages, page_table, q_start, kv_len, n)
    pq, q0, q1 = _heads(call, q, dtype, n, None, dim, "q")
    heads = q.shape[1]
    if out is None:
        out = torch.empty((n, heads, dim), dtype=dtype, device=q.device)
    po, o0, o1 = _heads(call, out, dtype, n, heads, dim, "out")
    pl = 0
    if lse is not None:
        pl = call.ptr(lse, torch.float32, "lse")
        if lse.shape != (n, heads) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous [T][heads]")
    scale = dim ** -0.5 if scale is None else scale
    tail = (q0, q1, o0, o1, heads, window, 1 if causal else 0, scale)
    args = _ATTEND.pack(*cache, pq, po, pl, 0, 0, *tail)
    need = lib.ckks_clear_attend_work_bytes(args)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=q.device)
        args = _ATTEND.pack(*cache, pq, po, pl, work.data_ptr(), need, *tail)
    _check(lib.ckks_clear_attend(args, call.stream()))
    return out


def ckks_clear_logits(logits, out=None, tokens=None, token_start=None, n_prompt=None, repetition=None, frequency=None, presence=None,
                      bias_ids=None, bias=None, bias_start=None, mask=None):
    """logits [R][V] (or [V]) under the rules -> out (logits' type or float32; new if None, may be logits itself)."""
    call, code = _Call(), _type(logits, "logits")
    pl = call.ptr(logits, logits.dtype, "logits")
    rows, vocab, ls = _rows(logits, "logits")
    out = _out(out, logits, logits.dtype, "out")
    po, oc = call.ptr(out, out.dtype, "out"), _type(out, "out")
    pm = ms = 0
    if mask is not None:
        pm = call.ptr(mask, torch.int32, "mask")
        mr, words, ms = _rows(mask, "mask")
        if mr != rows or words < (vocab + 31) // 32:
            raise ValueError("mask must hold one bit for each logit, 32 to a word")
    n_tokens = tokens.numel() if tokens is not None else 0
    n_biases = bias_ids.numel() if bias_ids is not None else 0
    _check(lib.ckks_clear_logits(
        _LOGITS.pack(pl, po, call.vec(tokens, torch.int32, None, "tokens"), call.vec(token_start, torch.int32, rows + 1, "token_start"),
                     call.vec(n_prompt, torch.int32, rows, "n_prompt"), call.vec(repetition, torch.float32, rows, "repetition"),
                     call.vec(frequency, torch.float32, rows, "frequency"), call.vec(presence, torch.float32, rows, "presence"),
                     call.vec(bias_ids, torch.int32, None, "bias_ids"), call.vec(bias_start, torch.int32, rows + 1, "bias_start"),
                     call.vec(bias, torch.float32, n_biases, "bias"), pm, ls, _rows(out, "out")[2], ms,
                     rows, vocab, n_tokens, n_biases, code, oc), call.stream()))
    return out
