"""CPU-only checks of the steps in the clear: argument structs as the header has them, and refusals, none of which reaches a GPU."""
import os
import struct
import subprocess

import pytest
import torch

from paper_2604_09975_amd import binding as B
from paper_2604_09975_amd import clear as K

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 40          # an address that nothing dereferences


def last():
    return B.lib.ckks_last_error().decode()


def test_structs_as_a_c_compiler_lays_them_out(tmp_path):
    """Size and the offset of the last field of each struct; the header is plain C."""
    fields = {"norm": "reserved", "norm_grad": "weight_dtype", "append": "flags", "attend": "scale", "logits": "out_dtype"}
    src = '#include <stddef.h>\n#include <stdio.h>\n#include "ckks_clear.h"\nint main(void) {\n'
    src += "".join(f'printf("%zu %zu\\n", sizeof(ckks_clear_{n}_t), offsetof(ckks_clear_{n}_t, {f}));\n' for n, f in fields.items())
    (tmp_path / "s.c").write_text(src + "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    got = [tuple(map(int, l.split())) for l in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.splitlines()]
    pages, batch = K._PAGES, K._BATCH
    formats = ["=6Q2q4IfI", "=10Q3q4I", "=" + pages + batch + "7Q8q4I", "=" + pages + batch + "5Q4q3If", "=12Q3q6I"]
    for (size, offset), fmt in zip(got, formats):
        assert struct.calcsize(fmt) == size and size - 4 == offset


def test_null_arguments_are_errors():
    for n in ("layer_norm", "layer_norm_grad", "cache_append", "attend", "logits"):
        assert getattr(B.lib, "ckks_clear_" + n)(None, None) == -1
        assert "null" in last() and n in last()
    assert B.lib.ckks_clear_attend_work_bytes(None) == 0


def norm(**k):
    a = dict(x=P, w=0, b=0, y=2 * P, mean=0, rstd=0, xs=64, ys=64, rows=4, cols=64, dtype=1, wtype=0, eps=1e-5)
    a.update(k)
    return B.lib.ckks_clear_layer_norm(K._NORM(*a.values(), 0), None)


@pytest.mark.parametrize("bad", [dict(x=0), dict(y=0), dict(cols=0), dict(rows=1 << 31), dict(dtype=3), dict(wtype=2), dict(dtype=0, wtype=1), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(mean=3 * P), dict(y=P + 2), dict(y=P, ys=128), dict(ys=63), dict(ys=0), dict(w=2 * P + 64),
                                 dict(mean=2 * P, rstd=3 * P), dict(mean=3 * P, rstd=3 * P + 4)])
def test_layer_norm_refusals(bad):
    assert norm(**bad) == -1 and "ckks_clear_layer_norm" in last()


def test_no_rows_is_no_work():
    assert norm(rows=0, x=0, y=0) == 0
    assert attend(n_tokens=0) == 0 and append(n_tokens=0) == 0 and logits(rows=0) == 0


def grad(**k):
    a = dict(dy=P, x=2 * P, w=0, mean=3 * P, rstd=4 * P, dx=5 * P, dw=6 * P, db=7 * P, work=8 * P, bytes=1 << 20, dys=64, xs=64, dxs=64, rows=4, cols=64,
             dtype=2, wtype=0)
    a.update(k)
    return B.lib.ckks_clear_layer_norm_grad(K._NORM_GRAD(*a.values()), None)


@pytest.mark.parametrize("bad", [dict(dy=0), dict(x=0), dict(mean=0), dict(bytes=16), dict(work=0), dict(work=8 * P + 1), dict(dx=2 * P), dict(dx=P + 2),
                                 dict(dw=5 * P), dict(db=8 * P + 8), dict(dxs=10), dict(cols=0), dict(dtype=9), dict(work=2 * P)])
def test_layer_norm_grad_refusals(bad):
    assert grad(**bad) == -1 and "ckks_clear_layer_norm_grad" in last()


def test_work_bytes_cover_all_sizes():
    for cols in (1, 8, 64, 2048, 2049, 8192, 16384, 16385, 100000):
        sizes = [B.lib.ckks_clear_layer_norm_grad_work_bytes(rows, cols, 0) for rows in (0, 1, 5, 100, 10**4, 10**6)]
        assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[1] >= 8 * cols


CACHE = dict(k=P, v=2 * P, ks0=2048, ks1=1024, ks2=64, vs0=2048, vs1=1024, vs2=64, n_pages=10, page=16, kv_heads=2, dim=64, dtype=1, r0=0,
             q_start=3 * P, kv_len=4 * P, table=5 * P, ts=4, n_seq=2, n_tokens=5, width=4, r1=0)
BAD_CACHE = [dict(dim=0), dict(dim=60), dict(dim=264), dict(kv_heads=0), dict(page=0), dict(dtype=7), dict(n_seq=0), dict(q_start=0), dict(kv_len=0), dict(table=0),
             dict(k=0), dict(v=0), dict(width=1 << 27, page=16), dict(ks0=1 << 32), dict(vs0=-1), dict(ks2=1 << 31), dict(vs2=1 << 28, page=16), dict(n_tokens=1 << 31)]


def append(**k):
    a = dict(CACHE, new_k=6 * P, new_v=7 * P, q=8 * P, q_out=9 * P, cos=10 * P, sin=11 * P, positions=0, k0=128, k1=64, v0=128, v1=64, q0=256, q1=64, o0=256, o1=64,
             heads=4, rot=64, n_pos=64, flags=0)
    a.update(k)
    return B.lib.ckks_clear_cache_append(K._APPEND(*a.values()), None)


@pytest.mark.parametrize("bad", BAD_CACHE + [dict(new_k=0), dict(new_v=0), dict(q_out=0), dict(heads=0), dict(rot=63), dict(rot=66), dict(cos=0), dict(sin=0),
                                             dict(flags=2), dict(new_k=P), dict(q_out=8 * P + 2), dict(q_out=6 * P), dict(k=11 * P), dict(positions=P),
                                             dict(q_out=8 * P, o0=300), dict(table=2 * P)])
def test_append_refusals(bad):
    assert append(**bad) == -1 and "ckks_clear_cache_append" in last()


def attend(**k):
    a = dict(CACHE, q=6 * P, out=7 * P, lse=0, work=8 * P, bytes=1 << 30, q0=256, q1=64, o0=256, o1=64, heads=4, window=0, flags=1, scale=0.125)
    a.update(k)
    return B.lib.ckks_clear_attend(K._ATTEND(*a.values()), None)


@pytest.mark.parametrize("bad", BAD_CACHE + [dict(q=0), dict(out=0), dict(heads=3), dict(heads=0), dict(heads=1 << 17), dict(flags=2), dict(flags=0, window=5),
                                             dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(out=6 * P), dict(out=P),
                                             dict(lse=7 * P), dict(lse=6 * P), dict(out=4 * P)])
def test_attend_refusals(bad):
    assert attend(**bad) == -1 and "ckks_clear_attend" in last()


def test_attend_workspace():
    """Few rows over a long axis are split, and the workspace for it is asked for."""
    a = dict(CACHE, width=8192, ts=8192, q=6 * P, out=7 * P, lse=0, work=0, bytes=0, q0=256, q1=64, o0=256, o1=64, heads=4, window=0, flags=1, scale=0.125)
    need = B.lib.ckks_clear_attend_work_bytes(K._ATTEND(*a.values()))
    assert need > 0 and need % (5 * 4 * (64 + 1) * 4) == 0
    for k in (dict(), dict(work=8 * P, bytes=need - 1), dict(work=8 * P + 4, bytes=need), dict(work=7 * P, bytes=need)):
        assert attend(**dict(a, **k)) == -1
    assert B.lib.ckks_clear_attend_work_bytes(K._ATTEND(*dict(a, width=4).values())) == 0
    assert B.lib.ckks_clear_attend_work_bytes(K._ATTEND(*dict(a, heads=3).values())) == 0


def logits(**k):
    a = dict(logits=P, out=2 * P, tokens=3 * P, token_start=4 * P, n_prompt=0, rep=5 * P, freq=0, pres=0, bias_ids=6 * P, bias_start=7 * P, bias=8 * P, mask=9 * P,
             ls=100, os=100, ms=4, rows=3, vocab=100, n_tokens=10, n_biases=5, dtype=2, out_dtype=2)
    a.update(k)
    return B.lib.ckks_clear_logits(K._LOGITS(*a.values()), None)


@pytest.mark.parametrize("bad", [dict(logits=0), dict(out=0), dict(tokens=0), dict(token_start=0), dict(bias=0), dict(bias_ids=0), dict(bias_start=0), dict(dtype=4),
                                 dict(out_dtype=1), dict(dtype=0, out_dtype=2), dict(os=99), dict(out=P + 2), dict(out=P, out_dtype=0), dict(out=P, os=101),
                                 dict(out=9 * P), dict(out=3 * P), dict(n_tokens=1 << 30), dict(n_biases=1 << 30), dict(vocab=1 << 31), dict(rows=1 << 30, vocab=1 << 20)])
def test_logits_refusals(bad):
    assert logits(**bad) == -1 and "ckks_clear_logits" in last()


def test_binding_refuses_what_is_no_device_tensor(monkeypatch):
    monkeypatch.setattr(K, "_device", lambda: 0)
    x = torch.zeros(4, 8)
    for call in (lambda: K.ckks_clear_layer_norm(x), lambda: K.ckks_clear_logits(x), lambda: K.ckks_clear_layer_norm(None),
                 lambda: K.ckks_clear_layer_norm(x.to(torch.float64)), lambda: K.ckks_clear_layer_norm_grad(x, x, x, x)):
        with pytest.raises(TypeError):
            call()
