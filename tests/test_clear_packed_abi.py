"""CPU-only checks of the cache of 8 bits and of the draw: argument structs as the header has them, and refusals, none of which
reaches a GPU."""
import os
import random
import struct
import subprocess

import pytest
import torch

from paper_2604_09975_amd import binding as B
from paper_2604_09975_amd import clear as K
from tests.test_clear_abi import P, last
from tests.test_clear_overlap import READ, ask, cells, layout

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_structs_as_a_c_compiler_lays_them_out(tmp_path):
    fields = {"packed": "dtype", "packed_append": "eps", "packed_attend": "scale", "packed_read": "v_out_stride", "sample": "reserved"}
    src = '#include <stddef.h>\n#include <stdio.h>\n#include "ckks_clear.h"\nint main(void) {\n'
    src += "".join(f'printf("%zu %zu\\n", sizeof(ckks_clear_{n}_t), offsetof(ckks_clear_{n}_t, {f}));\n' for n, f in fields.items())
    (tmp_path / "s.c").write_text(src + "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    got = [tuple(map(int, l.split())) for l in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.splitlines()]
    packed, batch = K._PACKED, K._BATCH
    formats = ["=" + packed, "=" + packed + batch + "9Q8q5If", "=" + packed + batch + "5Q4q3If", "=" + packed + batch + "2Q4q", "=8Qq4I"]
    for (size, offset), fmt, tail in zip(got, formats, (4, 4, 4, 16, 4)):
        assert struct.calcsize(fmt) == size and size - tail == offset


def test_null_arguments_are_errors():
    for n in ("packed_append", "packed_attend", "packed_read", "sample"):
        assert getattr(B.lib, "ckks_clear_" + n)(None, None) == -1
        assert "null" in last() and n in last()
    assert B.lib.ckks_clear_packed_attend_work_bytes(None) == 0


PACKED = dict(k=P, v=2 * P, kz=20 * P, vz=21 * P, ks0=2048, ks1=1024, ks2=64, vs0=2048, vs1=1024, vs2=64, kz0=64, kz1=32, kz2=2, vz0=64, vz1=32, vz2=2,
              n_pages=10, page=16, kv_heads=2, dim=64, form=16, dtype=1, q_start=3 * P, kv_len=4 * P, table=5 * P, ts=4, n_seq=2, n_tokens=5, width=4, r1=0)
BAD = [dict(dim=0), dict(dim=60), dict(dim=264), dict(kv_heads=0), dict(kv_heads=1 << 17), dict(page=0), dict(dtype=7), dict(form=0), dict(form=18), dict(n_seq=0),
       dict(q_start=0), dict(kv_len=0), dict(table=0), dict(k=0), dict(v=0), dict(kz=0), dict(vz=0), dict(width=1 << 27, page=16), dict(ks0=1 << 32), dict(vs0=-1),
       dict(ks2=1 << 31), dict(vs2=1 << 28), dict(kz0=1 << 32), dict(vz1=-2), dict(vz2=1 << 28), dict(n_tokens=1 << 31)]


def append(**k):
    a = dict(PACKED, new_k=6 * P, new_v=7 * P, q=8 * P, q_out=9 * P, k_norm=12 * P, q_norm=13 * P, cos=10 * P, sin=11 * P, positions=0, k0=128, k1=64, v0=128, v1=64,
             q0=256, q1=64, o0=256, o1=64, heads=4, rot=64, n_pos=64, flags=0, norm_dtype=0, eps=1e-6)
    a.update(k)
    return B.lib.ckks_clear_packed_append(K._PACKED_APPEND(*a.values()), None)


Q = dict(q=8 * P, q_out=8 * P)   # 4 heads of 64 in place, 16 bits


@pytest.mark.parametrize("bad", BAD + [
    dict(new_k=0), dict(new_v=0), dict(q_out=0), dict(heads=0), dict(heads=1 << 17), dict(rot=63), dict(rot=66), dict(cos=0), dict(sin=0), dict(flags=2),
    dict(norm_dtype=2), dict(norm_dtype=9), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(q=0), dict(q=0, q_out=0),
    dict(new_k=P), dict(new_v=20 * P), dict(q_out=8 * P + 2), dict(q_out=6 * P), dict(q_out=21 * P), dict(q_out=P), dict(k=11 * P), dict(kz=10 * P), dict(positions=P),
    dict(positions=20 * P), dict(k_norm=9 * P), dict(q_norm=2 * P), dict(table=21 * P), dict(q_out=8 * P, o0=300),
    # queries in place that share entries with the new keys or values
    dict(Q, new_k=8 * P, k0=256), dict(Q, new_v=8 * P + 2 * 128, v0=256), dict(Q, q0=512, o0=512, new_k=8 * P + 2 * 248, k0=512),
    # pages in one another's places
    dict(v=P), dict(v=P + 8), dict(kz=P), dict(vz=20 * P + 1), dict(kz=P + 2047, ks0=4096, kz0=4096), dict(kz=P + 63, ks2=80, ks1=1280, ks0=2560, kz2=80, kz1=1280, kz0=2560),
    # rows of an output that overlap
    dict(o0=0), dict(o1=63), dict(ks0=0), dict(ks1=0), dict(vs2=63), dict(kz2=1), dict(vz0=62), dict(vz1=0)])
def test_append_refusals(bad):
    assert append(**bad) == -1 and "ckks_clear_packed_append" in last()


def attend(**k):
    a = dict(PACKED, q=6 * P, out=7 * P, lse=0, work=8 * P, bytes=1 << 30, q0=256, q1=64, o0=256, o1=64, heads=4, window=0, flags=1, scale=0.125)
    a.update(k)
    return B.lib.ckks_clear_packed_attend(K._PACKED_ATTEND(*a.values()), None)


@pytest.mark.parametrize("bad", BAD + [
    dict(q=0), dict(out=0), dict(heads=3), dict(heads=0), dict(heads=1 << 17), dict(flags=2), dict(flags=0, window=5), dict(scale=0.0), dict(scale=float("inf")),
    dict(scale=float("nan")), dict(out=6 * P), dict(out=P), dict(out=20 * P), dict(out=21 * P), dict(lse=7 * P), dict(lse=20 * P), dict(out=4 * P), dict(o0=0), dict(o1=63)])
def test_attend_refusals(bad):
    assert attend(**bad) == -1 and "ckks_clear_packed_attend" in last()


def test_attend_workspace():
    """Few rows over a long axis are split, and the workspace for it is asked for."""
    a = dict(PACKED, width=8192, ts=8192, q=6 * P, out=7 * P, lse=0, work=0, bytes=0, q0=256, q1=64, o0=256, o1=64, heads=4, window=0, flags=1, scale=0.125)
    for dtype in (0, 1, 2):
        a["dtype"] = dtype
        need = B.lib.ckks_clear_packed_attend_work_bytes(K._PACKED_ATTEND(*a.values()))
        assert need > 0 and need % (5 * 4 * (64 + 1) * 4) == 0
        for k in (dict(), dict(work=8 * P, bytes=need - 1), dict(work=8 * P + 4, bytes=need), dict(work=7 * P, bytes=need), dict(work=20 * P, bytes=need)):
            assert attend(**dict(a, **k)) == -1
        assert B.lib.ckks_clear_packed_attend_work_bytes(K._PACKED_ATTEND(*dict(a, heads=3).values())) == 0


def read(**k):
    a = dict(PACKED, k_out=6 * P, v_out=7 * P, k0=128, k1=64, v0=128, v1=64)
    a.update(k)
    return B.lib.ckks_clear_packed_read(K._PACKED_READ(*a.values()), None)


@pytest.mark.parametrize("bad", BAD + [dict(k_out=P), dict(v_out=2 * P), dict(k_out=20 * P), dict(v_out=21 * P), dict(k_out=3 * P), dict(v_out=5 * P), dict(k_out=7 * P),
                                       dict(v_out=6 * P + 2 * 64), dict(k0=0), dict(v1=63), dict(v0=100)])
def test_read_refusals(bad):
    assert read(**bad) == -1 and "ckks_clear_packed_read" in last()


def sample(**k):
    a = dict(logits=P, token=2 * P, prob=3 * P, u=4 * P, temperature=5 * P, top_p=6 * P, min_p=7 * P, top_k=8 * P, stride=100, rows=3, vocab=100, dtype=2, reserved=0)
    a.update(k)
    return B.lib.ckks_clear_sample(K._SAMPLE(*a.values()), None)


@pytest.mark.parametrize("bad", [dict(logits=0), dict(token=0), dict(u=0), dict(dtype=3), dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(rows=1 << 31), dict(token=P),
                                 dict(token=P + 2 * 299), dict(prob=2 * P), dict(prob=2 * P + 8), dict(prob=4 * P), dict(token=8 * P), dict(prob=5 * P), dict(token=6 * P + 4), dict(prob=7 * P)])
def test_sample_refusals(bad):
    assert sample(**bad) == -1 and "ckks_clear_sample" in last()


def test_no_work_is_none():
    assert append(n_tokens=0) == 0 and attend(n_tokens=0) == 0 and read(n_tokens=0) == 0 and sample(rows=0, logits=0) == 0
    assert read(k_out=0, v_out=0) == 0


def test_shared_bytes_of_runs_of_different_lengths_are_found_exactly(tmp_path):
    rng, asked, want = random.Random(3), [], []
    for _ in range(6000):
        a, b = layout(rng, 3), layout(rng, 3)
        if rng.random() < 0.6:
            b = [(rng.randint(1, 4), s) for _, s in a]
        m, n = rng.randint(1, 12), rng.randint(1, 12)
        p, q = 1000, 1000 + rng.randint(-120, 120)
        asked.append([p, m, 3] + [x for d in a for x in d] + [q, n, 3] + [x for d in b for x in d])
        want.append(bool(set(cells(p, m, a)) & set(cells(q, n, b))))
    got = ask(tmp_path, READ + 'int main() { Runs a, b; while (read(a) && read(b)) puts(share_any(a, b) ? "1" : "0"); }', asked)
    assert 1000 < sum(want) < 5000 and [g == "1" for g in got] == want


def test_binding_refuses_what_is_no_device_tensor(monkeypatch):
    monkeypatch.setattr(K, "_device", lambda: 0)
    k, z, x = torch.zeros(2, 1, 4, 32, dtype=torch.int8), torch.zeros(2, 1, 4, 1, dtype=torch.uint8), torch.zeros(3, 1, 32)
    i = torch.zeros(2, 2, dtype=torch.int32)
    for call in (lambda: K.ckks_clear_packed_append(x, x, k, k, z, z, i, i[0], i[0]), lambda: K.ckks_clear_packed_attend(x, k, k, z, z, i, i[0], i[0]),
                 lambda: K.ckks_clear_packed_read(k, k, z, z, i, i[0], i[0], 3), lambda: K.ckks_clear_sample(x[:, 0], x[:, 0, 0]), lambda: K.ckks_clear_sample(None, None)):
        with pytest.raises(TypeError):
            call()
