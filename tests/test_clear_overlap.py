"""CPU-only checks of which arrays of the steps in the clear may lie in one another: every call here is refused, none reaches a GPU."""
import itertools
import os
import random
import subprocess

import pytest

from tests.test_clear_abi import P, append, attend, last

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_09975_amd", "csrc")


def cells(at, run, dims):
    """Bytes of an array of runs."""
    got = []
    for index in itertools.product(*(range(n) for n, _ in dims)):
        start = at + sum(i * s for i, (_, s) in zip(index, dims))
        got.extend(range(start, start + run))
    return got


def ask(tmp_path, body, lines):
    """Answers of a C++ program that reads numbers line by line."""
    (tmp_path / "t.cpp").write_text('#include <cstdio>\n#include "clear_extent.h"\nusing namespace ckks;\n' + body)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-Wno-missing-braces", "-I", CSRC, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    text = "".join(" ".join(map(str, l)) + "\n" for l in lines)
    return subprocess.run([str(tmp_path / "t")], input=text, capture_output=True, text=True, check=True).stdout.split()


READ = """
static bool read(Runs &r) {
    long long at, run, v[6];
    if (scanf("%lld %lld %d", &at, &run, &r.dims) != 3) return false;
    for (int i = 0; i < 2 * r.dims; ++i)
        if (scanf("%lld", v + i) != 1) return false;
    r.at = (const void *)at, r.run = run;
    for (int i = 0; i < r.dims; ++i) r.dim[i].n = v[2 * i], r.dim[i].stride = v[2 * i + 1];
    return true;
}
"""


def layout(rng, n):
    return [(rng.randint(1, 4), rng.choice((0, 3, 4, 5, 8, 11, 12, 16, 24, 31, 32, 40, 64, 96, -8, -20, -64))) for _ in range(n)]


def test_shared_entries_are_found_exactly(tmp_path):
    rng, asked, want = random.Random(1), [], []
    for _ in range(6000):
        n, run = rng.choice((2, 3)), rng.randint(1, 9)
        a, b = layout(rng, n), layout(rng, n)
        if rng.random() < 0.6:  # most often the same strides, as for columns of one array
            b = [(rng.randint(1, 4), s) for _, s in a]
        p, q = 1000, 1000 + rng.randint(-120, 120)
        asked.append([p, run, n] + [x for d in a for x in d] + [q, run, n] + [x for d in b for x in d])
        want.append(bool(set(cells(p, run, a)) & set(cells(q, run, b))))
    got = ask(tmp_path, READ + 'int main() { Runs a, b; while (read(a) && read(b)) puts(share(a, b) ? "1" : "0"); }', asked)
    assert 1000 < sum(want) < 5000 and [g == "1" for g in got] == want


def test_arrays_that_meet_themselves_are_found_exactly(tmp_path):
    rng, asked, want = random.Random(2), [], []
    for _ in range(6000):
        n, run = rng.choice((2, 3)), rng.randint(1, 9)
        a = layout(rng, n)
        asked.append([1000, run, n] + [x for d in a for x in d])
        all_of_it = cells(1000, run, a)
        want.append(len(set(all_of_it)) < len(all_of_it))
    got = ask(tmp_path, READ + 'int main() { Runs a; while (read(a)) puts(share_within(a) ? "1" : "0"); }', asked)
    assert 1000 < sum(want) < 5000 and [g == "1" for g in got] == want


def test_layouts_of_use_are_settled_quickly(tmp_path):
    """Queries beside keys of 10^6 tokens: columns of one array, heads side by side in either order, a head's query, key and value
    together; and the same with one entry shared.  Nothing here may run out of tries."""
    t, h, d, asked, want = 10**6, 128, 256, [], []
    row = 3 * h * d
    for qs, ks, at in (((row, d), (row, d), h * d), ((row, 3 * d), (row, 3 * d), d), ((d, 3 * t * d), (d, 3 * t * d), t * d), ((2 * h * d, d), (2 * h * d, d), h * d),
                       ((row, 2 * d), (row, d), (2 * h - 1) * d)):
        for less, hit in ((0, False), (2, True)):
            asked.append([0, d, 2, t, qs[0], h, qs[1], at - less, d, 2, t, ks[0], h, ks[1]])
            want.append(hit)
    assert [g == "1" for g in ask(tmp_path, READ + 'int main() { Runs a, b; while (read(a) && read(b)) puts(share(a, b) ? "1" : "0"); }', asked)] == want


Q = dict(q=8 * P, q_out=8 * P)   # 4 heads of 64 in place, 16 bits


@pytest.mark.parametrize("bad", [
    dict(Q, new_k=8 * P, k0=256), dict(Q, new_v=8 * P, v0=256),                          # the very queries
    dict(Q, new_k=8 * P + 2 * 64, k0=256), dict(Q, new_v=8 * P + 2 * 64 * 2, v0=256),    # some of their heads
    dict(Q, q0=512, o0=512, new_k=8 * P + 2 * 248, k0=512),                              # columns that reach into the last head
    dict(Q, q0=512, o0=512, new_k=8 * P + 2 * 392, k0=512),                              # ... into the next token's first
    dict(Q, q0=384, o0=384, q1=96, o1=96, new_k=8 * P + 2 * 60, k0=384, k1=96),          # ... into a head that they lie beside
    dict(Q, new_k=8 * P + 2 * 256, k0=512),                                              # other strides
])
def test_keys_and_values_that_share_entries_with_queries_in_place(bad):
    assert append(**bad) == -1 and "overlaps" in last()


@pytest.mark.parametrize("bad", [
    dict(v=P), dict(v=P + 2 * 8), dict(v=P + 2 * 2048), dict(v=P + 2 * 1024),                     # the keys' places, some of them, the next page's
    dict(ks0=4096, vs0=4096, v=P + 2 * 2040), dict(ks2=128, vs2=128, v=P + 2 * 60),               # beside the keys, but not quite
    dict(v=P + 2 * 1024 * 5, vs0=1024, vs1=0),                                                    # other strides
])
def test_values_in_the_places_of_keys(bad):
    assert append(**bad) == -1 and "overlaps" in last()


@pytest.mark.parametrize("bad", [dict(o0=0), dict(o1=0), dict(o0=192), dict(o1=63), dict(o0=64, o1=128), dict(o0=200, o1=64), dict(o0=-255)])
def test_rows_of_an_output_that_overlap(bad):
    """(5 tokens of 4 heads of 64)"""
    for call in (append, attend):
        assert call(**bad) == -1 and "overlap" in last()


@pytest.mark.parametrize("bad", [dict(ks0=0), dict(ks1=0), dict(vs1=0), dict(ks2=0), dict(vs2=63), dict(ks0=1984), dict(vs1=1000), dict(ks1=32, ks2=64)])
def test_pages_that_overlap_are_not_written(bad):
    assert append(**bad) == -1 and "overlap" in last()
