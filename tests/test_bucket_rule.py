"""The distances at which the buckets of a relative position bias begin, for every number of buckets and every largest
distance that the calls take, against the rule in whole numbers: the smallest n with n^s >= e^(s - t) d^t."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2010_04902_b200", "csrc")


@pytest.fixture(scope="module")
def starts_of(tmp_path_factory):
    where = tmp_path_factory.mktemp("rule")
    source, lib = os.path.join(where, "rule.cpp"), os.path.join(where, "rule.so")
    with open(source, "w") as fh:
        fh.write('#include "bucket_rule.h"\n'
                 'extern "C" void all_starts(int nb, int from, int to, uint16_t* out) {\n'
                 '    for (int d = from; d <= to; ++d, out += nb - nb / 2) bz::bucket_starts(nb, d, out);\n}\n')
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-I", CSRC, "-o", lib, source], check=True)
    fn = ctypes.CDLL(lib).all_starts

    def starts(nb, lo, hi):
        out = np.zeros((hi - lo + 1, nb - nb // 2), np.uint16)
        fn(nb, lo, hi, ctypes.c_void_p(out.ctypes.data))
        return out.astype(np.int64)

    return starts


def reached(n, nb, d, t):
    e = nb // 2
    s = nb - e
    return n ** s >= e ** (s - t) * d ** t


@pytest.mark.parametrize("nb,d,t,want", [(73, 905, 26, 348), (109, 1549, 20, 184), (187, 1839, 1, 97), (226, 188, 73, 158)])
def test_bounds_just_above_a_whole_number(starts_of, nb, d, t, want):
    assert reached(want, nb, d, t) and not reached(want - 1, nb, d, t)
    assert starts_of(nb, d, d)[0, t] == want


def test_every_rule(starts_of):
    closest = 1.0
    for nb in range(2, 257):
        e = nb // 2
        s = nb - e
        d = np.arange(e + 1, 2049)
        got = starts_of(nb, e + 1, 2048)
        x = e * (d[:, None].astype(np.longdouble) / e) ** (np.arange(s).astype(np.longdouble)[None] / s)
        n = np.rint(x)
        off = (x - n) / n
        sure = np.abs(off) > 1e-9     # extended precision decides
        assert (got[sure] == np.ceil(x[sure])).all(), nb
        for i, t in zip(*np.nonzero(~sure)):
            k = int(n[i, t])
            want = k if reached(k, nb, int(d[i]), int(t)) else k + 1
            assert got[i, t] == want, (nb, int(d[i]), int(t))
            if want == k + 1:
                closest = min(closest, float(off[i, t]))
    assert closest > 2e-11            # what the rule's slack relies on
