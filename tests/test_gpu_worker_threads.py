"""Two host threads that call the worker's operators at the same time with different sizes: no call may fail for what the
other one asked for.  The threads are native, so that nothing makes them take turns."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2010_04902_b200 import binding as bz

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <atomic>
#include <thread>
#include "bz.h"
struct Bias { const void* scores; const float* table; int distance; const float* stats; const void* dprobs; void* dscores; float* dtable; void* ws; size_t bytes; void* stream; };
struct Distill { const void* logits; const float* teacher; const int32_t* index; int t; float* loss; float* stats; void* stream; };
template <typename F> static int both(int n, F call) {
    std::atomic<int> failed{0}, ready{0};
    auto run = [&](int which) {
        for (++ready; ready < 2;) {}
        for (int i = 0; i < n; ++i) failed += call(which) != BZ_OK;
    };
    std::thread a(run, 0), b(run, 1);
    a.join(), b.join();
    return failed;
}
extern "C" int bias_twice(const Bias* p, int n, int64_t heads, int64_t tq, int64_t tk, int buckets) {
    const int64_t strides[3] = {heads * tq * tk, tq * tk, tk};
    return both(n, [&](int k) {
        const Bias& c = p[k];
        return bz_bias_softmax_backward(c.scores, strides, BZ_BF16, 1, heads, tq, tk, c.table, buckets, c.distance, 1, 0, 1.f, nullptr, nullptr, c.stats,
                                        c.dprobs, strides, c.dscores, strides, c.dtable, c.ws, c.bytes, c.stream);
    });
}
extern "C" int glu_twice(const void* x, const void* w, void* h0, void* h1) {
    return both(1, [&](int k) { return bz_glu(x, 64, w, w, 64, 64, 32, 64, BZ_BF16, BZ_ACT_SILU, k ? h1 : h0, 32, nullptr, nullptr, 0, nullptr); });
}
extern "C" int glu_in_a_new_thread(const void* x, const void* w, void* h) {
    int st = 1;
    std::thread([&] { st = bz_glu(x, 64, w, w, 64, 64, 32, 64, BZ_BF16, BZ_ACT_SILU, h, 32, nullptr, nullptr, 0, nullptr); }).join();
    return st;
}
extern "C" int distill_twice(const Distill* p, int n, int64_t m, int64_t v) {
    return both(n, [&](int k) {
        const Distill& c = p[k];
        return bz_distill(c.logits, v, BZ_BF16, m, v, c.teacher, c.index, c.t, 1.f, nullptr, c.loss, c.stats, nullptr, 0, c.stream);
    });
}
"""
FIRST = r"""
import ctypes, sys
import torch
from paper_2010_04902_b200 import binding as bz
bz.lib()
x, w = torch.ones(64, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(32, 64, dtype=torch.bfloat16, device="cuda")
h = torch.zeros(2, 64, 32, dtype=torch.bfloat16, device="cuda")
torch.cuda.synchronize()
P = ctypes.c_void_p
failed = ctypes.CDLL(sys.argv[1]).glu_twice(P(x.data_ptr()), P(w.data_ptr()), P(h[0].data_ptr()), P(h[1].data_ptr()))
torch.cuda.synchronize()
print("failed", failed, "same", torch.equal(h[0], h[1]))
"""
P, I, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t


class Bias(ctypes.Structure):
    _fields_ = [("scores", P), ("table", P), ("distance", I), ("stats", P), ("dprobs", P), ("dscores", P), ("dtable", P), ("ws", P), ("bytes", SZ), ("stream", P)]


class Distill(ctypes.Structure):
    _fields_ = [("logits", P), ("teacher", P), ("index", P), ("t", I), ("loss", P), ("stats", P), ("stream", P)]


@pytest.fixture(scope="module")
def threads(tmp_path_factory):
    bz.lib()
    where = tmp_path_factory.mktemp("threads")
    source, out = os.path.join(where, "threads.cpp"), os.path.join(where, "threads.so")
    with open(source, "w") as fh:
        fh.write(SOURCE)
    pkg = os.path.join(ROOT, "paper_2010_04902_b200")
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-pthread", "-I", os.path.join(ROOT, "include"), "-o", out, source,
                    "-L", pkg, "-l:libbz.so", "-Wl,-rpath," + pkg], check=True)
    return ctypes.CDLL(out)


def test_windows_of_different_size(threads):
    h, tq, tk = 2, 1, 256
    table = torch.randn(32, h, device="cuda")
    calls, held, want = (Bias * 2)(), [], []
    for k, distance in enumerate((336, 200)):
        scores, dprobs = torch.randn(1, h, tq, tk, device="cuda").to(torch.bfloat16), torch.randn(1, h, tq, tk, device="cuda").to(torch.bfloat16)
        _, stats = bz.bias_softmax(scores, table, distance)
        want.append(bz.bias_softmax_backward(scores, table, stats, dprobs, distance))
        ds, dt = torch.zeros_like(scores), torch.zeros_like(table)
        ws = torch.empty(bz.lib().bz_bias_softmax_workspace_bytes(1, h, tq, tk, 32), dtype=torch.uint8, device="cuda")
        s = torch.cuda.Stream()
        held.append((scores, dprobs, stats, ds, dt, ws, s))
        calls[k] = Bias(scores.data_ptr(), table.data_ptr(), distance, stats.data_ptr(), dprobs.data_ptr(), ds.data_ptr(), dt.data_ptr(), ws.data_ptr(),
                        ws.numel(), s.cuda_stream)
    torch.cuda.synchronize()
    assert threads.bias_twice(calls, 10000, ctypes.c_int64(h), ctypes.c_int64(tq), ctypes.c_int64(tk), 32) == 0
    torch.cuda.synchronize()
    for (_, _, _, ds, dt, _, _), (ds0, dt0) in zip(held, want):
        assert torch.equal(ds, ds0) and torch.equal(dt, dt0)


def test_teachers_of_different_size(threads):
    m, v = 160, 9000
    calls, held, want = (Distill * 2)(), [], []
    for k, t in enumerate((1000, 1)):
        logits, teacher = torch.randn(m, v, device="cuda").to(torch.bfloat16), torch.randn(m, t, device="cuda")
        index = torch.randint(0, v, (m, t), dtype=torch.int32, device="cuda")
        want.append(bz.distill(logits, teacher, index))
        loss, stats, s = torch.zeros(m, device="cuda"), torch.zeros(m, 2, device="cuda"), torch.cuda.Stream()
        held.append((logits, teacher, index, loss, stats, s))
        calls[k] = Distill(logits.data_ptr(), teacher.data_ptr(), index.data_ptr(), t, loss.data_ptr(), stats.data_ptr(), s.cuda_stream)
    torch.cuda.synchronize()
    assert threads.distill_twice(calls, 10000, ctypes.c_int64(m), ctypes.c_int64(v)) == 0
    torch.cuda.synchronize()
    for (_, _, _, loss, stats, _), (loss0, stats0) in zip(held, want):
        assert torch.equal(loss, loss0) and torch.equal(stats, stats0)


def test_first_call_of_a_thread(threads):
    """Nothing has made the device's context current in a new thread before the call."""
    x, w = torch.randn(64, 64, device="cuda").to(torch.bfloat16), torch.randn(32, 64, device="cuda").to(torch.bfloat16)
    want, h = bz.glu(x, w, w), torch.zeros(64, 32, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    assert threads.glu_in_a_new_thread(P(x.data_ptr()), P(w.data_ptr()), P(h.data_ptr())) == bz.OK
    torch.cuda.synchronize()
    assert torch.equal(h, want)


def test_first_calls_of_a_process(threads):
    """Both threads need the driver's tensor-map encoder, which nobody has looked up yet."""
    for _ in range(5):
        r = subprocess.run([sys.executable, "-c", FIRST, threads._name], cwd=ROOT, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-2000:]
        assert r.stdout.strip() == "failed 0 same True"
