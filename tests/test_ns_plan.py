"""Scales and work space of the Newton-Schulz orthogonalisation (csrc/ns_plan.h), compiled with the host compiler."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_15207_amd", "csrc")
CODE = r"""
#include "ns_plan.h"
using namespace hift;
extern "C" int scales(const double* co, double r, float* x, float* a, float* b, double* next) {
  const double c[3] = {co[0], co[1], co[2]};
  NsScales s;
  if (!ns_scales(c, r, &s)) return 0;
  *x = s.x; *a = s.a; *b = s.b; *next = s.r_next;
  return 1;
}
extern "C" int launches(int count, int few, const long long* s, int* out) {  // side, how many, which ...
  int n = 0;
  ns_launches(count, few != 0, [&](int i, int64_t* r, int64_t* c) { *r = s[2 * i]; *c = s[2 * i + 1]; }, [&](const int* which, int k, int side, bool) {
    out[n++] = side;
    out[n++] = k;
    for (int i = 0; i < k; ++i) out[n++] = which[i];
  });
  return n;
}
extern "C" size_t bytes(int count, const long long* s) {
  return ns_workspace_bytes(count, [&](int i, int64_t* r, int64_t* c) { *r = s[2 * i]; *c = s[2 * i + 1]; });
}
extern "C" size_t one(long long r, long long c) { return ns_bytes(r, c); }
extern "C" size_t shared(int side) { return ns_shared_bytes(side); }
extern "C" double span(int n, const long long* count, const double* length) {
  NsTiles runs[16];
  for (int i = 0; i < n; ++i) runs[i] = {(int64_t)count[i], length[i]};
  return ns_span(runs, n);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("ns")
    src, so = d / "ns.cpp", d / "ns.so"
    src.write_text(CODE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.span.restype = ctypes.c_double
    lib.bytes.restype = lib.one.restype = lib.shared.restype = ctypes.c_size_t
    lib.one.argtypes = [ctypes.c_longlong] * 2
    return lib


def scales(lib, co, r):
    c = (ctypes.c_double * 3)(*co)
    x, a, b, n = ctypes.c_float(), ctypes.c_float(), ctypes.c_float(), ctypes.c_double()
    ok = lib.scales(c, ctypes.c_double(r), ctypes.byref(x), ctypes.byref(a), ctypes.byref(b), ctypes.byref(n))
    return (x.value, a.value, b.value, n.value) if ok else None


@pytest.mark.parametrize("co", [(3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (0.0, 0.0, 1.0), (0.0, 1.0, 0.0),
                                (-2.0, 3.0, -1.5), (4.0, 0.0, -2.0)])
def test_scales_keep_every_factor_in_range(plan, co):
    r = 1.001
    for _ in range(8):
        got = scales(plan, co, r)
        if got is None:
            break
        x, a, b, nxt = got
        t = np.linspace(0.0, r, 20001)
        q = np.abs(co[0] + co[1] * t ** 2 + co[2] * t ** 4)
        for scale, most in ((x, r), (a, r * r), (b, q.max())):
            assert scale == 2.0 ** round(np.log2(scale)) and scale * most <= 32768.0 * (1 + 1e-6) and scale * most > 16383.0 * (1 - 1e-6)
        assert nxt >= (t * q).max()
        assert nxt <= max(1e-3, (t * q).max()) * 1.01
        r = nxt


def test_coefficients_that_let_values_grow_are_refused(plan):
    for co, r in (((1e4, 0.0, 0.0), 1.0), ((float("nan"), 0.0, 0.0), 1.0), ((0.0, 0.0, 0.0), 1.0), ((1.0, 1.0, 1.0), 2000.0), ((float("inf"), 0.0, 0.0), 1.0)):
        assert scales(plan, co, r) is None


def test_work_space_and_launches(plan):
    def call(f, shapes, *first):
        return f(*first, len(shapes), (ctypes.c_longlong * (2 * max(len(shapes), 1)))(*[v for s in shapes for v in s]))

    assert call(plan.bytes, []) == 0 and call(plan.bytes, [(0, 5), (5, 0)]) == 0
    assert plan.one(65, 300) == plan.one(300, 65) and plan.one(1, 1) % 16 == 0
    def launches(shapes, few=0):
        out = (ctypes.c_int * (4 * len(shapes) + 8))()
        n, at, got = plan.launches(len(shapes), few, (ctypes.c_longlong * (2 * len(shapes)))(*[v for s in shapes for v in s]), out), 0, []
        while at < n:
            got.append((out[at], list(out[at + 2:at + 2 + out[at + 1]])))
            at += 2 + out[at + 1]
        return got

    # what fits LDS: a workgroup a matrix and no work space, but along with others where there are any
    small = [(8, 8)] * 40
    assert launches(small) == [(0, list(range(0, 16))), (0, list(range(16, 32))), (0, list(range(32, 40)))] and call(plan.bytes, small) == 0
    assert launches([(256, 64), (0, 9), (64, 256), (64, 64), (17, 500)]) == [(0, [0, 2, 3, 4])]
    for too_large in ((64, 300), (96, 100), (128, 128), (17, 800)):
        assert launches([(8, 8), too_large]) == [(64, [1, 0])]
    small[0] = (64, 300)
    assert launches(small) == [(64, list(range(0, 16))), (64, list(range(16, 32))), (64, list(range(32, 40)))]
    assert call(plan.bytes, small) == plan.shared(128) + 15 * plan.one(8, 8) + plan.one(64, 300)
    # tiles of either size apart, the longest first, nothing for a side of 0, and no more than fits together
    mixed = [(64, 64), (4096, 4096), (0, 7), (4096, 11008), (100, 300)]
    assert launches(mixed) == [(256, [3, 1]), (64, [4, 0])] and launches([(64, 64), (600, 900)]) == [(64, [1, 0])]
    # products to a step differ, where large ones are worth launches of their own
    assert launches([(64, 64), (600, 900), (2048, 2048)], 1) == [(256, [2]), (64, [1, 0])] and launches([(600, 900)], 1) == [(128, [0])]
    assert launches([(64, 64), (600, 900), (1024, 2048)], 1) == [(128, [2, 1]), (64, [0])]
    for few in (0, 1):  # every matrix once
        some = [(64, 64), (600, 900), (2048, 2048), (512, 512), (511, 4096), (0, 9), (5000, 1300), (1300, 900)]
        assert sorted(i for _, which in launches(some, few) for i in which) == [0, 1, 2, 3, 4, 6, 7]
    assert call(plan.bytes, mixed) == plan.shared(256) + plan.one(4096, 4096) + plan.one(4096, 11008)
    large = [(16384, 16384), (16384, 16384), (64, 64)]
    assert launches(large) == [(256, [0]), (256, [1]), (64, [2])]
    assert launches([(1024, 1024)] * 6) == [(128, [0, 1, 2, 3, 4, 5])]
    assert call(plan.bytes, large) == plan.shared(256) + plan.one(16384, 16384)


@pytest.mark.parametrize("runs", [[], [(1, 5.0)], [(256, 3.0)], [(257, 3.0)], [(3088, 7.0)], [(408, 11.0), (544, 4.0)], [(1, 100.0), (1000, 1.0)],
                                  [(0, 4.0), (70, 2.5)], [(i + 1, 1.0 + 0.37 * i) for i in range(16)], [(200 + 31 * i, 9.0 - 0.5 * i) for i in range(16)]])
def test_span_is_that_of_a_tile_by_tile_assignment(plan, runs):
    import heapq
    free = [0.0] * 256
    for count, length in sorted(runs, key=lambda r: -r[1]):
        for _ in range(count):
            heapq.heapreplace(free, free[0] + length)
    n = len(runs)
    got = plan.span(n, (ctypes.c_longlong * max(n, 1))(*[c for c, _ in runs]), (ctypes.c_double * max(n, 1))(*[l for _, l in runs]))
    assert got == pytest.approx(max(free), rel=1e-12)
