"""Asking for LDS beyond 64 KB (csrc/lds_allowed.h), compiled with the host compiler over a runtime of counters."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_15207_amd", "csrc")
CODE = r"""
#include "lds_allowed.h"
#include <thread>
static int device;
static std::atomic<int> asked{0};
static hipError_t answer = hipSuccess;
extern "C" hipError_t hipGetDevice(int* d) { *d = device; return hipSuccess; }
extern "C" hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { ++asked; return answer; }
static hift::LdsAllowed one, other;
static int kernel;
extern "C" int ask(int which, int on, int bytes, int fail) {  // how often the runtime was asked; below 0: the call failed
  device = on;
  answer = fail ? hipErrorInvalidValue : hipSuccess;
  asked = 0;
  const hipError_t e = (which ? other : one)(&kernel, bytes);
  return e == hipSuccess ? asked.load() : -1 - asked.load();
}
extern "C" int threads(int n) {
  hift::LdsAllowed fresh;
  device = 0;
  answer = hipSuccess;
  asked = 0;
  std::thread t[16];
  for (int i = 0; i < n; ++i) t[i] = std::thread([&] { for (int k = 0; k < 1000; ++k) fresh(&kernel, 100000); });
  for (int i = 0; i < n; ++i) t[i].join();
  return asked;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("lds")
    src, so = d / "lds.cpp", d / "lds.so"
    src.write_text(CODE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-shared", "-fPIC", "-pthread", "-Wl,-Bsymbolic", "-I", CSRC, "-I", "/opt/rocm/include", str(src), "-o", str(so)],
                   check=True)
    return ctypes.CDLL(str(so))


def test_once_on_each_device(lib):
    assert [lib.ask(0, 0, 100000, 0) for _ in range(3)] == [1, 0, 0]
    assert [lib.ask(0, 3, 100000, 0) for _ in range(2)] == [1, 0]               # another device
    assert lib.ask(0, 0, 100000, 0) == 0
    assert lib.ask(1, 0, 100000, 0) == 1                                        # another kernel
    assert [lib.ask(0, 70, 100000, 0) for _ in range(2)] == [1, 1]              # beyond those that are remembered: every time


def test_a_refusal_is_not_remembered(lib):
    assert lib.ask(1, 5, 100000, 1) == -2
    assert lib.ask(1, 5, 100000, 0) == 1
    assert lib.ask(1, 5, 100000, 1) == 0


def test_threads_at_once(lib):
    assert 1 <= lib.threads(8) <= 8


def test_kernels_are_allowed_through_it():
    """No source keeps a flag of its own for it."""
    for name in sorted(os.listdir(CSRC)):
        if name.endswith(".hip"):
            code = open(os.path.join(CSRC, name)).read()
            assert "static bool" not in code, name
