"""Rotary calls of one context from several host threads (the binding lets go of the interpreter's lock): each gets its own theta's frequencies.
api_cache.cu compiled for the CPU against `packed_threads.cpp`."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2408_15562_b200", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("packed_threads") / "libpackedthreads.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-pthread", "-Wl,-Bsymbolic", "-DatomicCAS(p,a,b)=((void)(p),(void)(a),(void)(b))",
                           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-I/usr/local/cuda/include",
                           "-x", "c++", os.path.join(CSRC, "api_cache.cu"), os.path.join(HERE, "packed_threads.cpp"), "-o", out])
    lib = ctypes.CDLL(out)
    lib.rotary_calls_at_once.restype = ctypes.c_long
    return lib


@pytest.mark.parametrize("threads", [1, 2, 4])
def test_every_thread_gets_its_own_frequencies(lib, threads):
    assert lib.rotary_calls_at_once(threads, 20000) == 0
