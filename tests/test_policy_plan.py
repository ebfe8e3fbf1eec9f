"""The 4-bit head's choice of tile (csrc/plan.h), compiled with the host compiler, at sizes where either shape was
measured faster. The choice changes no result, so the parity tests cannot see a wrong one."""

import ctypes
import os
import subprocess

import pytest

from plan_shim import FP4_KERNELS, fp4_kernel

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_14220_amd", "csrc")


@pytest.fixture(scope="module")
def small_tiles(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text('#include "plan.h"\nextern "C" bool small_tiles(int64_t T, int64_t V, int64_t cus) '
                                "{ return tim::fp4_small_tiles(T, V, cus); }\n")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o",
                    str(d / "plan.so"), str(d / "shim.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "plan.so"))
    lib.small_tiles.argtypes = [ctypes.c_int64] * 3
    lib.small_tiles.restype = ctypes.c_bool
    return lib.small_tiles


@pytest.mark.parametrize("T,V,small", [
    (333, 50257, True), (200, 50257, False), (256, 50257, False), (512, 50257, False), (200, 32000, True),
    (256, 32000, True), (512, 32000, False), (200, 151936, False), (512, 151936, False), (2000, 151936, False)])
def test_choice(small_tiles, T, V, small):
    assert small_tiles(T, V, 256) == small


def test_without_a_device(small_tiles):
    assert not small_tiles(333, 50257, 0)


@pytest.mark.parametrize("T,d,V,esize,kernel", [
    (1, 384, 151936, 4, "short"), (2000, 256, 151936, 4, "short"), (1, 512, 151936, 4, "rows16"),
    (16, 512, 1, 4, "rows16"), (17, 512, 1, 4, "rows32"), (33, 2048, 151936, 4, "rows64"), (65, 2048, 151936, 4, "rows128"),
    (128, 2048, 151936, 4, "rows128"), (129, 2048, 331, 4, "small"), (333, 1536, 50257, 2, "small"),
    (200, 4096, 50257, 4, "large_once"), (256, 4096, 151936, 4, "large_once"), (257, 4096, 151936, 4, "small"),
    (500, 4096, 32001, 4, "large"), (442, 4096, 151936, 4, "large_past"), (883, 4096, 151936, 2, "large"),
    (884, 4096, 151936, 2, "large_past"), (2000, 4096, 151936, 4, "large_past")])
def test_kernel(T, d, V, esize, kernel):
    assert fp4_kernel(T, d, V, esize) == kernel


def test_every_kernel_is_chosen_somewhere():
    seen = {fp4_kernel(T, d, V, 4) for T in (1, 20, 40, 100, 200, 333, 500, 2000) for d in (256, 1536) for V in (32001, 50257, 151936)}
    assert seen == set(FP4_KERNELS)
