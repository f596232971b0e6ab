"""A C caller of the paged cache (tests/c_abi/cache_after_reset.c) that ends its context and goes on with another one."""
import os
import shutil
import subprocess

import pytest

from tests.test_c_caller import CUDA, ROOT


def _compile(tmp_path):
    from paper_2607_26475_b200 import build
    lib = build.build()
    exe = str(tmp_path / "cache_after_reset")
    cmd = [shutil.which("gcc") or "gcc", "-std=c99", "-Wall", "-Werror", "-O1", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(CUDA, "include"), os.path.join(ROOT, "tests", "c_abi", "cache_after_reset.c"), "-o", exe, lib,
           "-L", os.path.join(CUDA, "lib64"), "-lcudart", "-Wl,-rpath," + os.path.dirname(lib),
           "-Wl,-rpath," + os.path.join(CUDA, "lib64")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe


def test_cache_caller_compiles_and_links(tmp_path):
    assert os.path.exists(_compile(tmp_path))


@pytest.mark.gpu
def test_cache_calls_run_again_after_a_device_reset(tmp_path):
    r = subprocess.run([_compile(tmp_path)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "AFTER RESET OK" in r.stdout
