"""csrc/ops_api.cpp compiled for the host over a stand-in for the HIP runtime and the kernels (tests/host/): what the operators around the
cache refuse and what they launch, without a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = tmp_path_factory.mktemp("ops") / "ops_check"
    src = os.path.join(ROOT, "tests", "host", "ops_check.cpp")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused", "-fsanitize=address,undefined", "-D__HIP_PLATFORM_AMD__",
                    "-I" + os.path.join(ROCM, "include"), src, "-o", str(exe)], check=True)
    return exe


@pytest.mark.parametrize("name", ["rotate_refusals", "rope_freqs", "pack_refusals", "shared_memory", "many_units", "attn_plan", "no_exceptions"])
def test_host_side(program, name):
    r = subprocess.run([str(program), name], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr[-2000:]


@pytest.mark.parametrize("name", ["backward_frequencies", "chunk_rows", "large_launches", "rotation_shared_memory", "far_lists", "rope_parts_ends", "many_chunks", "large_rotations"])
def test_ranges(program, name):
    r = subprocess.run([str(program), name], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok") and not r.stderr, r.stdout + r.stderr[-2000:]
