"""csrc/pages_api.cpp compiled for the host over a stand-in for the HIP runtime and the kernels (tests/host/): what the calls over caches in pages
refuse, and that the launches they lay out hold whatever lengths the kernels find, without a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = tmp_path_factory.mktemp("pages") / "pages_check"
    src = os.path.join(ROOT, "tests", "host", "pages_check.cpp")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused", "-fsanitize=address,undefined", "-D__HIP_PLATFORM_AMD__",
                    "-I" + os.path.join(ROCM, "include"), src, "-o", str(exe)], check=True)
    return exe


@pytest.mark.parametrize("name", ["append_refusals", "cache_refusals", "attn_refusals", "plans"])
def test_host_side(program, name):
    r = subprocess.run([str(program), name], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok") and not r.stderr, r.stdout + r.stderr[-2000:]


def test_groups_without_room(program):
    r = subprocess.run([str(program), "dropped_groups"], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok") and not r.stderr, r.stdout + r.stderr[-2000:]
