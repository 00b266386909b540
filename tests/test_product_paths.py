"""Which kernels products and their gradients go to, on the CPU: the library's own checks, plan and working memory,
with the launches written down."""
import os
import subprocess

import pytest

from tests.test_host_code import CLANGXX, CSRC, INC, ROOT

HIPCC = "/opt/rocm/bin/hipcc"


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not (os.path.exists(CLANGXX) and os.path.exists(HIPCC)):
        pytest.skip("no ROCm compilers")
    at = tmp_path_factory.mktemp("paths")
    obj, exe = str(at / "product_paths.o"), str(at / "product_paths")
    subprocess.check_call([HIPCC, "--offload-host-only", "-O1", "-std=c++17", *INC[2:], "-x", "hip", "-c",
                           os.path.join(ROOT, "tests", "host", "product_paths.cpp"), "-o", obj], stderr=subprocess.DEVNULL)
    subprocess.check_call([CLANGXX, obj, "-Wl,--unresolved-symbols=ignore-all", "-o", exe])       # (no device code)
    return exe


def test_reach_of_loads_and_room(program):
    """Whatever is loaded to LDS directly, copies among it, lies below 2 GiB from where its tile begins, and working
    memory is written within the bytes that the sizes ask for."""
    r = subprocess.run([program, "draw", "300000"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "ALL OK" in r.stdout, r.stderr[:4000]
