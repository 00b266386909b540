"""Streams of the calls on a list of tensors: who waits for whom, on the CPU."""
import os
import subprocess

import pytest

from tests.test_host_code import CLANGXX, CSRC, INC, ROOT, _run


def test_order_of_calls(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc"
    if not (os.path.exists(CLANGXX) and os.path.exists(hipcc)):
        pytest.skip("no ROCm compilers")
    objs = [str(tmp_path / (src + ".o")) for src in ("dd_api", "dd_train")]
    for src, obj in zip(("dd_api", "dd_train"), objs):
        subprocess.check_call([hipcc, "--offload-host-only", "-O1", "-std=c++17", *INC[2:], "-c",
                               os.path.join(CSRC, src + ".hip"), "-o", obj], stderr=subprocess.DEVNULL)
    exe = str(tmp_path / "train_streams")
    subprocess.check_call([CLANGXX, "-O1", "-std=c++17", *INC, os.path.join(ROOT, "tests", "host", "train_streams.cpp"),
                           *objs, "-pthread", "-Wl,--unresolved-symbols=ignore-all", "-o", exe])   # (no device code)
    _run(exe)
