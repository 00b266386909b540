"""AddressSanitizer + UBSan build of the host code behind the weight update's
and the norm's entry points, linked with stubs for the device passes and run
on the CPU.  Any sanitizer report ends the program with a non-zero status."""
import os
import subprocess

from tests.test_sanitizers import CLANGXX, HERE, HIPCC, ROOT, SAN_ENV, _need


def test_train_host_layer_under_asan_ubsan(tmp_path):
    _need(HIPCC)
    _need(CLANGXX)
    csrc = os.path.join(ROOT, "paper_2006_03318_amd", "csrc")
    inc = ["-I", os.path.join(ROOT, "include"), "-I", csrc]
    objs = []
    for src in ("dd_api", "dd_train"):          # host code only; sanitizers on the host pass
        objs.append(str(tmp_path / (src + ".o")))
        subprocess.check_call([HIPCC, "--offload-host-only", "-O1", "-g", "-std=c++17",
                               "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                               "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"] + inc +
                              ["-c", os.path.join(csrc, src + ".hip"), "-o", objs[-1]],
                              stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    exe = str(tmp_path / "train_host")
    subprocess.check_call([CLANGXX, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include"] + inc +
                          [os.path.join(HERE, "train_host_driver.cpp")] + objs +
                          ["-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-pthread", "-o", exe])
    supp = tmp_path / "lsan.supp"               # allocations the HIP runtime keeps for the process
    supp.write_text("leak:libamdhip64\nleak:libhsa-runtime64\nleak:libhsakmt\nleak:libdrm\n")
    env = dict(SAN_ENV, LSAN_OPTIONS="suppressions=%s" % supp, HIP_VISIBLE_DEVICES="")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ALL OK" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])
