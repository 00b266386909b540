"""Which kernels products and their gradients go to, on the CPU: the library's own checks, plan and working memory,
with the launches written down."""
import os
import random
import subprocess

import pytest

from tests.product_cases import CASES
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
    memory is written within the bytes that the sizes ask for.  A gradient wanted alone has the tiles and parts that it
    has beside the other where operands load directly."""
    r = subprocess.run([program, "draw", "300000"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "ALL OK" in r.stdout, r.stderr[:4000]


def ask(program, calls):
    """(status, bytes written, bytes needed, bytes by sizes, what was launched) of each call."""
    r = subprocess.run([program], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[:4000]
    lines = [line.split(" ", 4) for line in r.stdout.splitlines()]
    assert len(lines) == len(calls)
    return [(*map(int, line[:4]), line[4].split(": ", 1)[1] if ": " in line[4] else "") for line in lines]


@pytest.mark.parametrize("rows,k,n", [(65536, 4096, 50257), (16384, 2048, 50257), (8192, 1024, 1024), (4096, 1000, 1003)])
def test_gradients_ask_for_no_more_than_they_use(program, rows, k, n):
    """Copies that the two products share take the place of their own: of all strides and layouts one uses what the
    sizes ask for, and that is little more than the operands."""
    got = ask(program, [("grad", rows, k, n, pad, turned, 0, 7) for pad in (0, 1, 3, 8) for turned in (0, 1)])
    asked = {g[3] for g in got}
    assert len(asked) == 1 and max(g[1] for g in got) >= 0.95 * asked.pop()
    assert got[0][3] <= 1.1 * 2 * (rows * n + rows * k + k * n)


def test_calls_need_what_they_write(program):
    """By their strides and addresses: aligned ones no copies, the others no more than they make."""
    calls = [(op, rows, k, n, pad, turned, 0, 7) for op in ("fwd", "grad") for rows, k, n in ((65536, 4096, 50257), (8192, 1024, 1024), (4096, 1000, 1003), (300, 2000, 520))
             for pad in (0, 1, 8) for turned in (0, 1)]
    for c, (status, written, need, by_sizes, _) in zip(calls, ask(program, calls)):
        assert status == 0 and written <= need <= min(1.01 * written + 16, by_sizes), c


def test_every_path_has_a_case(program):
    """The cases that a GPU runs go where their list says, and no drawn call finds a path that none of them takes."""
    got = ask(program, [(*c[:6], 0, 7) for c in CASES])
    assert [g[0] for g in got] == [0] * len(CASES)
    assert [(c[:6], g[4]) for c, g in zip(CASES, got)] == [(c[:6], c[6]) for c in CASES]
    taken = {(part, c[5]) for c in CASES for part in c[6].split()}
    rng = random.Random(5)

    def size(most):
        n = int(2 ** rng.uniform(0, most))
        return n if rng.random() < 0.5 else (n + 7) // 8 * 8
    calls = [(rng.choice(("fwd", "grad")), size(16), size(14), size(14), rng.choice((0, 0, 0, 8, 1, 3)), rng.randint(0, 1), rng.randint(0, 1), 7)
             for _ in range(100000)]
    new = {(part, c[5]): c for c, g in zip(calls, ask(program, calls)) if g[0] == 0 for part in g[4].split() if (part, c[5]) not in taken}
    assert not new, new
