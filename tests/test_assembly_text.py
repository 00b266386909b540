"""Assembly text in the kernels' sources, into which the compiler does not look: what it overwrites is
named, and it waits by itself for what the hardware does not."""
import glob
import os
import re

import pytest

from tests.test_host_code import CSRC


def blocks():
    """(file, instructions, what is named as overwritten) of every asm statement."""
    out = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            src = re.sub(r"//.*", "", f.read())
        for m in re.finditer(r"asm volatile\((.*?)\);", src, re.S):
            parts = re.split(r":(?=(?:[^\"]*\"[^\"]*\")*[^\"]*$)", m[1])
            text = "".join(re.findall(r'"([^"]*)"', parts[0]))
            out.append((os.path.basename(path), [i.strip() for i in text.replace("\\t", "").split("\\n") if i.strip()],
                        parts[3] if len(parts) > 3 else ""))
    return out


def test_there_are_some():
    assert sum("lds" in i for _, text, _ in blocks() for i in text) >= 1


@pytest.mark.parametrize("file,text,clobbers", blocks())
def test_registers_that_the_text_writes_are_named(file, text, clobbers):
    for i in text:
        if re.match(r"s_\w+ m0\b", i):
            assert '"m0"' in clobbers, (file, i)


@pytest.mark.parametrize("file,text,clobbers", blocks())
def test_loads_wait_for_their_scalar_operands(file, text, clobbers):
    """Five wait states between a vector instruction that writes a scalar register, which may be the one before
    the text, and the load that reads it; one between m0 and a load to LDS."""
    states, since_m0 = 0, None
    for i in text:
        if i.startswith("buffer_load"):
            assert states >= 5, (file, i)
            if i.endswith("lds"):
                assert since_m0 is not None and since_m0 >= 1, (file, i)
        n = re.match(r"s_nop (\d+)", i)
        wait = int(n[1]) + 1 if n else 1
        states += wait
        since_m0 = 0 if re.match(r"s_\w+ m0\b", i) else None if since_m0 is None else since_m0 + wait
