"""The loads to LDS that are written out, as compiled: their waits do not rest on where the
compiler happens to place them.  Assembly only, no GPU."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2606_02916_amd import build
from tests import helpers


def compiled(src):
    """The gfx950 instructions of each kernel of a source, built as the library is."""
    out = os.path.join(tempfile.mkdtemp(prefix="gglds_"), "k.s")
    subprocess.run([build.HIPCC, *build.FLAGS, "-Wno-align-mismatch", "--cuda-device-only", "-S", src, "-o", out],
                   check=True)
    text, kernels = open(out).read(), {}
    for m in re.finditer(r"^(\w+):\s*; @\w+$(.*?)^\.Lfunc_end", text, re.S | re.M):
        lines = (line.split(";")[0].split("//")[0].strip() for line in m[2].splitlines())
        kernels[m[1]] = [x for x in lines if x and not x.endswith(":") and not x.startswith(".")]
    return kernels


@pytest.fixture(scope="module")
def loads():
    return compiled(os.path.join(helpers.ROOT, "tests", "device", "lds_loads.hip"))


@pytest.mark.parametrize("kernel", ["m0_16", "m0_16_at", "m0_4"])
def test_the_compiler_sets_its_own_place_again(loads, kernel):
    """m0 has the place in LDS: between a load that is written out and the compiler's next one
    it is written again."""
    code = loads[kernel]
    at = [i for i, x in enumerate(code) if x.startswith("global_load_lds")]
    assert len(at) == 3
    for a, b in zip(at, at[1:]):
        assert any(re.search(r"\bm0,", x) for x in code[a + 1:b]), code[a:b + 1]


def test_a_base_from_lanes_is_waited_for(loads):
    """A scalar register that a vector instruction wrote is read by a vector load five wait
    states later at the earliest; no hardware waits for that."""
    code = loads["base_from_lanes"]
    load = next(i for i, x in enumerate(code) if x.startswith("global_load_lds"))
    m = re.search(r"s\[(\d+):(\d+)\]", code[load])
    base, wrote = {f"s{m[1]}", f"s{m[2]}"}, 0
    states = 0
    for x in reversed(code[:load]):
        if x.startswith("v_readfirstlane_b32") and x.split()[1].rstrip(",") in base:
            wrote += 1
            assert states >= 5, code[:load + 1]
        states += int(x.split()[1]) + 1 if x.startswith("s_nop") else 1
    assert wrote == 2


def test_waits_count_no_loads_of_the_compilers():
    """In the weights' gradient loads to LDS are followed by loads that the compiler makes, as
    many as it likes: a wait before a barrier that leaves some under way might leave those to LDS."""
    kernels = compiled(os.path.join(build.CSRC, "product_grad.hip"))
    waits = {name: [re.search(r"vmcnt\((\d+)\)", x)[1] for x, y in zip(code, code[1:])
                    if y == "s_barrier" and x.startswith("s_waitcnt") and "vmcnt" in x]
             for name, code in kernels.items() if any(x.startswith("global_load_lds") for x in code)}
    assert len(waits) == 1 and len(*waits.values()) >= 3
    assert set(*waits.values()) == {"0"}, waits
