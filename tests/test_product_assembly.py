"""What the assembly in the products' kernels relies on, read from the compiler's output (built from source, no GPU)."""
import os
import re
import subprocess

import pytest


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    """The kernels' instructions, line by line, with the compiler's marks around what comes from asm statements."""
    from paper_2603_13606_amd import build
    out = tmp_path_factory.mktemp("asm") / "product.s"
    cmd = [build.HIPCC, *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, "ep_product.hip"), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return [line.strip() for line in out.read_text().splitlines()]


def blocks(listing):
    """Instructions of the asm statements, and those of the compiler."""
    inside, asm, own = None, [], []
    for line in listing:
        if line.startswith(";;#ASMSTART"):
            inside = []
        elif line.startswith(";;#ASMEND"):
            asm.append(inside)
            inside = None
        else:
            code = line.split(";")[0].split("//")[0].strip()
            if code and not code.startswith(".") and not code.endswith(":"):
                (own if inside is None else inside).append(code)
    return asm, own


def test_loads_in_assembly_wait_for_their_descriptor(listing):
    """Five wait states lie between whatever the compiler has put in front, which may be a vector instruction that writes the
    descriptor's registers, and the load that reads them; one between the write of m0 and its use."""
    asm, _ = blocks(listing)
    loads = [b for b in asm if any(i.startswith("buffer_load") for i in b)]
    assert len(loads) > 100
    for b in loads:
        states, since_m0 = 0, None
        for i in b:
            nop = re.match(r"s_nop (\d+)", i)
            n = int(nop[1]) + 1 if nop else 1
            if i.startswith("buffer_load"):
                assert states >= 5 and since_m0 is not None and since_m0 >= 1, b
            states += n
            since_m0 = 0 if re.match(r"s_\w+ m0,", i) else since_m0 + n if since_m0 is not None else None


def test_m0_is_used_by_the_loads_in_assembly_alone(listing):
    _, own = blocks(listing)
    assert len(own) > 10000
    assert [i for i in own if re.search(r"\bm0\b", i) or re.search(r"\blds\b", i)] == []
