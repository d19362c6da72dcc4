"""Loads into LDS that the kernels of the matrix product write by hand, in the assembly built for gfx950: every one of them goes where M0 was set for it, and no fragment
is read between a barrier's wait and the barrier.  No GPU is needed."""
import os
import re
import subprocess

import pytest

from paper_2207_10741_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CSRC = os.path.join(os.path.dirname(build.__file__), "csrc")


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    """{kernel's mangled name: its instructions and labels in order}"""
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path_factory.mktemp("asm") / "large.s")
    subprocess.run([HIPCC, *build.HIPCC_FLAGS, "-w", "-I", os.path.join(build.ROOT, "include"), "-I", CSRC, "-DFC_LARGE_PART=0", "--cuda-device-only", "-S",
                    os.path.join(CSRC, "fc_linear_large.hip"), "-o", out], check=True, stderr=subprocess.DEVNULL)
    found, name = {}, None
    for line in open(out):
        start = re.match(r"(_Z\w+):", line)
        text = line.split(";", 1)[0].strip()
        if start:
            name = start.group(1)
            found[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name and text and (text.endswith(":") or not text.startswith(".")):
            found[name].append(text)
    return {n: c for n, c in found.items() if "k_linear_large" in n}


def test_every_load_into_lds_is_aimed(code):
    """M0 holds where a load goes; it is set once for each, by the code that writes the load, and by nobody else."""
    assert len(code) == 1
    for name, lines in code.items():
        loads, aimed = 0, False
        for text in lines:
            if text.endswith(":"):
                assert not aimed, name                  # (no place control comes to lies between the two)
            elif re.match(r"s_mov_b32 m0,", text):
                assert not aimed, "%s: M0 is set twice before a load" % name
                aimed = True
            elif text.startswith("buffer_load") and text.endswith(" lds"):
                assert aimed, "%s: `%s` goes where another load went" % (name, text)
                aimed = False
                loads += 1
            else:
                assert not re.search(r"\bm0\b", text), "%s: `%s`" % (name, text)
        # rows of x for two stages, of w for one, six pieces behind the first barrier or seven; then sixteen a stage
        assert loads >= 24 + 6 + 6 * 16, name


def test_fragments_are_read_behind_the_barrier(code):
    """A stage's barrier follows the wait for its loads with no read of LDS between: what is read behind it is everyone's."""
    for name, lines in code.items():
        inside = [i for i, text in enumerate(lines) if text == "s_barrier"]
        assert len(inside) >= 8, name
        for i in inside[:-1]:
            before = lines[max(i - 12, 0):i]
            waits = [j for j, text in enumerate(before) if text.startswith("s_waitcnt") and "vmcnt" in text]
            assert waits, name
            assert not any(text.startswith("ds_read") or text.startswith("buffer_load") for text in before[waits[-1]:]), name
