"""Loads into LDS go where M0 says, which they may read one wait state after it was written at the earliest: the compiler sees to that for loads of its own,
loads written by hand have to by themselves.  The listing of the whole built library is gone through.  No GPU is needed."""
import os
import re
import subprocess

import pytest

from paper_2207_10741_amd import binding
from tests.test_kernel_waits import OBJDUMP, _device_code


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    """{kernel's mangled name: its instructions in order}"""
    if not (os.path.exists(OBJDUMP) and os.path.exists(binding.LIB_PATH)):
        pytest.skip("needs the built library and llvm-objdump")
    tmp, found = tmp_path_factory.mktemp("code"), {}
    for i, code in enumerate(_device_code(binding.LIB_PATH)):
        path = str(tmp / ("%d.elf" % i))
        with open(path, "wb") as f:
            f.write(code)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", path], check=True, capture_output=True, text=True).stdout
        for line in text.splitlines():
            if line.startswith("<"):
                at = found.setdefault(line.strip("<>:"), [])
            elif line.startswith("\t"):
                at.append(line.split("//", 1)[0].strip())
    return found


def _is_lds_load(text):
    return text.startswith(("buffer_load", "global_load")) and (text.endswith(" lds") or " lds " in text or "_lds_" in text)


def _writes_m0(text):
    return re.match(r"[sv]_\w+ m0\b", text) is not None


def test_a_wait_state_lies_between_m0_and_the_load(listing):
    loads, early = 0, []
    for name, code in listing.items():
        for before, text in zip(code, code[1:]):
            if _is_lds_load(text):
                loads += 1
                if _writes_m0(before):
                    early.append("%s: `%s`, `%s`" % (name, before, text))
    assert loads > 1000                                     # (the listing is one)
    assert not early, "%d: %s" % (len(early), "\n".join(early[:10]))


def test_every_load_of_the_large_tiles_is_aimed(listing):
    """All instances of the kernel: M0 is set once for each load, and between the two stands a product or the copy of the scalar offset."""
    large = {name: code for name, code in listing.items() if "k_linear_large" in name}
    assert len(large) == 4
    for name, code in large.items():
        loads, aimed = 0, False
        for text in code:
            if _writes_m0(text):
                assert not aimed, "%s: M0 is set twice before a load" % name
                aimed = True
            elif _is_lds_load(text):
                assert aimed, "%s: `%s` goes where another load went" % (name, text)
                aimed, loads = False, loads + 1
            elif aimed:
                assert not text.startswith(("s_cbranch", "s_branch", "s_barrier", "s_endpgm")), "%s: `%s`" % (name, text)
        assert loads >= 24 + 6 + 6 * 16, name
