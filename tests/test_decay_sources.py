"""What the sources of decayed linear attention and draft verification promise, and what the assembler reports for them (no GPU)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_30386_b200 import build

SOURCES = ["decay_chunked.cu", "decay_seq.cu", "verify_draft.cu"]


def _code(name):
    text = open(os.path.join(build.CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


@pytest.mark.parametrize("name", [*SOURCES, "decay_common.cuh"])
def test_nothing_is_read_past_what_an_earlier_kernel_may_still_be_writing(name):
    code = _code(name)
    assert not re.search(r"\.nc\b|__ldg|__restrict__", code)
    if name in SOURCES:  # every kernel waits for the stream, or says that it reads nothing before it has
        assert len(re.findall(r"__global__", code)) <= len(re.findall(r"stream_order_(?:wait|begin)\(\)", code))


@pytest.mark.skipif(not (shutil.which("nvcc") or os.path.exists(build._nvcc())), reason="no nvcc")
def test_the_chunked_kernel_keeps_everything_in_registers(tmp_path):
    out = subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-Xptxas=-v", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                          "-c", os.path.join(build.CSRC, "decay_chunked.cu"), "-o", str(tmp_path / "decay_chunked.o")],
                         capture_output=True, text=True, check=True).stderr
    found = re.findall(r"(\d+) bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads", out)
    assert len(found) == len(re.findall(r"Compiling entry function", out)) > 0
    assert [f for f in found if f != ("0", "0", "0")] == []
