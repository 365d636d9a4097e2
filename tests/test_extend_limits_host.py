"""The ABI's limits of a call and the sizes of the arrays that its kernels take are one number: a build in which they differ
does not compile."""
import os
import subprocess

import pytest

from paper_2609_30884_gb300 import build

HEADER = os.path.join(build.INCLUDE, "crf.h")


@pytest.mark.parametrize("name,value", [("CRF_MAX_CHUNKS", 128), ("CRF_MAX_TABLES", 512)])
def test_a_raised_limit_does_not_compile_alone(tmp_path, name, value):
    try:
        nvcc = build.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    text = open(HEADER).read()
    line = f"#define {name} {value}"
    assert text.count(line) == 1
    # the sources find the header two folders up
    csrc = tmp_path / "pkg" / "csrc"
    (tmp_path / "include").mkdir()
    csrc.mkdir(parents=True)
    for f in os.listdir(build.CSRC):
        if f.endswith((".h", ".cuh")) or f == "api_extend.cu":
            (csrc / f).write_text(open(os.path.join(build.CSRC, f)).read())

    def compiles(header):
        (tmp_path / "include" / "crf.h").write_text(header)
        cmd = [nvcc, *build.ARCH, "-std=c++17", "--expt-relaxed-constexpr", "-c", str(csrc / "api_extend.cu"), "-o", str(tmp_path / "a.o")]
        return subprocess.run(cmd, capture_output=True, text=True)

    assert compiles(text).returncode == 0
    r = compiles(text.replace(line, f"#define {name} {value + 1}"))
    assert r.returncode != 0 and "limits of the ABI" in r.stderr
