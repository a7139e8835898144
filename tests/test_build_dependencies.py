"""An incremental build compiles every unit again whose text, or that of a file it includes, has changed: what the build takes for a unit's files against
what the compiler reads."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2502_11407_amd", "csrc")
sys.path.insert(0, CSRC)


@pytest.fixture(scope="module")
def kernel_build():
    import build
    assert os.path.dirname(os.path.abspath(build.__file__)) == CSRC
    return build


def units(kernel_build):
    """The host's sources, and a generated unit of every kind."""
    kinds = {}
    for path in kernel_build.generate():
        kinds.setdefault(re.sub(r"_?\d*\.hip$", "", os.path.basename(path)), path)
    assert {"inst", "conv", "chains", "fused", "fusedchains", "lm", "gated"} <= set(kinds)
    return list(kinds.values()) + [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith(".cpp")]


def test_units_depend_on_all_that_they_include(kernel_build):
    for unit in units(kernel_build):
        r = subprocess.run([kernel_build.HIPCC, "--offload-arch=gfx950", "-std=c++17", "-I", CSRC, "--offload-host-only", "-x", "hip", "-MM", unit],
                           capture_output=True, text=True, cwd=CSRC)
        assert r.returncode == 0, r.stderr[-2000:]
        read = r.stdout.split(":", 1)[1].replace("\\\n", " ").split()
        read = {os.path.realpath(os.path.join(CSRC, f)) for f in read}
        assert len(read) > 1, unit
        assert read <= {os.path.realpath(f) for f in kernel_build.dependencies(unit)}, unit


def test_a_changed_header_is_seen(kernel_build, tmp_path):
    """Through other headers, from either folder, and also where two include each other."""
    (tmp_path / "a.cpp").write_text('#include <map>\n  #  include "b.hpp"\nint x;\n')
    (tmp_path / "b.hpp").write_text('#pragma once\n#include "a.hpp"\n#include "gemm_kernel.hpp"\n')
    (tmp_path / "a.hpp").write_text('#include "b.hpp"\n')
    found = {os.path.realpath(f) for f in kernel_build.dependencies(str(tmp_path / "a.cpp"))}
    assert found == {os.path.realpath(p) for p in (tmp_path / "a.cpp", tmp_path / "b.hpp", tmp_path / "a.hpp", os.path.join(CSRC, "gemm_kernel.hpp"))}
    (tmp_path / "a.hpp").write_text('#include "b.hpp"\n#include "more.hpp"\n')
    (tmp_path / "more.hpp").write_text("")
    assert str(tmp_path / "more.hpp") in kernel_build.dependencies(str(tmp_path / "a.cpp"))
    with pytest.raises(FileNotFoundError):
        (tmp_path / "a.cpp").write_text('#include "not there.hpp"\n')
        kernel_build.dependencies(str(tmp_path / "a.cpp"))
