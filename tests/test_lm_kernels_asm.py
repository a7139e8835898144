"""The compiled kernels of the gated layers and of the scores, read from the compiler's own output for this repository's sources (device code only, no GPU
needed): hand-written waits of the LDS reads issued from assembly, and registers."""
import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_asm_read_contract import CSRC, _functions, check_function  # noqa: E402

sys.path.insert(0, CSRC)
import build as kernel_build  # noqa: E402
import lattice  # noqa: E402


def _assembly(tmp_path, d, ends):
    src, out = tmp_path / ("%s%d.hip" % (ends[0], d["id"])), tmp_path / ("%s%d.s" % (ends[0], d["id"]))
    body = ['#include "lm_registry.hpp"', "namespace gensor {", "typedef %s C_X;" % lattice.cfg_type(d)]
    body += ["hipError_t l_%s(const %s& a, hipStream_t st) { return launch_end<C_X, %s>(a, st); }" % ((k,) + kernel_build.LM_ENDS[k]) for k in ends]
    src.write_text("\n".join(body + ["}\n"]))
    extra = kernel_build.CONV_FLAGS if lattice.chains(d) > 1 else []
    r = subprocess.run([kernel_build.HIPCC] + kernel_build.FLAGS + extra + ["-x", "hip", "--cuda-device-only", "-S", str(src), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return out.read_text()


def _all(tmp_path, jobs):
    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        return list(ex.map(lambda job: (job[0], _assembly(tmp_path, *job)), jobs))


def test_reads_from_assembly_are_waited_for(tmp_path):
    """Directly staged tiles with row-major weights, one type (the other's code differs in the products only)."""
    picked = lambda L: [d for d in L if d["direct"] and d["bsrc"] == "NC" and d["asrc"] == "KC" and d["dt"] == "bf16" and d["out"] == "bf16"]
    jobs = [(d, ["gated"]) for d in picked(lattice.gated())] + [(d, ["gated_grad"]) for d in picked(lattice.fused())]
    assert len(jobs) == 3 + 4
    for d, text in _all(tmp_path, jobs):
        functions = _functions(text)
        assert len(functions) == 1
        for f in functions:
            violations, reads = check_function(f)
            assert reads > 0 and not violations, (d["id"], violations[:3])


def test_registers(tmp_path):
    """The 256x256 tiles' two waves per SIMD have 256 registers each.  The scores' reduction, whose workgroups stay, spills a few once a tile, the others next
    to nothing, and none in the loop over k."""
    jobs = [(d, ["gated"]) for d in lattice.gated() if lattice.alternate(d) and d["dt"] == "f16"]
    jobs += [(d, lattice.lm_ends(d)) for d in lattice.fused() if lattice.alternate(d) and d["dt"] == "f16" and lattice.lm_ends(d)]
    for d, text in _all(tmp_path, jobs):
        names = re.findall(r"\.name:\s+(_ZN6gensor\S+)", text)
        regs = [int(x) for x in re.findall(r"\.vgpr_count:\s+(\d+)", text)]
        spills = [int(x) for x in re.findall(r"\.vgpr_spill_count:\s+(\d+)", text)]
        assert len(names) == len(regs) == len(spills) > 0
        for name, n, spilled in zip(names, regs, spills):
            assert n <= 256 and spilled <= (32 if "5Score" in name else 4), (name, n, spilled)
