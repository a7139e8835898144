"""The compiled kernels of the products that are consumed in place, read from the compiler's own output for this repository's sources (device
code only, no GPU needed): hand-written waits of the LDS reads issued from assembly, and registers."""
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


def _assembly(tmp_path, d, kinds):
    src, out = tmp_path / ("f%d.hip" % d["id"]), tmp_path / ("f%d.s" % d["id"])
    body = ['#include "fused_registry.hpp"', "namespace gensor {", "typedef %s C_X;" % lattice.cfg_type(d)]
    body += ["hipError_t l_%s(const FusedArgs& a, hipStream_t st) { return launch_fused<C_X, %s>(a, st); }" % (k, lattice.FUSED_KINDS[k]) for k in kinds]
    src.write_text("\n".join(body + ["}\n"]))
    extra = kernel_build.CONV_FLAGS if lattice.chains(d) > 1 else []
    r = subprocess.run([kernel_build.HIPCC] + kernel_build.FLAGS + extra + ["-x", "hip", "--cuda-device-only", "-S", str(src), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return out.read_text()


def _all(tmp_path, insts, kinds_of):
    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        return list(ex.map(lambda d: (d, _assembly(tmp_path, d, kinds_of(d))), insts))


def test_reads_from_assembly_are_waited_for(tmp_path):
    """Directly staged tiles with a transposed 16-bit operand, whole tiles and groups, one type (the other's code differs in the products only)."""
    insts = [d for d in lattice.fused() if d["direct"] and (d["bsrc"] == "NC" or d["asrc"] == "MC") and d["dt"] == "bf16" and d["out"] == "bf16"]
    assert len(insts) == 8
    for d, text in _all(tmp_path, insts, lambda d: d["kinds"]):
        functions = _functions(text)
        assert len(functions) >= 3
        for f in functions:
            violations, reads = check_function(f)
            assert reads > 0 and not violations, (d["id"], violations[:3])


def test_registers(tmp_path):
    """The 256x256 tiles' two waves per SIMD have 256 registers each.  The logits' reduction, whose workgroups stay, spills a few once a tile, the
    others next to nothing (what is requested early for the epilogue), and none in the loop over k."""
    insts = [d for d in lattice.fused() if lattice.alternate(d) and d["dt"] == "f16"]
    for d, text in _all(tmp_path, insts, lambda d: d["kinds"]):
        names = re.findall(r"\.name:\s+(_ZN6gensor\S+)", text)
        regs = [int(x) for x in re.findall(r"\.vgpr_count:\s+(\d+)", text)]
        spills = [int(x) for x in re.findall(r"\.vgpr_spill_count:\s+(\d+)", text)]
        assert len(names) == len(regs) == len(spills)
        for name, n, spilled in zip(names, regs, spills):
            assert n <= 256 and spilled <= (16 if "FusedILi1E" in name else 4), (name, n, spilled)
