"""What the scores' join takes for one of the largest logits has been stored: tests/score_order.cpp walks the kernels' own rules over whole tokens on the
host, with everything that was not stored above all logits."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_set_that_is_read_has_been_stored(tmp_path):
    sys.path.insert(0, os.path.join(ROOT, "paper_2502_11407_amd", "csrc"))
    import build as kernel_build
    exe = str(tmp_path / "score_order")
    r = subprocess.run([kernel_build.HIPCC] + kernel_build.FLAGS + ["-x", "hip", os.path.join(ROOT, "tests", "score_order.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-1000:]
