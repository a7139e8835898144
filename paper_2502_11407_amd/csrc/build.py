"""Build libgensor.so for gfx950: one translation unit per group of kernel instances
(generated from lattice.py), the registry table, the constructor and the C ABI."""
import functools
import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.dirname(HERE)
GEN = os.path.join(HERE, "_build")
LIB = os.path.join(PKG, "libgensor.so")
PROBE_LIB = os.path.join(PKG, "libgensor_probe.so")     # the benchmark's MFMA-only probe, a library of its own
sys.path.insert(0, HERE)
import lattice  # noqa: E402

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-I", HERE,
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument"]
# patch-staged convolutions and tiles of several sums per output: accumulators stay in plain VGPRs (no copies to and from
# AGPRs around the tap loop, or in every k tile)
CONV_FLAGS = ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]
PER_TU = 4


def _write_if_changed(path, text):
    if os.path.exists(path) and open(path).read() == text:
        return
    with open(path, "w") as f:
        f.write(text)


def generate():
    os.makedirs(GEN, exist_ok=True)
    L = lattice.lattice()
    tus = []
    # translation units hold instances of one kernel template only (they are built with different flags)
    conv = [d for d in L if d["units"] or lattice.conv_rows(d)]
    small = [d for d in L if lattice.chains(d) > 1]
    ordered = [d for d in L if not (d["units"] or lattice.conv_rows(d) or lattice.chains(d) > 1)]
    ordered += [None] * (-len(ordered) % PER_TU) + small
    ordered += [None] * (-len(ordered) % PER_TU) + conv
    for t in range(0, len(ordered), PER_TU):
        group = [d for d in ordered[t:t + PER_TU] if d is not None]
        src = ['#include "registry.hpp"', "namespace gensor {"]
        for d in group:
            src.append("typedef %s C_%d;" % (lattice.cfg_type(d), d["id"]))
            launcher = "launch_conv_instance" if d["units"] else "launch_conv_rows" if lattice.conv_rows(d) else "launch_instance"
            src.append("hipError_t launch_%d(const KernelArgs& a, hipStream_t st) { return %s<C_%d>(a, st); }" % (d["id"], launcher, d["id"]))
            if lattice.splittable(d):
                src.append("hipError_t launch_split_%d(const KernelArgs& a, hipStream_t st) { return launch_instance<C_%d, true>(a, st); }"
                           % (d["id"], d["id"]))
        src.append("}  // namespace gensor\n")
        kind = "conv" if group[0]["units"] or lattice.conv_rows(group[0]) else "chains" if lattice.chains(group[0]) > 1 else "inst"
        path = os.path.join(GEN, "%s_%03d.hip" % (kind, t // PER_TU))
        _write_if_changed(path, "\n".join(src))
        tus.append(path)
    tus += generate_fused()
    tus += generate_lm()
    for f in os.listdir(GEN):                      # units of an earlier lattice
        if f.endswith(".hip") and os.path.join(GEN, f) not in tus and f not in ("registry.hip", "fused_registry.hip", "lm_registry.hip"):
            os.remove(os.path.join(GEN, f))
            if os.path.exists(os.path.join(GEN, f[:-4] + ".o")):
                os.remove(os.path.join(GEN, f[:-4] + ".o"))
    reg = ['#include "registry.hpp"', "#if !defined(__HIP_DEVICE_COMPILE__)", "namespace gensor {"]
    for d in L:
        reg.append("hipError_t launch_%d(const KernelArgs&, hipStream_t);" % d["id"])
        if lattice.splittable(d):
            reg.append("hipError_t launch_split_%d(const KernelArgs&, hipStream_t);" % d["id"])
    reg.append("const InstanceDesc g_instances[] = {")
    reg += ["  {%s, launch_%d, %s}," % (instance_fields(d), d["id"], ("launch_split_%d" % d["id"]) if lattice.splittable(d) else "nullptr") for d in L]
    reg.append("};")
    reg.append("const int g_num_instances = %d;" % len(L))
    reg.append("}  // namespace gensor")
    reg.append("#endif\n")
    path = os.path.join(GEN, "registry.hip")
    _write_if_changed(path, "\n".join(reg))
    tus.append(path)
    return tus


def instance_fields(d):
    """The members of an InstanceDesc in front of its launches."""
    es = 4 if d["dt"] == "f32" else 2
    kg = (64 // d["mb"]) * (16 // es)
    a_bytes = d["bm"] * d["bk"] * es if d["asrc"] == "KC" else d["bk"] * (d["bm"] * es + (0 if d["direct"] else lattice.pad_m(d)))
    b_bytes = d["bn"] * d["bk"] * es if (d["bsrc"] == "KC" or d["direct"]) else d["bk"] * (d["bn"] * es + lattice.pad_n(d))
    lds = 0 if d["units"] or lattice.conv_rows(d) else (a_bytes + b_bytes) * d["stages"] + (b_bytes if lattice.alternate(d) else 0)
    threads = (d["bm"] // d["wm"]) * (d["bn"] // d["wn"]) * 64
    return ", ".join(str(x) for x in (
        d["id"], lattice.DT[d["dt"]], lattice.DT[d["out"]], d["bm"], d["bn"], d["bk"], d["wm"], d["wn"], d["mb"],
        d["vm"], d["vn"], lattice.BSRC[d["bsrc"]], lattice.ASRC[d["asrc"]], d["vec"], d["stages"], d["direct"], lds, threads, kg, d["units"]))


def generate_fused():
    """Units and table of the products that are consumed in place."""
    L = lattice.fused()
    tus = []
    # (a unit holds tiles built with the same flags)
    chains = [d for d in L if lattice.chains(d) > 1]
    for kind, group in (("fused", [d for d in L if lattice.chains(d) == 1]), ("fusedchains", chains)):
        for d in group:
            src = ['#include "fused_registry.hpp"', "namespace gensor {", "typedef %s C_%d;" % (lattice.cfg_type(d), d["id"])]
            src += ["hipError_t fused_%d_%s(const FusedArgs& a, hipStream_t st) { return launch_fused<C_%d, %s>(a, st); }"
                    % (d["id"], k, d["id"], lattice.FUSED_KINDS[k]) for k in d["kinds"]]
            src.append("}  // namespace gensor\n")
            path = os.path.join(GEN, "%s_%03d.hip" % (kind, d["id"]))
            _write_if_changed(path, "\n".join(src))
            tus.append(path)
    reg = ['#include "fused_registry.hpp"', "#if !defined(__HIP_DEVICE_COMPILE__)", "namespace gensor {"]
    reg += ["hipError_t fused_%d_%s(const FusedArgs&, hipStream_t);" % (d["id"], k) for d in L for k in d["kinds"]]
    reg.append("const FusedDesc g_fused[] = {")
    reg += ["  {{%s, nullptr, nullptr}, {%s}}," % (instance_fields(d), ", ".join(
        "fused_%d_%s" % (d["id"], k) if k in d["kinds"] else "nullptr" for k in lattice.FUSED_KINDS)) for d in L]
    reg += ["};", "const int g_num_fused = %d;" % len(L), "}  // namespace gensor", "#endif\n"]
    path = os.path.join(GEN, "fused_registry.hip")
    _write_if_changed(path, "\n".join(reg))
    return tus + [path]


LM_ENDS = {"score": ("ScoreArgs", "Score"), "teach": ("FusedArgs", "Teach"), "gated_grad": ("GatedArgs", "GatedGrad"), "gated": ("GatedArgs", "Gated")}


def generate_lm():
    """Units and tables of the ends of lm_kernel.hpp: those of the tiles above, and the tiles of two products at once."""
    units, reg = [], ['#include "lm_registry.hpp"', "#if !defined(__HIP_DEVICE_COMPILE__)", "namespace gensor {"]
    fused, gated = lattice.fused(), lattice.gated()
    for name, group in (("lm", fused), ("gated", gated)):
        for d in group:
            ends = ["gated"] if name == "gated" else lattice.lm_ends(d)
            if not ends:
                continue
            src = ['#include "lm_registry.hpp"', "namespace gensor {", "typedef %s C_%d;" % (lattice.cfg_type(d), d["id"])]
            for k in ends:
                src.append("hipError_t %s_%d_%s(const %s& a, hipStream_t st) { return launch_end<C_%d, %s>(a, st); }" % (name, d["id"], k, LM_ENDS[k][0], d["id"], LM_ENDS[k][1]))
                reg.append("hipError_t %s_%d_%s(const %s&, hipStream_t);" % (name, d["id"], k, LM_ENDS[k][0]))
            path = os.path.join(GEN, "%s%s_%03d.hip" % (name, "chains" if lattice.chains(d) > 1 else "", d["id"]))
            _write_if_changed(path, "\n".join(src + ["}  // namespace gensor\n"]))
            units.append(path)
    reg.append("const LmEnds g_lm_ends[] = {")
    reg += ["  {%s}," % ", ".join("lm_%d_%s" % (d["id"], k) if k in lattice.lm_ends(d) else "nullptr" for k in ("score", "teach", "gated_grad")) for d in fused]
    reg += ["};", "const GatedDesc g_gated[] = {"]
    reg += ["  {{%s, nullptr, nullptr}, gated_%d_gated}," % (instance_fields(d), d["id"]) for d in gated]
    reg += ["};", "const int g_num_gated = %d;" % len(gated), "}  // namespace gensor", "#endif\n"]
    path = os.path.join(GEN, "lm_registry.hip")
    _write_if_changed(path, "\n".join(reg))
    return units + [path]


@functools.lru_cache(maxsize=None)
def _included(path, modified):
    with open(path) as f:
        return re.findall(r'^\s*#\s*include\s+"([^"]+)"', f.read(), re.M)


def dependencies(src):
    """The unit and every file of this repository that it includes, by itself or through others."""
    found, todo = [], [os.path.abspath(src)]
    while todo:
        path = todo.pop()
        if path in found:
            continue
        found.append(path)
        for name in _included(path, os.stat(path).st_mtime_ns):
            near = os.path.normpath(os.path.join(os.path.dirname(path), name))
            todo.append(near if os.path.exists(near) else os.path.join(HERE, name))
    return found


def _compile(src):
    obj = os.path.join(GEN, os.path.basename(src).rsplit(".", 1)[0] + ".o")
    if os.path.exists(obj) and all(os.path.getmtime(obj) >= os.path.getmtime(d) for d in dependencies(src)):
        return obj
    # host sources: no fused multiply-add contraction, so the constructor's double arithmetic
    # is the plain IEEE sequence its tests compare against
    extra = ["-ffp-contract=off"] if src.endswith(".cpp") else []
    if os.path.basename(src).startswith(("conv_", "chains_", "fusedchains_", "lmchains_", "gatedchains_")):
        extra += CONV_FLAGS
    cmd = [HIPCC] + FLAGS + extra + ["-x", "hip", "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed on %s:\n%s" % (src, err))
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(force=False, jobs=None):
    tus = generate()
    tus += [os.path.join(HERE, "gensor_api.cpp"), os.path.join(HERE, "constructor.cpp"), os.path.join(HERE, "scan_kernels.cpp"),
            os.path.join(HERE, "gensor_fused.cpp"), os.path.join(HERE, "gensor_lm.cpp")]
    probe = os.path.join(HERE, "probe.cpp")
    if force:
        for f in os.listdir(GEN):
            if f.endswith(".o"):
                os.remove(os.path.join(GEN, f))
    jobs = jobs or min(8, os.cpu_count() or 1)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, tus + [probe]))
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs[:-1], check=True)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", PROBE_LIB, objs[-1]], check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
