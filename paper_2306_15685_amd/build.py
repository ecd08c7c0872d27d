"""Builds the HIP library in-tree for gfx950 (hipcc cross-compiles without a GPU)."""
from __future__ import annotations

import functools
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SRC = os.path.join(CSRC, "cbd.hip")              # the decoder
HEADER = os.path.join(HERE, "..", "include", "cbd.h")
# translation units and what each includes
SOURCES = {
    SRC: [os.path.join(CSRC, f) for f in ("cbd_device.hpp", "cbd_lean.hpp", "cbd_parts.hpp", "cbd_team.hpp", "cbd_host.hpp", "word_index.hpp")],
    os.path.join(CSRC, "cbd_layer.hip"): [os.path.join(CSRC, f) for f in ("cbd_host.hpp", "cbd_score.hpp")],
    os.path.join(CSRC, "cbd_sample.hip"): [os.path.join(CSRC, f) for f in ("cbd_host.hpp", "cbd_score.hpp")],
}
LIB = os.path.join(HERE, "libcbdec.so")
LIB_PROFILE = os.path.join(HERE, "libcbdec_prof.so")   # diagnostic build: phase stamps in the lean frame code
LIB_SPREAD = os.path.join(HERE, "libcbdec_spread.so")   # test build: teams of workgroups as if spread over several dies

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the kernels already combine a wave's updates into one atomic issued by one lane; the compiler's own
    # wave-level combining of atomics would only wrap each of them in more code
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
    "-Wall", "-Wno-unused-result", "-pthread",
]


def build(force: bool = True, verbose: bool = False, profile: bool = False, spread: bool = False) -> str:
    """Compile libcbdec.so.  With force=False only the units whose sources are newer than their objects.
    profile=True builds libcbdec_prof.so instead: the same code with -DCBD_PROFILE, in which thread 0 of every
    workgroup stamps the phases of the lean frames (bench.py --phases reads the sums); not the product build.
    spread=True builds libcbdec_spread.so: the same code with -DCBD_TEAM_SPREAD, in which teams use device-wide barriers
    throughout (tests/test_gpu_team.py); not the product build either."""
    lib = LIB_PROFILE if profile else LIB_SPREAD if spread else LIB
    newest = lambda files: max(os.path.getmtime(f) for f in files)  # noqa: E731
    if not force and os.path.exists(lib) and os.path.getmtime(lib) >= newest([HEADER] + [f for s, d in SOURCES.items() for f in (s, *d)]):
        return lib
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [*HIPCC_FLAGS, *(["-DCBD_PROFILE"] if profile else []), *(["-DCBD_TEAM_SPREAD"] if spread else [])]
    objects = os.path.join(HERE, "_build", os.path.splitext(os.path.basename(lib))[0])
    os.makedirs(objects, exist_ok=True)

    def compile_unit(src: str) -> str:
        obj = os.path.join(objects, os.path.splitext(os.path.basename(src))[0] + ".o")
        if not force and os.path.exists(obj) and os.path.getmtime(obj) >= newest([src, HEADER, *SOURCES[src]]):
            return obj
        run([hipcc, *flags, "-c", "-o", obj + ".tmp", src])
        os.replace(obj + ".tmp", obj)
        return obj

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with ThreadPoolExecutor(len(SOURCES)) as pool:
        objs = list(pool.map(compile_unit, SOURCES))
    run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-pthread", "-o", lib + ".tmp", *objs])
    os.replace(lib + ".tmp", lib)
    return lib


@functools.lru_cache(maxsize=None)   # (it takes a minute)
def resource_usage() -> dict:
    """Compiles the device code of all units once more with the compiler's resource remarks on and returns, per kernel,
    {"vgprs", "vgpr_spill", "scratch", "lds"} (name = demangled-ish substring of the kernel symbol)."""
    import re
    import tempfile
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in HIPCC_FLAGS if f not in ("-Wall", "-Wno-unused-result")]
    with tempfile.TemporaryDirectory() as tmp:
        def remarks(src: str) -> str:
            cmd = [hipcc, *flags, "--cuda-device-only", "-c", "-Rpass-analysis=kernel-resource-usage",
                   "-o", os.path.join(tmp, os.path.basename(src) + ".o"), src]
            return subprocess.run(cmd, check=True, capture_output=True, text=True).stderr

        with ThreadPoolExecutor(len(SOURCES)) as pool:
            out = "".join(pool.map(remarks, SOURCES))
    usage, cur = {}, None
    for line in out.splitlines():
        m = re.search(r"remark: Function Name: (\S+)", line)
        if m:
            cur = usage.setdefault(m.group(1), {})
            continue
        for key, pat in (("vgprs", r"remark:\s+VGPRs: (\d+)"), ("vgpr_spill", r"VGPRs Spill: (\d+)"),
                         ("scratch", r"ScratchSize \[bytes/lane\]: (\d+)"), ("lds", r"LDS Size \[bytes/block\]: (\d+)")):
            m = re.search(pat, line)
            if m and cur is not None:
                cur[key] = int(m.group(1))
    return usage


if __name__ == "__main__":
    print(build(force=True, verbose=True, profile="--profile" in sys.argv[1:], spread="--spread" in sys.argv[1:]))
