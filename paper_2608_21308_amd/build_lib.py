"""Build the HIP library libe2ttt.so in-tree for gfx950 (hipcc, no JIT)."""
from __future__ import annotations

import glob
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libe2ttt.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]

# Flags of single files.  The delta rule's kernels live on MFMA results that the
# vector units take up at once: kept out of the accumulation registers, they need
# no moves (a sixth of the chain's instructions).
FILE_FLAGS = {n: ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]
              for n in ("delta_prep.hip", "delta_fwd.hip", "delta_bwd.hip", "delta_grads.hip")}


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _run(cmd: list[str], verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    # the host pass does not know the packed-fp32 feature; that warning is harmless
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        sys.stderr.write(out + "\n")
        raise RuntimeError("hipcc failed (%d): %s" % (res.returncode, cmd[-3]))
    if verbose and out.strip():
        print(out)


def build(verbose: bool = False, extra: list[str] | None = None) -> str:
    """Compile every source to an object in parallel (one hipcc per file), then link."""
    from concurrent.futures import ThreadPoolExecutor
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    flags = [f for f in HIPCC_FLAGS if f != "-shared"] + list(extra or [])
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    jobs = []
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src)[:-4] + ".o")
        own = FILE_FLAGS.get(os.path.basename(src), [])
        jobs.append((src, obj, [hipcc, *flags, *own, *inc, "-c", src, "-o", obj]))
    workers = max(1, min(len(jobs), int(os.environ.get("MAX_JOBS", "0")) or (os.cpu_count() or 1)))
    with ThreadPoolExecutor(max_workers=workers) as ex:
        for f in [ex.submit(_run, cmd, verbose) for _, _, cmd in jobs]:
            f.result()
    tmp = LIB + ".tmp%d" % os.getpid()
    _run([hipcc, *HIPCC_FLAGS, *(extra or []), *[o for _, o, _ in jobs], "-o", tmp], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
