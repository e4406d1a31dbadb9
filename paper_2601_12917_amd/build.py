"""Compiles the HIP sources under csrc/ into libzgr.so (gfx950) next to this file."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libzgr.so")
SOURCES = ["api.hip", "perturb.hip", "forward.hip", "ceilings.hip", "cloud.hip", "backward.hip", "product.hip", "rotate.hip", "heads.hip",
           "dropout.hip", "sublayer_api.hip"]
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-shared", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]

STEP_KERNEL_SOURCES = ("perturb.hip", "forward.hip", "forward.h", "product.hip", "product.h", "planes.h", "act.h", "rng.h", "wave.h", "internal.h")


def source_digest() -> str:
    """sha256 over the sources of the client step's kernels (perturbation passes and forward pass, with the headers
    they include): identifies the device code that hardware-counter figures were taken on.  The host runtime, the
    cloud-side kernels and the micro-benchmarks are not part of it."""
    import hashlib
    h = hashlib.sha256()
    for name in sorted(os.listdir(CSRC)):
        if name in STEP_KERNEL_SOURCES:
            h.update(name.encode())
            h.update(open(os.path.join(CSRC, name), "rb").read())
    return h.hexdigest()


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, src.replace(".hip", ".o"))
        cmd = [hipcc] + [f for f in FLAGS if f != "-shared"] + ["-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for cmd, p in procs:
        out, _ = p.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l and "warning generated" not in l and "warnings generated" not in l)
        if verbose or p.returncode:
            print(" ".join(cmd)); print(out)
        if p.returncode:
            raise RuntimeError("hipcc failed")
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objs + ["-o", LIB]
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
