"""Builds the HIP shared library (gfx950) in-tree: paper_2602_06036_amd/libdflash.so."""
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "csrc", "dflash.hip")
SRCS = [SRC] + [os.path.join(HERE, "csrc", f) for f in ("kvq_attn.hip", "kvq.hip")]
OUT = os.path.join(HERE, "libdflash.so")

FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function"]


def build(verbose: bool = True) -> str:
    """The sources side by side, each an object of its own, then the library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SRCS]
        cmds = [[hipcc] + FLAGS + ["-c", s, "-o", o] for s, o in zip(SRCS, objs)]
        running = []
        for cmd in cmds:
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True))
        done = [r.communicate() + (r.returncode,) for r in running]
        if all(rc == 0 for _, _, rc in done):
            link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objs + ["-o", OUT]
            if verbose:
                print(" ".join(link), flush=True)
            res = subprocess.run(link, capture_output=True, text=True)
            done.append((res.stdout, res.stderr, res.returncode))
    # the host pass prints a harmless "not a recognized feature" note for -packed-fp32-ops
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for _, e, _ in done for l in e.splitlines() if noise not in l)
    if err.strip() and verbose:
        print(err, file=sys.stderr)
    if any(rc for _, _, rc in done):
        raise RuntimeError("hipcc failed:\n" + err)
    return OUT


if __name__ == "__main__":
    build()
