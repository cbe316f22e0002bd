"""Compile the HIP library for gfx950 into paper_2401_06197_amd/libdcnv4.so (in-tree).

hipcc cross-compiles without a GPU.  Run as `python -m paper_2401_06197_amd.build`.
"""
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SOURCES = [os.path.join(HERE, "csrc", name) for name in ("dcnv4.hip", "dcnv4_norm.hip", "dcnv4_loss.hip")]
LIB = os.path.join(HERE, "libdcnv4.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed-fp32 instructions out of scalar float code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"),
]


def build(verbose: bool = False) -> str:
    """Each source to an object of its own, side by side, then one library of them."""
    # the host pass does not know the device-only target feature and says so; that is harmless
    noise = "is not a recognized feature for this target"
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SOURCES]
        steps = [[[HIPCC] + FLAGS + ["-c", "-o", obj, src] for src, obj in zip(SOURCES, objects)],
                 [[HIPCC, "--offload-arch=gfx950", "-shared", "-o", LIB] + objects]]
        for cmds in steps:
            runs = [subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True) for cmd in cmds]
            said = [run.communicate()[1] for run in runs]
            for cmd, run, text in zip(cmds, runs, said):
                err = "\n".join(l for l in text.splitlines() if noise not in l)
                if run.returncode != 0:
                    raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + err)
                if verbose and err.strip():
                    print(err)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
