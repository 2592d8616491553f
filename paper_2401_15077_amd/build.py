"""Build libeagle.so (hipcc, gfx950) in-tree."""
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libeagle.so")
SOURCES = ["eagle.hip", "operators.hip"]
HEADERS = ["kernels.h", "kernels2.h", "plans.h", "common.h", "host.h", "operators.h", "rows.h", "rope.h", "chunk_attn.h", "logit_rules.h", os.path.join("..", "..", "include", "eagle.h")]


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 into libeagle.so.  Raises on failure."""
    if not force and not needs_build():
        return LIB
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Wno-unused-result", "-Wno-unused-command-line-argument"]
    noise = "is not a recognized feature for this target"
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        jobs = [subprocess.Popen(["hipcc", *flags, "-c", os.path.join(CSRC, s), "-o", o], stderr=subprocess.PIPE, text=True) for s, o in zip(SOURCES, objects)]
        for source, job in zip(SOURCES, jobs):
            err = "\n".join(l for l in job.communicate()[1].splitlines() if noise not in l)
            if verbose or job.returncode:
                print(err)
            if job.returncode:
                raise RuntimeError(f"hipcc failed on {source}:\n" + err)
        res = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", LIB], capture_output=True, text=True)
        if res.returncode:
            raise RuntimeError("hipcc failed to link:\n" + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
