"""Build the gfx950 shared library (hipcc cross-compiles without a GPU)."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "csrc", "pcr_lib.hip")                # the decoder, the loader, records
SRC_TRAIN = os.path.join(HERE, "csrc", "pcr_train.hip")        # the operators behind the decode
LIB = os.path.join(HERE, "libpcr.so")

HIPCC_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build():
    """Compile csrc/ into libpcr.so (always recompiles)."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    compile_only = [hipcc, "-c"] + [f for f in HIPCC_FLAGS if f != "-shared"]
    sources = (SRC, SRC_TRAIN)
    objects = [s[:-len(".hip")] + ".o" for s in sources]
    running = [subprocess.Popen(compile_only + ["-o", o, s]) for s, o in zip(sources, objects)]
    failed = [p.args for p in running if p.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(1, failed[0])
    subprocess.check_call([hipcc] + HIPCC_FLAGS + ["-o", LIB] + objects)
    return LIB


if __name__ == "__main__":
    print(build())
