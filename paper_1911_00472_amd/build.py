"""Build the gfx950 shared library (hipcc cross-compiles without a GPU) and the Python module over its operators for PyTorch tensors."""
import os
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "csrc", "pcr_lib.hip")                # the decoder, the loader, records
SRC_TRAIN = os.path.join(HERE, "csrc", "pcr_train.hip")        # the operators behind the decode
SRC_DISTILL = os.path.join(HERE, "csrc", "pcr_distill.hip")
SRC_BIND = os.path.join(HERE, "csrc", "pcr_bind.cpp")          # their arguments, as a Python module
LIB = os.path.join(HERE, "libpcr.so")
MODULE = os.path.join(HERE, "_train.so")

HIPCC_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _module_command():
    import torch
    home = os.path.dirname(torch.__file__)
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
            "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(home, "include"), "-I" + os.path.join(home, "include", "torch", "csrc", "api", "include"),
            "-c", "-o", SRC_BIND[:-len(".cpp")] + ".o", SRC_BIND], os.path.join(home, "lib")


def build_library():
    """Compile csrc/ into libpcr.so (always recompiles): the C ABI, which needs neither PyTorch nor Python's headers."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    compile_only = [hipcc, "-c"] + [f for f in HIPCC_FLAGS if f != "-shared"]
    sources = (SRC, SRC_TRAIN, SRC_DISTILL)
    objects = [s[:-len(".hip")] + ".o" for s in sources]
    running = [subprocess.Popen(compile_only + ["-o", o, s]) for s, o in zip(sources, objects)]
    failed = [p.args for p in running if p.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(1, failed[0])
    subprocess.check_call([hipcc] + HIPCC_FLAGS + ["-o", LIB] + objects)
    return LIB


def build():
    """Compile csrc/ into libpcr.so and _train.so (always recompiles).  What keeps the module from being made is raised when the library is; a module of
    another library is not left beside it."""
    compiling, late = None, None
    try:
        module, torch_lib = _module_command()
        compiling = subprocess.Popen(module)
    except (ImportError, OSError) as e:
        late = e
    try:
        build_library()
    finally:
        failed = compiling is not None and compiling.wait() != 0
    if (late is not None or failed) and os.path.exists(MODULE):
        os.remove(MODULE)
    if late is not None:
        raise late
    if failed:
        raise subprocess.CalledProcessError(1, module)
    subprocess.check_call([module[0], "-shared", "-o", MODULE, module[module.index("-o") + 1], "-L" + HERE, "-lpcr", "-Wl,-rpath,$ORIGIN", "-L" + torch_lib, "-ltorch_python", "-ltorch_cpu", "-lc10"])
    return LIB


if __name__ == "__main__":
    print(build())
