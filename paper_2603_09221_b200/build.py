"""Build step of the CUDA library: nvcc, sm_100a only, in-tree output next to this file."""
from __future__ import annotations

import contextlib
import glob
import os
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libttc_lqr.so")
STEP = os.path.join(_HERE, "_step.so")
NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "-Xcompiler", "-fPIC",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale(artefact=LIB):
    if not os.path.exists(artefact):
        return True
    t = os.path.getmtime(artefact)
    deps = glob.glob(os.path.join(CSRC, "*")) + glob.glob(os.path.join(_HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


@contextlib.contextmanager
def _in_place(artefact):
    """A path beside `artefact` to write to, which takes its place once it is whole: another process may load it meanwhile."""
    stem, end = os.path.splitext(os.path.basename(artefact))
    fd, path = tempfile.mkstemp(prefix=stem + ".", suffix=end, dir=os.path.dirname(artefact))
    os.close(fd)
    try:
        yield path
        os.chmod(path, 0o755)
        os.replace(path, artefact)
    except BaseException:
        os.unlink(path)
        raise


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every ``csrc/*.cu`` (side by side) into ``libttc_lqr.so``; rebuilds when a source is newer."""
    if force or _stale():
        nvcc = [os.environ.get("NVCC", "nvcc")] + NVCC_FLAGS
        with tempfile.TemporaryDirectory() as tmp:
            objects, jobs = [], []
            for src in sources():
                objects.append(os.path.join(tmp, os.path.basename(src) + ".o"))
                cmd = nvcc + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", objects[-1], src]
                jobs.append((cmd, subprocess.Popen(cmd)))
            failed = [subprocess.CalledProcessError(job.returncode, cmd) for cmd, job in jobs if job.wait()]
            if failed:
                raise failed[0]
            with _in_place(LIB) as path:
                subprocess.run(nvcc + ["-shared", "-o", path] + objects, check=True)
    return LIB


def step_command(output):
    """The compiler's call for ``_step.so`` (``csrc/step_binding.cpp``): a Python module against torch's own headers and libraries."""
    import sysconfig
    import torch
    root = os.path.dirname(torch.__file__)
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
           os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    cmd += ["-isystem" + i for i in inc] + ["-o", output, os.path.join(CSRC, "step_binding.cpp"), "-L" + os.path.join(root, "lib")]
    return cmd + ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch", "-ltorch_python"]


def build_step_binding(force: bool = False) -> str:
    """Compile ``_step.so``, the short way into the calls for single tokens."""
    if force or _stale(STEP):
        with _in_place(STEP) as path:
            subprocess.run(step_command(path), check=True)
    return STEP
