"""Compiles the HIP library for gfx950 and the Python extension in-tree:  python -m paper_2410_21120_amd.build"""
import importlib.util
import os
import subprocess
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libfusedinf.so")
TENSORS = os.path.join(HERE, "_tensors.so")   # the decoder operators on PyTorch tensors (argument marshalling; host code)
SOURCES = ["fi_plan.cpp", "fi_api.cpp", "fi_sched.cpp", "fi_server.cpp", "fi_kernels.hip", "fi_chain.hip", "fi_stem.hip", "fi_kwave.hip", "fi_patch.hip", "fi_stream.hip", "fi_pool.hip", "fi_ops.cpp", "fi_rope.hip", "fi_attn.hip", "fi_q4.hip", "fi_fp4.hip", "fi_fp4_f32.hip", "fi_beam.hip", "fi_pages.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def sources():
    return [os.path.join(CSRC, s) for s in SOURCES]


def stale() -> bool:
    if not os.path.exists(OUT) or not os.path.exists(TENSORS):
        return True
    t = min(os.path.getmtime(OUT), os.path.getmtime(TENSORS))
    headers = [os.path.join(CSRC, h) for h in ("fi_internal.h", "fi_device.h", "fi_ops.h", "fi_ops_device.h", "fi_tree_device.h", "fi_fp4_device.h", "fi_tensors.cpp")]
    deps = sources() + headers + [os.path.join(HERE, "..", "include", "fusedinf.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def _start(cmd):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(process, what):
    out = "\n".join(l for l in process.communicate()[0].splitlines() if "packed-fp32-ops" not in l)
    if process.returncode != 0:
        raise RuntimeError(what + " failed:\n" + out)
    if out.strip():
        print(out)


def _start_tensors():
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    return _start([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I" + sysconfig.get_paths()["include"],
                   "-isystem", os.path.join(torch, "include"), "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
                   os.path.join(CSRC, "fi_tensors.cpp"), "-L" + os.path.join(torch, "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python", "-o", TENSORS])


def build_tensors() -> str:
    _finish(_start_tensors(), "g++")
    return TENSORS


def build(force: bool = True) -> str:
    if not force and not stale():
        return OUT
    tensors = _start_tensors()
    try:
        # (the sources side by side: one after the other they take five minutes, eight at a time one and a half)
        with tempfile.TemporaryDirectory(dir=HERE, prefix=".objects-") as folder, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            objects = [os.path.join(folder, os.path.basename(s) + ".o") for s in sources()]
            done = [pool.submit(lambda s, o: _finish(_start([HIPCC, *FLAGS, "-x", "hip", "-c", s, "-o", o]), "hipcc"), *pair) for pair in zip(sources(), objects)]
            for compiled in done:
                compiled.result()
            _finish(_start([HIPCC, "--offload-arch=gfx950", "-shared", *objects, "-o", OUT]), "hipcc")
    finally:
        _finish(tensors, "g++")
    return OUT


if __name__ == "__main__":
    print("built", build())
