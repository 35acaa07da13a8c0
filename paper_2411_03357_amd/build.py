"""Builds libpgcm.so (HIP kernels + C ABI) for gfx950 with hipcc, and the Python binding's native
marshalling with the host compiler, in-tree."""
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpgcm.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
KV_MARSHAL = os.path.join(HERE, "_kv_marshal.so")    # a torch extension; the rest does without torch
SOURCES = ["pgcm_kernels.hip", "pgcm_bitsliced.hip", "pgcm_host.hip", "pgcm_bounce.hip", "pgcm_pipe.hip",
           "pgcm_seq.cpp", "pgcm_kv.hip", "pgcm_kv_attend.hip", "pgcm_kv_cache.hip", "pgcm_kv_choose.hip",
           "pgcm_kv8_cache.hip", "pgcm_kv_window.hip", "pgcm_kv_window_few.hip",
           "pgcm_kv_window_many.hip"]
HEADERS = ["pgcm_kernels.h", "pgcm_types.h", "pgcm_arrive.h", "pgcm_contexts.h", "pgcm_one_launch.h",
           "pgcm_spans.h", "pgcm_routes.h", "pgcm_host_ivs.h", "pgcm_bitsliced_gen.h",
           "pgcm_kv_common.h", "pgcm_kv8_common.h", "pgcm_kv_window.h",
           os.path.join("..", "..", "include", "pgcm.h"),
           os.path.join("..", "..", "include", "pgcm_seq.h"),
           os.path.join("..", "..", "include", "pgcm_bounce.h"),
           os.path.join("..", "..", "include", "pgcm_pipe.h"),
           os.path.join("..", "..", "include", "pgcm_kv.h"),
           os.path.join("..", "..", "include", "pgcm_kv8.h")]

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
    "-Wall", "-Wno-unused-command-line-argument",
    # keep the compiler from forming packed-FP32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the leading kernel arguments come in registers instead of being loaded from host memory
    "-mllvm", "-amdgpu-kernarg-preload-count=14",
    # one lane's atomic stays one instruction, whose result is waited for where it is used
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found")
    return exe


def _torch():
    """the torch that is installed, or None: the cipher and its binding do without"""
    try:
        import torch
    except ImportError:
        return None
    return torch


def _built_for(torch) -> bytes:
    return b"built for torch " + torch.__version__.encode() + b"\0"


def is_stale() -> bool:
    torch = _torch()
    built = (LIB, MARSHAL) if torch is None else (LIB, MARSHAL, KV_MARSHAL)
    if not all(os.path.exists(b) for b in built):
        return True
    if torch is not None:
        with open(KV_MARSHAL, "rb") as f:
            if _built_for(torch) not in f.read():
                return True
    t = min(os.path.getmtime(b) for b in built)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS + ["marshal.cpp", "kv_marshal.cpp"]] + \
        [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def _host_build(source, target, *more) -> None:
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        raise RuntimeError("no host C++ compiler")
    tmp = target + ".tmp%d" % os.getpid()
    proc = subprocess.run([cxx, "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
                           "-Wall", "-I" + sysconfig.get_paths()["include"],
                           os.path.join(CSRC, source), "-o", tmp, *more],
                          stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if proc.returncode != 0:
        raise RuntimeError("compiling %s failed:\n%s" % (source, proc.stdout))
    os.replace(tmp, target)


def build_marshal() -> None:
    _host_build("marshal.cpp", MARSHAL)
    torch = _torch()
    if torch is None:       # no tensors, so none of the operators that take them
        return
    at = os.path.dirname(torch.__file__)
    _host_build("kv_marshal.cpp", KV_MARSHAL, "-isystem", os.path.join(at, "include"),
                "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi(), '-DBUILT_FOR="%s"' % torch.__version__,
                "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10")


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [hipcc()] + FLAGS + [os.path.join(CSRC, s) for s in SOURCES] + ["-o", tmp]
    if verbose:
        print(" ".join(cmd))
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in proc.stdout.splitlines() if "packed-fp32-ops" not in l)
    if proc.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)
    os.replace(tmp, LIB)
    build_marshal()
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
