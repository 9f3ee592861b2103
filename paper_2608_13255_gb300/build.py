"""Build libgeocache.so (CUDA for sm_103a) in-tree with nvcc.

The library is compiled from ``csrc/*.cu`` with one ``-gencode`` for sm_103a,
each translation unit in parallel, and linked with the static CUDA runtime so
that the shared object only needs the driver at run time.  Beside it stands
``geocache_rows_binding.so``, a module of the running interpreter (g++, its
headers and those of a CUDA torch) through which Python calls the operators on
rows.  The library does not need it: where one of these is missing the library is
built alone, and the calls on rows say why they have no module.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIBDIR = os.path.join(PKG, "_lib")
LIB = os.path.join(LIBDIR, "libgeocache.so")
BINDING = os.path.join(LIBDIR, "geocache_rows_binding.so")
BINDING_FOR = os.path.join(LIBDIR, "geocache_rows_binding.for")  # the interpreter and the torch it was built for

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-O2", "--expt-relaxed-constexpr"]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libgeocache.so")


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _binding_source():
    return os.path.join(CSRC, "geocache_rows_binding.cpp")


def _deps():
    return (_sources() + [_binding_source()] + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh"))
            + glob.glob(os.path.join(INCLUDE, "*.h")) + [os.path.abspath(__file__)])


def source_hash() -> str:
    """Hash of every file the library is compiled from (identifies a kernel
    version, e.g. to tell whether stored profiler counters still apply)."""
    import hashlib
    h = hashlib.sha256()
    for d in sorted(_deps()):
        if d == os.path.abspath(__file__):
            continue
        h.update(os.path.basename(d).encode())
        with open(d, "rb") as f:
            h.update(f.read())
    return h.hexdigest()[:16]


def _torch_dir() -> str:
    import importlib.util
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec and spec.origin else ""


def binding_for() -> str:
    """The interpreter and the torch that a module built now would be for."""
    import importlib.metadata
    try:
        torch_version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        torch_version = "none"
    return "%s, torch %s" % (sysconfig.get_config_var("SOABI"), torch_version)


def binding_needs() -> str:
    """What the module's build lacks here ("" if nothing)."""
    torch_dir = _torch_dir()
    for what, there in (("g++", shutil.which("g++")), ("Python.h", os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))),
                        ("torch", torch_dir), ("a CUDA torch", os.path.exists(os.path.join(torch_dir, "lib", "libc10_cuda.so")))):
        if not there:
            return what
    return ""


def binding_was_for() -> str:
    """The interpreter and the torch that the module was built for."""
    try:
        with open(BINDING_FOR) as f:
            return f.read()
    except OSError:
        return "another build"


def binding_is_stale() -> bool:
    """Whether the module is missing or older than its sources, or was built for another interpreter or torch."""
    if not os.path.exists(BINDING) or binding_was_for() != binding_for():
        return True
    t = os.path.getmtime(BINDING)
    return any(os.path.getmtime(d) > t for d in _deps())


def library_is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(d) > t for d in _deps() if d != _binding_source())


def is_stale() -> bool:
    return library_is_stale() or (binding_is_stale() and not binding_needs())


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    """Compile and link libgeocache.so if any source changed; return its path.
    Processes that build at the same time (one per rank) take turns on a lock
    file, so that none links objects another is still writing."""
    if not force and not is_stale():
        return LIB
    import fcntl
    os.makedirs(LIBDIR, exist_ok=True)
    with open(os.path.join(LIBDIR, ".build.lock"), "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        if not force and not is_stale():  # another process built it meanwhile
            return LIB
        return _build_locked(verbose, extra_flags, force)


def _build_locked(verbose, extra_flags, force) -> str:
    cc = nvcc()
    library, lacks = force or library_is_stale(), binding_needs()
    binding = not lacks and (force or binding_is_stale())
    objs, procs = [], []
    for src in _sources() if library else []:
        obj = os.path.join(LIBDIR, os.path.basename(src)[:-3] + ".o")
        cmd = [cc, *ARCH, *NVCC_FLAGS, *extra_flags, "-I", INCLUDE, "-I", CSRC, "-c", src, "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        objs.append(obj)
    torch_dir = _torch_dir()
    binding_obj = os.path.join(LIBDIR, "geocache_rows_binding.o")
    if binding:
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I", INCLUDE, "-I", os.path.join(torch_dir, "include"),
               "-I", os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
               "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(cc))), "include"),
               "-I", sysconfig.get_paths()["include"], "-c", _binding_source(), "-o", binding_obj]
        procs.append((_binding_source(), subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode:
            sys.stderr.write(out.decode(errors="replace"))
        if p.returncode:
            failed.append(src)
    if library and not any(src != _binding_source() for src in failed):
        tmp = LIB + ".tmp%d" % os.getpid()
        subprocess.check_call([cc, *ARCH, "-shared", "-cudart", "static", "-o", tmp, *objs])
        os.replace(tmp, LIB)
    if failed:
        raise RuntimeError("compiling failed on: " + ", ".join(failed))
    if binding:
        tmp = BINDING + ".tmp%d" % os.getpid()
        subprocess.check_call(["g++", "-shared", "-o", tmp, binding_obj, "-L", LIBDIR, "-lgeocache", "-Wl,-rpath,$ORIGIN",
                               "-L", os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"])
        os.replace(tmp, BINDING)
        with open(BINDING_FOR, "w") as f:
            f.write(binding_for())
    elif lacks:
        sys.stderr.write("geocache_rows_binding.so is not built: it needs %s\n" % lacks)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
