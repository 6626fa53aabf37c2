"""Builds libwinof4.so (host plan + gfx950 HIP kernels) in-tree with hipcc, and
the binding's _marshal.so with the host compiler.

The library is a plain C ABI (include/winof4.h) that links nothing of torch;
_marshal.so checks torch tensors for the binding and links both.  ``build()``
always recompiles.
"""
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libwinof4.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
SOURCES = ["plan.cpp", "plan_device.hip", "wino_kernels.hip", "wino_fused.hip", "direct_conv.hip", "wino_float.hip", "probe.hip",
           "w4_quantize.cpp", "w4_matvec.hip", "kv4_append.hip", "kv4_attention.hip", "prompt_attention.hip",
           "w8_quantize.hip", "w8_matmul.hip", "w8_experts.hip", "route_experts.hip"]
ARCH = "gfx950"
# Packed fp32 instructions are disabled for every HIP translation unit; the
# host pass prints a harmless note that it does not know the feature.
HIP_FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Wall", "-Wno-unused-function"]


def hipcc():
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def marshal_commands(out):
    """Compile and link commands of _marshal.so; the library has to be there for the second."""
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(hipcc())))
    obj = os.path.join(PKG, "_build", "marshal.cpp.o")
    compile_ = ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__",
                f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"]]
    for p in include_paths() + [os.path.join(rocm, "include")]:
        compile_ += ["-isystem", p]
    link = ["g++", "-shared", "-o", out, obj, "-L", PKG, "-l:libwinof4.so", "-Wl,-rpath,$ORIGIN"]
    for p in library_paths()[:1]:
        link += ["-L", p]
    return compile_ + ["-c", os.path.join(CSRC, "marshal.cpp"), "-o", obj], link + ["-ltorch_python", "-ltorch_cpu", "-lc10"]


def build_marshal(verbose=False):
    """_marshal.so, once the library is in place.  The library needs hipcc alone: without torch or a host compiler only
    the Python binding of the decoder operators is missing, and says so when it is called."""
    try:
        for cmd in marshal_commands(MARSHAL + ".tmp"):
            if verbose:
                print(" ".join(cmd), flush=True)
            r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            if r.returncode != 0:
                sys.stderr.write(r.stdout)
                raise RuntimeError("compilation or link failed for marshal.cpp")
    except (ImportError, FileNotFoundError) as e:
        sys.stderr.write(f"_marshal.so is not built, the decoder operators have no Python binding: {e}\n")
        if os.path.exists(MARSHAL):
            os.remove(MARSHAL)              # of other sources
        return
    os.replace(MARSHAL + ".tmp", MARSHAL)


def build(verbose=False, jobs=None):
    cc = hipcc()
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs, procs = [], []
    for src in SOURCES:
        obj = os.path.join(objdir, src + ".o")
        cmd = [cc] + HIP_FLAGS + ["-I", os.path.join(ROOT, "include"), "-c", os.path.join(CSRC, src), "-o", obj]
        if src.endswith(".cpp"):
            cmd.insert(1, "-x")
            cmd.insert(2, "hip")
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        msgs = [l for l in out.splitlines() if "packed-fp32-ops" not in l]
        if p.returncode != 0:
            failed.append(src)
            sys.stderr.write("\n".join(msgs) + "\n")
        elif verbose and msgs:
            print("\n".join(msgs))
    if failed:
        raise RuntimeError("compilation failed for " + ", ".join(failed))
    tmp = LIB + ".tmp"
    cmd = [cc, "-shared", f"--offload-arch={ARCH}", "-o", tmp] + objs
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout)
        raise RuntimeError("link failed")
    os.replace(tmp, LIB)
    build_marshal(verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
