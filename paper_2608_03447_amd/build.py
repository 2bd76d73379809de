"""Build ``libasd.so`` (the C-ABI verifier library) for gfx950 with hipcc.

The library is built in-tree next to this file.  Every HIP source is compiled
with packed FP32 instructions disabled and without FMA contraction, so the
binary32/binary64 operations of the verifier are exactly the ones written.

The build embeds a hash of the sources it compiled in ``asd_version()``; the
binding refuses a library whose hash differs from the sources beside it, so a
stale build is never tested, benchmarked or smoke-checked by mistake.
"""
import concurrent.futures
import hashlib
import os
import re
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIBRARY = os.path.join(HERE, "libasd.so")
# The decoding operators around the verifier, and the header they share.
DECODE_SOURCES = [os.path.join(CSRC, "asd_decode_api.cpp"), os.path.join(CSRC, "asd_cache.hip"),
                  os.path.join(CSRC, "asd_attend.hip"), os.path.join(CSRC, "asd_sample.hip")]
DECODE_HEADERS = [os.path.join(CSRC, "asd_decode.h"), os.path.join(CSRC, "asd_tokens.h")]
SOURCES = [os.path.join(CSRC, "asd_api.cpp"), os.path.join(CSRC, "asd_kernels.hip"), *DECODE_SOURCES]
# The verifier's sources and headers; with DECODE_SOURCES and DECODE_HEADERS, every file whose
# code goes into the library.
HASHED_SOURCES = [os.path.join(CSRC, "asd_kernels.hip"), os.path.join(CSRC, "asd_plan.h"),
                  os.path.join(CSRC, "asd_api.cpp"), os.path.join(ROOT, "include", "asd.h")]
# Those that decide what the verifier's kernels do: their code, and the plan of their launches.
VERIFIER_SOURCES = HASHED_SOURCES[:3]
# The binding's native marshalling (a CPython module over torch's C++ tensors).
BINDING = os.path.join(HERE, "_asd_binding.so")
BINDING_SOURCES = [os.path.join(CSRC, "asd_binding.cpp"), os.path.join(ROOT, "include", "asd.h")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-I" + os.path.join(ROOT, "include"),
]


def source_hash(paths=None) -> str:
    """SHA-256 (first 16 hex digits) of the library's sources with comments and
    whitespace removed: an edit to a comment keeps the hash, any code edit
    changes it."""
    h = hashlib.sha256()
    for p in (HASHED_SOURCES + DECODE_SOURCES + DECODE_HEADERS if paths is None else paths):
        with open(p) as f:
            text = f.read()
        text = re.sub(r"/\*.*?\*/", " ", text, flags=re.S)
        text = re.sub(r"//[^\n]*", " ", text)
        h.update(" ".join(text.split()).encode())
    return h.hexdigest()[:16]


def build_library(verbose: bool = False, output: str = LIBRARY, extra_flags=()) -> str:
    tag = '-DASD_SOURCE_HASH="%s"' % source_hash()
    with tempfile.TemporaryDirectory() as objects, \
            concurrent.futures.ThreadPoolExecutor(len(SOURCES)) as pool:
        def compile_one(source):
            obj = os.path.join(objects, os.path.basename(source) + ".o")
            cmd = [HIPCC, *HIP_FLAGS, tag, *extra_flags, "-c", source, "-o", obj]
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.run(cmd, check=True)
            return obj

        link = [HIPCC, "--offload-arch=gfx950", "-shared", *pool.map(compile_one, SOURCES), "-o",
                output + ".tmp"]
        if verbose:
            print(" ".join(link), flush=True)
        subprocess.run(link, check=True)
    os.replace(output + ".tmp", output)
    return output


def binding_hash() -> str:
    """Of the binding's sources and of the torch and Python whose layouts it is compiled for."""
    import torch

    built_for = "%s %s %d %s" % (source_hash(BINDING_SOURCES), torch.__version__,
                                 torch._C._GLIBCXX_USE_CXX11_ABI, sys.implementation.cache_tag)
    return hashlib.sha256(built_for.encode()).hexdigest()[:16]


def build_binding(verbose: bool = False, output: str = BINDING) -> str:
    """The native marshalling, against the installed torch (host code only)."""
    import sysconfig

    import torch

    base = os.path.dirname(torch.__file__)
    include = [os.path.join(base, "include"),
               os.path.join(base, "include", "torch", "csrc", "api", "include"),
               "/opt/rocm/include", sysconfig.get_paths()["include"]]
    cmd = ["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
           "-DUSE_ROCM", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           '-DASD_BINDING_HASH="%s"' % binding_hash()]
    for path in include:
        cmd += ["-isystem", path]
    cmd += [BINDING_SOURCES[0], "-o", output + ".tmp", "-L" + os.path.join(base, "lib"), "-lc10",
            "-lc10_hip", "-ltorch_cpu", "-ltorch_python"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(output + ".tmp", output)
    return output


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_binding(verbose=True))
