"""Build libscalesim.so (HIP for gfx950) in the package directory.

    python -m paper_2601_21473_amd.build        # or build() from Python
"""
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
SOURCES = ["ss_kernels.hip", "ss_pool.hip", "ss_distance.hip", "ss_loader.hip", "ss_cache.hip",
           "ss_attention.hip", "ss_adapter.hip"]
LIB = os.path.join(HERE, "libscalesim.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Wall", "-Werror=return-type",
    # keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


# Host-side AddressSanitizer and UndefinedBehaviorSanitizer (the device code
# is built as usual): for tests of the library's host code, loaded with the
# sanitizer runtime preloaded.
SANITIZE_FLAGS = ["-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host",
                  "-fsanitize=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]


def build(verbose: bool = False, out: str = LIB, sanitize: bool = False) -> str:
    srcs = [os.path.join(CSRC, s) for s in SOURCES]
    flags = [*FLAGS, *(SANITIZE_FLAGS if sanitize else [])]
    tmp = out + ".tmp"

    def hipcc(*args):
        cmd = [HIPCC, *flags, *args]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + r.stdout + r.stderr)

    with tempfile.TemporaryDirectory() as d, ThreadPoolExecutor(len(srcs)) as pool:
        objects = [os.path.join(d, s + ".o") for s in SOURCES]
        list(pool.map(lambda so: hipcc("-c", so[0], "-o", so[1]), zip(srcs, objects)))
        hipcc(*objects, "-o", tmp)
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
