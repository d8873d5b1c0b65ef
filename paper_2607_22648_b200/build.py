"""Build the CUDA library in-tree with nvcc for sm_100a (no JIT cache: the .so sits next to the sources)."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libptstore.so")
SOURCES = ["ptstore.cu", "fetch_static.cu", "copy_probe.cu", "plan.cu", "kvcache.cu", "attend.cu", "attend_lse.cu", "latent.cu", "expanded.cu", "weights.cu", "evict.cu"]
NVCC_FLAGS = ["-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC",
              "-shared", "-cudart", "shared", "--threads", "0"]


def _source_hash():
    """Hash of every source and header the library is built from (file times do not survive a copy of the tree)."""
    import hashlib
    h = hashlib.sha256()
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for f in sorted(os.listdir(root)):
            h.update(f.encode())
            h.update(open(os.path.join(root, f), "rb").read())
    h.update(" ".join(NVCC_FLAGS).encode())
    return h.hexdigest()


def build(force=False, verbose=False):
    """Compile csrc/*.cu into libptstore.so unless it was already built from exactly these sources."""
    stamp = LIB + ".srchash"
    want = _source_hash()
    if not force and os.path.exists(LIB) and os.path.exists(stamp) and open(stamp).read().strip() == want:
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB + ".tmp"] + \
          [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.check_call(cmd)
    os.replace(LIB + ".tmp", LIB)
    with open(stamp, "w") as f:
        f.write(want)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
