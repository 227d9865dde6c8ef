"""Build the HIP library libmesh_attn.so in-tree for gfx950.

Every translation unit under csrc/ is compiled with hipcc and linked into one
shared library next to this file; the Python binding loads it from there.
"""

import glob
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJDIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmesh_attn.so")
ARCH = "gfx950"

# Packed FP32 VALU forms are kept out of generated code.
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Wno-unused-command-line-argument", f"-I{INCLUDE}", f"-I{CSRC}"]


# Per-file additions.  The backward kernels keep dK, dV (or dQ) and the score
# tiles live together; MFMA results in VGPR form keep the compiler from
# parking score accumulators in AGPRs and copying them back for the softmax.
# The forward is scheduled with the target's own register-pressure trackers:
# its float32-output kernel then fits 256 registers without a spill, and the
# bf16-output kernel's schedule runs 0.5-1.6 % faster.
# The attention over the cache keeps every join's own restore of the execution
# mask: in a kernel that is no longer built (float32 O, tiles of 64 rows) the
# compiler left one out, and a register saved inside a nested branch of the fold
# was restored for the inner branch's lanes alone and then used in an address.
# The present kernels' assembly has no join that runs vector instructions before
# its restore, with this flag or without; what the register allocator puts there
# changes with any edit, so the flag stays.
# (The backward under a score rule, which has a few spilled registers too, is built
# the same way.)
EXTRA = {"cache_fwd.hip": ["-mllvm", "-amdgpu-remove-redundant-endcf=0"],
         "score_bwd.hip": ["-mllvm", "-amdgpu-remove-redundant-endcf=0"],
         "tile_bwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
         "tile_fwd.hip": ["-mllvm", "-amdgpu-use-amdgpu-trackers"]}


def hipcc():
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found; ROCm is required to build")
    return exe


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")) +
                  glob.glob(os.path.join(CSRC, "*.cpp")))


def _compile(src):
    obj = os.path.join(OBJDIR, os.path.basename(src) + ".o")
    cmd = [hipcc(), *COMMON, *EXTRA.get(os.path.basename(src), []), "-c",
           src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}{r.stderr}")
    return obj


def build(verbose=True):
    """Compile every source and link libmesh_attn.so (always rebuilds)."""
    os.makedirs(OBJDIR, exist_ok=True)
    srcs = sources()
    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs,
           "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
