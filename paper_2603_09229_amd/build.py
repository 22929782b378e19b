"""Compile the HIP sources under csrc/ into libflashkm.so (gfx950 only), in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libflashkm.so"

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-fno-gpu-rdc", "-Wall", "-Wno-unused-function",
    # MFMA accumulators in ordinary VGPRs: the argmin epilogue reads them with VALU
    # instructions, which cannot address AGPRs (saves one copy per accumulator element)
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    # packed-fp32 VALU forms are kept out of the generated code on purpose
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    f"-I{ROOT / 'include'}", f"-I{CSRC}",
]
# the HSA runtime (already a dependency of the HIP runtime) is asked for the cache sizes
LIBS = ["-L/opt/rocm/lib", "-lhsa-runtime64"]


def sources() -> list[Path]:
    return sorted(CSRC.glob("*.hip"))


def build(verbose: bool = True) -> Path:
    """Always recompiles, one compiler a source on the machine's processors; raises on any compiler error."""
    with tempfile.TemporaryDirectory(dir=PKG, prefix=".build") as tmp:
        def run(cmd):
            if verbose:
                print(" ".join(cmd), flush=True)
            proc = subprocess.run(cmd, capture_output=True, text=True)
            # the host pass warns that it does not know the packed-fp32 feature: harmless
            noise = "is not a recognized feature for this target"
            err = "\n".join(l for l in proc.stderr.splitlines() if noise not in l)
            if verbose and err.strip():
                print(err, file=sys.stderr)
            if proc.returncode != 0:
                raise RuntimeError(f"hipcc failed ({proc.returncode}):\n{err}")

        # the longest first, with the headers they include: what is left at the end is short
        def length(source):
            text = source.read_text()
            return len(text) + sum(h.stat().st_size for h in CSRC.glob("*.h") if f'"{h.name}"' in text)

        todo = sorted(sources(), key=length, reverse=True)
        objects = [str(Path(tmp) / (s.name + ".o")) for s in todo]
        with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(lambda so: run([HIPCC, *(f for f in FLAGS if f != "-shared"), "-c", "-o", so[1], str(so[0])]), zip(todo, objects)))
        made = str(Path(tmp) / LIB.name)
        run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", made, *objects, *LIBS])
        os.replace(made, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
