"""Build libtim.so (the C-ABI library) for gfx950 with hipcc, in-tree.

    python -m paper_2605_14220_amd.build            # build
    python -m paper_2605_14220_amd.build --asm DIR  # also keep the device assembly in DIR
"""

from __future__ import annotations

import argparse
import concurrent.futures
import os
import shutil
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libtim.so")
SOURCES = ["lmhead.hip", "lmgrad.hip", "rmsnorm.hip", "mismatch.hip", "seqstats.hip", "ppo.hip", "tim_api.hip",
           "mxfp4.hip", "mxfp4_logits.hip", "rules.hip", "policy_api.hip", "grouping.hip", "embedding.hip", "adapters.hip",
           "adapters_expand.hip", "adapters_pass.hip", "vocab_api.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    # Every floating-point operation is written out explicitly (fmaf where a
    # fused multiply-add is meant); the compiler may not contract a * b + c.
    "-ffp-contract=off",
    # Keep the compiler from forming packed fp32 arithmetic.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall",
    "-Wno-unused-function",
]


def build(asm_dir: str | None = None, verbose: bool = False, defines=(), out: str = LIB) -> str:
    """Compile the library (`defines`: extra NAME=VALUE preprocessor definitions passed to hipcc)."""
    if shutil.which(HIPCC) is None and not os.path.exists(HIPCC):
        raise RuntimeError(f"hipcc not found at {HIPCC}")
    tmp = out + ".tmp"
    compile_flags = [f for f in FLAGS if f != "-shared"]
    includes = ["-I", INCLUDE, "-I", CSRC]
    if asm_dir:
        os.makedirs(asm_dir, exist_ok=True)
        compile_flags.insert(0, "-save-temps")
        asm_dir = os.path.abspath(asm_dir)

    def run(cmd, cwd=None):
        if verbose:
            print(" ".join(cmd))
        r = subprocess.run(cmd, cwd=cwd, capture_output=True, text=True)
        log = "\n".join(line for line in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in line)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed ({r.returncode}):\n{log}")
        if verbose and log.strip():
            print(log)

    # each source by itself, several at a time
    with tempfile.TemporaryDirectory(dir=os.path.dirname(os.path.abspath(out))) as objects:
        obj = {s: os.path.join(objects, s.replace(".hip", ".o")) for s in SOURCES}

        def compile_one(s):
            run([HIPCC, *compile_flags, *[f"-D{x}" for x in defines], *includes, "-c", os.path.join(CSRC, s), "-o",
                 obj[s]], asm_dir)

        with concurrent.futures.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(compile_one, sorted(SOURCES, key=lambda s: not s.startswith("adapters"))))
        run([HIPCC, *FLAGS, *[obj[s] for s in SOURCES], "-o", tmp])
    os.replace(tmp, out)
    return out


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--asm", default=None, help="directory for -save-temps output")
    ap.add_argument("-v", "--verbose", action="store_true")
    ap.add_argument("-D", dest="defines", action="append", default=[], help="NAME=VALUE preprocessor definition")
    ap.add_argument("-o", dest="out", default=LIB)
    args = ap.parse_args(argv)
    print(build(args.asm, args.verbose, args.defines, args.out))


if __name__ == "__main__":
    sys.exit(main())
