"""Compile the HIP sources into paper_2407_01781_amd/libfvdb_hotpath.so (gfx950 only)."""
from __future__ import annotations

import glob
import importlib.util
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfvdb_hotpath.so")
SOURCES = ["attention_bwd.hip", "attention.hip", "attention_step.hip", "conv_wgrad_bf16.hip", "conv_wgrad_f16.hip", "conv.hip", "conv_bwd.hip", "conv_leaf.hip", "conv_lowdepth.hip",
           "grid.hip", "kmap.hip", "conv_wgrad_pairs.hip", "conv_wgrad_lists.hip", "block.hip", "scan.hip", "sequences.hip", "pool.hip", "lib.hip"]      # the ones that take longest first
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument"]
# Sources whose kernels must not spill registers: their rows sit in registers across divergent branches, and a spill in
# such a branch has been stored for the branch's lanes only (wrong gradients at 3 channels).
NO_SCRATCH = {"scan.hip", "block.hip"}
# Here scalar registers may be kept in lanes of vector registers (and a frame be reserved for it), vector registers may not.
NO_VECTOR_SPILL = {"attention.hip", "attention_bwd.hip", "attention_step.hip"}

# by its path: this file is run without its package, too, which loads the library
_spec = importlib.util.spec_from_file_location("_matrix_waits", os.path.join(HERE, "matrix_waits.py"))
_matrix_waits = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(_matrix_waits)


def _spills(src: str, lines) -> list:
    """The compiler's remarks on kernels of a source that keep vector registers in memory."""
    if src in NO_SCRATCH:
        return [l for l in lines if "ScratchSize [bytes/lane]:" in l and not l.split("ScratchSize [bytes/lane]:")[1].strip().startswith("0")]
    found, kernel, spilled = [], "", False
    for l in lines:
        kernel = l.split("Function Name:")[1].split()[0] if "Function Name:" in l else kernel
        frame = "ScratchSize [bytes/lane]:" in l and not l.split("ScratchSize [bytes/lane]:")[1].strip().startswith("0")
        spilled = frame if "ScratchSize [bytes/lane]:" in l else spilled
        # without a frame they are in accumulation registers
        if spilled and "VGPRs Spill:" in l and not l.split("VGPRs Spill:")[1].strip().startswith("0"):
            found.append(kernel + l)
    return found


def _newest_source_mtime() -> float:
    m = 0.0
    for root, _, files in os.walk(CSRC):
        for f in files:
            m = max(m, os.path.getmtime(os.path.join(root, f)))
    m = max(m, os.path.getmtime(os.path.join(os.path.dirname(HERE), "include", "fvdb_hotpath.h")))
    return m


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile every source to an object (in parallel, one hipcc per file) and link the shared library."""
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    from concurrent.futures import ThreadPoolExecutor
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    compile_flags = [f for f in FLAGS if f != "-shared"]

    def compile_one(src):
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        cmd = [hipcc] + compile_flags + ["-c", os.path.join(CSRC, src), "-o", obj]
        if src in NO_SCRATCH or src in NO_VECTOR_SPILL:
            cmd.append("-Rpass-analysis=kernel-resource-usage")
        cmd.append("-save-temps=obj")
        if verbose:
            print(" ".join(cmd))
        res = subprocess.run(cmd, capture_output=True, text=True)
        early, temps = None, [t for e in ("-h*", ".hip-h*") for t in glob.glob(obj[:-2] + e)]
        for t in temps:
            if res.returncode == 0 and t.endswith("gfx950.s"):
                with open(t) as f:
                    early = _matrix_waits.early_reads(f.read())
            os.remove(t)
        return obj, res, early

    with ThreadPoolExecutor(min(8, len(SOURCES))) as ex:
        results = list(ex.map(compile_one, SOURCES))
    errs = []
    for src, (obj, res, early) in zip(SOURCES, results):
        lines = [l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l]
        if (src in NO_SCRATCH or src in NO_VECTOR_SPILL) and res.returncode == 0:
            spills = _spills(src, lines)
            if spills:
                raise RuntimeError(f"{src}: a kernel spills registers\n" + "\n".join(spills))
            lines = []
        err = "\n".join(lines)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + err)
        if early is None or early:
            raise RuntimeError(f"{src}: matrix results are read too early, or there is no assembly to look at\n" + "\n".join(early or []))
        if err.strip():
            errs.append(err)
    link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + [obj for obj, _, _ in results] + ["-o", LIB]
    if verbose:
        print(" ".join(link))
    res = subprocess.run(link, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stderr)
    if verbose and errs:
        print("\n".join(errs))
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
