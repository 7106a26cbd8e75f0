"""Build the gfx950 HIP library libbytecomp.so in-tree with hipcc.

Every source under csrc/ is compiled for gfx950 only, with
-ffp-contract=off (no fused multiply-add contraction: the operators'
results are defined by separate fp32 roundings) and with packed fp32
instructions disabled.
"""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbytecomp.so")
BUILD = os.path.join(HERE, "_build")
SOURCES = ["api.hip", "kernels_sign.hip", "kernels_topk.hip", "kernels_randk.hip", "kernels_agg_sparse.hip",
           "kernels_agg_sign.hip", "kernels_resid.hip", "kernels_part.hip", "kernels_quant.hip",
           "kernels_dgc.hip", "noalloc.hip", "cpu_ops.hip", "plan_sim.hip", "api_layers.hip",
           "kernels_layernorm.hip", "kernels_linear.hip", "kernels_ortho.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-I", os.path.join(HERE, "..", "include")]


def build(verbose: bool = False, jobs: int = 5) -> str:
    os.makedirs(BUILD, exist_ok=True)
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(BUILD, src.replace(".hip", ".o"))
        objs.append(obj)
        cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        if len(procs) >= jobs:
            _wait(procs.pop(0))
    while procs:
        _wait(procs.pop(0))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs, "-L/opt/rocm/lib",
           "-lrocprofiler-sdk-roctx", "-Wl,-rpath,/opt/rocm/lib"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


def _wait(item):
    src, p = item
    out, _ = p.communicate()
    text = out.decode(errors="replace")
    if p.returncode != 0:
        sys.stderr.write(text)
        raise RuntimeError(f"hipcc failed on {src}")
    if text.strip():
        # host-pass warnings about the packed-fp32 target feature are expected
        lines = [ln for ln in text.splitlines() if "packed-fp32-ops" not in ln]
        if any(ln.strip() for ln in lines):
            sys.stderr.write("\n".join(lines) + "\n")


if __name__ == "__main__":
    build(verbose=True)
