"""Builds libcodec.so (HIP kernels + host planner + C ABI) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import json
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libcodec.so")
SOURCES = ["planner.cpp", "api.cpp", "operators.cpp", "pages.cpp", "device.hip"]     # device.hip includes every kernel
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
         # scalar fp32 code must not be fused into packed-fp32 instructions on this target
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # accumulators of the matrix instructions in ordinary registers, where the softmax works on them:
         # kernels that may use 512 registers per lane (256 channels) would keep them in accumulation
         # registers and copy them back and forth in every block
         "-mllvm", "-amdgpu-mfma-vgpr-form",
         "-Wall", "-Wno-unused-command-line-argument"]


COST_TABLE_JSON = os.path.join(PKG, "cost_table_mi355x.json")
COST_TABLE_INC = os.path.join(CSRC, "cost_table_generated.inc")


def generate_cost_tables(json_path: str = COST_TABLE_JSON, inc_path: str = COST_TABLE_INC) -> str:
    """Writes the built-in cost tables of the planner (C++ initialisers) from the profiler's JSON.

    The JSON is what ``python -m paper_2505_17694_amd.profile`` writes on the target GPU; the planner
    includes the generated file, so the table the library plans with is the measured one by construction.
    """
    with open(json_path) as f:
        tables = json.load(f)

    def init(t):
        rows, lens, cost = t["row_grid"], t["len_grid"], t["cost"]
        assert len(cost) == len(rows) and all(len(c) == len(lens) for c in cost), "table shape"
        assert all(isinstance(x, int) and x > 0 for c in cost for x in c), "costs are positive integers"
        body = ",\n         ".join(", ".join(str(x) for x in c) for c in cost)
        return ("{\n        {%s},\n        {%s},\n        {%s}}"
                % (", ".join(map(str, rows)), ", ".join(map(str, lens)), body))

    text = ("// Generated by build.py from %s (the cost-table profiler's output); do not edit.\n"
            "// Unit: %s.\n"
            "static const CostTable narrow_table = %s;\n"
            "static const CostTable wide_table = %s;\n"
            % (os.path.basename(json_path), tables.get("unit", "ns"), init(tables["narrow"]), init(tables["wide"])))
    old = None
    if os.path.exists(inc_path):
        with open(inc_path) as f:
            old = f.read()
    if old != text:
        with open(inc_path, "w") as f:
            f.write(text)
    return inc_path


def build_library(verbose: bool = False) -> str:
    generate_cost_tables()
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [hipcc] + FLAGS + ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", tmp]
    cmd += ["-x", "hip"] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err, file=sys.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
