"""Build libhapmoe.so (HIP, gfx950) in-tree with hipcc."""
import concurrent.futures
import os
import subprocess
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libhapmoe.so")
SOURCES = ["api.hip", "cost_tables.hip", "stage_dp.hip", "type_dp.hip", "width_dp.hip", "latency_dp.hip", "best_plan.hip",
           "op_api.hip", "route.hip", "combine.hip", "adamw.hip", "expert_matmul.hip",
           "route_balanced.hip", "layer_norm.hip", "embed.hip", "dropout.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off", "-fno-fast-math",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


CLOCKS_LIB = os.path.join(PKG, "libhapmoe_clocks.so")


def build(force=True, verbose=False, section_clocks=False):
    """Compile every HIP source of the library; returns the .so path.
    section_clocks: the diagnostic variant (libhapmoe_clocks.so) whose stage-DP
    kernel records where its time goes (hapmoe_section_clocks)."""
    lib = CLOCKS_LIB if section_clocks else LIB
    if not force and os.path.exists(lib):
        return lib
    tmp = lib + ".tmp"
    extra = ["-DHAPMOE_SECTION_CLOCKS"] if section_clocks else []

    def run(*args):
        cmd = [HIPCC, *FLAGS, *args]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    # a process a source: one after another they take minutes
    with tempfile.TemporaryDirectory() as at, concurrent.futures.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        objects = [os.path.join(at, s + ".o") for s in SOURCES]
        for done in [pool.submit(run, *extra, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), "-c", "-o", o,
                                 os.path.join(PKG, "csrc", s)) for s, o in zip(SOURCES, objects)]:
            done.result()
        run("-shared", "-o", tmp, *objects)
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    import sys
    print(build(verbose=True, section_clocks="--section-clocks" in sys.argv))
