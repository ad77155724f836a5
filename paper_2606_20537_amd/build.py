"""Build libcapsule.so (host ABI + gfx950 kernels) in-tree with hipcc.

The library is always rebuilt when ``build()`` is called; loading code uses
whatever is already built.  Usage: ``python -m paper_2606_20537_amd.build``.
"""
import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB_PATH = os.path.join(PKG, "_build", "libcapsule.so")
SOURCES = ["capsule_host.cpp", "capsule_copy.hip", "linattn_scan.hip", "linattn_seg.hip", "linattn_step.hip", "gdn_scan.hip", "gdn_step.hip", "gdn_noalloc.hip", "kv_fp8.hip", "append.hip",
           "kvb_host.cpp", "kvb_append.hip", "kvb_attend.hip", "kvb_prefill.hip", "kvb_select.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# gfx950 only.  Packed-fp32 instructions are disabled for all device code.
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-fvisibility=hidden", "-Wall", "-Wno-unused-function",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def build(out_path: str = LIB_PATH, extra_flags=(), verbose: bool = False) -> str:
    os.makedirs(os.path.dirname(out_path), exist_ok=True)
    tmp = out_path + ".tmp%d" % os.getpid()
    cmd = [HIPCC, *FLAGS, *extra_flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", tmp, *[os.path.join(CSRC, s) for s in SOURCES]]
    res = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the packed-fp32 feature; that warning is harmless
    noise = "'-packed-fp32-ops' is not a recognized feature"
    msgs = [l for l in (res.stdout + res.stderr).splitlines() if noise not in l]
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + "\n".join(msgs))
    if verbose and msgs:
        print("\n".join(msgs))
    os.replace(tmp, out_path)
    return out_path


if __name__ == "__main__":
    print(build(verbose=True))
