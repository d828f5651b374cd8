"""Builds libcsd.so (hand-written HIP for gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcsd.so")
SOURCES = ["csd_api.hip", "csd_draft.hip", "csd_accept.hip", "csd_forward.hip", "csd_attention.hip", "csd_chain.hip", "csd_rows.hip", "csd_tall.hip", "csd_f32.hip",
           "csd_paged.hip", "csd_paged_attn.hip", "csd_paged_few.hip", "csd_paged_many.hip", "csd_paged_chunk.hip", "csd_pages.hip", "csd_sample.hip"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def build(verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 and link the C-ABI shared library."""
    cmd = [hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           # plain kernel arguments in scalar registers when a wave starts (as many dwords as there is room for)
           "-mllvm", "-amdgpu-kernarg-preload-count=16",
           "-Wall", "-Wno-unused-function", "-Rpass-analysis=kernel-resource-usage",
           "-o", LIB] + os.environ.get("CSD_HIPCC_FLAGS", "").split() + [os.path.join(CSRC, s) for s in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    lines = (res.stdout + res.stderr).splitlines()
    remarks = [l for l in lines if "-Rpass-analysis=kernel-resource-usage" in l]
    others = [l for l in lines if l not in remarks and "packed-fp32-ops" not in l]
    if verbose or res.returncode != 0:
        # the host pass does not know the packed-fp32 feature and says so; that is harmless
        print("\n".join(others))
    if res.returncode != 0:
        raise RuntimeError("hipcc failed")
    # a kernel that spills registers is a performance bug: say so at build time
    name = None
    for l in remarks:
        if "Function Name:" in l or " Name: " in l:
            name = l.split("Name:")[1].split("[")[0].strip()
        if "VGPRs Spill:" in l:
            n = int(l.split("VGPRs Spill:")[1].split("[")[0])
            if n > 0:
                print(f"warning: kernel {name} spills {n} VGPRs")
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
