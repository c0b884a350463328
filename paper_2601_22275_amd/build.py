"""Builds libvmonarch.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libvmonarch.so")
# (source, object, flags of its own): flash2.hip and seq_mfma.hip are compiled once per head dimension
SOURCES = [(s, s.replace(".hip", ".o"), []) for s in ("api.hip", "generic.hip", "flash.hip", "flash_kv.hip", "frame.hip", "lpass.hip",
                                                      "backward.hip", "backward_mfma.hip", "f32.hip", "rotary.hip", "seq_api.hip", "seq_general.hip", "seq_token.hip", "seq_bwd.hip")]
SOURCES += [("flash2.hip", f"flash2_{d}.o", [f"-DVM_FLASH2_D={d}"]) for d in (64, 128)]
SOURCES += [("seq_mfma.hip", f"seq_mfma_{d}.o", [f"-DVM_SEQ_D={d}"]) for d in (64, 128)]
FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fvisibility=hidden",
    # keep the compiler from forming packed fp32 VALU instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-value", "-Wno-unknown-warning-option",
]
# per-file extras: the blocked-softmax kernels keep MFMA results in vector registers; their
# logits are never NaN (masking uses large finite values), which spares the v_max x, x, x that
# would otherwise quiet a possible signalling NaN in front of every maximum
EXTRA = {"flash2.hip": ["-fno-honor-nans", "-Wno-inline-asm"],
         "flash.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-fno-honor-nans"],
         "flash_kv.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-fno-honor-nans"],
         "frame.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-fno-honor-nans"],
         "f32.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
         "seq_mfma.hip": ["-Wno-inline-asm"],
         "seq_token.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
         "seq_bwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
         "seq_general.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
         "backward_mfma.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    procs = []
    for src, obj, flags in SOURCES:
        obj = os.path.join(CSRC, obj)
        cmd = [hipcc, *FLAGS, *EXTRA.get(src, []), *flags, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0:
            sys.stderr.write(out)
            raise RuntimeError(f"hipcc failed on {src}")
        if verbose and out.strip():
            print(out)
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
