"""TEST INFRASTRUCTURE ONLY: compiles the 4-bit key/value cache's kernels and C ABI against the CPU stand-in for the HIP runtime,
with AddressSanitizer and UBSan, into tests/emu/_build/kv/emu_kv_driver.  A call is cut into few pieces (QP_KV_FEW, QP_KV_MANY), so
that a launch is a handful of emulated blocks and small contexts are still split and joined."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
EMU = os.path.dirname(HERE)
sys.path.insert(0, EMU)
import build_emu  # noqa: E402

FLAGS = ["-DQP_KV_FEW=12", "-DQP_KV_MANY=10", "-DQP_KV_LEAST=1", "-DQP_KV_SPAN_FILL=30", "-DQP_KV_COPY_BLOCKS=4", "-DQP_KV_GRID=5"]


def build():
    """The driver's path, or None without a host clang++."""
    cxx = build_emu.find_cxx()
    if cxx is None:
        return None
    out = os.path.join(EMU, "_build", "kv")
    os.makedirs(out, exist_ok=True)
    flags = ["-std=c++20", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer",
             "-fno-rtti", "-ffp-contract=off", "-pthread", "-Wno-unused-value", "-I", HERE, "-I", os.path.join(build_emu.ROOT, "include"),
             "-I", build_emu.CSRC, *FLAGS]
    units = [(s, ["-x", "c++"]) for s in sorted(glob.glob(os.path.join(build_emu.CSRC, "kv", "*.hip")))]
    units += [(os.path.join(EMU, "emu_rt.cpp"), []), (os.path.join(HERE, "emu_kv_driver.cpp"), [])]

    def cc(unit):
        src, lang = unit
        obj = os.path.join(out, os.path.basename(src) + ".o")
        subprocess.run([cxx, *flags, *lang, "-c", src, "-o", obj], check=True, capture_output=True)
        return obj

    with ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(cc, units))
    exe = os.path.join(out, "emu_kv_driver")
    subprocess.run([cxx, *flags, *objs, "-o", exe], check=True, capture_output=True)
    return exe


if __name__ == "__main__":
    print(build())
