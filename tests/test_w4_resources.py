"""The streaming 4-bit kernels' registers and LDS, as the compiler reports them, against the number of
workgroups per CU that the choice of K parts counts on (CPU only: hipcc cross-compiles)."""
import os
import re
import subprocess

from paper_2608_14385_amd import build

LDS, REGISTERS = 160 << 10, 512   # of a CU, and of a SIMD for each of a wave's 64 lanes


def compiled(tmp_path):
    """{template arguments: (registers, LDS)} of w4_stream_kernel's instantiations."""
    cmd = [build._hipcc(), *build.HIPCC_FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage",
           "-c", os.path.join(build.CSRC, "w4.hip"), "-o", str(tmp_path / "w4.o")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found, name = {}, None
    for line in r.stderr.splitlines():
        if m := re.search(r"Function Name: (\S+)", line):
            m = re.search(r"w4_stream_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELb([01])ELb([01])E", m[1])
            name = tuple(map(int, m.groups())) if m else None
            regs = 0
        elif m := re.search(r" (VGPRs|AGPRs): (\d+)", line):
            regs = (regs + 3) // 4 * 4 + int(m[2])   # accumulation registers follow at the next four
        elif (m := re.search(r"LDS Size.*: (\d+)", line)) and name:
            found[name] = regs, int(m[1])
    return found


def test_resident_workgroups(tmp_path):
    kernels = compiled(tmp_path)
    assert len(kernels) >= 20, kernels
    src = ['#include "ops.h"']
    for (mats, nr, ntt, g32, _, wide), (regs, lds) in kernels.items():
        resident = min(REGISTERS // ((regs + 7) // 8 * 8), LDS // lds)   # registers are given out by eight
        src.append(f"static_assert(deamoe::stream_resident({mats}, {nr}, {ntt}, {32 * g32}, {wide}) == {resident}, "
                   f'"{mats} {nr} {ntt} {g32} {wide}: {regs} registers, {lds} bytes");')
    (tmp_path / "check.hip").write_text("\n".join(src) + "\n")
    r = subprocess.run([build._hipcc(), *build.HIPCC_FLAGS, "-I", build.CSRC, "-fsyntax-only", str(tmp_path / "check.hip")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
