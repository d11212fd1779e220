"""Which forward kernel of the norm a row length takes is decided on its shared memory in 64 bits: no length that the
call accepts passes for one that fits.  The size is compiled from the library's own header and compared
with the same sum in Python's whole numbers."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DIMS = sorted({1, 7, 128, 129, 4001, 45504, 45505, 45568, 45569, 51200, 51201, 1 << 20, (1 << 31) - 1}
              | {d + o for d in (1 << 30, 954437184, 954437185, 1908874368, 1431655765) for o in (-1, 0, 1, 128, 45000, 51000)})


@pytest.mark.skipif(shutil.which("g++") is None or shutil.which("nvcc") is None, reason="no compiler")
def test_bytes_of_a_row_do_not_wrap(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('#include <cstdio>\n#include "mx_launch.h"\nint main() {\n  const long long dims[] = {' + ", ".join(f"{d}LL" for d in DIMS) +
                   '};\n  for (long long d : dims)\n    for (int bf16 = 0; bf16 < 2; ++bf16)\n'
                   '      std::printf("%llu %d\\n", (unsigned long long)mx::norm_row_bytes(bf16, d), mx::norm_row_bytes(bf16, d) <= mx::kNormRowBytes);\n}\n')
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc")))), "include")
    subprocess.check_call(["g++", "-std=c++17", str(src), "-o", str(exe), "-isystem", cuda, "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2310_10537_b200", "csrc")])
    lines = iter(subprocess.check_output([str(exe)], text=True).split("\n"))
    for d in DIMS:
        for bf16 in (False, True):
            padded = -(-d // 128) * 128
            want = 4 * (padded + padded // 8 if bf16 else padded)
            assert next(lines).split() == [str(want), str(int(want <= 200 * 1024))], (d, bf16)
