"""The fields of mx_route_t that the gradient does not use may hold anything: no call ends the process.

Each call runs in a process of its own that sees no GPU, so that arguments which pass every check end in
MX_ERR_CUDA at the launch."""
import os
import subprocess
import sys

import pytest

import paper_2310_10537_b200 as mx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALL = """
import ctypes, sys
import numpy as np
sys.path.insert(0, sys.argv[1])
import paper_2310_10537_b200 as mx
groups, topk_groups, group_score, shift = map(int, sys.argv[2:])
buf = np.zeros(1 << 14, np.uint8)
p = buf.ctypes.data + (-buf.ctypes.data) % 256
r = mx.binding.mx_route_t(2, 0, groups, topk_groups, group_score, 1, 1.0)
o = mx.binding.mx_opts_t(mx.MX_F32, mx.MX_SCALES_SWIZZLED, None, 0)
print(mx.lib().mx_route_backward(p, p, p, 4, 16, ctypes.byref(r), p + shift, ctypes.byref(o)))
"""


@pytest.mark.parametrize("groups,topk_groups,group_score", [(32, 1, 0), (17, 9, 7), (0, 0, 0), (-1, -1, -1), (1, 1, 0)])
def test_backward_ignores_the_groups(groups, topk_groups, group_score):
    for shift, want in ((4, mx.MX_ERR_ALIGN), (0, mx.MX_ERR_CUDA)):
        p = subprocess.run([sys.executable, "-c", CALL, ROOT, *map(str, (groups, topk_groups, group_score, shift))], capture_output=True,
                           text=True, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
        assert p.returncode == 0 and int(p.stdout) == want, (p.returncode, p.stdout, p.stderr)
