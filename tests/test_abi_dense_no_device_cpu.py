"""Calls of the dense block, its norm and mx8 on a machine without a usable GPU: an error status, not the end of the process. Each runs in
a process of its own that sees no device, with addresses that nothing reads."""
import os
import subprocess
import sys

import pytest

from paper_2609_34077_gb300 import build
from paper_2609_34077_gb300 import mcft as M

CALLS = {
    "forward": "L.mcft_ffn_forward(D, a[0], T, a[1], a[2], None, a[4], 1 << 40, None)",
    "forward with a checkpoint": "L.mcft_ffn_forward(D, a[0], T, a[1], a[2], a[3], a[4], 1 << 40, None)",
    "gradient": "L.mcft_ffn_grad(D, a[0], T, a[1], a[2], None, None, a[3], a[5], dtype, 0, a[4], 1 << 40, None)",
    "gradient from checkpoints": "L.mcft_ffn_grad(D, a[0], T, a[1], None, a[2], a[6], a[3], a[5], dtype, 0, a[4], 1 << 40, None)",
    "norm": "L.mcft_residual_rmsnorm_mx8(D, a[0], a[1], T, a[2], C.c_float(0.0), a[3], a[4], a[5], a[6], a[7], None)",
    "norm gradient": "L.mcft_rmsnorm_grad(D, a[0], None, a[1], a[2], a[3], T, a[4], a[5], a[6], 0, a[7], 1 << 40, None)",
    "mx8": "L.mcft_mx8_quantize(a[0], T, 128, 128, dtype, a[1], None)",
    "mx8 back": "L.mcft_mx8_dequantize(a[0], T, 128, dtype, a[1], 128, None)",
}


@pytest.mark.parametrize("name", CALLS)
def test_an_error_without_a_device(name):
    build.build()
    code = f"""
import ctypes as C
from paper_2609_34077_gb300 import mcft as M
L, a = M.lib(), [C.c_void_p((i + 1) << 20) for i in range(9)]
for dtype in (0, 1):
    D = C.byref(M.LayerDesc(128, 0, 0, 192, 0, 0, dtype))
    for T in (1, 40, 300, 5000):
        assert {CALLS[name]} == M.MCFT_ERR_CUDA, (dtype, T)
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=build.ROOT, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""),
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-500:]
