"""Where the device's status word cannot be had, a call ends there, before it launches anything that would write to it.  In a process that
sees no device, so that nothing runs anywhere."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALLS = {
    "fwd": "L.hdt_self_attn_fwd(A, A, None, 2, 100, 100, A, A, A, A, 32, 128, 1, A, A, 2, 64, dtype, 0.0, A, 1 << 24, None)",
    "bwd": "L.hdt_self_attn_bwd(A, A, None, 2, 100, 100, A, A, A, A, 32, 128, 1, A, A, A, A, A, A, A, 2, 64, dtype, 0.0, A, 1 << 24, None)",
}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("dtype", [0, 1])
def test_no_status_word(call, dtype):
    code = f"import paper_2407_08330_b200 as P; L, A, dtype = P.lib(), 0x10000, {dtype}; print({CALLS[call]}, L.hdt_last_error(), P.hdt_launch_count())"
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""}, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert r.stdout.startswith("-5 ") and "g_device_status" in r.stdout and r.stdout.split()[-1] == "0", r.stdout
