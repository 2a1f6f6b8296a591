"""The host code of the language side (rotary axes, windowed attention, the cross entropy over a vocabulary, blocks with these) under AddressSanitizer and
UndefinedBehaviorSanitizer, against stand-in launchers that touch what the kernels touch (tests/host_sanitize/).  Host only: no GPU code is built or run."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2407_20761_amd as ob
from test_host_sanitizers import CSRC, HERE

BATCHES = [[1], [5, 1, 64], [1100], [5000, 30, 2500, 4097, 4096], [20] * 300 + [200] * 70]


def _segments(lens):
    s = ob.Segments(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=None)
    s.c.cu_dev = 0x1000
    return s


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"), reason="needs g++ and the ROCm headers")
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    # (one stand-in for the row gather: that of the language side)
    stubs = tmp_path / "stubs.cpp"
    text = open(os.path.join(HERE, "stubs.cpp")).read().replace("../../", os.path.dirname(os.path.dirname(HERE)) + "/")
    lines = [l for l in text.splitlines() if not l.startswith("void launch_rows_gather(")]
    assert len(lines) == len(text.splitlines()) - 1
    stubs.write_text("\n".join(lines))
    exe = str(tmp_path / "host_sanitize")
    srcs = [str(stubs)] + [os.path.join(HERE, f) for f in ("language_driver.cpp", "language_stubs.cpp")] + \
           [os.path.join(CSRC, f) for f in ("gemm_plan.cpp", "attention_plan.cpp", "api.cpp", "rotary_axes_api.cpp", "window_api.cpp", "block_attn_api.cpp", "lm_loss_api.cpp")]
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           *srcs, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "all checks passed" in r.stdout
    # the build under the sanitizers lays its buffers out as the shipped library does
    sizes = [line.split() for line in r.stdout.splitlines() if line.startswith(("loss", "window", "attn"))]
    assert len(sizes) == 10 + 60 + 15
    for kind, *v in sizes:
        v = [int(t) for t in v]
        if kind == "loss":
            assert ob.ob_lm_loss_workspace_bytes(ob.make_lm_loss_desc(v[0], v[1]), v[2]) == v[3]
        elif kind == "window":
            seg = _segments(BATCHES[v[0]])
            assert ob.ob_varlen_attn_window_bwd_plan(seg, v[1], 2, 64, v[2], 33)[2] == v[3]
            assert ob.ob_varlen_attn_window_bwd_workspace_bytes(seg, v[1], 2, 64, v[2], 33) == v[4]
        else:
            desc = ob.ob_block_desc(128, 8, 1, 64, 128, ob.OB_RMSNORM, ob.OB_SWIGLU, ob.OB_MASK_SEG_CAUSAL, ob.OB_BF16, 0, 1e4, 1e-5, 0)
            lens = {9: [9], 1700: [1700], 2341: [40, 1, 2300]}[v[2]]
            assert ob.ob_block_attn_workspace_bytes(desc, ob.BlockAttn(v[0], v[1]), _segments(lens)) == v[3]
