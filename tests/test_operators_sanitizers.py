"""Host-side sanitizer build (AddressSanitizer + UndefinedBehaviorSanitizer; CPU only, no GPU code is instrumented) of the
operators' boundary: argument checks and workspace sizes, every path that returns before a launch."""
import os
import shutil
import subprocess

import pytest

from tests.test_host_sanitizers import ENV, SAN, run


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_operators_boundary_under_sanitizers(tmp_path):
    from paper_2604_15180_amd import build as hip_build
    hip_build.build(force=False)
    objs = [os.path.join(hip_build.OBJDIR, u + ".o") for u in hip_build.UNITS if u not in ("prep", "cache", "decode_cache4")]
    assert all(os.path.exists(o) for o in objs)
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Wno-unused-command-line-argument", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    sources = [os.path.join(hip_build.CSRC, u + ".hip") for u in ("prep", "cache", "decode_cache4")] + [os.path.join(SAN, "operators_main.cpp")]
    outs = [str(tmp_path / (os.path.basename(s) + ".o")) for s in sources]
    procs = [subprocess.Popen(["hipcc"] + flags + ["-c", s, "-o", o], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
             for s, o in zip(sources, outs)]
    for pr in procs:
        _, err = pr.communicate()
        assert pr.returncode == 0, err[-4000:]
    exe = str(tmp_path / "operators_san")
    run(["hipcc", "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize"] + outs + objs + ["-o", exe])
    res = run([exe], env=ENV)
    assert res.stdout.strip().endswith("ok") and "runtime error" not in res.stderr, res.stderr[-2000:]
