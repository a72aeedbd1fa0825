"""The attention layers' host-side validation under the address and undefined-behaviour sanitizers (no GPU)."""
import os
import shutil

import pytest

from test_sanitizers import ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
def test_attention_validation_under_sanitizers(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    exe = str(tmp_path / "kv_san")
    cmd = [hipcc, "--cuda-host-only", "-O1", "-g", "-std=c++17", "-x", "hip", "-Xarch_host", "-fsanitize=address", "-Xarch_host",
           "-fsanitize=undefined", "-fno-omit-frame-pointer", os.path.join(ROOT, "paper_2505_14969_amd", "csrc", "api_kv.hip"),
           os.path.join(SAN, "kv_driver.cpp"), "-o", exe]
    assert "0 mismatches" in _run(cmd, exe, tmp_path)
