"""The rules on sizes and strides by which the attention operators choose their kernels, as host code under AddressSanitizer and UBSan."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1202_3173_b200", "csrc")


def test_rules(tmp_path):
    cuda = "/usr/local/cuda/include"
    if not shutil.which("g++") or not os.path.isdir(cuda):
        pytest.skip("needs g++ and the CUDA headers")
    exe = str(tmp_path / "attention_rules")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-I", cuda,
                           os.path.join(ROOT, "tests", "native", "attention_rules.cpp"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-4000:]
    status, checks = out.stdout.split()
    assert status == "ok" and int(checks) > 500
