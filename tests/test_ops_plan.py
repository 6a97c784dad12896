"""CPU check of the rule by which the norm's gradient reads its inputs: by the bytes that it has of them."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_22932_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_inputs_past_the_caches_are_streamed(tmp_path):
    exe = str(tmp_path / "ops_plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", CSRC, "-I", "/opt/rocm/include", "-o", exe,
                    os.path.join(HERE, "ops_plan.cpp")], check=True)
    d, cached = 4096, 32 << 20
    calls, want = [], []
    for h_bf16 in (0, 1):
        for dres in (0, 1):
            row = d * (2 + (2 if h_bf16 else 4) * (1 + dres))           # dy is bf16
            for T in (1, cached // row, cached // row + 1, 1 << 18):
                calls.append(f"{T} {d} {h_bf16} {dres}\n")
                want.append(int(T * row > cached))
    out = subprocess.run([exe], input="".join(calls), capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == want
