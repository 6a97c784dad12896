"""CPU check of the arithmetic behind the E4M3 codes: the kernels' own functions against IEEE results."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_22932_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("program", ["ops_codes", "ops_root"])
def test_codes_arithmetic(tmp_path, program):
    exe = str(tmp_path / program)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fopenmp", "-ffp-contract=off", "-I", CSRC, "-o", exe,
                    os.path.join(HERE, program + ".cpp"), "-lm"], check=True)
    env = dict(os.environ)
    env.setdefault("OMP_NUM_THREADS", str(min(8, os.cpu_count() or 1)))
    out = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600).stdout.split()
    assert len(out) >= 4 and len(out) % 2 == 0, out
    assert not any(int(n) for n in out[1::2]), out
