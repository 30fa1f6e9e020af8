"""The bookkeeping of attention's rings of bulk copies (csrc/ring.cuh), compiled for the host."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_no_copy_outlives_a_wait_that_ran_out(tmp_path):
    program = str(tmp_path / "ring_model")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-o", program, os.path.join(HERE, "ring_model.cpp")], check=True)
    res = subprocess.run([program], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
    assert int(res.stdout) > 10000
