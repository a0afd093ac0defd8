"""The checks of vectors of ciphertexts at equal distances (host build of the same header)."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_no_accepted_stride_passes_64_bits_and_layouts_in_use_are_accepted(tmp_path):
    exe = str(tmp_path / "ctarray_check")
    subprocess.run(["g++", "-O1", "-std=c++17", "-o", exe, os.path.join(HERE, "ctarray_check.cpp")], check=True)
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
