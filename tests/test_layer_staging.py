"""CPU-only: the offsets by which products and prompt attention read memory, at every ragged end."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_nothing_is_read_beyond_an_operand(tmp_path):
    exe = tmp_path / "places"
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2412_04788_amd", "csrc"),
                           os.path.join(ROOT, "tests", "staging_places.cpp"), "-o", str(exe)])
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
    assert int(run.stdout) > 1_000_000
