"""How attention on caches is launched (compiled for the host; no GPU)."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2605_08123_amd", "csrc")


def build(tmp_path, name):
    exe = str(tmp_path / name)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, "-o", exe, os.path.join(HERE, name + ".cpp")], check=True)
    return exe


def test_joins_within_32_bits_of_threads(tmp_path):
    """cache_joins.cpp: every launch of a join has fewer than 2^32 threads."""
    run = subprocess.run([build(tmp_path, "cache_joins")], capture_output=True, text=True)
    print(run.stdout)
    assert run.returncode == 0, run.stdout
