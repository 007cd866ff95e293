"""A row's walk over its edges (edge_steps.hpp, the loop of the mean over the
microscaled store) built for the CPU: rows of up to 2^31 - 1 edges end."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_edge_once(tmp_path):
    exe = str(tmp_path / "edge_steps_main")
    native = os.path.join(ROOT, "tests", "native")
    subprocess.check_call(["g++", "-O2", "-std=c++20", "-Wall", "-I" + os.path.join(native, "hip_cpu"),
                           "-I" + os.path.join(ROOT, "paper_2010_05337_amd", "csrc"),
                           os.path.join(native, "edge_steps_main.cpp"), "-o", exe])
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=240)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout
