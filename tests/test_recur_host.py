"""The recurrence's arithmetic that host and device share, checked on the host (csrc/host_check_recur_main.cpp)."""
import subprocess

from paper_2312_17241_amd import build


def test_arithmetic_shared_by_host_and_device():
    res = subprocess.run([build.build_host_recur()], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
