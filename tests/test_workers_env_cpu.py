"""Threads that outlive a call and a caller that changes its environment meanwhile (tests/native/env_cpu.cpp)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2401_14351_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
@pytest.mark.parametrize("keep", [None, "0", "3"])
def test_environment_may_change_between_calls(tmp_path, keep):
    exe = tmp_path / "env_cpu"
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{ROOT}/include", f"-I{CSRC}", os.path.join(ROOT, "tests", "native", "env_cpu.cpp"),
                    os.path.join(CSRC, "common.cpp"), os.path.join(CSRC, "workers.cpp"), "-o", str(exe), "-lpthread", "-ldl"], check=True)
    env = {k: v for k, v in os.environ.items() if k != "SLLM_IDLE_WORKERS"}
    if keep is not None:
        env["SLLM_IDLE_WORKERS"] = keep
    for _ in range(2):
        r = subprocess.run([str(exe), "3000"], capture_output=True, text=True, env=env, timeout=120)
        assert r.returncode == 0, (r.returncode, r.stderr)
        idle = int(r.stdout.split()[1])
        assert idle <= (64 if keep is None else int(keep))
