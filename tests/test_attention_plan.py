"""How attention's keys are shared out is plain integer logic in csrc/attention_plan.hpp: tests/attention_plan_check.cpp runs it over
lengths up to the longest, also built so that an integer that overflows ends it."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("flags", [["-O2"], ["-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all"]], ids=["plain", "undefined"])
def test_keys_are_shared_out(tmp_path, flags):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    exe = tmp_path / "attention_plan_check"
    cmd = [gxx, "-std=c++17", "-Wall", "-Wextra", *flags, os.path.join(HERE, "attention_plan_check.cpp"), "-o", str(exe)]
    built = subprocess.run(cmd, capture_output=True, text=True)
    if built.returncode != 0 and len(flags) > 1:
        pytest.skip("sanitizer runtime not available to this compiler")
    assert built.returncode == 0, built.stderr
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)       # the sanitizer runtime has to come first in the link order
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
    assert r.stdout.split()[0] == "ok"
