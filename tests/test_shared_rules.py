"""The rules by which the append's workgroups share the ring and the eviction's wait for one another, from the headers that the kernels are built with."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rules_under_the_sanitizers(tmp_path):
    exe = str(tmp_path / "shared_rules")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g"]
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", *san, os.path.join(ROOT, "tests", "shared_rules_main.cpp"), "-o", exe], check=True)
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "ok:" in r.stdout
