"""Which tokens the sequences of a batch have, on the host, under the sanitizers."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tokens_of_sequences_under_the_sanitizers(tmp_path):
    exe = str(tmp_path / "pcache_tokens")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g"]
    subprocess.run(["g++", "-std=c++17", "-O2", *san, os.path.join(ROOT, "tests", "pcache_tokens_main.cpp"), "-pthread", "-o", exe], check=True)
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "ok:" in r.stdout
