"""Host side of the weights and the eviction: the order in which rows are moved in place, the workspace, refusals, none of which needs a GPU."""
import os
import subprocess

import paper_2605_12471_amd as kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_moving_in_place_under_the_sanitizers(tmp_path):
    exe = str(tmp_path / "evict_model")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g"]
    subprocess.run(["g++", "-std=c++17", "-O1", *san, os.path.join(ROOT, "tests", "evict_model_main.cpp"), "-o", exe], check=True)
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "ok:" in r.stdout


def test_null_handles():
    assert kv.kvfold_cache_weigh(None, 0, 16, 1, None, None, 16, 16) == -1
    assert kv.kvfold_evict_workspace_bytes(None, 10) == 0
    assert kv.kvfold_cache_evict(None, 0, 16, 1, 0, 0, None, 0, None, None, 16, 1000) == -1
