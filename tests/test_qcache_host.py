"""Host side of the cache held in 8 bits: its layout, what can be rewound, plans and refusals, none of which needs a GPU."""
import ctypes
import os
import subprocess

import pytest

import paper_2605_12471_amd as kv
from paper_2605_12471_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def config(**kw):
    cfg = binding.make_config(2, 8, 2, 128, 64, 1000, kv.KVFOLD_BF16)
    for name, value in kw.items():
        setattr(cfg, name, value)
    return cfg


def test_layout_rewinding_and_plans_under_the_sanitizers(tmp_path):
    exe = str(tmp_path / "qcache_model")
    csrc = os.path.join(ROOT, "paper_2605_12471_amd", "csrc")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g"]
    subprocess.run(["g++", "-std=c++17", "-O2", *san, os.path.join(ROOT, "tests", "qcache_model_main.cpp"), os.path.join(csrc, "kvfold_plan.cpp"),
                    os.path.join(csrc, "qcache_plan.cpp"), "-lm", "-pthread", "-o", exe], check=True)
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "ok:" in r.stdout


def test_bytes_are_about_half_of_the_bf16_caches():
    cfg = binding.make_config(32, 32, 8, 128, 256, 131072, kv.KVFOLD_BF16)
    codes, scales, ring = 2 * 8 * 131072 * 128, 8 * 2048 * 8, 2 * 8 * 2 * 64 * 128 * 2
    assert kv.kvfold_qcache_bytes_required(cfg) == 32 * (codes + scales + ring)
    assert kv.kvfold_qcache_bytes_required(cfg) < 0.503 * kv.kvfold_cache_bytes_required(cfg)
    assert kv.kvfold_qcache_bytes_required(config(capacity_tokens=1, chunk_tokens=1)) == 2 * (2 * 2 * 64 * 128 + 256 + 2 * 2 * 2 * 64 * 128 * 2)


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=8), -1), (dict(n_layers=0), -1), (dict(chunk_tokens=2000), -1), (dict(softmax_scale=float("nan")), -1), (dict(kv_buffer=0x1001), -1),
    (dict(dtype=kv.KVFOLD_F32), -5), (dict(dtype=2), -5), (dict(head_dim=96), -5), (dict(n_q_heads=7), -5), (dict(capacity_tokens=1 << 31), -5),
    (dict(kv_buffer=0x10000, kv_buffer_bytes=1000), -6),
])
def test_create_refuses_before_touching_the_gpu(change, status):
    cfg = config(**change)
    rc, h = kv.kvfold_qcache_create(cfg)
    assert rc == status and h is None
    assert status == -6 or kv.kvfold_qcache_bytes_required(cfg) == 0


def test_null_handles():
    assert kv.load_library().kvfold_qcache_create(None, None) == -1
    assert kv.kvfold_qcache_create(None)[0] == -1
    assert kv.kvfold_qcache_destroy(None) == 0
    assert kv.kvfold_qcache_length(None, 0) == -1
    assert kv.kvfold_qcache_truncate(None, 0, 0) == -1
    assert kv.kvfold_qcache_step(None, 0, 16, 16, 16, 1, 0, None, None, 16) == -1
    assert kv.kvfold_qcache_append(None, 0, 16, 16, 8, 8, 1, 0) == -1
    assert kv.kvfold_qcache_read(None, 0, 0, 1, 16, 16) == -1
    assert kv.kvfold_qcache_bytes_required(config(n_layers=0)) == 0
