"""Host side of the cache in pages: refusals, bytes, plans, and the reference's own rules, none of which needs a GPU."""
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2605_12471_amd as kv
import pcache_ref as R
from paper_2605_12471_amd import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def config(**kw):
    cfg = binding.make_pconfig(2, 8, 2, 128, 64, 1000, kv.KVFOLD_BF16)
    for name, value in kw.items():
        setattr(cfg, name, value)
    return cfg


def test_refusals_sequences_and_plans_under_the_sanitizers(tmp_path):
    exe = str(tmp_path / "pcache_model")
    csrc = os.path.join(ROOT, "paper_2605_12471_amd", "csrc")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g"]
    subprocess.run(["g++", "-std=c++17", "-O2", *san, os.path.join(ROOT, "tests", "pcache_model_main.cpp"), os.path.join(csrc, "kvfold_plan.cpp"),
                    os.path.join(csrc, "pcache_plan.cpp"), "-lm", "-pthread", "-o", exe], check=True)
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "ok:" in r.stdout


def test_bytes():
    assert kv.kvfold_pcache_bytes_required(config()) == 2 * 2 * 1000 * 2 * 64 * 128 * 2
    assert kv.kvfold_pcache_bytes_required(config(dtype=kv.KVFOLD_F32, page_tokens=16)) == 2 * 2 * 1000 * 2 * 16 * 128 * 4


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=8), -1), (dict(n_layers=0), -1), (dict(n_pages=0), -1), (dict(n_pages=-3), -1), (dict(page_tokens=0), -1), (dict(device=-1), -1),
    (dict(softmax_scale=float("nan")), -1), (dict(softmax_scale=float("inf")), -1), (dict(softmax_scale=-0.5), -1), (dict(kv_buffer=0x1001), -1), (dict(dtype=2), -5),
    (dict(head_dim=96), -5), (dict(head_dim=256), -5), (dict(n_q_heads=7), -5), (dict(page_tokens=48), -5), (dict(page_tokens=8), -5), (dict(page_tokens=512), -5),
    (dict(n_pages=1 << 26), -5), (dict(n_layers=(1 << 31) - 1, n_pages=1 << 24, n_kv_heads=32000, n_q_heads=32000), -5),
    (dict(kv_buffer=0x10000, kv_buffer_bytes=1000), -6)])
def test_create_refuses_before_touching_the_gpu(change, status):
    cfg = config(**change)
    rc, h = kv.kvfold_pcache_create(cfg)
    assert rc == status and h is None
    assert status == -6 or kv.kvfold_pcache_bytes_required(cfg) == 0


def test_null_handles():
    lib, b = kv.load_library(), binding.make_batch(1, 1, 1, 1)
    assert lib.kvfold_pcache_create(None, None) == -1
    assert kv.kvfold_pcache_create(None)[0] == -1
    assert kv.kvfold_pcache_destroy(None) == 0
    assert kv.kvfold_pcache_view(None, 0)[0] == -1
    assert kv.kvfold_pcache_workspace_bytes(None, b) == 0
    assert lib.kvfold_pcache_step(None, 0, b, 16, 16, 16, 16, None, 256, 1 << 20, None) == -1
    assert lib.kvfold_pcache_append(None, 0, 16, 16, 0, 16, 1, None) == -1
    assert lib.kvfold_pcache_assign(None, 1, 16, 16, 16, 16, 16, 1, 16, 16, 16, 16, 1, 16, 16, None) == -1
    assert kv.kvfold_pcache_bytes_required(config(n_layers=0)) == 0


def test_the_reference_itself():
    """A plain softmax in 64 bits beside torch's, causal and with rows that see nothing; the places of a small batch by hand."""
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(shape, generator=g, dtype=torch.float64) for shape in ((3, 4, 8), (7, 2, 8), (7, 2, 8)))
    seen = np.arange(7)[None, :] <= 4 + np.arange(3)[:, None]
    out, lse, mean_abs, span = R.attend(q, k, v, seen, 0.3)
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), *(t.repeat_interleave(2, 1).transpose(0, 1) for t in (k, v)), attn_mask=torch.tensor(seen),
                                                            scale=0.3).transpose(0, 1)
    # (two evaluations in 64 bits of sums of some ten terms of order one: 2^-53 a rounding, well below a hundred of them)
    assert np.abs(out - want.numpy()).max() < 100 * 2.0 ** -53 * 8 and (mean_abs >= np.abs(out) - 1e-12).all() and (span > 0).all()
    logits = torch.einsum("nhd,lhd->hnl", q, k.repeat_interleave(2, 1)) * 0.3
    assert np.abs(lse - torch.logsumexp(logits.masked_fill(~torch.tensor(seen), -torch.inf), -1).numpy()).max() < 1e-13
    seen[1] = False
    out, lse, _, _ = R.attend(q, k, v, seen, 0.3)
    assert (out[1] == 0).all() and np.isneginf(lse[:, 1]).all() and np.isfinite(lse[:, [0, 2]]).all()
    assert R.assign([3, 0, 16], [1, 17, 1], [9, 8, 7, 6], 4, [[1, -1], [-1, -1], [2, -1]], 16, 21) == (
        [[1, -1], [6, 7], [2, 8]], [4, 17, 17], [0, 1, 18, 19], [19] + list(range(96, 112)) + [112, 128, -1, -1], [3] + list(range(17)) + [16, -1, -1], 1, 0)


def test_what_matrix_instructions_written_by_hand_read_is_there(tmp_path):
    """attn_prompt_kernel's matrix instructions are asm, so that the compiler adds no wait states in front of them: in its machine code no register that one reads is written by a
    vector instruction among the two before it."""
    asm = str(tmp_path / "attn_prompt.s")
    flags = [f for f in build.HIPCC_FLAGS if not f.startswith("-Rpass")]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, "attn_prompt.hip"), "-o", asm],
                   check=True, capture_output=True)
    kernels = re.findall(r"^(_ZN6kvfold18attn_prompt_kernel\w+):(.*?)s_endpgm", open(asm).read(), re.S | re.M)
    assert len(kernels) == 2
    for name, text in kernels:
        ins = [line.strip() for line in text.split("\n") if line.startswith("\t") and not line.strip().startswith((";", "."))]
        matrix = [j for j, line in enumerate(ins) if line.startswith("v_mfma")]
        assert len(matrix) > 100
        for j in matrix:
            reads = re.findall(r"([av])\[(\d+):(\d+)\]", ins[j])[1:]
            states = 0
            for line in ins[max(0, j - 5):j][::-1]:
                if states >= 2:
                    break
                write = re.match(r"(v_\w+) ([av])(?:(\d+)|\[(\d+):(\d+)\])", line)
                if write and not line.startswith(("v_mfma", "v_cmp")):
                    low, high = int(write[3] or write[4]), int(write[3] or write[5])
                    assert not any(f == write[2] and int(a) <= high and low <= int(b) for f, a, b in reads), (name, line, ins[j])
                nop = re.match(r"s_nop (\d+)", line)
                states += int(nop[1]) + 1 if nop else 0 if line.startswith("s_waitcnt") else 1
