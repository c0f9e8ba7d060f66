"""Register budget of the layer norm and 8-bit kernels (CPU; compiles for gfx950): no
scratch memory, and the waves that hide their latencies.  The 8-bit layer's largest tile
holds 128 sums and 96 operands a lane of its 256 registers: what it spills are values
that a tile needs once, none in its loop over K."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_resources import CSRC, HIPCC, ROOT

SOURCES = ("norm.hip", "norm_grad.hip", "gemm_q8.hip")


def _kernels(src, tmp):
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-S", "--offload-device-only",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", os.path.join(CSRC, src), "-o", os.path.join(str(tmp), src + ".s")]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(os.path.join(str(tmp), src + ".s")) as f:
        text = f.read()
    out = {}
    for part in text.split("; -- Begin function ")[1:]:
        m = re.search(r"; ScratchSize: (\d+).*?; Occupancy: (\d+)", part, re.S)
        if m:
            out[part.split(None, 1)[0]] = (int(m.group(1)), int(m.group(2)), part)
    return out


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_no_spills(tmp_path):
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        found = dict(zip(SOURCES, ex.map(lambda s: _kernels(s, tmp_path), SOURCES)))
    counts = {"row_kernel": 0, "norm_grad_kernel": 0, "norm_grad_few_kernel": 0, "gemm_q8_pipe_kernel": 0,
              "gemm_q8_rows_kernel": 0, "gemm_q8_strip_kernel": 0}
    for kernels in found.values():
        for name, (scratch, waves, body) in kernels.items():
            for k in counts:
                counts[k] += re.search(r"\d" + k, name) is not None
            if "PipeCfgILi256ELi256E" in name:
                assert scratch <= 128 and waves == 2, (name, scratch, waves)
                # the steady loop: the block that multiplies two half stages and loads one
                blocks = re.split(r"^\.LBB\S+:", body, flags=re.M)
                loops = [b for b in blocks if b.count("v_mfma") >= 64 and "global_load_lds" in b]
                assert loops and not any("scratch_" in b for b in loops), name
            else:
                assert scratch == 0, (name, scratch)
            if "StripCfg" in name:
                assert waves >= 4, (name, waves)
            if "PipeCfgILi128ELi128E" in name or "PipeCfgILi64ELi64ELi2ELi2ELi2E" in name:
                assert waves >= 4, (name, waves)
    assert all(counts.values()), counts


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_strips_have_the_waves_they_ask_for(tmp_path):
    """A strip kernel's workgroups of four waves are as many a CU as StripCfg reckons, by the
    LDS of W's columns and by the registers: so many waves a SIMD."""
    found = 0
    for name, (scratch, waves, _) in _kernels("gemm_q8.hip", tmp_path).items():
        m = re.search(r"StripCfgILi(\d+)ELi(\d+)ELi(\d+)E", name)
        if not m:
            continue
        found += 1
        bf16, ks, tn = map(int, m.groups())
        lds = (ks + 1) // 2 * 16 * tn * 128 + 2 * 16 * tn * 4
        regs = 4 * (ks + 2 * tn) + 2 * tn * (1 if bf16 else 2) + 24
        assert scratch == 0 and waves >= min(160 * 1024 // lds, 512 // regs), (name, waves)
    assert found == 2 * 2 * 5 * 2  # types, with and without GELU, steps of K, columns
