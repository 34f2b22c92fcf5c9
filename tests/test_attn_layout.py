"""Packed attention's tiles in LDS, checked lane by lane on the CPU: what each
copy instruction fills, what each fragment read takes, and their banks."""

import os
import subprocess

import pytest

from paper_2410_17243_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_attn_tile_layout(tmp_path):
    try:
        cc = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    exe = str(tmp_path / "attn_layout_check")
    r = subprocess.run([cc, *build.HIPCC_FLAGS, os.path.join(HERE, "attn_layout_check.hip"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout
