"""The package without its extension: what does not need it still works, what does says what is missing."""
import os
import shutil
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
PKG = ROOT / "paper_2506_23906_b200"

USE = """
import torch
import paper_2506_23906_b200 as mmv
assert mmv.workspace_bytes(mmv.OP_SEG_SCAN, mmv.F16_TO_F32, mmv.SEG_FLAGS_U8, 1000) > 0 and mmv.status_string(0)
x = torch.zeros(2, 1, 8, dtype=torch.bfloat16)
for _ in range(2):
    try:
        mmv.linear_attention_step(x, x, x, torch.zeros(1), torch.zeros(2, 1, 8, 8))
    except ImportError as e:
        print("refused:", e)
"""


@pytest.mark.parametrize("extension", ["missing", "of another build"])
def test_segmented_operators_do_not_need_the_extension(tmp_path, extension):
    pytest.importorskip("torch")
    if not (PKG / "libmmv.so").exists():
        pytest.skip("not built")
    pkg = tmp_path / PKG.name
    pkg.mkdir()
    shutil.copy(PKG / "__init__.py", pkg)
    os.symlink(PKG / "libmmv.so", pkg / "libmmv.so")
    if extension != "missing":
        (pkg / "_serve.so").write_bytes(b"no library at all")
    run = subprocess.run([sys.executable, "-c", USE], cwd=tmp_path, env=dict(os.environ, PYTHONPATH=str(tmp_path)), capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr
    assert run.stdout.count("refused:") == 2 and "_serve.so" in run.stdout
