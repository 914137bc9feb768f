"""The package without the binding module of the paged and sampling calls: the other calls do not need it."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = "paper_2609_34538_gb300"

SCRIPT = f"""
import torch, {PACKAGE} as das
assert das.status_string(0) and das.wave_widths(9, 3, 2)
assert das.LIB.das_greedy_accept(None, None, 1, 1, 1, None, None, None, None) == das.DAS_ERR_INVALID_ARG
t = torch.zeros(1, dtype=torch.int32)
try:
    das.das_page_assign(t, t, t, t, t, t, t)
except ImportError as e:
    print("refused:", e)
"""


@pytest.mark.parametrize("left", ["nothing", "a file that is no library"])
def test_older_calls_do_not_need_the_binding_module(tmp_path, left):
    src = os.path.join(ROOT, PACKAGE)
    dst = tmp_path / PACKAGE
    dst.mkdir()
    for name in os.listdir(src):
        if name.endswith(".py") or name == "libdas.so":
            shutil.copy(os.path.join(src, name), dst / name)
    if left != "nothing":
        (dst / "_calls.so").write_bytes(b"no library")
    r = subprocess.run([sys.executable, "-c", SCRIPT], cwd=tmp_path, capture_output=True, text=True, timeout=300,
                       env={**os.environ, "PYTHONPATH": str(tmp_path)})
    assert r.returncode == 0, r.stderr
    assert "refused:" in r.stdout and "_calls.so" in r.stdout
