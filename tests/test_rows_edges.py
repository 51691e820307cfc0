"""Row operators at the edges of what they accept, on the CPU: workspace sizes
of empty batches, and the definitions' answers for rows without a distribution."""
import subprocess
import sys

import pytest

ROWS = [(1 << 19) - 1, 1 << 19, (1 << 31) - 2]
COLS = [1, 16384, 16385, 131072, 1 << 20]


def _run(code):
    """Code that used to end the process runs in one of its own."""
    out = subprocess.run([sys.executable, "-c", "from paper_2607_22922_amd import ifvs as B\nlib = B.lib()\n" + code],
                         capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, (out.returncode, out.stderr[-500:])
    return out.stdout


def test_gradient_workspace_of_an_empty_batch():
    out = _run(f"print([lib.ifvs_embed_workspace(r, 64, 0, bag) for r in {ROWS} for bag in (1, 16)])")
    assert out.strip() == str([0] * 6)
