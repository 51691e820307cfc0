"""Row operators at the edges of what they accept, on the CPU: workspace sizes
of empty batches, and the definitions' answers for rows without a distribution."""
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import ifvs_rows_oracle as R
from paper_2607_22922_amd import ifvs

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


@pytest.mark.parametrize("fn", ["ifvs_log_probs_workspace(0, {}, 5)", "ifvs_distill_workspace(0, {})"])
def test_row_workspaces_of_an_empty_batch(fn):
    out = _run("print([" + ", ".join("lib." + fn.format(c) for c in COLS) + "])")
    assert out.strip() == str([0] * len(COLS))


def test_empty_batches_of_long_rows_do_nothing():
    """The whole calls, with nothing to read: NULL arrays and no workspace."""
    out = _run("""
import ctypes
f = ctypes.c_float(1.0)
for cols in (16385, 131072, 1 << 20):
    print(lib.ifvs_log_probs(0, cols, None, cols, 1, None, f, None, 1, 5, None, None, None, None, None, 0, None),
          lib.ifvs_distill_loss(0, cols, None, cols, 1, None, 3, None, None, None, f, None, None, None, cols, None, 0,
                                None))
""")
    assert out.split() == ["0"] * 6


@pytest.mark.parametrize("with_lse", [False, True])
def test_definition_leaves_out_rows_without_a_distribution(with_lse):
    """A padding row's teacher has no distribution either (its logits are all
    -inf, its sum's logarithm -inf or undefined): loss and gradient stay 0.  A
    NaN among the row's present teacher logits shows, and so does an undefined
    sum beside a student that has a distribution."""
    x = np.full((5, 6), -np.inf)
    x[4] = np.arange(6)
    ids = np.tile([1, 3], (5, 1))
    t = np.array([[-np.inf, -np.inf], [-np.inf, -np.inf], [0.5, 1.0], [np.nan, 1.0], [0.5, 1.0]])
    lse = np.array([-np.inf, np.nan, np.inf, 0.0, -np.inf])
    loss, grad = R.distill(x, ids, t, teacher_lse=lse if with_lse else None)
    assert np.all(loss[:3] == 0) and np.all(grad[:3] == 0)
    assert np.isnan(loss[3]) and np.isnan(loss[4]) == with_lse


@pytest.mark.parametrize("wide,values,want", [
    (torch.int8, [-128, -1, 127], [-128, -1, 127]), (torch.uint8, [0, 255], [0, 255]),
    (torch.int16, [-32768, 32767], [-32768, 32767]), (torch.uint16, [0, 65535], [0, 65535]),
    (torch.uint32, [7, 2**32 - 1], [7, 2**31 - 1]), (torch.int64, [-2**40, 3, 2**32 + 3], [-1, 3, 2**31 - 1])])
def test_whole_numbers_become_32_bits(wide, values, want):
    """Narrow types keep their values; numbers past 32 bits stay outside."""
    t = torch.tensor(values, dtype=torch.int64).to(wide)
    got = ifvs._small_arg(t, "ids", torch.int32, (len(values),), t.device)
    assert got.dtype == torch.int32 and got.tolist() == want


@pytest.mark.parametrize("bad", [torch.float32, torch.bool, torch.complex64])
def test_other_types_are_no_ids(bad):
    t = torch.zeros(3).to(bad)
    with pytest.raises(ifvs.IfvsError):
        ifvs._small_arg(t, "ids", torch.int32, (3,), t.device)
