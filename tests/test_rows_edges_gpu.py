"""Row operators on the GPU at the edges of what they accept, against their
64-bit definitions: empty batches, logits far from 0, ties behind ragged ends,
rows and teachers without a distribution, narrow ids.  Tolerances are those of
test_rows_gpu.py."""
import pytest
import torch

from tests._gpu_util import say
from tests.test_rows_gpu import INF, TYPES, _check_distill, _check_log_probs, _gen, _row_view, _teacher

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2607_22922_amd import ifvs
    return ifvs


@pytest.mark.parametrize("rows", [(1 << 19) - 1, 1 << 19, (1 << 20) + 3])
def test_gradient_of_no_slots_clears_large_tables(B, rows):
    out = torch.full((rows, 9), 3.0, device="cuda")
    B.embed_gradient(torch.empty(0, 9, device="cuda"), torch.empty(0, 2, device="cuda", dtype=torch.int32), rows,
                     out=out)
    torch.cuda.synchronize()
    assert torch.all(out == 0)
    out.fill_(3.0)
    B.embed_gradient(torch.empty(0, 9, device="cuda"), torch.empty(0, 2, device="cuda", dtype=torch.int32), rows,
                     out=out, accumulate=True)
    torch.cuda.synchronize()
    assert torch.all(out == 3)


@pytest.mark.parametrize("cols", [1, 16385, 131072, 1 << 20])
def test_empty_batches_of_long_rows(B, cols):
    x = torch.empty(0, cols, device="cuda")
    ids = torch.empty(0, 2, device="cuda", dtype=torch.int32)
    assert [tuple(o.shape) for o in B.log_probs(x, ids, 4)] == [(0, 2), (0,), (0, 4), (0, 4)]
    loss, grad = B.distill_loss(x, ids, torch.empty(0, 2, device="cuda"))
    assert loss.shape == (0,) and grad.shape == (0, cols)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [2001, 2047, 4091, 16383, 35003, 40001])
def test_alternatives_of_ties_with_ragged_ends(B, dtype, cols):
    """Long ties behind a lower or masked start, at every alignment: a row's
    first and last elements lie outside its whole vectors."""
    say(f"[ragged ties] {dtype} cols={cols}")
    leads = [l for l in (1, 255, 256, 512, 1024, 2048, 8200, 20000) if l < cols - 1100]
    for shift in range(8):
        x = torch.zeros(2 * len(leads) * (cols + 3) + shift, device="cuda", dtype=dtype)
        x = x[shift:].view(2 * len(leads), cols + 3)[:, :cols]
        for i, lead in enumerate(leads):
            x[2 * i, :lead] = -1.0
            x[2 * i + 1, :lead] = -INF
        _check_log_probs(B, x, 1.0, None, None, 10 if shift % 2 else 32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [0, 3])
def test_alternatives_of_ties_in_ragged_chunks(B, dtype, shift):
    """The same in rows of many chunks of 16384 columns: the tie starts in a
    later round of its chunk, at the threads that hold the chunk's ends."""
    say(f"[ragged ties in chunks] {dtype} shift={shift}")
    cols = (1 << 20) - 5
    x = torch.zeros(2 * cols + shift, device="cuda", dtype=dtype)[shift:].view(2, cols)
    x[0, :30 * 16384 + 8192] = -1.0
    x[1, :47 * 16384 + 4096] = -1.0
    _check_log_probs(B, x, 1.0, None, None, 10)
