"""Row operators on the GPU at the edges of what they accept, against their
64-bit definitions: empty batches, logits far from 0, ties behind ragged ends,
rows and teachers without a distribution, narrow ids.  Tolerances are those of
test_rows_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import ifvs_rows_oracle as R
from tests._gpu_util import say
from tests.test_rows_gpu import (HALF, INF, TINY, TYPES, U, _check_distill, _check_log_probs, _close, _gen, _np,
                                 _row_view, _teacher)

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


def _far_rows(dtype, cols, n, seed):
    """Rows with finite masks far below 0 (whole rows, a stretch that fills
    wavefronts and chunks, every other column, all columns but one), rows far
    from 0 on either side and rows of large logits of both signs.  fp16 holds
    what it can (65504)."""
    masks = [-1e9, -1e10, -1e12, -1e20, -1e30] if dtype != torch.float16 else [-6e4, -6.5e4]
    x = _row_view(n, cols, dtype, _gen(seed))
    i = 0
    for m in masks:
        x[i] = m
        x[i + 1, cols // 8:cols - cols // 8] = m
        x[i + 2, ::2] = m
        x[i + 3, :] = m
        x[i + 3, cols // 3] = 0.5
        i += 4
    for far in (1e10, -3e15) if dtype != torch.float16 else (6e4, -3e4):
        x[i] = far
        x[i + 1] = x[i + 1].float() * (abs(far) / 16.0)
        i += 2
    return x, i


FAR_ROWS = 24
# 1 / tau large takes ordinary logits as far (fp16 masks reach 2^30 at 1e-4)
FAR_TAUS = [1.0, 1e-4, 1e-6, 1e-9]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tau", FAR_TAUS)
@pytest.mark.parametrize("cols", [50, 3001, 40001])
def test_log_probs_far_from_zero(B, dtype, tau, cols):
    say(f"[far logprobs] {dtype} tau={tau} cols={cols}")
    x, _ = _far_rows(dtype, cols, FAR_ROWS, cols)
    given = torch.tensor([[0, cols // 2, cols - 1, -1, cols // 3]], device="cuda",
                         dtype=torch.int32).repeat(FAR_ROWS, 1)
    _check_log_probs(B, x, tau, None, given, 12)


def _check_far_distill(B, x, ids, t, tau, lse, weight):
    """The bounds of test_rows_gpu.py's check, but the other columns' shares of
    the rest are taken from their logits' differences: far below the row's
    maximum their q is 0 in 64 bits too, while the rest's gradient
    -weight tau P q_v / Q is not.  With zo = (largest other - x) / tau a share
    2^(x c - b) / S is off by u (3 zo + 6) (exponent and power), S by
    u (3 E[zo] + 132), its product with the constant and the difference from
    tau q by u each."""
    loss, grad = B.distill_loss(x, ids, t, tau, lse, weight)
    only, _ = B.distill_loss(x, ids, t, tau, lse, weight, want_grad=False)
    mine = x.clone()
    loss2, grad2 = B.distill_loss(mine, ids, t, tau, lse, weight)
    loss3, grad3 = B.distill_loss(mine, ids, t, tau, lse, weight, grad_out=mine)
    torch.cuda.synchronize()
    bits = lambda a: a.contiguous().view(torch.int32 if a.dtype == torch.float32 else torch.int16)
    assert torch.equal(bits(loss), bits(only)) and torch.equal(bits(loss2), bits(loss3))
    assert torch.equal(bits(grad2), bits(grad3)), "the gradient in place differs"
    x64, t64, at, wt = _np(x), _np(t), _np(ids), _np(weight)
    tau = float(np.float32(tau))
    w_loss, w_grad = R.distill(x64, at, t64, tau, None if lse is None else _np(lse), wt)
    n, cols = x64.shape
    loss_tol, grad_tol = np.zeros(n), np.zeros((n, cols))
    for i in range(n):
        lq = R.log_softmax(x64[i], tau)
        if lq is None:
            continue
        z = (x64[i].max() - x64[i]) / tau
        q = np.exp(lq)
        lse_tol = U * (3 * (q[q > 0] * z[q > 0]).sum() + 132)
        lp = R.log_softmax(t64[i], tau) if lse is None else t64[i] / tau - float(lse[i])
        p = np.exp(lp)
        target = np.zeros(cols)
        np.add.at(target, at[i], p)
        loss_tol[i] = (p * (lse_tol + 2 * U * np.where(np.isfinite(z[at[i]]), z[at[i]], 0))).sum()
        rel = np.where(q > 0, lse_tol + U * (3 * np.where(q > 0, z, 0) + 6), 0)
        tol = q * rel + U * (q + target)
        others = np.isfinite(x64[i])
        others[at[i]] = False
        left = max(0.0, 1 - p.sum())
        if lse is not None and others.any() and left > 0:
            zo = z[others] - z[others].min()
            qo = np.exp(-zo) / np.exp(-zo).sum()
            rest_tol = U * (3 * (qo * zo).sum() + 132)
            loss_tol[i] += left * (lse_tol + rest_tol + 4 * U * z[others].min())
            tol[others] += left * qo * (rest_tol + U * (3 * zo + 8))
        # below fp32's normal range (tau^2 may be 1e-75) rounding costs up to 2^-126, as for gradients
        loss_tol[i] = tau * tau * loss_tol[i] + U * abs(np.nan_to_num(w_loss[i], posinf=0)) + 1e-12 * tau * tau \
            + TINY[torch.float32]
        grad_tol[i] = wt[i] * tau * tol + (HALF[x.dtype] * (1 + 1e-3) + 2 * U) * np.abs(w_grad[i]) + TINY[x.dtype]
    _close(_np(loss), w_loss, loss_tol, "loss")
    _close(_np(loss2), w_loss, loss_tol, "the copy's loss")
    _close(_np(grad), w_grad, grad_tol, "gradient")
    _close(_np(grad2), w_grad, grad_tol, "the copy's gradient")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("tau", [1.0, 1e-4, 1e-9])
@pytest.mark.parametrize("cols,n", [(50, 28), (3001, 28), (40001, 28), (40001, 131), (9001, 514)])
def test_distill_far_from_zero(B, dtype, rest, tau, cols, n):
    """The far columns are others, named ones, or both; named ones of ordinary
    size among others that are all far below."""
    say(f"[far distill] {dtype} tau={tau} cols={cols} n={n} rest={rest}")
    x, far = _far_rows(dtype, cols, n, cols)
    gen = _gen(cols + 1)
    ids = torch.rand(n, cols, generator=gen, device="cuda").topk(6, 1).indices.to(torch.int32)
    t = tau * torch.randn(n, 6, generator=gen, device="cuda")
    # a teacher that takes some half of its probability to the named columns
    lse = torch.logsumexp(t / tau, 1) + 0.7
    x[0, ids[0].long()] = torch.randn(6, generator=gen, device="cuda").to(dtype)
    if dtype != torch.float16:
        x[4, ids[4].long()] = torch.randn(6, generator=gen, device="cuda").to(dtype)
    weight = torch.rand(n, generator=gen, device="cuda") + 0.5
    _check_far_distill(B, x, ids, t, tau, lse if rest else None, weight)


@pytest.mark.parametrize("cols,n", [(50, 9), (3001, 9), (40001, 9), (40001, 131)])
def test_distill_of_teachers_far_from_zero(B, cols, n):
    """A teacher whose logits are all masked with one finite value follows a
    uniform distribution over its slots; distances of any size are teachers."""
    say(f"[far teacher] cols={cols} n={n}")
    gen = _gen(cols)
    x = _row_view(n, cols, torch.float32, gen)
    ids, t, _ = _teacher(x, 6, 1.0, gen)
    low = torch.finfo(torch.float32).min
    for i, far in enumerate((low, -1e30, -1e20, -1e17, 1e16, 3e38)):
        t[i] = far
    t[6, :3] = low
    t[7] = 1e15 + torch.arange(6, device="cuda") * 6.7e7          # steps of one fp32 unit
    _check_distill(B, x, ids, t, 1.0)
    _check_distill(B, x, ids, t, 3.0)


@pytest.mark.parametrize("cols,n", [(50, 8), (3001, 8), (40001, 8), (40001, 131)])
@pytest.mark.parametrize("rest", [False, True])
def test_distill_leaves_out_padding_rows(B, rest, cols, n):
    """Rows without a column above -inf, as a padded batch holds them, are left
    out whatever their teacher's sum is; a row with a distribution is not, and
    NaN among teacher logits shows."""
    say(f"[padding rows] cols={cols} n={n} rest={rest}")
    gen = _gen(cols)
    x = _row_view(n, cols, torch.float32, gen)
    ids, t, lse = _teacher(x, 6, 1.0, gen)
    n_valid = torch.full((n,), cols, device="cuda", dtype=torch.int32)
    n_valid[0] = n_valid[1] = 0
    lse[0], lse[1] = -INF, float("nan")
    x[2:5] = -INF
    t[2:4] = -INF
    lse[2], lse[3] = -INF, INF
    t[4, 1] = float("nan")
    lse[5] = -INF
    loss, grad = B.distill_loss(x, ids, t, 1.0, lse if rest else None, None, n_valid)
    torch.cuda.synchronize()
    assert torch.all(loss[:4] == 0) and torch.all(grad[:4] == 0)
    assert bool(torch.isnan(loss[4])) and bool(torch.isnan(loss[5])) == rest
    _check_distill(B, x, ids, t, 1.0, lse if rest else None, None, n_valid)


@pytest.mark.parametrize("wide", [torch.int8, torch.uint8, torch.int16, torch.uint16, torch.uint32, torch.int64])
def test_ids_of_any_whole_type(B, wide):
    """Ids, lengths and slots of every whole-number type name what 32-bit ones
    name (255 of uint8 is a column, not an absent slot)."""
    x = torch.randn(6, 300, generator=_gen(1), device="cuda")
    top = 256 if wide not in (torch.int8,) else 128
    ids = torch.randint(0, top, (6, 3), generator=_gen(2), device="cuda", dtype=torch.int32)
    ids[0, 0] = top - 1
    nv = torch.tensor([100, 120, 5, 77, 1, 90], device="cuda", dtype=torch.int32)
    t = torch.randn(6, 3, generator=_gen(3), device="cuda")
    ids2, nv2 = ids.to(wide), nv.to(wide)
    want = (B.embed_lookup(x, ids.clamp(max=5)), B.embed_gradient(x, ids, 300), *B.log_probs(x, ids, 4, n_valid=nv),
            *B.log_probs(x, ids, 0)[:2], *B.distill_loss(x, ids, t, n_valid=nv), *B.distill_loss(x, ids, t))
    got = (B.embed_lookup(x, ids.clamp(max=5).to(wide)), B.embed_gradient(x, ids2, 300),
           *B.log_probs(x, ids2, 4, n_valid=nv2), *B.log_probs(x, ids2, 0)[:2],
           *B.distill_loss(x, ids2, t, n_valid=nv2), *B.distill_loss(x, ids2, t))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
    if wide in (torch.int8, torch.int16, torch.int64):
        absent = torch.full((6, 1), -1, device="cuda", dtype=wide)
        assert torch.all(B.embed_lookup(x, absent) == 0) and torch.all(B.log_probs(x, absent)[0] == -INF)


@pytest.mark.parametrize("kind", ["uniform", "skew"])
@pytest.mark.parametrize("rows,dim", [(45000, 961), (8192, 2048), (300000, 33)])
def test_gradients_around_the_longest_one_launch_sort(B, rows, dim, kind):
    """One launch sorts as many slots as the clear beside it allows (one more
    for every 32 KB beyond 16384), a radix sort the next: an absent slot more
    changes nothing."""
    limit = 16384 + min(rows * dim * 4 // 32768, 16384)
    say(f"[longest one-launch sort] {rows} x {dim}, {limit} slots, {kind}")
    gen = _gen(rows)
    grad = torch.randn(limit + 1, dim, generator=gen, device="cuda")
    ids = torch.randint(-1, rows, (limit + 1, 1), generator=gen, device="cuda", dtype=torch.int32)
    if kind == "skew":
        ids[torch.rand(limit + 1, 1, generator=gen, device="cuda") < 0.3] = rows // 3
    ids[limit] = -1
    one, two = B.embed_gradient(grad[:limit], ids[:limit], rows), B.embed_gradient(grad, ids, rows)
    want = torch.zeros(rows + 1, dim, device="cuda", dtype=torch.float64)
    size = torch.zeros_like(want)
    flat = ids[:, 0].long() % (rows + 1)
    want.index_add_(0, flat, grad.double())
    size.index_add_(0, flat, grad.double().abs())
    count = torch.bincount(flat, minlength=rows + 1)[:rows, None]
    torch.cuda.synchronize()
    assert torch.equal(one.view(torch.int32), two.view(torch.int32))
    # as many fp32 additions as the row has slots, one rounding of the result
    assert torch.all((one.double() - want[:rows]).abs() <= (count + 2) * U * size[:rows])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("tau", [3e-38, 2e30, 1e38, 1.3e38, 3e38])
@pytest.mark.parametrize("cols,n", [(50, 20), (3001, 20), (40001, 20), (40001, 131)])
def test_temperatures_at_the_ends_of_fp32(B, rest, tau, cols, n):
    """Temperatures whose reciprocal is barely a number, with logits of that
    size; masks of -inf.  (tau^2 times a divergence may pass fp32's range.)"""
    say(f"[extreme tau] {tau} cols={cols} n={n} rest={rest}")
    gen = _gen(cols)
    x = _row_view(n, cols, torch.float32, gen, scale=min(tau, 5e37) if tau > 1 else 1e-37)
    x[1, ::3] = -INF
    x[2] = 0.0
    x[3] = torch.finfo(torch.float32).min
    ids = torch.rand(n, cols, generator=gen, device="cuda").topk(6, 1).indices.to(torch.int32)
    t = torch.randn(n, 6, generator=gen, device="cuda") * (5e37 if tau > 1e37 else tau)
    lse = torch.logsumexp(t / tau, 1) + 0.7
    weight = torch.rand(n, generator=gen, device="cuda")
    _check_log_probs(B, x, tau, None, ids, 12)
    _check_far_distill(B, x, ids, t, tau, lse if rest else None, weight)
