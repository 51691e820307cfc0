"""The row operators on the GPU against their 64-bit definitions
(oracle/ifvs_rows_oracle.py): element types, row lengths from one column to
many, odd sizes and strides, masks, ties and rows without a distribution.

Tolerances, from the arithmetic the header promises (u = 2^-24, one fp32
rounding).  With z = (x - max) / tau an exponent is off by at most 2u |z| (the
constant log2(e) / tau) + u |z| (its multiply-add), its power of two by 2 ulp
(4u), a thread adds at most 128 powers one after another in fp32 (128u), the
rest is 64 bits: log S is off by u (3 E|z| + 132), E the mean under q.  A log
probability adds 2u |z| and its own rounding.  The result's rounding is half a
step of its type."""
import numpy as np
import pytest
import torch

from oracle import ifvs_rows_oracle as R
from tests._gpu_util import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# half of the smallest subnormal step: what rounding costs below the normal range
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}
TYPES = [torch.float32, torch.float16, torch.bfloat16]
INF = float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2607_22922_amd import ifvs
    return ifvs


def _np(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _close(got, want, tol, what):
    """|got - want| <= tol element by element; NaN and infinities in the same
    places.  Every result is fp32 or narrower: a value past fp32's largest
    (3.4e38, as the logarithm of a lowest-value mask divided by a small tau)
    rounds to infinity."""
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    want = np.where(np.abs(want) > np.finfo(np.float32).max, np.copysign(np.inf, want), want)
    tol = np.broadcast_to(tol, want.shape)
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), f"{what}: infinities differ"
    err = np.abs(got[fin] - want[fin])
    bad = err > tol[fin]
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} off, worst {float((err - tol[fin]).max()):.3e} over "
                           f"its tolerance (error {float(err[np.argmax(err - tol[fin])]):.3e}, "
                           f"value {float(want[fin][np.argmax(err - tol[fin])]):.6e})")


def _row_view(n, cols, dtype, gen, pad=0, shift=0, scale=2.5):
    """[n, cols] random rows `pad` elements apart more than needed, the first
    one `shift` elements into its buffer."""
    buf = torch.randn(n * (cols + pad) + shift, generator=gen, device="cuda") * scale
    buf = buf.to(dtype)
    return buf[shift:].view(n, cols + pad)[:, :cols]


# ------------------------------------------------------------------- embedding
def _lookup_tol(table, ids, scale, bag, dtype, want):
    size = R.embed_lookup(np.abs(table), ids, abs(scale))
    return (bag + 2) * U * size + HALF[dtype] * np.abs(want) * (1 + 1e-3) + TINY[dtype]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,n,bag,pad,shift", [
    (1, 1, 1, 1, 0, 0), (5, 3, 7, 2, 0, 0), (100, 64, 33, 1, 0, 0), (1000, 100, 257, 3, 4, 1), (50, 961, 70, 4, 3, 1),
    (4096, 384, 256, 2, 0, 0), (37, 2048, 9, 16, 8, 8), (300, 5000, 5, 1, 1, 3), (65, 257, 1000, 1, 0, 1)])
def test_embed_lookup(B, dtype, rows, dim, n, bag, pad, shift):
    say(f"[lookup] {dtype} rows={rows} dim={dim} n={n} bag={bag}")
    gen = _gen(rows + dim)
    table = _row_view(rows, dim, dtype, gen, pad, shift, 1.0)
    ids = torch.randint(-2, rows + 2, (n, bag), generator=gen, device="cuda", dtype=torch.int32)
    out = B.embed_lookup(table, ids, 1.75)
    into = torch.full((n, dim + 5), 7.0, device="cuda", dtype=dtype)
    B.embed_lookup(table, ids, 1.75, out=into[:, 2:2 + dim])
    torch.cuda.synchronize()
    t, i = _np(table), _np(ids)
    want = R.embed_lookup(t, i, 1.75)
    _close(_np(out), want, _lookup_tol(t, i, 1.75, bag, dtype, want), "lookup")
    assert torch.equal(into[:, 2:2 + dim], out)
    assert torch.all(into[:, :2] == 7) and torch.all(into[:, 2 + dim:] == 7)


@pytest.mark.parametrize("dtype,out_dtype", [(torch.float32, torch.float32), (torch.float16, torch.float16),
                                             (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                             (torch.float16, torch.float32)])
@pytest.mark.parametrize("rows,dim,n,bag,pad,shift,kind", [
    (1, 1, 1, 1, 0, 0, "any"), (5, 3, 7, 2, 0, 0, "any"), (300, 64, 33, 1, 0, 0, "any"),
    (1000, 100, 257, 3, 4, 1, "any"), (50, 961, 70, 4, 3, 1, "any"), (37, 128, 2000, 2, 0, 0, "any"),
    (3000, 40, 5000, 1, 0, 0, "one"), (200, 33, 4097, 2, 1, 1, "skew"), (70000, 8, 300, 1, 0, 0, "any"),
    (20, 16, 50, 3, 0, 0, "absent"), (9, 700, 1, 16, 0, 0, "any"), (150000, 24, 9001, 1, 0, 0, "skew"),
    (600000, 5, 300, 2, 0, 0, "any"), (600000, 9, 9001, 1, 0, 0, "skew"), (1500, 12, 70001, 2, 1, 0, "any"),
    (77, 20, 150000, 1, 0, 0, "skew"), (5000, 36, 33000, 1, 0, 0, "skew"), (3000, 6, 140001, 1, 0, 0, "one"),
    (90, 1100, 1024, 1, 0, 0, "skew"), (90, 70, 1025, 1, 1, 0, "skew"), (50, 600, 512, 2, 0, 1, "one"),
    (130000, 600, 20000, 1, 0, 0, "skew")])
def test_embed_gradient(B, dtype, out_dtype, rows, dim, n, bag, pad, shift, kind):
    say(f"[gradient] {dtype}->{out_dtype} rows={rows} dim={dim} n={n} bag={bag} {kind}")
    gen = _gen(rows + dim)
    grad = _row_view(n, dim, dtype, gen, pad, shift, 1.0)
    # past 16384 slots (32768 beside a large table) or 512K rows the sort takes several launches
    ids = torch.randint(-2, rows + 2, (n, bag), generator=gen, device="cuda", dtype=torch.int32)
    if kind == "one":
        ids[:] = rows - 1
    elif kind == "skew":                       # one row in half of the slots
        ids[torch.rand(n, bag, generator=gen, device="cuda") < 0.5] = rows // 2
    elif kind == "absent":
        ids[:] = -1
    out = B.embed_gradient(grad, ids, rows, 0.75, dtype=out_dtype)
    again = B.embed_gradient(grad, ids, rows, 0.75, dtype=out_dtype)
    base = _row_view(rows, dim, out_dtype, gen, 3, 1, 1.0)
    acc = torch.full((rows, dim + 3), 5.0, device="cuda", dtype=out_dtype)
    acc[:, :dim] = base
    B.embed_gradient(grad, ids, rows, 0.75, out=acc[:, :dim], accumulate=True, dtype=out_dtype)
    torch.cuda.synchronize()
    g, i = _np(grad), _np(ids)
    want = R.embed_gradient(g, i, rows, 0.75)
    size = R.embed_gradient(np.abs(g), i, rows, 0.75)
    count = R.embed_gradient(np.ones((n, 1)), i, rows, 1.0)
    tol = (count + 2) * U * size + HALF[out_dtype] * np.abs(want) * (1 + 1e-3) + TINY[out_dtype]
    tol = np.where(count > 0, tol, 0.0)                 # rows that nothing names are exactly 0
    _close(_np(out), want, tol, "gradient")
    assert torch.equal(out, again), "two equal calls differ"
    old = _np(base)
    tol = (count + 2) * U * size + (HALF[out_dtype] * (1 + 1e-3) + U) * np.abs(old + want) + TINY[out_dtype]
    tol = np.where(count > 0, tol, 0.0)                 # untouched rows keep their bits
    _close(_np(acc[:, :dim]), old + want, tol, "accumulated")
    assert torch.all(acc[:, dim:] == 5)


@pytest.mark.parametrize("dtype,out_dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                             (torch.float16, torch.float32)])
@pytest.mark.parametrize("rows,dim,pad", [(300, 33, 3), (5000, 520, 8), (41, 1, 1)])
def test_embed_gradient_into_strided_rows(B, dtype, out_dtype, rows, dim, pad):
    """Rows further apart than their length: cleared and written, what lies
    between them is left."""
    gen = _gen(rows)
    grad = _row_view(60, dim, dtype, gen)
    ids = torch.randint(-1, rows, (60, 2), generator=gen, device="cuda", dtype=torch.int32)
    buf = torch.full((rows, dim + pad), 9.0, device="cuda", dtype=out_dtype)
    out = buf[:, 1:1 + dim]
    assert B.embed_gradient(grad, ids, rows, 1.5, out=out) is out
    want = B.embed_gradient(grad, ids, rows, 1.5, dtype=out_dtype)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert torch.all(buf[:, :1] == 9) and torch.all(buf[:, 1 + dim:] == 9)


def test_embed_gradient_of_no_slots_clears(B):
    out = torch.full((50, 7), 3.0, device="cuda")
    B.embed_gradient(torch.empty(0, 7, device="cuda"), torch.empty(0, 2, device="cuda", dtype=torch.int32), 50, out=out)
    torch.cuda.synchronize()
    assert torch.all(out == 0)


def test_ids_beyond_32_bits_name_no_row(B):
    table = torch.randn(8, 4, device="cuda")
    ids = torch.tensor([[1 << 32, 3], [-(1 << 32) + 1, -1]], device="cuda")
    out = B.embed_lookup(table, ids)
    torch.cuda.synchronize()
    assert torch.equal(out[0], table[3]) and torch.all(out[1] == 0)


def test_offsets_past_32_bits(B):
    """A table of 2^31 + elements: the last rows are found."""
    rows, dim = (1 << 21) + 5, 1031
    table = torch.zeros(rows, dim, device="cuda", dtype=torch.bfloat16)
    table[-3:] = 1.5
    ids = torch.tensor([[rows - 1], [0], [rows - 3], [rows]], device="cuda", dtype=torch.int32)
    out = B.embed_lookup(table, ids, 2.0)
    g = torch.ones(4, dim, device="cuda", dtype=torch.bfloat16)
    B.embed_gradient(g, ids, rows, 2.0, out=table)
    torch.cuda.synchronize()
    assert torch.all(out[0] == 3) and torch.all(out[1] == 0) and torch.all(out[2] == 3) and torch.all(out[3] == 0)
    hit = torch.nonzero(table[:, -1])[:, 0]
    assert hit.tolist() == [0, rows - 3, rows - 1] and torch.all(table[hit] == 2)
    assert int(torch.count_nonzero(table[:, 0])) == 3


# --------------------------------------------------------------- log probabilities
def _row_stats(logits, tau, n_valid):
    """Per row: z = (x - max) / tau (valid, finite places), tolerance of log S."""
    n, cols = logits.shape
    z = np.zeros((n, cols))
    lse_tol = np.zeros(n)
    for i in range(n):
        m = R.row_length(n_valid, i, cols)
        lp = R.log_softmax(logits[i, :m], tau)
        if lp is None or np.isnan(lp).any():
            continue
        zi = (logits[i, :m] - logits[i, :m].max()) / tau
        q = np.exp(lp)
        live = q > 0
        lse_tol[i] = U * (3 * (q[live] * -zi[live]).sum() + 132)
        z[i, :m] = np.where(np.isneginf(zi), 0, zi)
    return z, lse_tol


def _check_log_probs(B, logits, tau=1.0, n_valid=None, given=None, n_top=0):
    out, ent, ids, top = B.log_probs(logits, given, n_top, tau, n_valid)
    again = B.log_probs(logits, given, n_top, tau, n_valid)
    torch.cuda.synchronize()
    x = _np(logits)
    nv = None if n_valid is None else _np(n_valid)
    gv = None if given is None else _np(given)
    tau = float(np.float32(tau))                 # the call takes it in 32 bits
    w_out, w_ent, w_ids, w_top = R.log_probs(x, tau, nv, gv, n_top)
    z, lse = _row_stats(x, tau, nv)
    if given is not None:
        zg = np.take_along_axis(z, np.clip(gv, 0, x.shape[1] - 1), 1)
        _close(_np(out), w_out, lse[:, None] + 2 * U * np.abs(zg) + U * np.abs(np.where(np.isfinite(w_out), w_out, 0)),
               "given")
    # entropy: log S and sum e z / S, each term relative 3|z| + 132 + the product's own rounding
    q = np.exp(np.where(z < 0, z, 0) - np.log(np.maximum(np.exp(z).sum(1, keepdims=True), 1)))
    tol = lse + U * (q * np.abs(z) * (3 * np.abs(z) + 134)).sum(1) + lse * np.abs(np.nan_to_num(w_ent)) \
        + U * np.abs(np.nan_to_num(w_ent))
    _close(_np(ent), w_ent, tol, "entropy")
    if n_top:
        assert np.array_equal(_np(ids), w_ids), f"alternatives differ: {_np(ids)[:2]} {w_ids[:2]}"
        zt = np.take_along_axis(z, np.clip(w_ids, 0, None), 1)
        _close(_np(top), w_top, lse[:, None] + 2 * U * np.abs(zt) + U * np.abs(np.where(np.isfinite(w_top), w_top, 0)),
               "alternatives")
    for a, b in zip((out, ent, ids, top), again):
        assert a is None or torch.equal(a.view(torch.int32), b.view(torch.int32)), "two equal calls differ"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,cols,n_given,n_top,pad,shift,tau", [
    (1, 1, 1, 1, 0, 0, 1.0), (3, 2, 2, 5, 0, 0, 0.5), (5, 7, 3, 3, 1, 1, 1.0), (9, 42, 10, 32, 0, 0, 1.0),
    (70, 64, 1, 1, 0, 0, 2.0), (4, 100, 0, 0, 3, 2, 1.0), (6, 1000, 100, 20, 0, 1, 0.7), (3, 1023, 1, 32, 1, 0, 1.0),
    (5, 4096, 7, 10, 0, 0, 1.0), (3, 4099, 1, 0, 0, 3, 1.0), (2, 8193, 1, 7, 0, 0, 1.0), (2, 50001, 1, 32, 0, 0, 1.0),
    (1, 131072, 1, 20, 0, 0, 0.8), (300, 700, 1, 5, 0, 0, 1.0), (2, 40000, 1024, 1, 7, 5, 1.3),
    (270, 40001, 2, 9, 1, 1, 1.0), (3, 28000, 1, 32, 0, 2, 1.0)])
def test_log_probs(B, dtype, n, cols, n_given, n_top, pad, shift, tau):
    say(f"[logprobs] {dtype} n={n} cols={cols} given={n_given} top={n_top}")
    gen = _gen(n + cols)
    logits = _row_view(n, cols, dtype, gen, pad, shift)
    given = torch.randint(-1, cols + 1, (n, n_given), generator=gen, device="cuda", dtype=torch.int32)
    _check_log_probs(B, logits, tau, None, given if n_given else None, n_top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [50, 3001, 40001])
def test_log_probs_of_ragged_and_masked_rows(B, dtype, cols):
    """Columns past a row's length hold NaN and infinities; inside, masks of
    -inf and of the type's lowest value, whole rows of them, and far rows."""
    say(f"[logprobs masks] {dtype} cols={cols}")
    gen = _gen(cols)
    x = _row_view(14, cols, dtype, gen)
    low = torch.finfo(dtype).min
    n_valid = torch.tensor([cols, 0, 1, 2, cols // 2, cols - 1, cols + 9, -3, cols, cols, cols, cols, cols, cols],
                           device="cuda", dtype=torch.int32)
    for i in range(14):
        m = min(max(int(n_valid[i]), 0), cols)
        x[i, m:] = torch.tensor([float("nan"), INF, -INF], device="cuda").to(dtype).repeat(cols // 3 + 1)[:cols - m]
    x[3, 0] = -INF
    x[4, :cols // 4] = -INF
    x[8] = -INF
    x[9] = low
    x[10, 1:] = low
    x[11] = -INF
    x[11, cols - 1] = -1.5
    x[12] = x[12] * 0.25 + (1000 if dtype != torch.bfloat16 else 4096)
    x[13, ::2] = low
    given = torch.stack([torch.zeros(14), torch.full((14,), cols - 1), torch.full((14,), cols // 2),
                         torch.full((14,), -1)], 1).to("cuda", torch.int32)
    _check_log_probs(B, x, 1.0, n_valid, given, 12)
    _check_log_probs(B, x, 0.3, n_valid, given, 32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [33, 1000, 33000])
def test_log_probs_of_undefined_rows(B, dtype, cols):
    x = _row_view(4, cols, dtype, _gen(cols))
    x[0, cols // 2] = float("nan")
    x[1, 3] = INF
    x[2, cols - 1] = float("nan")
    given = torch.tensor([[0, -1], [3, 1], [5, 6], [7, 8]], device="cuda", dtype=torch.int32)
    _check_log_probs(B, x, 1.0, None, given, 4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [40, 2000, 35000])
def test_alternatives_of_tied_rows(B, dtype, cols):
    """Rows of one value, of few values, of zeros of both signs, and rows whose
    best columns all lie side by side."""
    say(f"[ties] {dtype} cols={cols}")
    gen = _gen(cols)
    x = torch.zeros(7, cols, device="cuda")
    x[1] = torch.randint(0, 3, (cols,), generator=gen, device="cuda").float()
    x[2, ::3] = -0.0
    x[3, cols // 2:cols // 2 + 40] = 4.0
    x[4] = -torch.arange(cols, device="cuda") / 64.0
    x[5] = torch.arange(cols, device="cuda") / 64.0
    # thousands of equal best columns, all held by a few threads
    x[6] = torch.where(torch.arange(cols, device="cuda") // 8 % 256 < 32, 1.0, -1.0 - torch.rand(cols, device="cuda"))
    _check_log_probs(B, x.to(dtype), 1.0, None, None, 32)
    _check_log_probs(B, x.to(dtype), 1.0, None, None, 1)


# ------------------------------------------------------------------- distillation
def _check_distill(B, logits, ids, t, tau=1.0, lse=None, weight=None, n_valid=None):
    loss, grad = B.distill_loss(logits, ids, t, tau, lse, weight, n_valid)
    loss2, grad2 = B.distill_loss(logits, ids, t, tau, lse, weight, n_valid)
    loss3, none = B.distill_loss(logits, ids, t, tau, lse, weight, n_valid, want_grad=False)
    torch.cuda.synchronize()
    x = _np(logits)
    c = lambda a: None if a is None else _np(a)
    nv, wt = c(n_valid), c(weight)
    tau32, tau = tau, float(np.float32(tau))     # the call takes it in 32 bits
    w_loss, w_grad = R.distill(x, _np(ids), _np(t), tau, c(lse), wt, nv)
    z, lt = _row_stats(x, tau, nv)
    n, cols = x.shape
    loss_tol, grad_tol = np.zeros(n), np.zeros((n, cols))
    for i in range(n):
        w = 1.0 if wt is None else wt[i]
        if w == 0 or not np.isfinite(w_loss[i]):
            # an infinite loss (a listed column of probability 0) still has a gradient
            if not np.isposinf(w_loss[i]):
                continue
        m = R.row_length(nv, i, cols)
        lq = R.log_softmax(x[i, :m], tau)
        if lq is None:
            continue
        q = np.exp(lq)
        there = [k for k in range(ids.shape[1]) if 0 <= int(ids[i, k]) < m]
        at = _np(ids)[i, there]
        tt = _np(t)[i, there]
        if lse is None:
            lp = R.log_softmax(tt, tau) if there else np.zeros(0)
        else:
            lp = tt / tau - float(lse[i])
        p = np.exp(lp)
        rel = lt[i] + U * (3 * np.abs(z[i, :m]) + 6)
        loss_tol[i] = (p * (lt[i] + 2 * U * np.abs(z[i, at]))).sum()
        target = np.zeros(m)
        np.add.at(target, at, p)
        tol = q * rel + U * (q + target)
        if lse is not None:
            others = np.ones(m, dtype=bool)
            others[at] = False
            others &= q > 0
            left = max(0.0, 1 - p.sum())
            if others.any() and left > 0:
                zo = np.abs(z[i, :m][others])
                mo = zo.min()
                qo = q[others] / q[others].sum()
                rest_tol = U * (3 * (qo * (zo - mo)).sum() + 132)
                loss_tol[i] += left * (lt[i] + rest_tol + 4 * U * mo)
                share = left * qo
                tol[others] += share * (rest_tol + U * (3 * (zo - mo) + 6)) + U * share
        # the sum's rounding of its own; in 64 bits the rest's cancellation stays below u
        loss_tol[i] = tau * tau * loss_tol[i] + U * abs(np.nan_to_num(w_loss[i], posinf=0)) + 1e-12
        grad_tol[i, :m] = w * tau * tol + (HALF[logits.dtype] * (1 + 1e-3) + 2 * U) * np.abs(w_grad[i, :m]) \
            + TINY[logits.dtype]
    _close(_np(loss), w_loss, loss_tol, "loss")
    _close(_np(grad), w_grad, grad_tol, "gradient")
    assert none is None
    for a, b in ((loss, loss2), (loss, loss3)):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32)), "two equal calls differ"
    bits = torch.int32 if grad.dtype == torch.float32 else torch.int16
    assert torch.equal(grad.contiguous().view(bits), grad2.contiguous().view(bits)), "two equal calls differ"
    # In place of the logits.  (Rows are cut at 16-byte boundaries, so the same
    # values at another alignment are summed in another order: the reference is
    # this copy's own result.)
    mine = torch.zeros(n, cols + 3, device="cuda", dtype=logits.dtype)[:, :cols]
    mine.copy_(logits)
    loss4, grad4 = B.distill_loss(mine, ids, t, tau32, lse, weight, n_valid)
    loss5, grad5 = B.distill_loss(mine, ids, t, tau32, lse, weight, n_valid, grad_out=mine)
    torch.cuda.synchronize()
    _close(_np(loss4), w_loss, loss_tol, "the copy's loss")
    _close(_np(grad4), w_grad, grad_tol, "the copy's gradient")
    assert grad5.data_ptr() == mine.data_ptr()
    assert torch.equal(loss5.view(torch.int32), loss4.view(torch.int32)), "the loss in place differs"
    assert torch.equal(grad5.contiguous().view(bits), grad4.contiguous().view(bits)), "the gradient in place differs"


def _teacher(x, k, tau, gen, n_valid=None):
    """The k largest of the logits plus noise, and the log of the teacher's sum."""
    t = x.float() + 0.5 * torch.randn(x.shape, generator=gen, device="cuda")
    if n_valid is not None:
        t = torch.where(torch.arange(x.shape[1], device="cuda")[None] < n_valid[:, None], t, -INF)
    top, at = torch.topk(t, k, dim=1)
    return at.to(torch.int32), top.contiguous(), torch.logsumexp(t / tau, 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n,cols,k,pad,shift,tau", [
    (1, 1, 1, 0, 0, 1.0), (3, 2, 1, 0, 0, 2.0), (5, 7, 7, 1, 1, 1.0), (9, 42, 10, 0, 0, 1.0), (70, 64, 5, 0, 0, 4.0),
    (6, 1000, 100, 0, 1, 0.7), (3, 1023, 30, 1, 0, 1.0), (5, 4096, 64, 0, 0, 2.0), (3, 4099, 8, 0, 3, 1.0),
    (2, 8193, 1024, 0, 0, 1.0), (2, 50001, 32, 0, 0, 2.0), (1, 131072, 64, 0, 0, 1.0), (300, 700, 12, 0, 0, 1.0),
    (2, 40000, 20, 7, 5, 1.0), (130, 40001, 17, 1, 1, 1.0), (515, 5001, 9, 0, 1, 2.0), (513, 20003, 9, 2, 0, 1.0)])
def test_distill(B, dtype, rest, n, cols, k, pad, shift, tau):
    say(f"[distill] {dtype} n={n} cols={cols} k={k} rest={rest}")
    gen = _gen(n + cols)
    x = _row_view(n, cols, dtype, gen, pad, shift)
    ids, t, lse = _teacher(x, k, tau, gen)
    weight = torch.rand(n, generator=gen, device="cuda") + 0.5
    _check_distill(B, x, ids, t, tau, lse if rest else None, weight)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("cols,n", [(50, 14), (3001, 14), (40001, 14), (40001, 131), (9001, 514)])
def test_distill_of_ragged_and_masked_rows(B, dtype, rest, cols, n):
    """Rows left out by weight, length or mask (with NaN where nothing is
    read), absent and repeated teacher slots, a listed column of probability 0
    (an infinite loss), undefined rows and teachers."""
    say(f"[distill masks] {dtype} cols={cols} rest={rest}")
    gen = _gen(cols)
    x = _row_view(n, cols, dtype, gen)
    n_valid = torch.full((n,), cols, device="cuda", dtype=torch.int32)
    n_valid[1], n_valid[2], n_valid[3] = 0, 1, cols // 2
    clean = torch.where(torch.isfinite(x.float()), x.float(), -30.0)
    ids, t, lse = _teacher(clean, 6, 1.0, gen, torch.clamp(n_valid, min=6))
    weight = torch.rand(n, generator=gen, device="cuda") + 0.5
    weight[4] = 0.0
    x[4] = float("nan")
    for i in (1, 2, 3):
        x[i, int(n_valid[i]):] = float("nan")
    ids[5] = -1
    ids[6, 1] = ids[6, 0]
    ids[6, 2] = ids[6, 0]
    ids[6, 3] = cols
    x[7] = -INF
    x[8, ids[8, 2].long()] = -INF
    x[9, cols // 3] = float("nan")
    t[10, 1] = float("nan")
    x[11] = torch.finfo(dtype).min
    x[12] = x[12] * 0.25 + (1000 if dtype != torch.bfloat16 else 4096)
    t[13, 5] = -INF
    _check_distill(B, x, ids, t, 1.0, lse if rest else None, weight, n_valid)


@pytest.mark.parametrize("rest", [False, True])
def test_distill_of_repeated_and_undefined_teachers(B, rest):
    """Slots that name one column many times, among more slots than a
    wavefront's lanes; sums of the teacher that are not finite."""
    gen = _gen(5)
    x = _row_view(6, 900, torch.float32, gen)
    ids, t, lse = _teacher(x, 200, 1.0, gen)
    ids[0] = ids[0, 0]
    ids[1, 100:] = ids[1, :100]
    ids[2, 199] = ids[2, 0]
    lse = lse + 1.0                            # repeats must not take more than everything
    lse[4], lse[5] = float("nan"), INF
    _check_distill(B, x, ids, t - (5.0 if rest else 0.0), 1.0, lse if rest else None)


@pytest.mark.parametrize("dtype", TYPES)
def test_the_longest_rows(B, dtype):
    """2^20 columns: the most chunks that a join takes."""
    say(f"[longest] {dtype}")
    cols = B.MAX_COLS
    x = torch.randn(cols, generator=_gen(1), device="cuda").to(dtype).view(1, cols)
    x[0, cols - 1] = 9.0
    ids, t, lse = _teacher(x, 5, 1.0, _gen(2))
    given, ent, top, logp = B.log_probs(x, ids, 4)
    loss, grad = B.distill_loss(x, ids, t, 1.0, lse)
    torch.cuda.synchronize()
    lp = torch.log_softmax(x.double(), 1)
    assert int(top[0, 0]) == cols - 1
    # as _row_stats: u (3 E|z| + 132) with E|z| < 10, and the value's rounding
    tol = U * (3 * 10 + 132 + 3 * 20)
    assert torch.all((given.double() - torch.gather(lp, 1, ids.long())).abs() <= tol)
    assert torch.all((logp.double() - torch.gather(lp, 1, top.long())).abs() <= tol)
    assert abs(float(ent) + float((lp.exp() * lp).sum())) <= 20 * tol
    w_loss, w_grad = R.distill(_np(x), _np(ids), _np(t), 1.0, _np(lse))
    assert abs(float(loss) - w_loss[0]) <= 4 * tol
    assert np.all(np.abs(_np(grad) - w_grad) <= (2 * tol + HALF[dtype] * 1.001) * np.abs(w_grad) + TINY[dtype] + U * 1e-6)


def test_more_rows_than_one_grid_counts(B):
    n = (1 << 22) + 37
    x = torch.randn(n, 3, generator=_gen(4), device="cuda")
    ids = torch.randint(0, 3, (n, 1), generator=_gen(5), device="cuda", dtype=torch.int32)
    t = torch.zeros(n, 1, device="cuda")
    given, ent, top, logp = B.log_probs(x, ids, 1)
    loss, grad = B.distill_loss(x, ids, t)
    torch.cuda.synchronize()
    lp = torch.log_softmax(x.double(), 1)
    at = torch.gather(lp, 1, ids.long())
    tol = U * (3 * 12 + 8)                     # three terms a row, |z| below 12
    assert torch.all((given.double() - at).abs() <= tol)
    assert torch.equal(top[:, 0].long(), x.argmax(1))
    assert torch.all((loss.double() + at[:, 0]).abs() <= tol)
    hot = torch.zeros_like(lp).scatter_(1, ids.long(), 1.0)
    assert torch.all((grad.double() - (lp.exp() - hot)).abs() <= tol)


@pytest.mark.parametrize("cols", [200, 3001, 40001])
def test_logits_past_32_bits(B, cols):
    """Rows whose offsets pass 2^31 elements give what the same rows close
    together give; a gradient written in place leaves the space between."""
    n, ld = 5, 600_000_000
    near = torch.empty(n, cols + 8 - cols % 8, device="cuda", dtype=torch.bfloat16)[:, :cols]
    near.copy_(torch.randn(n, cols, generator=_gen(cols), device="cuda"))
    room = torch.empty((n - 1) * ld + cols + 1, device="cuda", dtype=torch.bfloat16)
    far = room.as_strided((n, cols), (ld, 1))
    far.copy_(near)
    room.as_strided((n,), (ld,), cols).fill_(7.0)
    ids, t, lse = _teacher(near, 5, 1.0, _gen(2))
    one, two = B.log_probs(near, ids, 4), B.log_probs(far, ids, 4)
    room_near = torch.empty(n, near.stride(0), device="cuda", dtype=torch.bfloat16)
    loss, grad = B.distill_loss(near, ids, t, 1.0, lse, grad_out=room_near[:, :cols])
    loss2, grad2 = B.distill_loss(far, ids, t, 1.0, lse, grad_out=far)
    torch.cuda.synchronize()
    for a, b in zip(one, two):
        assert torch.equal(a, b)
    assert torch.equal(loss, loss2) and torch.equal(grad, grad2)
    assert grad2.data_ptr() == far.data_ptr() and torch.all(room.as_strided((n,), (ld,), cols) == 7)


def test_empty_batches(B):
    x = torch.empty(0, 7, device="cuda")
    ids = torch.empty(0, 2, device="cuda", dtype=torch.int32)
    assert B.embed_lookup(torch.ones(3, 7, device="cuda"), ids).shape == (0, 7)
    assert [tuple(o.shape) for o in B.log_probs(x, ids, 4)] == [(0, 2), (0,), (0, 4), (0, 4)]
    loss, grad = B.distill_loss(x, ids, torch.empty(0, 2, device="cuda"))
    assert loss.shape == (0,) and grad.shape == (0, 7)


def test_distill_far_from_the_teachers_columns(B):
    """The listed columns hold nearly all of the student's probability: the
    rest's share (e^-60) is summed by itself, not as a difference."""
    x = torch.randn(3, 5000, device="cuda")
    x[:, 7] += 60
    ids = torch.full((3, 1), 7, device="cuda", dtype=torch.int32)
    t = torch.full((3, 1), -0.5, device="cuda")
    _check_distill(B, x, ids, t, 1.0, torch.zeros(3, device="cuda"))


# ------------------------------------------------------------ streams and graphs
def _run_all(B, st):
    return [B.embed_lookup(st["table"], st["ids"], 0.5), B.embed_gradient(st["g"], st["ids"], st["table"].shape[0]),
            *B.log_probs(st["x"], st["given"], 9, n_valid=st["nv"]),
            *B.distill_loss(st["x"], st["tid"], st["t"], 2.0, st["lse"], n_valid=st["nv"])]


def _state(seed, cols):
    gen = _gen(seed)
    x = torch.randn(37, cols, generator=gen, device="cuda").to(torch.bfloat16)
    tid, t, lse = _teacher(x[:, :cols // 2], 11, 2.0, gen)
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen, device="cuda", dtype=torch.int32)
    return dict(table=torch.randn(500, 96, generator=gen, device="cuda"), ids=ints(-1, 500, 3000, 2),
                g=torch.randn(3000, 96, generator=gen, device="cuda"), x=x, given=ints(0, cols, 37, 3),
                nv=ints(cols // 2, cols + 1, 37), tid=tid, t=t, lse=lse)


@pytest.mark.parametrize("cols", [300, 50003])
def test_captured_calls_replay(B, cols):
    """Two graphs of all calls, replayed in turn and side by side on two
    streams with new inputs each time and eager calls between."""
    say(f"[graph] cols={cols}")
    states = [_state(1, cols), _state(2, cols)]
    for st in states:
        _run_all(B, st)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for st in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_run_all(B, st))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for step in range(3):
        for k, st in enumerate(states):
            fresh = _state(10 * step + k, cols)
            for name in st:
                st[name].copy_(fresh[name])
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for st, got in zip(states, outs):
            want = _run_all(B, st)
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                bits = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
                assert torch.equal(a.view(bits), b.view(bits)), (step, a.shape)


def test_calls_follow_the_current_stream(B):
    st = _state(3, 5000)
    want = _run_all(B, st)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    late = {k: torch.empty_like(v) for k, v in st.items()}
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        for k in late:
            late[k].copy_(st[k])
        got = _run_all(B, late)
    s.synchronize()
    for a, b in zip(got, want):
        bits = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
        assert torch.equal(a.view(bits), b.view(bits))


def test_wrapper_refusals(B):
    x = torch.randn(4, 10, device="cuda")
    ids = torch.zeros(4, 2, device="cuda", dtype=torch.int32)
    t = torch.zeros(4, 2, device="cuda")
    for call in (lambda: B.log_probs(x.cpu()), lambda: B.log_probs(x.double()), lambda: B.log_probs(x[0]),
                 lambda: B.log_probs(x, ids[:3]), lambda: B.log_probs(x, ids.cpu()), lambda: B.log_probs(x, n_top=33),
                 lambda: B.log_probs(x, ids[:, 0]), lambda: B.distill_loss(x, ids[:, 0], t),
                 lambda: B.log_probs(x, ids.float()), lambda: B.log_probs(x, n_valid=ids[:, 0][:2]),
                 lambda: B.distill_loss(x, ids, t[:, :1]), lambda: B.distill_loss(x, ids, t, tau=0.0),
                 lambda: B.distill_loss(x, ids, t, grad_out=torch.empty(4, 9, device="cuda")),
                 lambda: B.distill_loss(x, ids, t, grad_out=torch.empty(10, 4, device="cuda").t()),
                 lambda: B.embed_lookup(x, ids, float("nan")), lambda: B.embed_lookup(x, ids[None]),
                 lambda: B.embed_lookup(x, ids, out=torch.empty(4, 9, device="cuda")),
                 lambda: B.embed_gradient(x, ids[:3], 5), lambda: B.embed_gradient(x, ids, 0),
                 lambda: B.embed_gradient(x, ids, 5, accumulate=True),
                 lambda: B.embed_gradient(x, ids, 5, dtype=torch.float16)):
        with pytest.raises(B.IfvsError) as e:
            call()
        assert e.value.status == B.E_INVALID


@pytest.mark.parametrize("dtype", TYPES)
def test_any_layout_is_taken(B, dtype):
    """Transposed, broadcast and stepped logits and tables: the lookup and its
    gradient give what their contiguous copies give, bit for bit, the row
    operators what their definitions give."""
    x = torch.randn(40, 30, device="cuda").to(dtype)
    views = [x.t(), x[::2], x[:, ::3], x[:1].expand(7, 30), x[3:4]]
    for v in views:
        n, cols = v.shape
        ids = torch.zeros(n, 2, device="cuda", dtype=torch.int64) + torch.tensor([1, 4], device="cuda")
        t = torch.randn(2, n, device="cuda").t()
        c = v.contiguous()
        assert torch.equal(B.embed_lookup(v, ids), B.embed_lookup(c, ids))
        assert torch.equal(B.embed_gradient(v, ids, 9), B.embed_gradient(c, ids, 9))
        _check_log_probs(B, v, 1.0, None, ids, 3)
        if not (v.stride(0) == 0 and n > 1):              # a broadcast row has no place for a gradient
            _check_distill(B, v, ids, t)
        else:
            _check_distill(B, c, ids, t)
            a, b = B.distill_loss(v, ids, t), B.distill_loss(c, ids, t)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
