"""The row operators' 64-bit definitions pinned by something other than
themselves: scipy's log_softmax and entropy, one-hot matrix products, central
differences, and the divergence over a full teacher; then the refusals of the
C entry points, which run before anything touches a GPU."""
import ctypes
import math

import numpy as np
import pytest
from scipy.special import log_softmax, rel_entr
from scipy.stats import entropy as sp_entropy

from oracle import ifvs_rows_oracle as R


def test_lookup_and_gradient_are_one_hot_products():
    rng = np.random.default_rng(1)
    table = rng.normal(size=(13, 5))
    ids = rng.integers(-2, 16, size=(9, 3))          # -2, -1 and 13.. are absent
    hot = np.zeros((9, 13))
    for i in range(9):
        for j in ids[i]:
            if 0 <= j < 13:
                hot[i, j] += 1
    assert np.allclose(R.embed_lookup(table, ids, 1.7), 1.7 * hot @ table, rtol=1e-12, atol=1e-12)
    g = rng.normal(size=(9, 5))
    assert np.allclose(R.embed_gradient(g, ids, 13, 1.7), 1.7 * hot.T @ g, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_log_probs_match_scipy(tau):
    rng = np.random.default_rng(2)
    x = rng.normal(size=(6, 40)) * 3
    x[2, 5:30] = -np.inf
    n_valid = np.array([40, 1, 40, 17, 0, 90])
    given = rng.integers(0, 40, size=(6, 4))
    given[0, 0], given[3, 1] = -1, 17
    out, ent, ids, top = R.log_probs(x, tau, n_valid, given, 8)
    for i, m in enumerate((40, 1, 40, 17, 0, 40)):
        if m == 0:
            assert np.isneginf(out[i]).all() and ent[i] == 0 and (ids[i] == -1).all() and np.isneginf(top[i]).all()
            continue
        ref = log_softmax(x[i, :m] / tau)
        for g in range(4):
            want = ref[given[i, g]] if 0 <= given[i, g] < m else -np.inf
            assert out[i, g] == want or abs(out[i, g] - want) < 1e-12
        assert abs(ent[i] - sp_entropy(np.exp(ref))) < 1e-12
        live = int((~np.isneginf(x[i, :m])).sum())
        want = sorted(range(m), key=lambda v: (-x[i, v], v))[:min(8, live)]
        assert list(ids[i, :len(want)]) == want and (ids[i, len(want):] == -1).all()


def test_alternatives_break_ties_to_the_lower_column():
    x = np.array([[1.0, 3.0, 3.0, 0.0, -0.0, 3.0, 1.0]])
    assert list(R.log_probs(x, n_top=6)[2][0]) == [1, 2, 5, 0, 6, 3]


def _cases():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(5, 12)) * 2
    ids = np.array([[3, 1, 7], [0, -1, 5], [2, 2, 4], [11, 12, -7], [6, 9, 8]])
    t = rng.normal(size=(5, 3)) * 2
    full = rng.normal(size=(5, 12))
    lse = np.log(np.exp(t / 2.0).sum(1) + np.exp(full).sum(1))
    n_valid = np.array([12, 8, 12, 12, 7])
    weight = np.array([1.0, 0.5, 2.0, 0.0, 1.5])
    return x, ids, t, lse, n_valid, weight


@pytest.mark.parametrize("rest", [False, True])
def test_distillation_gradient_is_the_losss_difference(rest):
    x, ids, t, lse, n_valid, weight = _cases()
    kw = dict(tau=2.0, teacher_lse=lse if rest else None, row_weight=weight, n_valid=n_valid)
    _, grad = R.distill(x, ids, t, **kw)
    h = 1e-5
    for v in range(x.shape[1]):
        up, down = x.copy(), x.copy()
        up[:, v] += h
        down[:, v] -= h
        diff = (R.distill(up, ids, t, **kw)[0] - R.distill(down, ids, t, **kw)[0]) / (2 * h) * weight
        # a central difference is off by h^2 |L'''| / 6 + rounding 1e-16 / h
        assert np.allclose(grad[:, v], diff, rtol=0, atol=1e-8), v


def test_distillation_of_a_whole_teacher_is_the_divergence():
    """With every column listed both forms are tau^2 KL(teacher || student)."""
    rng = np.random.default_rng(4)
    x, t = rng.normal(size=(3, 9)), rng.normal(size=(3, 9))
    ids = np.stack([rng.permutation(9) for _ in range(3)])
    tau = 1.5
    p = np.exp(log_softmax(t / tau, axis=1))
    q = np.exp(log_softmax(x / tau, axis=1))
    want = tau ** 2 * np.array([rel_entr(p[i], q[i][ids[i]]).sum() for i in range(3)])
    lse = np.log(np.exp(t / tau).sum(1))
    assert np.allclose(R.distill(x, ids, t, tau)[0], want, rtol=1e-12)
    assert np.allclose(R.distill(x, ids, t, tau, teacher_lse=lse)[0], want, rtol=1e-10)


# ----------------------------------------------------------------- refusals
P = ctypes.c_void_p(0x1000)          # never read: every call below is refused first
W = 1 << 40                          # workspace bytes claimed


@pytest.fixture(scope="module")
def B():
    from paper_2607_22922_amd import ifvs
    return ifvs


def _refused(B, fn, args):
    st = getattr(B.lib(), fn)(*args)
    msg = B.lib().ifvs_last_error().decode()
    assert st == B.E_INVALID and msg and msg != "no error", (fn, args, st, msg)


LOOKUP = dict(rows=10, dim=8, table=P, table_ld=8, dtype=0, n=4, bag=2, ids=P, scale=1.0, out=P, out_ld=8, stream=None)
GRAD = dict(rows=10, dim=8, n=4, bag=2, ids=P, scale=1.0, grad=P, grad_ld=8, dtype=1, accumulate=0, table_grad=P,
            out_ld=8, out_dtype=0, ws=P, ws_bytes=W, stream=None)
LOGP = dict(n=4, cols=50, logits=P, ld=50, dtype=0, n_valid=None, tau=1.0, given=P, n_given=1, n_top=5, given_out=P,
            entropy=P, top_ids=P, top=P, ws=P, ws_bytes=W, stream=None)
DISTILL = dict(n=4, cols=50, logits=P, ld=50, dtype=2, n_valid=None, n_teacher=3, ids=P, t=P, lse=None, tau=1.0,
               weight=None, loss=P, grad=P, grad_ld=50, ws=P, ws_bytes=W, stream=None)
ODD = ctypes.c_void_p(0x1001)
COMMON_ROWS = [("n", -1), ("n", 1 << 31), ("cols", 0), ("cols", (1 << 20) + 1), ("logits", None), ("logits", ODD),
               ("ld", 49), ("dtype", 3), ("dtype", -1), ("n_valid", ODD), ("tau", 0.0), ("tau", -1.0),
               ("tau", math.nan), ("tau", math.inf), ("tau", 1e-44)]
EMBED = [("rows", 0), ("rows", (1 << 31) - 1), ("dim", 0), ("dim", 65537), ("bag", 0), ("bag", 17),
         ("n", -1), ("n", (1 << 29) + 1), ("ids", None), ("ids", ODD), ("scale", math.nan), ("scale", math.inf),
         ("dtype", 3), ("out_ld", 7)]
REFUSALS = (
    [("ifvs_embed_lookup", LOOKUP, k, v) for k, v in EMBED + [("table", None), ("table", ODD), ("table_ld", 7),
                                                              ("out", None), ("out", ODD)]] +
    [("ifvs_embed_gradient", GRAD, k, v) for k, v in EMBED + [
        ("grad", None), ("grad", ODD), ("grad_ld", 7), ("table_grad", None), ("table_grad", ODD), ("out_dtype", 2),
        ("out_dtype", 7), ("accumulate", 2), ("accumulate", -1)]] +
    [("ifvs_log_probs", LOGP, k, v) for k, v in COMMON_ROWS + [
        ("n_given", -1), ("n_given", 1025), ("n_top", -1), ("n_top", 33), ("given", None), ("given_out", None),
        ("given_out", ODD), ("entropy", ODD), ("top_ids", None), ("top", None), ("top", ODD)]] +
    [("ifvs_distill_loss", DISTILL, k, v) for k, v in COMMON_ROWS + [
        ("n_teacher", 0), ("n_teacher", 1025), ("ids", None), ("ids", ODD), ("t", None), ("lse", ODD),
        ("weight", ODD), ("loss", None), ("grad", ODD), ("grad_ld", 49)]])


@pytest.mark.parametrize("fn,good,field,value", REFUSALS, ids=lambda v: None if isinstance(v, dict) else str(v))
def test_bad_arguments_are_refused(B, fn, good, field, value):
    args = dict(good)
    args[field] = value
    _refused(B, fn, list(args.values()))


def test_small_and_misaligned_workspaces_are_refused(B):
    """Where a call needs scratch: one byte too few, none, and off by 8."""
    lib = B.lib()
    for fn, good, need in (
            ("ifvs_embed_gradient", dict(GRAD, n=100000, rows=5000), lib.ifvs_embed_workspace(5000, 8, 100000, 2)),
            ("ifvs_log_probs", dict(LOGP, n=2, cols=1 << 20, ld=1 << 20), lib.ifvs_log_probs_workspace(2, 1 << 20, 5)),
            ("ifvs_distill_loss", dict(DISTILL, n=2, cols=1 << 20, ld=1 << 20, grad_ld=1 << 20),
             lib.ifvs_distill_workspace(2, 1 << 20))):
        assert need >= 0
        if need == 0:
            continue
        for ws, have in ((P, need - 1), (None, need), (ctypes.c_void_p(0x1008), need)):
            _refused(B, fn, list(dict(good, ws=ws, ws_bytes=have).values()))


def test_workspace_sizes_out_of_range(B):
    lib = B.lib()
    assert lib.ifvs_embed_workspace(0, 8, 4, 1) == -1 and lib.ifvs_embed_workspace(8, 8, 4, 17) == -1
    assert lib.ifvs_log_probs_workspace(4, 0, 1) == -1 and lib.ifvs_log_probs_workspace(4, 9, 33) == -1
    assert lib.ifvs_distill_workspace(-1, 9) == -1 and lib.ifvs_distill_workspace(1, (1 << 20) + 1) == -1


def test_empty_calls_do_nothing(B):
    lib = B.lib()
    assert lib.ifvs_embed_lookup(*dict(LOOKUP, n=0).values()) == B.OK
    assert lib.ifvs_embed_gradient(*dict(GRAD, n=0, accumulate=1).values()) == B.OK
    assert lib.ifvs_log_probs(*dict(LOGP, n=0).values()) == B.OK
    assert lib.ifvs_distill_loss(*dict(DISTILL, n=0).values()) == B.OK


def test_index_calls_need_a_handle(B):
    lib = B.lib()
    assert lib.ifvs_score_candidates(None, 1, P, 0, P, 4, P, None) == B.E_STATE
    assert lib.ifvs_distill_step(None, 1, P, P, None, P, 4, 2, P, 1.0, 0.0, 0.1, P, None, None) == B.E_STATE
    assert b"NULL" in lib.ifvs_last_error()
