"""The row operators where the framework itself uses them: candidate scores
against the search's distances, the distillation training step against
automatic differentiation in 64 bits, a learned table of predicate weights
trained through lookup, training step and table gradient, and the training
loop with both."""
import math

import numpy as np
import pytest
import torch

from oracle import ifvs_rows_oracle as R
from oracle.ifvs_oracle import fingerprint, hashed_rows
from tests._gpu_util import say
from tests.test_train_gpu import LR, _close, _np, _problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2607_22922_amd import ifvs
    return ifvs


@pytest.mark.parametrize("M,dsub,cluster_cols", [(16, 4, ()), (16, 4, (0,)), (48, 2, (0,)), (5, 2, ()), (3, 7, (0,))])
@pytest.mark.parametrize("f16", [False, True])
def test_candidate_scores_are_the_searchs_distances(B, M, dsub, cluster_cols, f16):
    say(f"[score] M={M} dsub={dsub} cols={cluster_cols} f16={f16}")
    idx, ix, q, w_z, cand, preds, _ = _problem(B, 3 + M, M, dsub, cluster_cols, nq=9, n_cand=700)
    dt = B.LUT_F16 if f16 else B.LUT_F32
    alpha, wf = idx.select_codebook(q, preds, w_z)
    lut = idx.build_lut(q, alpha, wf, dt)
    ids, dist = idx.search(preds, lut, 16, dt)
    got = idx.score_candidates(lut, ids, dt)
    scores = idx.score_candidates(lut, cand, dt)
    torch.cuda.synchronize()
    want = torch.where(ids >= 0, -dist, torch.full_like(dist, -math.inf))
    assert torch.equal(got, want)                         # bit for bit, clustered or not
    codes = ix["codes"].long()
    there = (cand >= 0) & (cand < codes.shape[0])
    rows = codes[cand.clamp(0, codes.shape[0] - 1).long()]                      # [nq][n_cand][M]
    d64 = torch.gather(lut.double(), 2, rows.permute(0, 2, 1)).sum(1)
    fin = torch.isfinite(d64) & there
    # M fp32 additions of table entries
    assert torch.all((scores.double() + d64).abs()[fin] <= M * 2.0 ** -24 * d64[fin])
    assert torch.all(scores[~there] == -math.inf)


def _reference(ix, q, w_z, cand, preds, teacher, tau, lam):
    """Losses and gradients of the mean loss by automatic differentiation in 64 bits."""
    bank = ix["bank"].cpu().double().requires_grad_(True)
    W = ix["W"].cpu().double().requires_grad_(True)
    C = ix["C_pq"].cpu().double()
    codes = ix["codes"].cpu().long()
    wz = None if w_z is None else w_z.cpu().double().requires_grad_(True)
    M, K, d = C.shape
    r = W.shape[1]
    losses = []
    nq = q.shape[0]
    for i in range(nq):
        rows = hashed_rows(fingerprint(_np(q[i]), preds[i]), ix["h"], bank.shape[0], ix["hash_seed"])
        alpha = sum(bank[int(row)] for row in rows).view(M, r)
        delta = torch.einsum("mt,mtcj->mcj", alpha, W)
        w = torch.ones(M * d, dtype=torch.float64) if wz is None else torch.log1p(torch.exp(wz[i]))
        lut = (w.view(M, 1, d) * (q[i].cpu().double().view(M, 1, d) - C - delta) ** 2).sum(2)
        c = cand[i].cpu().long()
        there = (c >= 0) & (c < codes.shape[0])
        slots = torch.nonzero(there)[:, 0]
        loss = torch.zeros((), dtype=torch.float64)
        k = slots[slots < teacher.shape[1]]
        if k.numel():
            dist = lut[torch.arange(M)[None], codes[c[slots]]].sum(1)
            logq = torch.log_softmax(-dist / tau, 0)
            logp = torch.log_softmax(-teacher[i].cpu().double()[k] / tau, 0)
            where = torch.searchsorted(slots, k)
            loss = tau ** 2 * (torch.exp(logp) * (logp - logq[where])).sum()
        losses.append(loss + lam * (delta ** 2).mean())
    total = torch.stack(losses)
    total.mean().backward()
    return (total.detach().numpy(), bank.grad.numpy(), W.grad.numpy(), None if wz is None else wz.grad.numpy())


@pytest.mark.parametrize("M,dsub,cluster_cols,nq,n_cand,n_teacher,with_wz", [
    (16, 4, (), 12, 24, 4, True), (16, 4, (0,), 12, 24, 24, True), (48, 2, (0,), 5, 42, 10, False),
    (8, 16, (), 4, 1500, 100, True), (5, 2, (), 150, 12, 5, True)])
def test_distill_step_against_automatic_differentiation(B, M, dsub, cluster_cols, nq, n_cand, n_teacher, with_wz):
    say(f"[distill step] M={M} dsub={dsub} nq={nq} n_cand={n_cand} teacher={n_teacher}")
    idx, ix, q, w_z, cand, preds, _ = _problem(B, 5 + M, M, dsub, cluster_cols, nq=nq, n_cand=n_cand,
                                               with_wz=with_wz)
    cand[2, :n_teacher] = -1                               # no teacher slot: anchor term only
    tau, lam = 2.0, 0.05
    gen = torch.Generator(device="cuda").manual_seed(7)
    teacher = torch.rand(nq, n_teacher, generator=gen, device="cuda") * 8 + 1
    want = _reference(ix, q, w_z, cand, preds, teacher, tau, lam)
    bank0, W0 = idx.read_params()
    loss, dwz = idx.distill_step(q, preds, w_z, cand, teacher, tau, lam, LR, want_dwz=with_wz)
    bank1, W1 = idx.read_params()
    torch.cuda.synchronize()
    _close(_np(loss), want[0], "loss", rel=1e-4)
    _close(_np((bank0 - bank1) / LR), want[1], "bank gradient")
    _close(_np((W0 - W1) / LR), want[2], "W gradient")
    if with_wz:
        _close(_np(dwz), want[3], "w_z gradient")


def test_distill_step_is_deterministic_and_grows_its_buffers(B):
    outs = []
    for first in (False, True):
        idx, ix, q, w_z, cand, preds, _ = _problem(B, 33, 16, 4, (0,), bank_rows=3, n_cand=64)
        teacher = torch.linspace(1, 9, 12 * 4, device="cuda").view(12, 4)
        if first:       # a step with fewer candidates and no learning rate before
            idx.distill_step(q, preds, w_z, cand[:, :8], teacher, 1.0, 0.0, 0.0)
        loss, dwz = idx.distill_step(q, preds, w_z, cand, teacher, 0.8, 0.05, 1.0, want_dwz=True)
        bank, W = idx.read_params()
        torch.cuda.synchronize()
        outs.append([t.clone() for t in (loss, dwz, bank, W)])
    for a, b in zip(*outs):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))


def test_distill_step_refusals(B):
    idx, ix, q, w_z, cand, preds, _ = _problem(B, 9, 8, 4, ())
    bank0, W0 = idx.read_params()
    t = torch.ones(12, 4, device="cuda")
    for args in ((cand, t, 0.0, 0.1, 1.0), (cand, t, 1e-44, 0.1, 1.0), (cand, t, 1.0, -1.0, 1.0),
                 (cand, t, 1.0, 0.1, float("nan")), (cand[:, :3], t, 1.0, 0.1, 1.0), (cand[:5], t, 1.0, 0.1, 1.0),
                 (cand, t[:5], 1.0, 0.1, 1.0), (cand, t[:, :0], 1.0, 0.1, 1.0)):
        with pytest.raises(B.IfvsError) as e:
            idx.distill_step(q, preds, w_z, *args)
        assert e.value.status == B.E_INVALID
    plain = B.Index(ix["codes"], ix["C_pq"], ix["attrs"], max_batch=12, max_k=8)
    with pytest.raises(B.IfvsError) as e:
        plain.distill_step(q, preds, None, cand, t, 1.0, 0.1, 1.0)
    assert e.value.status == B.E_STATE
    with pytest.raises(B.IfvsError) as e:
        plain.score_candidates(plain.build_lut(q), cand[:, :0])
    assert e.value.status == B.E_INVALID
    for call in (lambda: plain.score_candidates(plain.build_lut(q), cand[:5]),
                 lambda: idx.distill_step(q, preds, w_z[:5], cand, t, 1.0, 0.1, 1.0)):
        with pytest.raises(B.IfvsError) as e:
            call()
        assert e.value.status == B.E_INVALID
    torch.cuda.synchronize()
    bank1, W1 = idx.read_params()
    assert torch.equal(bank0, bank1) and torch.equal(W0, W1)


def test_operators_together(B):
    """Weights of predicates from a table (two rows each), the conditioned
    search's candidates scored with them, their distillation loss, its gradient
    by the training step carried back into the table: against differences of
    the 64-bit loss in a few table entries; and the candidates' log
    probabilities are those of the scores."""
    idx, ix, q, _, cand, preds, _ = _problem(B, 21, 16, 4, (0,), nq=10, n_cand=20, with_wz=False, scale=4.0)
    gen = torch.Generator(device="cuda").manual_seed(3)
    table = 0.3 * torch.randn(6, 64, generator=gen, device="cuda")
    ids = torch.randint(-1, 6, (10, 2), generator=gen, device="cuda", dtype=torch.int32)
    teacher = torch.rand(10, 5, generator=gen, device="cuda") * 8 + 1
    tau = 3.0
    w_z = B.embed_lookup(table, ids, 0.5) + 0.5
    alpha, wf = idx.select_codebook(q, preds, w_z)
    logits = idx.score_candidates(idx.build_lut(q, alpha, wf), cand)
    slots = torch.arange(5, device="cuda", dtype=torch.int32).repeat(10, 1)
    given, entropy, best, best_logp = B.log_probs(logits, slots, 8, tau=tau)
    there = (cand >= 0) & (cand < ix["codes"].shape[0])
    loss0, _ = B.distill_loss(logits, torch.where(there[:, :5], slots, -1), -teacher, tau=tau)
    loss, dwz = idx.distill_step(q, preds, w_z, cand, teacher, tau, 0.0, 0.0, want_dwz=True)
    g_table = B.embed_gradient(dwz, ids, 6, 0.5)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss0)                        # the step's loss is the operator's
    ref = R.log_probs(_np(logits).astype(np.float64), tau, None, _np(slots), 8)
    assert np.array_equal(_np(best), ref[2])
    for got, want in ((given, ref[0]), (entropy, ref[1]), (best_logp, ref[3])):
        fin = np.isfinite(want)
        assert np.array_equal(np.isfinite(_np(got)), fin)
        # exponents and logarithms of about 20 terms: a few 2^-22 of |log p| + 1
        assert np.all(np.abs(_np(got)[fin] - want[fin]) <= 2.0 ** -20 * (1 + np.abs(want[fin])))

    def mean_loss(t):
        w = 0.5 + 0.5 * sum(torch.where(ids[:, j, None] >= 0, t[ids[:, j].clamp(min=0).long()], 0.0) for j in (0, 1))
        return _reference(ix, q, w, cand, preds, teacher, tau, 0.0)[0].mean()

    h = 1e-4
    t64 = table.double()
    for row, col in ((0, 0), (2, 17), (5, 63)):
        up, down = t64.clone(), t64.clone()
        up[row, col] += h
        down[row, col] -= h
        diff = (mean_loss(up) - mean_loss(down)) / (2 * h)
        # differences: h^2 of the third derivative; the gradient: fp32 sums as in the training tests
        assert abs(float(g_table[row, col]) - diff) <= 2e-4 * max(float(g_table.abs().max()), 1e-30)


def test_training_loop_distils_and_learns_predicate_weights(B):
    """The training loop with the distillation loss and a table of predicate
    weights: it runs, the conditioned search starts as plain PQ, and what it
    reports is finite."""
    from paper_2607_22922_amd import train
    out = train.main(["--config", "c1", "--bin", "0.1", "--train-queries", "64", "--test-queries", "32", "--batch",
                      "32", "--epochs", "2", "--n-neg", "16", "--loss", "distill", "--wz-rows", "128", "--lr-wz", "0.5"])
    assert out["recall@10_conditioned_before"] == out["recall@10_identity"]
    assert all(np.isfinite(out["loss_per_epoch"])) and len(out["loss_per_epoch"]) == 2
    for when in ("before", "after"):
        stats = out[f"candidates_{when}"]
        assert all(np.isfinite(v) for v in stats.values())
        assert stats["logprob_of_neighbours"] <= 0 and stats["entropy"] >= 0
        assert 0 <= stats["best_is_a_neighbour"] <= 1
    assert out["wz_table_rows_touched"] > 0
