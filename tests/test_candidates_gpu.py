"""Scores of listed candidates as callers may use them: several streams,
captured graphs, candidates and tables of any kind the wrapper takes."""
import pytest
import torch

from tests.test_train_gpu import _problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2607_22922_amd import ifvs
    return ifvs


def _scored(B, seed, cluster_cols=(0,), n_cand=300):
    idx, ix, q, w_z, cand, preds, _ = _problem(B, seed, 16, 4, cluster_cols, nq=9, n_cand=n_cand)
    alpha, wf = idx.select_codebook(q, preds, w_z)
    return idx, ix, idx.build_lut(q, alpha, wf), cand


def test_first_scores_on_two_streams(B):
    """The first call on a clustered index makes the order's inverse; a call on
    another stream right after it sees it whole."""
    idx, ix, lut, cand = _scored(B, 41)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(one):
        torch.cuda._sleep(20_000_000)
        a = idx.score_candidates(lut, cand)
    with torch.cuda.stream(two):
        b = idx.score_candidates(lut, cand)
    torch.cuda.synchronize()
    rows = ix["codes"].long()[cand.clamp(0, ix["codes"].shape[0] - 1).long()]
    want = -torch.gather(lut.double(), 2, rows.permute(0, 2, 1)).sum(1)
    there = (cand >= 0) & (cand < ix["codes"].shape[0])
    assert torch.equal(a, b)
    # 16 fp32 additions of table entries
    assert torch.all((a.double() - want).abs()[there] <= 16 * 2.0 ** -24 * want.abs()[there])
    assert torch.all(a[~there] == -float("inf"))


def test_scores_in_a_captured_graph(B):
    """The first call cannot be captured and says so; later ones can, and
    replay with new tables."""
    idx, _, lut, cand = _scored(B, 42)
    torch.cuda.synchronize()
    with pytest.raises(B.IfvsError) as e:
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            idx.score_candidates(lut, cand)
    assert e.value.status == B.E_STATE
    want = idx.score_candidates(lut, cand)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = idx.score_candidates(lut, cand)
    for step in range(3):
        lut.mul_(1.0 + step)
        want = idx.score_candidates(lut, cand)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), step


@pytest.mark.parametrize("cluster_cols", [(), (0,)])
def test_candidates_and_tables_of_any_layout(B, cluster_cols):
    """Wide ids (past 32 bits: absent), stepped ids and tables, and inputs of
    the step in other float types give what 32-bit contiguous ones give."""
    idx, ix, q, w_z, cand, preds, _ = _problem(B, 43, 16, 4, cluster_cols, nq=9, n_cand=40)
    alpha, wf = idx.select_codebook(q, preds, w_z)
    lut = idx.build_lut(q, alpha, wf)
    want = idx.score_candidates(lut, cand)
    assert torch.equal(idx.score_candidates(lut, cand.long()), want)
    assert torch.equal(idx.score_candidates(lut, cand.repeat_interleave(2, 1)[:, ::2]), want)
    assert torch.equal(idx.score_candidates(lut.repeat_interleave(2, 0)[::2], cand), want)
    wide = cand.long() + (1 << 32)
    assert torch.all(idx.score_candidates(lut, wide) == -float("inf"))
    teacher = torch.rand(9, 4, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") + 1
    half = q.half()
    ref = idx.distill_step(half.float(), preds, w_z, cand, teacher, 1.0, 0.1, 0.0, want_dwz=True)
    got = idx.distill_step(half, preds, w_z, cand.long(), teacher.double(), 1.0, 0.1, 0.0, want_dwz=True)
    torch.cuda.synchronize()
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


def test_training_loop_without_training_queries(B):
    """No training queries and no epochs: recall on the test queries alone."""
    from paper_2607_22922_amd import train
    out = train.main(["--config", "c1", "--bin", "0.1", "--train-queries", "0", "--test-queries", "32", "--batch",
                      "32", "--epochs", "0", "--n-neg", "16"])
    assert out["recall@10_conditioned_before"] == out["recall@10_identity"] == out["recall@10_conditioned_after"]
    assert out["candidates_before"] == {"logprob_of_neighbours": 0.0, "entropy": 0.0, "best_is_a_neighbour": 0.0}
