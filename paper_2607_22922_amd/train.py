"""Train the filter-aware conditioning (memory bank and W) on a synthetic
workload and measure what it does to recall (Section 2, training paragraph;
Section 3's train / test split of the query workload).

Usage:
    python -m paper_2607_22922_amd.train [--config c4] [--bin 0.01] ...

Every step runs in the library: positives are the exact filtered top-k of
the full-precision vectors (ifvs_exact_search), hard negatives the best
conditioned-ADC results that are not positives (ifvs_filtered_search with
the current parameters, re-mined every epoch), and ifvs_train_step updates
the bank and W.  With --loss distill the step is ifvs_distill_step: the exact
distances of the positives are the teacher.  With --wz-rows N the predicates'
weights are learned too: a predicate's w_z is a constant (w_f = 1 at the start)
plus the sum of the rows of an N-row table that its clauses hash to
(ifvs_embed_lookup), and the step's dL/dw_z goes back into those rows
(ifvs_embed_gradient).  Training starts from alpha = 0 (a zero bank) and w_f = 1,
as the paper does; W starts from the workload's random values (with W = 0
no gradient reaches the bank).  Prints one JSON line: the step throughput,
the loss per epoch and recall@k of the conditioned search on the training
queries and on held-out test queries before and after training (the
identity mode, plain PQ, is the "before" value), and what the student's
distribution over the training candidates says before and after
(ifvs_score_candidates, ifvs_log_probs): the mean log probability of the exact
neighbours, the entropy, and how often the most probable candidate is one.
"""
from __future__ import annotations

import argparse
import json
import math
import time

import torch


def _recall(ids, gt):
    hits = 0
    total = 0
    for a, b in zip(ids.tolist(), gt.tolist()):
        want = {v for v in b if v >= 0}
        hits += len(want & {v for v in a if v >= 0})
        total += len(want)
    return hits / max(1, total)


def clause_rows(preds, n_rows, max_clauses):
    """[n][max_clauses] int32: the table row of each clause (a hash of its
    column and bounds), -1 past a predicate's last."""
    rows = torch.full((len(preds), max_clauses), -1, dtype=torch.int32)
    for i, clauses in enumerate(preds):
        for j, clause in enumerate(clauses):
            key = 0
            for part in clause:
                key = (key * 1000003 + int(part) + 1) & ((1 << 61) - 1)
            rows[i, j] = key % n_rows
    return rows


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", default="c4")
    ap.add_argument("--N", type=int, default=None, help="base vectors (default: the config's)")
    ap.add_argument("--bin", type=float, default=0.01, help="selectivity bin of the training queries")
    ap.add_argument("--train-queries", type=int, default=2048)
    ap.add_argument("--test-queries", type=int, default=512)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--epochs", type=int, default=20)
    ap.add_argument("--n-neg", type=int, default=32, help="hard negatives per query")
    ap.add_argument("--tau", type=float, default=1.0)
    ap.add_argument("--lam", type=float, default=0.1, help="anchor regularizer weight")
    ap.add_argument("--lr", type=float, default=20.0)
    ap.add_argument("--loss", choices=("labels", "distill"), default="labels")
    ap.add_argument("--wz-rows", type=int, default=0, help="rows of the learned table of predicate weights (0: none)")
    ap.add_argument("--lr-wz", type=float, default=1.0, help="learning rate of that table")
    args = ap.parse_args(argv)

    from paper_2607_22922_amd import ifvs as B
    from workload import make_workload

    torch.cuda.set_device(0)
    dev = torch.device("cuda", 0)
    n_q = args.train_queries + args.test_queries
    t0 = time.time()
    w = make_workload(args.config, device=dev, n_queries=n_q, N=args.N, keep_x=True)
    torch.cuda.synchronize()
    gen_s = time.time() - t0
    k, batch = w.k, args.batch
    if args.bin not in w.bins:
        raise SystemExit(f"--bin must be one of {w.bins}")
    preds = w.preds[args.bin]
    bank0 = torch.zeros_like(w.bank)                       # alpha = 0 at the start
    idx = B.Index(w.codes, w.C_pq, w.attrs, bank0, w.W, w.r, w.h, w.hash_seed, max_batch=batch,
                  max_k=k + args.n_neg, cluster_cols=(0,))
    idx.load_vectors(w.x)
    w.x = None
    # Positives: the exact filtered top-k of every query.
    gt = torch.empty(n_q, k, dtype=torch.int32, device=dev)
    gt_dist = torch.empty(n_q, k, device=dev)
    for b0 in range(0, n_q, batch):
        sl = slice(b0, min(n_q, b0 + batch))
        ids, dist = idx.exact_search(w.queries[sl].contiguous(), preds[sl], k)
        gt[sl], gt_dist[sl] = ids, dist
    # Predicate weights from a table of rows, zero at the start (w_f = 1).
    wz_rows = wz_table = None
    if args.wz_rows > 0:
        wz_rows = clause_rows(preds, args.wz_rows, B.MAX_CLAUSES).to(dev)
        wz_table = torch.zeros(args.wz_rows, idx.dim, device=dev)

    def weights(sl):
        if wz_table is None:
            return None
        return B.embed_lookup(wz_table, wz_rows[sl]) + math.log(math.e - 1.0)

    train = range(0, args.train_queries)
    test = range(args.train_queries, n_q)

    def search(rows, kk, conditioned=True):
        out = torch.empty(len(rows), kk, dtype=torch.int32, device=dev)
        lo = rows.start
        for b0 in range(rows.start, rows.stop, batch):
            sl = slice(b0, min(rows.stop, b0 + batch))
            q = w.queries[sl].contiguous()
            if conditioned:
                alpha, wf = idx.select_codebook(q, preds[sl], weights(sl))
                lut = idx.build_lut(q, alpha, wf)
            else:
                lut = idx.build_lut(q)
            ids, _ = idx.search(preds[sl], lut, kk)
            out[b0 - lo:b0 - lo + ids.shape[0]] = ids
        return out

    def recall(rows, conditioned=True):
        ids = search(rows, k, conditioned)
        return _recall(ids, gt[rows.start:rows.stop])

    def candidates(sl, mined):
        """Positives, then the batch's hard negatives: mined results that are
        not positives, best first."""
        pos = gt[sl]
        is_pos = (mined[:, :, None] == pos[:, None, :]).any(dim=2) | (mined < 0)
        order = torch.argsort(is_pos.to(torch.int8), dim=1, stable=True)
        negs = torch.gather(mined, 1, order)[:, :args.n_neg]
        negs = torch.where(torch.gather(is_pos, 1, order)[:, :args.n_neg], torch.full_like(negs, -1), negs)
        return torch.cat([pos, negs], dim=1).contiguous()

    def distribution():
        """The student's distribution over the training queries' candidates."""
        mined = search(train, k + args.n_neg)
        logp = entropy = best = n = n_rows = 0.0
        for b0 in range(train.start, train.stop, batch):
            sl = slice(b0, min(train.stop, b0 + batch))
            q = w.queries[sl].contiguous()
            alpha, wf = idx.select_codebook(q, preds[sl], weights(sl))
            cand = candidates(sl, mined[sl.start - train.start:sl.stop - train.start])
            logits = idx.score_candidates(idx.build_lut(q, alpha, wf), cand)
            slots = torch.arange(k, device=dev, dtype=torch.int32).repeat(q.shape[0], 1)
            lp, h, top, _ = B.log_probs(logits, slots, 1, tau=args.tau)
            there = torch.isfinite(lp)
            logp += float(lp[there].sum())
            n += int(there.sum())
            entropy += float(h.sum())
            best += int(((top[:, 0] >= 0) & (top[:, 0] < k)).sum())
            n_rows += q.shape[0]
        return {"logprob_of_neighbours": logp / max(n, 1), "entropy": entropy / max(n_rows, 1),
                "best_is_a_neighbour": best / max(n_rows, 1)}

    before = {"train": recall(train), "test": recall(test)}
    identity = {"train": recall(train, False), "test": recall(test, False)}
    dist_before = distribution()
    losses, step_ms = [], 0.0
    n_steps = 0
    t_train = time.time()
    for epoch in range(args.epochs):
        mined = search(train, k + args.n_neg)             # current parameters
        ep_loss, ep_n = 0.0, 0
        for b0 in range(train.start, train.stop, batch):
            sl = slice(b0, min(train.stop, b0 + batch))
            cand = candidates(sl, mined[sl.start - train.start:sl.stop - train.start])
            q = w.queries[sl].contiguous()
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            w_z = weights(sl)
            if args.loss == "distill":
                loss, dwz = idx.distill_step(q, preds[sl], w_z, cand, gt_dist[sl], args.tau, args.lam, args.lr,
                                             want_dwz=w_z is not None)
            else:
                loss, dwz = idx.train_step(q, preds[sl], w_z, cand, k, args.tau, args.lam, args.lr,
                                           want_dwz=w_z is not None)
            if w_z is not None:
                B.embed_gradient(dwz, wz_rows[sl], args.wz_rows, -args.lr_wz, out=wz_table, accumulate=True)
            e1.record()
            torch.cuda.synchronize()
            step_ms += e0.elapsed_time(e1)
            n_steps += 1
            ep_loss += float(loss.sum())
            ep_n += loss.shape[0]
        losses.append(round(ep_loss / ep_n, 6))
    train_s = time.time() - t_train
    after = {"train": recall(train), "test": recall(test)}
    out = {
        "what": "iFVS conditioning trained with " + ("ifvs_distill_step" if args.loss == "distill" else "ifvs_train_step"),
        "config": args.config, "N": w.N, "bin": args.bin, "k": k,
        "train_queries": args.train_queries, "test_queries": args.test_queries,
        "epochs": args.epochs, "batch": batch, "n_neg": args.n_neg, "tau": args.tau, "lam": args.lam,
        "lr": args.lr, "bank_rows": int(w.bank.shape[0]), "r": w.r, "h": w.h,
        "train_step_queries_per_s": n_steps * batch / (step_ms / 1e3) if step_ms > 0 else None,
        "train_step_ms": step_ms / max(1, n_steps),
        "training_wall_s": round(train_s, 2), "generation_s": round(gen_s, 1),
        "loss_per_epoch": losses,
        f"recall@{k}_identity": identity,
        f"recall@{k}_conditioned_before": before,
        f"recall@{k}_conditioned_after": after,
        "candidates_before": dist_before,
        "candidates_after": distribution(),
    }
    if wz_table is not None:
        out.update(wz_rows=args.wz_rows, lr_wz=args.lr_wz,
                   wz_table_rows_touched=int((wz_table != 0).any(dim=1).sum()))
    print(json.dumps(out), flush=True)
    return out


if __name__ == "__main__":
    main()
