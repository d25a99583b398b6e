#!/usr/bin/env python3
"""Fine-tunes a fitted completion on link preferences and on rewards.

1. Fits S ~ max(0, W H) of a seeded community graph by SALSA sweeps.
2. Preferences: in each step some rows name a present and an absent column; the
   rows' scores are one matrix product, preference_loss compares the two
   columns' log-probabilities with those of the fitted model (factor_logprobs,
   which stores no scores) and gives the scores' gradient, the factors'
   gradients are two matrix products, clip_grad_norm bounds them, and a plain
   gradient step is taken.  (Both rows of a pair are one cell's here, so that
   their log-sum-exps cancel in the margin; pairs of different cells, or of
   sequences over several, take the same calls.)
3. Rewards: columns drawn from the model earn a reward where they are links;
   policy_loss with a KL term against the fitted model does the rest.

    python examples/tune_links.py [--cells 4096] [--steps 30]
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)


def fit(cells: int, rank: int, sweeps: int):
    from paper_2608_21607_gb300 import nmd, workloads

    S = workloads.communities(cells, cells, 8, 30.0, seed=3)
    W, H = workloads.init_factors(cells, cells, rank, 3)
    solver = nmd.Solver(S, rank, block_rows=1024, block_cols=1024, eta=0.5, gamma=0.9)
    solver.set_factors(W, H)
    for _ in range(sweeps):
        solver.sweep()
    return S, solver


def link_pairs(S, count: int, rng):
    """(rows, present columns, absent columns) of `count` rows that have links."""
    import numpy as np

    rows = rng.choice(np.flatnonzero(np.diff(S.row_ptr)), count)
    present = np.array([S.col_idx[rng.integers(S.row_ptr[i], S.row_ptr[i + 1])] for i in rows])
    absent = rng.integers(0, S.n, count)
    for k, i in enumerate(rows):
        while absent[k] in S.col_idx[S.row_ptr[i]:S.row_ptr[i + 1]]:
            absent[k] = rng.integers(0, S.n)
    return rows, present, absent


def step(factors, rows, logits, grad, rate: float, max_norm: float):
    """One gradient step on A = W and B = H^T from the gradient of logits = A[rows] B^T; returns the norm."""
    import torch

    from paper_2608_21607_gb300 import tuning

    A, B = factors
    grad = grad.float()
    dA = torch.zeros_like(A).index_add_(0, rows, grad @ B)
    dB = grad.t() @ A[rows]
    norm = tuning.clip_grad_norm([dA, dB], max_norm)
    A.sub_(dA, alpha=rate)
    B.sub_(dB, alpha=rate)
    return norm


def tune(S, solver, steps: int, pairs: int, rate: float = 20.0, seed: int = 0) -> dict:
    """Runs both stages; returns the share of preferred links and the mean reward before and after."""
    import numpy as np
    import torch

    from paper_2608_21607_gb300 import tuning

    W, H = solver.get_factors()
    A, B = torch.from_numpy(W).cuda(), torch.from_numpy(np.ascontiguousarray(H.T)).cuda()
    A0, B0 = A.clone(), B.clone()                       # the reference model
    rng = np.random.default_rng(seed)
    torch.manual_seed(seed)
    put = lambda v: torch.as_tensor(v, dtype=torch.int64, device="cuda")  # noqa: E731
    report = {"loss_before": solver.loss()["obj"]}

    # two sequences of one column per pair: present, absent
    offsets = torch.arange(2 * pairs + 1, device="cuda")
    checked = link_pairs(S, 4 * pairs, rng)

    def preferred():
        i, j, k = (put(v) for v in checked)
        return float((tuning.factor_logprobs(A[i], B, j) > tuning.factor_logprobs(A[i], B, k)).float().mean())

    report["preferred_before"] = preferred()
    for _ in range(steps):
        i, j, k = link_pairs(S, pairs, rng)
        rows, targets = put(np.repeat(i, 2)), put(np.stack([j, k], 1).reshape(-1))
        reference = tuning.factor_logprobs(A0[rows], B0, targets)
        logits = (A[rows] @ B.t()).bfloat16()
        out = tuning.preference_loss(logits, targets, offsets, reference, beta=0.5)
        step((A, B), rows, logits, out.grad, rate, 1.0)
    report["preferred_after"] = preferred()
    report["preference_loss"] = float(out.loss)

    links = torch.zeros((S.m, S.n), dtype=torch.bool, device="cuda")
    links[put(np.repeat(np.arange(S.m), np.diff(S.row_ptr))), put(S.col_idx)] = True
    live = put(np.flatnonzero(np.diff(S.row_ptr)))
    rewards = []
    for _ in range(steps):
        rows = live[torch.randint(0, live.numel(), (2 * pairs,), device="cuda")]
        logits = (A[rows] @ B.t()).bfloat16()
        targets = torch.multinomial(torch.softmax(logits.float(), 1), 1)[:, 0]
        reward = links[rows, targets].float()
        old = tuning.token_logprobs(logits, targets)
        reference = tuning.factor_logprobs(A0[rows], B0, targets)
        out = tuning.policy_loss(logits, targets, old, reference, reward - reward.mean(), kl_coef=0.01)
        step((A, B), rows, logits, out.grad, 4.0 * rate, 1.0)
        rewards.append(reward.mean())
    rewards = torch.stack(rewards).tolist()
    third = max(1, len(rewards) // 3)
    report["reward_before"], report["reward_after"] = sum(rewards[:third]) / third, sum(rewards[-third:]) / third
    report["kl"] = float(out.kl)
    solver.set_factors(A, B.t())                        # the tuned factors go on in the solver
    report["loss_after"] = solver.loss()["obj"]
    return report


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cells", type=int, default=4096)
    ap.add_argument("--rank", type=int, default=16)
    ap.add_argument("--sweeps", type=int, default=5)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--pairs", type=int, default=512)
    a = ap.parse_args(argv)
    S, solver = fit(a.cells, a.rank, a.sweeps)
    report = tune(S, solver, a.steps, a.pairs)
    for k, v in report.items():
        print("%-18s %.4f" % (k, v))
    return report


if __name__ == "__main__":
    main()
