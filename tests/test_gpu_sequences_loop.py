"""The operators of a fine-tuning loop together: chains by beam search, their states reordered, the best against the
worst chain of each group as a preference, the factors' gradients clipped, a Muon step on both factors.

A chain's score is the sum of its columns' log-probabilities: each of the two ways is off by TOL = u (128 + 4 R + 4 |lp|)
per column (u = 2^-24, R the spread of the row's logits) and the scores are rounded once per step.  The step is that of
the fp64 oracle on the same gradients, within 1e-4 of the update's norm: five steps of fp32 products on these matrices
(at most 500 x 24, kept away from rank deficiency by their noise) come out about 1e-6 off.
"""
import numpy as np
import pytest

import oracle as O
from gpu_common import require_gpu

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def gpu():
    return require_gpu()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("graph", [False, True])
def test_chains_preferences_and_step(dtype, graph):
    from paper_2608_21607_gb300 import tuning as t

    rng = np.random.default_rng(0)
    n, r, B, K, steps, end = 500, 24, 6, 4, 5, 7
    W = torch.from_numpy(rng.standard_normal((n, r)).astype(np.float32)).cuda()
    H = torch.from_numpy((0.5 * rng.standard_normal((r, n))).astype(np.float32)).cuda()
    start = torch.from_numpy(rng.integers(0, n, B)).cuda()

    # ---- chains
    last = start.repeat_interleave(K)
    scores = torch.full((B, K), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    done = torch.zeros((B, K), dtype=torch.bool, device="cuda")
    history = torch.full((B * K, steps + 3), -1, dtype=torch.int64, device="cuda")
    froms = torch.full((B * K, steps + 3), -1, dtype=torch.int64, device="cuda")
    rows = [history[:, :steps], froms[:, :steps]]
    for i in range(steps):
        logits = (W[last] @ H).to(dtype)
        kept = [v.clone() for v in (scores, done)]
        if graph:   # one step replayed
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                out = t.beam_select(logits, scores, finished=done, end=end)
            g.replay()
        else:
            out = t.beam_select(logits, scores, finished=done, end=end)
        best, parents, tokens, _ = O.tuning.beam_select(logits.double().cpu().numpy(), kept[0].cpu().numpy(), K,
                                                        kept[1].cpu().numpy(), end)
        assert np.array_equal(out.tokens.cpu().numpy(), tokens) and np.array_equal(out.parents.cpu().numpy(), parents)
        before = [v.clone() for v in rows]
        assert t.beam_reorder(rows, out.parents) is rows
        for v, b in zip(rows, before):
            assert np.array_equal(v.cpu().numpy(), O.tuning.beam_reorder(b.cpu().numpy(), parents))
        # a finished beam's further columns are left out (below zero)
        finished = done.gather(1, out.parents)
        history[:, i] = torch.where(finished, -1, out.tokens).view(-1)
        came = last.view(B, K).gather(1, out.parents)
        froms[:, i] = came.view(-1)
        scores, done = out.scores.clone(), out.finished.clone()
        last = out.tokens.clamp(min=0).view(-1)
    assert (history[:, steps:] == -1).all()

    # ---- a chain's score is the sum of its log-probabilities
    targets = history[:, :steps].reshape(-1).contiguous()
    logits = (W[froms[:, :steps].reshape(-1).clamp(min=0)] @ H).to(dtype)
    lp = t.token_logprobs(logits, targets).double().view(B * K, steps).sum(1).view(B, K)
    spread = float((logits.max(1).values - logits.min(1).values).max())
    tol = steps * (2 * U * (128 + 4 * spread + 4 * 30.0) + U * 150.0)
    assert torch.all((lp - scores.double()).abs() <= tol)

    # ---- the best against the worst of each group
    pick = torch.tensor([0, K - 1], device="cuda")
    chosen = history[:, :steps].view(B, K, steps)[:, pick].reshape(-1).contiguous()
    at = froms[:, :steps].view(B, K, steps)[:, pick].reshape(-1).clamp(min=0)
    offsets = torch.arange(2 * B + 1, device="cuda") * steps
    reference = t.factor_logprobs(W[at], H.t(), chosen)
    logits = (W[at] @ H).to(dtype)
    out = t.preference_loss(logits, chosen, offsets, reference, beta=0.5)
    assert abs(float(out.loss) - np.log(2.0)) < 0.05      # the reference is the model itself, up to the logits' type
    grad = out.grad.float()
    dW = torch.zeros_like(W).index_add_(0, at, grad @ H.t()) + 1e-6 * torch.randn_like(W)
    dH = W[at].t() @ grad + 1e-6 * torch.randn_like(H)
    norm = t.clip_grad_norm([dW, dH], 0.1)
    assert float(norm) > 0.0
    for weight, g in ((W, dW), (H, dH)):
        momentum = torch.zeros_like(g)
        want, m = O.tuning.muon_step(weight.double().cpu().numpy(), g.double().cpu().numpy(),
                                     momentum.double().cpu().numpy(), lr=0.02, weight_decay=0.01)
        start_weight = weight.double().cpu().numpy()
        t.muon_step(weight, g, momentum, lr=0.02, weight_decay=0.01)
        moved = np.linalg.norm(want - start_weight)
        assert moved > 0.0 and np.linalg.norm(weight.double().cpu().numpy() - want) <= 1e-4 * moved + U * np.linalg.norm(want)
        np.testing.assert_allclose(momentum.double().cpu().numpy(), m, rtol=1e-6, atol=1e-12)
