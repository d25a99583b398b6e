"""The fine-tuning operators at their edges, against the fp64 oracle (oracle/tuning.py) or a property of the definition.

Tolerances are those of test_gpu_tuning.py (counted from the formulas there) unless a test says otherwise.
"""
import numpy as np
import pytest

import oracle as O
from gpu_common import require_gpu
from paper_2608_21607_gb300 import nmd as N
from test_gpu_tuning import DTYPES, HALF, NORM_TOL, U, check, check_grad, cuda, make_grads, make_logits, tol_lp, tuning

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    return require_gpu()


def check_policy(r, x, y, lp, old, ref, adv, want, dtype, kl, temperature, borders=None):
    """Loss, terms and gradient of a policy batch against the oracle's, with the tolerances of test_policy_loss."""
    live = y >= 0
    e = tol_lp(x, y, lp, temperature) + U * np.abs(lp)
    w = O.tuning.policy_weights(y, borders)
    rho = np.where(live, np.exp(np.where(adv != 0, lp - old, 0.0)), 0.0)
    erho = rho * (e + U * (np.abs(lp) + np.abs(old) + 8))
    gap = np.where(live, ref - lp, 0.0)
    egap = e + U * (np.abs(gap) + np.abs(lp))
    ek = np.abs(np.expm1(gap)) * egap + 8 * U * (np.exp(gap) + np.abs(gap))
    eterm = w * (erho * np.abs(adv) + 4 * U * np.abs(rho * adv) + kl * ek)
    check("loss", r.loss.cpu().numpy(), want["loss"], eterm.sum() + 2 * U * np.sum(w * (np.abs(rho * adv) + 1)))
    check("kl", r.kl.cpu().numpy(), want["kl"], (w * ek).sum() + 4 * U * abs(want["kl"]))
    check("clipped", r.clipped.cpu().numpy(), want["clipped"], 4 * U)
    if r.grad is not None:
        dcoef = w * (erho * np.abs(adv) + 4 * U * np.abs(rho * adv) + kl * (np.exp(gap) * egap + 8 * U * np.exp(gap)))
        check_grad(r.grad, x, y, lp, want["coef"], dcoef, want["grad"], dtype, temperature)


def policy_values(lp, rng):
    """old, reference, advantages: ratios well away from the borders of the clipped range 0.8 to 1.3."""
    T = len(lp)
    return (np.float32(lp - rng.choice([-0.7, -0.1, 0.05, 0.6], T)), np.float32(lp + 0.4 * rng.standard_normal(T)),
            np.float32(rng.standard_normal(T)))


# a warp per row and a CTA per row, with and without a kernel of their own for the weights, and streamed rows
OUTSIDE = [(50, 200, "fp32"), (40, 5000, "bf16"), (1100, 60, "fp16"), (1030, 3000, "fp32"), (620, 25000, "bf16")]


@pytest.mark.parametrize("shape", OUTSIDE, ids=lambda s: "x".join(map(str, s)))
def test_policy_rows_outside_every_sequence(shape):
    """Live rows before the first border and past the last take no part, whatever they hold."""
    T, V, dtype = shape
    borders = [3, 3, T // 3, T - 4]
    g, x, y = make_logits(T + V, T, V, dtype, masked=0.2)
    rng = np.random.default_rng(T)
    out = np.r_[0:3, T - 4:T]
    y[out] = 1
    x[out] = rng.standard_normal((len(out), V))
    x[1, 1] = -200.0                       # log-probability -200 against a reference of 0: past fp32's range
    x[T - 2] = np.nan
    x[T - 1, 0] = np.inf
    g.copy_(torch.from_numpy(np.float32(x)))
    x = g.double().cpu().numpy()
    inside = y.copy()
    inside[out] = -1
    lp = O.tuning.token_logprobs(x, inside, 0.9)
    old, ref, adv = policy_values(lp, rng)
    given = [np.where(inside >= 0, v, np.float32(np.nan)) for v in (old, ref, adv)]
    for v, inf in zip(given, (-np.inf, np.inf, -np.inf)):
        v[0], v[1], v[T - 4] = 0.0, 0.0, inf
    given[2][1] = -1.0
    given[0][2], given[2][2] = -1e9, -1.0  # a ratio past fp32's range
    off = cuda(borders, torch.int64)
    args = dict(clip_low=0.2, clip_high=0.3, kl_coef=0.2, temperature=0.9)
    want = O.tuning.policy_loss(x, inside, old, ref, adv, borders, **args)
    for grad in (True, False):
        r = tuning().policy_loss(g, cuda(y, torch.int64), *map(cuda, given), offsets=off, grad=grad, **args)
        check_policy(r, x, inside, lp, old, ref, adv, want, dtype, 0.2, 0.9, borders)


@pytest.mark.parametrize("shape", [(50, 200, "fp32"), (40, 5000, "bf16"), (1100, 60, "fp16"), (620, 25000, "bf16")],
                         ids=lambda s: "x".join(map(str, s)))
def test_policy_advantage_of_zero(shape):
    """A row without an advantage has no first term, also where its ratio is past fp32's range."""
    T, V, dtype = shape
    g, x, y = make_logits(T + V, T, V, dtype, masked=0.2)
    rng = np.random.default_rng(V)
    lp = O.tuning.token_logprobs(x, y, 0.9)
    old, ref, adv = policy_values(lp, rng)
    none = rng.random(T) < 0.3
    adv[none] = 0.0
    old[none] = np.float32(lp[none] - 120.0)
    args = dict(clip_low=0.2, clip_high=0.3, kl_coef=0.2, temperature=0.9)
    want = O.tuning.policy_loss(x, y, old, ref, adv, **args)
    # such a row's ratio still counts as it is: nothing of it is cut off
    r = tuning().policy_loss(g, cuda(y, torch.int64), cuda(old), cuda(ref), cuda(adv), **args)
    check_policy(r, x, y, lp, old, ref, adv, want, dtype, 0.2, 0.9)


@pytest.mark.parametrize("shape", [(200_000, 2), (1500, 300), (1030, 9000)], ids=lambda s: "%dx%d" % s)
def test_policy_without_gradient_of_rows_all_left_out(shape):
    """Once the call's work on the stream is done, its workspace is free: what the caller writes there next stays."""
    T, V = shape
    x = torch.full((T, V), float("nan"), device="cuda", dtype=torch.bfloat16)
    y = torch.full((T,), -1, device="cuda", dtype=torch.int64)
    nan = torch.full((T,), float("nan"), device="cuda")
    ends = torch.tensor([0, T // 3, T], device="cuda")
    for off in (None, ends):
        for _ in range(5):
            p = tuning().policy_loss(x, y, nan, nan, nan, offsets=off, kl_coef=0.1, grad=False)
            assert p.grad is None
            kept = [float(v) for v in (p.loss, p.kl, p.clipped)], p.logps.any()
            del p
            tuning().policy_loss(x, y, nan, nan, nan, offsets=off, kl_coef=0.1, grad=False)
            reused = [torch.full((n,), 5.0, device="cuda") for n in (T, 2 * T, 4 * T, 4 * T + 64, 4 * T + 131)]
            assert all(bool((r == 5.0).all()) for r in reused)
            assert kept[0] == [0.0, 0.0, 0.0] and not kept[1]


# The streaming kernel's clusters: two, four, five and six CTAs a row in fp32 (from 36,864, 73,728, 98,304 and 122,880
# columns on), five and six in 16 bits (from 294,912 and 368,640); rows that six CTAs cannot hold are kept by a cluster
# of the row kernel (fp32 from 294,912 columns on) and, past what that holds, read twice
CLUSTERS = [(310, 40001, 0, 1, "fp32", True), (160, 90001, 7, 0, "fp32", False), (125, 100003, 0, 3, "fp32", True),
            (110, 139255, 9, 0, "fp32", True), (125, 300001, 0, 0, "bf16", True), (104, 370001, 0, 5, "fp16", False),
            (80, 300001, 3, 0, "fp32", True), (2, 400001, 0, 1, "fp32", False), (2, 400000, 0, 0, "fp32", True),
            (2, 900001, 0, 0, "bf16", True), (40, 400001, 0, 0, "fp32", False)]


@pytest.mark.parametrize("shape", CLUSTERS, ids=lambda s: "x".join(map(str, s)))
def test_policy_of_long_rows(shape):
    T, V, pad, shift, dtype, sequences = shape
    g, x, y = make_logits(V, T, V, dtype, pad=pad, shift=shift, banned=0.05, masked=0.3 if T > 2 else 0.0)
    rng = np.random.default_rng(T)
    lp = O.tuning.token_logprobs(x, y, 0.9)
    old, ref, adv = policy_values(lp, rng)
    borders = [0, T // 2, T // 2, T] if sequences else None
    args = dict(clip_low=0.2, clip_high=0.3, kl_coef=0.2, temperature=0.9)
    want = O.tuning.policy_loss(x, y, old, ref, adv, borders, **args)
    off = cuda(borders, torch.int64) if sequences else None
    given = [cuda(np.where(y >= 0, v, np.float32(np.nan))) for v in (old, ref, adv)]
    runs = [tuning().policy_loss(g, cuda(y, torch.int64), *given, offsets=off, **args) for _ in range(2)]
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    check("logps", runs[0].logps.cpu().numpy(), lp, tol_lp(x, y, lp, 0.9) + U * np.abs(lp))
    check_policy(runs[0], x, y, lp, old, ref, adv, want, dtype, 0.2, 0.9, borders)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_gradient_of_a_slice_takes_its_own_size(dtype):
    """The gradient's rows are less than a 128-byte line longer than the logits', however far apart those lie."""
    T, S, V = 6, 50, 1003
    g, x, y = make_logits(5, T, V, dtype)
    lp = O.tuning.token_logprobs(x, y)
    es = g.element_size()
    big = torch.zeros(T, S, V, dtype=g.dtype, device="cuda")
    wide = torch.zeros(T, 40 * V, dtype=g.dtype, device="cuda")
    for given in (big[:, -1, :], wide[:, :V], wide[:, 8:8 + V], wide.view(40 * T, V)[::40]):
        given.copy_(g)
        z = cuda(np.zeros(T))
        want = O.tuning.preference_loss(x, y, [0, 2, 6], np.zeros(T), 0.1)
        e = tol_lp(x, y, lp, 1.0) + U * np.abs(lp)
        r = tuning().preference_loss(given, cuda(y, torch.int64), cuda([0, 2, 6], torch.int64), z, beta=0.1)
        check_grad(r.grad, x, y, lp, want["coef"], np.full(T, 0.1 * 0.1 * e.sum()), want["grad"], dtype, 1.0)
        p = tuning().policy_loss(given, cuda(y, torch.int64), z, None, z + 1)
        for grad in (r.grad, p.grad):
            assert grad.untyped_storage().nbytes() < T * (V * es + 128)


def test_small_results_hold_nothing_else():
    """A scalar that is kept for a log does not keep the call's workspace."""
    g, _, y = make_logits(2, 3000, 40, "bf16")
    z, yt = cuda(np.zeros(3000)), cuda(y, torch.int64)
    r = tuning().preference_loss(g, yt, cuda(np.arange(3001) - np.arange(3001) % 3000, torch.int64), z)
    p = tuning().policy_loss(g, yt, z, z, z + 1, kl_coef=0.1)
    for scalar in (r.loss, p.loss, p.kl, p.clipped):
        assert scalar.dim() == 0 and scalar.untyped_storage().nbytes() <= 64


def test_written_gradients_count_as_changed():
    """Autograd finds that a tensor which it has saved was overwritten."""
    x, y = torch.randn(300, device="cuda"), torch.randn(7, 5, device="cuda").t()
    seen = [x._version, y._version]
    tuning().clip_grad_norm([x, y], 0.1)
    assert x._version > seen[0] and y._version > seen[1]
    out, seen = torch.empty_like(x), x._version
    was = out._version
    tuning().clip_grad_norm([x], 0.1, out=[out])
    assert out._version > was and x._version == seen
    w = torch.randn(300, device="cuda", requires_grad=True)
    saved = w * 1.0
    loss = (saved * saved).sum()
    tuning().clip_grad_norm([saved.detach()], 0.1)
    with pytest.raises(RuntimeError):
        loss.backward()
    with torch.inference_mode():
        z = torch.randn(300, device="cuda")
        tuning().clip_grad_norm([z], 0.1)
    assert abs(float(z.norm()) - 0.1) < 1e-5


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_log_probabilities_are_not_positive(dtype):
    """Rows whose target has all of the probability: log(1 - p) of a log-probability above 0 would be no number."""
    T, n, r = 400, 500, 64
    rng = np.random.default_rng(3)
    A = cuda(4.0 * rng.standard_normal((T, r))).to(DTYPES[dtype])
    B = cuda(4.0 * rng.standard_normal((n, r))).to(DTYPES[dtype])
    z = A.double() @ B.double().t()
    y = z.argmax(1)
    got = tuning().factor_logprobs(A, B, y)
    assert (got <= 0).all() and (got > -50).any()
    x = z.to(DTYPES[dtype])
    y = x.double().argmax(1)
    got = tuning().token_logprobs(x, y)
    assert (got <= 0).all()
    for V in (1, 3000):
        x = torch.full((T, V), -60.0, device="cuda", dtype=DTYPES[dtype])
        x[:, 0] = cuda(20.0 * rng.standard_normal(T)).to(x.dtype)
        got = tuning().token_logprobs(x, torch.zeros_like(y), temperature=0.3)
        assert (got <= 0).all()


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("max_norm", [1e-2, 1e-5, 1e-8])
def test_scales_below_the_normal_range(kind, max_norm):
    """max_norm / norm below fp32's smallest normal number: the scaled gradients keep their 24 bits."""
    grads = make_grads(6, [1000, 77, 8193], [kind], 1e37)
    old = [g.double().cpu().numpy() for g in grads]
    norm, want = O.tuning.clip_grad_norm(old, max_norm)
    assert max_norm / norm < 2.0 ** -126
    out = [torch.empty_like(g) for g in grads]
    tuning().clip_grad_norm(grads, max_norm, out=out)
    tuning().clip_grad_norm(grads, max_norm)
    for g, o, w in zip(grads, out, want):
        assert torch.equal(g, o)
        check("out", g.double().cpu().numpy(), w, (NORM_TOL + 4 * U + HALF[kind][0]) * np.abs(w) + 2.0 ** -126)


def test_written_tensors_that_overlap_are_refused():
    """A tensor that is written twice, or written while another is read from it, has no defined result."""
    clip = tuning().clip_grad_norm
    buf, other = torch.randn(4000, device="cuda"), torch.empty(4000, device="cuda")
    was = buf.clone()
    for grads, out in (([buf, buf], None), ([buf[:100], other, buf[99:200]], None),
                       ([buf[:10], buf[20:30]], [other[:10], other[9:19]]),
                       ([buf[:10], buf[10:20]], [buf[10:20], buf[:10]]),
                       ([buf[:100]], [buf[1:101]]), ([buf[100:200], buf[300:400]], [other[:100], buf[150:250]])):
        with pytest.raises(N.NmdError) as e:
            clip(grads, 0.1, out=out)
        assert e.value.status == N.NMD_ERR_INVALID
    assert torch.equal(buf, was)
    # neighbours, empty tensors anywhere, a gradient that is its own output, one that is read twice
    clip([buf[:100], buf[50:50], buf[100:201], buf[201:]], 0.1)
    assert abs(float(buf.norm()) - 0.1) < 1e-5
    clip([buf[:100], buf[100:200]], 1e-3, out=[buf[:100], other[:100]])
    assert abs(float((buf[:100].square().sum() + other[:100].square().sum()).sqrt()) - 1e-3) < 1e-7
    clip([was, was], 1.0, out=[other[:4000], torch.empty_like(was)])
    assert abs(float(other.norm()) - 0.5 ** 0.5) < 1e-5


@pytest.mark.parametrize("r", [100, 128, 192, 256])
def test_fp32_factor_scores_have_little_leaning(r):
    """Scores z near 100 made of positive products only, whose roundings towards zero all lean the same way.

    The r / 16 accumulations of the leading products lose half a unit of the sum so far on average, which grows evenly:
    2^-23 z (r / 16 + 1) / 4 in all.  The others are below 2^-7 of z together and there are five for each: 2^-23 z 5 (r /
    16) / 2 2^-7.  The target's own score (fp32, r / 32 additions in each lane) and the logarithm lean by u z at most.
    """
    rng = np.random.default_rng(r)
    A = cuda(np.sqrt(100 / r) * (0.5 + rng.random((600, r))))
    B = cuda(np.sqrt(100 / r) * (0.5 + rng.random((400, r))))
    y = rng.integers(0, 400, 600)
    a, b = A.double().cpu().numpy(), B.double().cpu().numpy()
    z = (a @ b.T).max()
    want = O.tuning.factor_logprobs(a, b, y)
    got = tuning().factor_logprobs(A, B, cuda(y, torch.int64)).cpu().numpy()
    leaning = abs(np.mean(got - want))
    assert leaning <= 2.0 ** -23 * z * ((r / 16 + 1) / 4 + 5 * (r / 16) / 2 * 2.0 ** -7) + U * z


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [16, 64, 500])
def test_short_rows_of_one_large_probability(V, dtype):
    """Rows in which one column has most of the probability, so that nothing averages its roundings.

    An exponent in (2, 4] is rounded to 2^-22, the exponential to about as much: 2^-22 / sqrt(12) (ln 2 and 1) each, of
    three quarters of the sum; the logarithm's and the result's roundings at 1.2 are 2^-23 / sqrt(12) each.  Together
    7.5e-8 in the root mean square; half as much again is allowed.
    """
    T = 4000
    rng = np.random.default_rng(V)
    x = rng.normal(3.0, 4.0, (T, 1)) - 30.0 - 5.0 * rng.random((T, V))
    for top in (1, 2):
        x[:, top] = x[:, 0] + 40.0 + rng.random(T)
        x[:, 5] = x[:, top] - 1.1
        g = cuda(x).to(DTYPES[dtype])
        y = np.full(T, 5)
        want = O.tuning.token_logprobs(g.double().cpu().numpy(), y)
        got = tuning().token_logprobs(g, cuda(y, torch.int64)).double().cpu().numpy()
        assert np.sqrt(np.mean((got - want) ** 2)) <= 1.1e-7
        x[:, top] = x[:, 0]
