"""The fine-tuning operators against the fp64 oracle (oracle/tuning.py).

Tolerances, with u = 2^-24 (fp32 rounding), R the spread max - min of a row's
finite z = x / temperature and lp its log-probability:

* log-probabilities: each term 2^(c (x - m)) carries the rounding of c, of the
  difference and of the product (u R each, 3 u R) and of the exponential (4 u); the sum adds at most
  64 u by its order and 40 u by the rescalings of ten merges; the logarithm and
  the last difference add 2 u (|lp| + R).  Together below
  u (128 + 4 R + 4 |lp|), called TOL(lp) here.
* factors: a score's products are exact for 16-bit factors and the fp32 additions
  lose at most (r + 8) 2 u sum |a b|; fp32 factors, as six products of three
  pieces, (6 r + 8) 2 u and 8 u for what the pieces leave out.  A log-probability
  takes twice the largest of that over its row's columns, over temperature.
* preference: a ratio sums TOL(lp) + u |lp| over its rows (the log-probability
  is stored in fp32 first), the margin takes beta of two of them, the logistic
  function has slope at most 1/4, and coefficients are rounded once.
* policy: the ratio's relative error is TOL(lp) + u (|lp| + |old| + 4), each
  row's terms are a few roundings more; the sums are in fp64.
* gradients: |g| p / tau times the relative error of p (that of lp), |dg| / tau,
  4 u |g| / tau for the last operations, and half a unit of the logits' type.
"""
import numpy as np
import pytest

import oracle as O
from gpu_common import require_gpu
from paper_2608_21607_gb300 import nmd as N

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = 2.0 ** -24
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# half a unit in the last place (relative), and the spacing below the normal range
HALF = {"fp32": (2.0 ** -24, 2.0 ** -149), "bf16": (2.0 ** -8, 2.0 ** -133), "fp16": (2.0 ** -11, 2.0 ** -24)}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    return require_gpu()


def tuning():
    from paper_2608_21607_gb300 import tuning as t
    return t


def make_logits(seed, T, V, dtype, *, pad=0, shift=0, banned=0.0, masked=0.0, scale=2.5):
    """(CUDA logits, the same in fp64, targets): rows of stride V + pad starting `shift` elements into the storage;
    rows that are left out hold NaN."""
    rng = np.random.default_rng(seed)
    x = (scale * rng.standard_normal((T, V))).astype(np.float32)
    y = rng.integers(0, V, T)
    if T:
        y[0] = V - 1
        y[T // 2] = 0
    if banned:
        cols = rng.permutation(V)[:int(banned * V)]
        x[:, cols] = -np.inf
        free = np.setdiff1d(np.arange(V), cols)
        y = free[rng.integers(0, len(free), T)]
    x[np.arange(T), y] = rng.normal(5.0, 2.0, T)
    out = rng.random(T) < masked
    y[out] = -1 - rng.integers(0, 200, out.sum())
    x[out] = np.nan
    store = torch.zeros(shift + T * (V + pad) + 64, dtype=DTYPES[dtype], device="cuda")
    g = store[shift:shift + T * (V + pad)].view(T, V + pad)[:, :V]
    g.copy_(torch.from_numpy(x))
    return g, g.double().cpu().numpy(), y


def spread(x, y, temperature):
    z = np.where(np.isfinite(x), x, np.nan) / temperature
    with np.errstate(all="ignore"):
        r = np.nan_to_num(np.nanmax(z, axis=1, initial=-1e30) - np.nanmin(z, axis=1, initial=1e30))
    return np.where(y >= 0, np.maximum(r, 0.0), 0.0)


def tol_lp(x, y, lp, temperature):
    return np.where(y >= 0, U * (128 + 4 * spread(x, y, temperature) + 4 * np.abs(lp)), 0.0)


def check(name, got, want, tol):
    got = np.asarray(got, np.float64)
    assert got.shape == np.shape(want), name
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.abs(got - want)[bad].max(), np.broadcast_to(tol, bad.shape)[bad].max())


def check_grad(got, x, y, lp, coef, dcoef, want, dtype, temperature):
    rel, least = HALF[dtype]
    e = tol_lp(x, y, lp, temperature)
    z = np.where((y >= 0)[:, None], x, 0.0) / temperature
    p = np.exp(z - z.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    tol = (np.abs(coef) * e)[:, None] * p + (dcoef + 4 * U * np.abs(coef))[:, None]
    tol = tol / temperature + rel * np.abs(want) * (1 + 1e-3) + 2 * least + 2.0 ** -126
    tol[y < 0] = 0.0
    check("grad", got.double().cpu().numpy(), want, tol)


def cuda(v, dtype=torch.float32):
    return torch.as_tensor(np.ascontiguousarray(v), dtype=dtype, device="cuda")


SHAPES = [  # T, V, pad, shift
    (1, 1, 0, 0), (5, 2, 0, 0), (9, 7, 0, 1), (33, 33, 3, 0), (6, 1023, 0, 3), (6, 1024, 0, 0), (7, 1025, 0, 0),
    (3, 4097, 7, 5), (70, 6000, 0, 0), (400, 2049, 0, 1), (2, 50001, 0, 0), (1, 139255, 0, 0), (3, 139255, 9, 2),
    (5, 300001, 0, 1),
]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_token_logprobs(shape, dtype):
    T, V, pad, shift = shape
    for temperature, banned, masked in ((1.0, 0.0, 0.0), (0.7, 0.2 if V > 8 else 0.0, 0.4)):
        g, x, y = make_logits(T + V, T, V, dtype, pad=pad, shift=shift, banned=banned, masked=masked)
        got = tuning().token_logprobs(g, cuda(y, torch.int64), temperature=temperature)
        want = O.tuning.token_logprobs(x, y, temperature)
        check("logps", got.cpu().numpy(), want, tol_lp(x, y, want, temperature) + U * np.abs(want))


@pytest.mark.parametrize("V", [40, 5000])
def test_logprobs_of_unusual_rows(V):
    low = torch.finfo(torch.float32).min
    x = torch.randn(9, V, device="cuda")
    y = torch.full((9,), 3, device="cuda", dtype=torch.int64)
    x[0, 5:] = low                    # masked with the lowest value
    x[1, :] = low                     # nothing but it: uniform
    x[2, 5:] = float("-inf")          # masked with -inf
    x[3, :] = float("-inf")           # nothing left
    x[4, 7] = float("nan")
    x[5, 7] = float("inf")
    x[6, 3] = float("-inf")           # the target itself is banned
    y[7] = V                          # past the last column
    x[8, :] = 3e38                    # near the largest value: uniform
    got = tuning().token_logprobs(x, y).cpu()
    few = torch.log_softmax(x[:, :5].double().cpu(), 1)[:, 3]
    assert abs(got[0] - few[0]) < 1e-5 and abs(got[2] - few[2]) < 1e-5
    assert abs(got[1] + np.log(V)) < 1e-5 and abs(got[8] + np.log(V)) < 1e-5
    assert torch.isnan(got[[3, 4, 5, 7]]).all() and got[6] == float("-inf")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("temperature", [1e-3, 0.05, 30.0, 3000.0])
def test_temperatures(dtype, temperature):
    """Sharp and flat distributions, with banned columns and large common offsets of the logits."""
    for V, shift in ((700, 0.0), (9000, 0.0), (9000, -3000.0), (9000, 900.0)):
        g, x, y = make_logits(V, 12, V, dtype, banned=0.1)
        g += shift
        x = g.double().cpu().numpy()
        got = tuning().token_logprobs(g, cuda(y, torch.int64), temperature=temperature)
        want = O.tuning.token_logprobs(x, y, temperature)
        check("logps", got.cpu().numpy(), want, tol_lp(x, y, want, temperature) + U * np.abs(want))


def test_no_rows_and_equal_bits():
    t = tuning()
    x = torch.empty(0, 12, device="cuda")
    y = torch.empty(0, device="cuda", dtype=torch.int64)
    v = torch.empty(0, device="cuda")
    assert t.token_logprobs(x, y).shape == (0,)
    r = t.preference_loss(x, y, torch.zeros(3, device="cuda", dtype=torch.int64), v)
    assert abs(float(r.loss) - np.log(2.0)) < 1e-6 and r.grad.shape == (0, 12)
    p = t.policy_loss(x, y, v, v, v, kl_coef=0.1)
    assert float(p.loss) == 0.0 and p.grad.shape == (0, 12)
    g, _, y = make_logits(1, 300, 5001, "bf16", masked=0.2)
    ref = cuda(np.zeros(300))
    runs = [t.preference_loss(g, cuda(y, torch.int64), cuda([0, 90, 150, 299, 300], torch.int64), ref)
            for _ in range(2)]
    for a, b in zip(*runs):
        assert torch.equal(a, b)


def make_factors(seed, T, n, r, dtype, scale=1.0):
    rng = np.random.default_rng(seed)
    f = scale * np.sqrt(2.5 / np.sqrt(r))
    A = cuda(f * rng.standard_normal((T, r))).to(DTYPES[dtype])
    B = cuda(f * rng.standard_normal((n, r))).to(DTYPES[dtype])
    y = rng.integers(0, n, T)
    y[0], y[-1] = n - 1, 0
    y[rng.random(T) < 0.2] = -3
    return A, B, y


def check_factors(A, B, y, dtype, temperature, got):
    a, b, r = A.double().cpu().numpy(), B.double().cpu().numpy(), A.shape[1]
    a = np.where((y >= 0)[:, None], a, 0.0)
    want = O.tuning.factor_logprobs(a, b, y, temperature)
    worst = (np.abs(a) @ np.abs(b).T).max(axis=1)
    ez = worst * ((6 * r + 8) * 2 * U + 8 * U if dtype == "fp32" else (r + 8) * 2 * U)
    tol = 2 * ez / temperature + tol_lp(a @ b.T, y, want, temperature) + U * np.abs(want)
    check("logps", got.cpu().numpy(), want, np.where(y >= 0, tol, 0.0))


FACTORS = [  # T, n, r
    (1, 1, 1), (1, 2, 3), (5, 127, 16), (128, 128, 64), (129, 129, 17), (300, 1000, 65), (7, 20001, 64),
    (1000, 257, 100), (33, 5000, 128), (257, 3001, 129), (64, 4097, 200), (513, 2500, 256), (2, 139255, 64),
    (40000, 40, 8),
]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", FACTORS, ids=lambda s: "x".join(map(str, s)))
def test_factor_logprobs(shape, dtype):
    T, n, r = shape
    for temperature in (1.0, 0.6):
        A, B, y = make_factors(T + n, T, n, r, dtype)
        got = tuning().factor_logprobs(A, B, cuda(y, torch.int64), temperature=temperature)
        check_factors(A, B, y, dtype, temperature, got)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_factor_layouts(dtype):
    """Every layout gives what contiguous factors give: H as it is stored (r x n), rows cut out of wider ones,
    unaligned starts, broadcast rows."""
    A, B, y = make_factors(3, 200, 777, 40, dtype)
    yt = cuda(y, torch.int64)
    H = B.t().contiguous()
    wide = torch.zeros(777, 64, dtype=B.dtype, device="cuda")
    odd = torch.zeros(777 * 41 + 1, dtype=B.dtype, device="cuda")[1:].view(777, 41)
    wide[:, 8:48] = B
    odd[:, 1:] = B
    want = tuning().factor_logprobs(A, B, yt)
    check_factors(A, B, y, dtype, 1.0, want)
    for given in (H.t(), wide[:, 8:48], odd[:, 1:]):
        assert torch.equal(tuning().factor_logprobs(A, given, yt), want)
    assert torch.equal(tuning().factor_logprobs(A.t().contiguous().t(), B, yt), want)
    same = A[5:6].expand(200, 40)
    check_factors(same, B, y, dtype, 1.0, tuning().factor_logprobs(same, B, yt))


def test_factor_rows_that_are_no_numbers():
    """A NaN or infinite row of A spoils its own result only, unless it is left out."""
    A, B, y = make_factors(4, 150, 300, 64, "bf16")
    y[:] = np.arange(150)
    y[9] = -1
    A[9], A[20], A[21, 3] = float("nan"), float("nan"), float("inf")
    yt = cuda(y, torch.int64)
    yt[33] = 300                          # past the last column
    got = tuning().factor_logprobs(A, B, yt).cpu()
    bad = torch.zeros(150, dtype=torch.bool)
    bad[[20, 21, 33]] = True
    assert torch.equal(torch.isnan(got), bad) and got[9] == 0.0
    A, B, y = make_factors(4, 3, 300, 64, "fp32")
    assert tuning().factor_logprobs(A[:0], B, torch.empty(0, dtype=torch.int64, device="cuda")).shape == (0,)


PREFERENCE = [  # T, V, pad, shift, borders
    (2, 5, 0, 0, [0, 1, 2]),
    (40, 300, 0, 1, [0, 0, 7, 7, 7, 30, 36]),            # empty sequences, rows past the last
    (64, 1500, 4, 0, [2, 9, 33, 40, 64]),                # rows before the first
    (31, 4099, 0, 0, list(range(0, 31, 2)) + [31]),
    (12, 139255, 0, 0, [0, 5, 12]),
    (1300, 77, 0, 0, [0, 640, 1300]),
]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("case", PREFERENCE, ids=lambda c: "%dx%d" % c[:2])
def test_preference_loss(case, dtype):
    T, V, pad, shift, borders = case
    if len(borders) % 2 == 0:
        borders = borders[:-1]
    for average, smoothing, temperature, masked in ((False, 0.0, 1.0, 0.0), (True, 0.15, 1.4, 0.5)):
        g, x, y = make_logits(T * V, T, V, dtype, pad=pad, shift=shift, masked=masked)
        lp = O.tuning.token_logprobs(x, y, temperature)
        rng = np.random.default_rng(T)
        ref = np.float32(lp + 0.4 * rng.standard_normal(T))
        beta = 0.3
        want = O.tuning.preference_loss(x, y, borders, ref, beta, smoothing, average, temperature)
        # left-out rows hold garbage
        given = np.where(y >= 0, ref, np.float32(np.nan))
        r = tuning().preference_loss(g, cuda(y, torch.int64), cuda(borders, torch.int64), cuda(given), beta=beta,
                                     label_smoothing=smoothing, average=average, temperature=temperature)
        e = tol_lp(x, y, lp, temperature) + U * np.abs(lp)
        check("logps", r.logps.cpu().numpy(), want["logps"], e)
        K = len(borders) - 1
        n = [max(1, int((y[borders[k]:borders[k + 1]] >= 0).sum())) if average else 1 for k in range(K)]
        er = np.array([e[borders[k]:borders[k + 1]].sum() / n[k] for k in range(K)])
        check("ratios", r.ratios.cpu().numpy(), want["ratios"], er + 2 * U * np.abs(want["ratios"]) + 1e-12)
        eh = beta * (er[0::2] + er[1::2])
        check("margins", r.margins.cpu().numpy(), want["margins"], eh + 2 * U * np.abs(want["margins"]) + 1e-12)
        check("loss", r.loss.cpu().numpy(), want["loss"], eh.mean() + 2 * U * abs(want["loss"]))
        dcoef = np.zeros(T)
        for k in range(K):
            dcoef[borders[k]:borders[k + 1]] = beta / (K // 2) * eh[k // 2] / 4 / n[k]
        check_grad(r.grad, x, y, lp, want["coef"], dcoef, want["grad"], dtype, temperature)
        only = tuning().preference_loss(g, cuda(y, torch.int64), cuda(borders, torch.int64), cuda(given), beta=beta,
                                        label_smoothing=smoothing, average=average, temperature=temperature,
                                        grad=False)
        assert only.grad is None and torch.equal(only.loss, r.loss) and torch.equal(only.logps, r.logps)


POLICY = [  # T, V, pad, shift, borders
    (1, 3, 0, 0, None),
    (50, 200, 0, 1, None),
    (50, 1024, 0, 0, [0, 0, 13, 50]),
    (65, 2500, 6, 0, [1, 40, 40, 60]),
    (9, 33000, 0, 0, None),
    (6, 139255, 0, 0, [0, 2, 6]),
    (3, 300001, 0, 1, None),
    (2100, 60, 0, 0, [0, 1000, 2100]),
]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("case", POLICY, ids=lambda c: "%dx%d" % c[:2])
def test_policy_loss(case, dtype):
    T, V, pad, shift, borders = case
    for kl, temperature, masked, with_ref in ((0.0, 1.0, 0.0, False), (0.2, 0.8, 0.4, True)):
        g, x, y = make_logits(T + V, T, V, dtype, pad=pad, shift=shift, masked=masked)
        rng = np.random.default_rng(V)
        lp = O.tuning.token_logprobs(x, y, temperature)
        # ratios well away from the borders of the clipped range
        old = np.float32(lp - rng.choice([-0.7, -0.1, 0.05, 0.6], T))
        ref = np.float32(lp + 0.4 * rng.standard_normal(T)) if with_ref else None
        adv = np.float32(rng.standard_normal(T))
        args = dict(clip_low=0.2, clip_high=0.3, kl_coef=kl, temperature=temperature)
        want = O.tuning.policy_loss(x, y, old, ref, adv, borders, **args)
        hide = lambda v: None if v is None else cuda(np.where(y >= 0, v, np.float32(np.nan)))  # noqa: E731
        off = None if borders is None else cuda(borders, torch.int64)
        r = tuning().policy_loss(g, cuda(y, torch.int64), hide(old), hide(ref), hide(adv), offsets=off, **args)
        e = tol_lp(x, y, lp, temperature) + U * np.abs(lp)
        check("logps", r.logps.cpu().numpy(), want["logps"], e)
        w = O.tuning.policy_weights(y, borders)
        live = y >= 0
        rho = np.where(live, np.exp(lp - old), 0.0)
        erho = rho * (e + U * (np.abs(lp) + np.abs(old) + 8))
        gap = np.where(live, ref - lp, 0.0) if with_ref else np.zeros(T)
        egap = e + U * (np.abs(gap) + np.abs(lp))
        ek = np.abs(np.expm1(gap)) * egap + 8 * U * (np.exp(gap) + np.abs(gap))
        eterm = w * (erho * np.abs(adv) + 4 * U * np.abs(rho * adv) + kl * ek)
        check("loss", r.loss.cpu().numpy(), want["loss"], eterm.sum() + 2 * U * np.sum(w * (np.abs(rho * adv) + 1)))
        check("kl", r.kl.cpu().numpy(), want["kl"], (w * ek).sum() + 4 * U * abs(want["kl"]))
        check("clipped", r.clipped.cpu().numpy(), want["clipped"], 4 * U)
        dcoef = w * (erho * np.abs(adv) + 4 * U * np.abs(rho * adv) + kl * (np.exp(gap) * egap + 8 * U * np.exp(gap)))
        check_grad(r.grad, x, y, lp, want["coef"], dcoef, want["grad"], dtype, temperature)
        only = tuning().policy_loss(g, cuda(y, torch.int64), hide(old), hide(ref), hide(adv), offsets=off, grad=False,
                                    **args)
        assert only.grad is None and torch.equal(only.loss, r.loss) and torch.equal(only.kl, r.kl)


# batches that fill the GPU take other kernels than the ones above: long rows stream through a ring of shared-memory
# slots (one CTA or a cluster of them per row), short ones take a warp each
LARGE = [(611, 30001, 0, 1, "bf16"), (620, 25000, 0, 0, "fp16"), (615, 12301, 3, 2, "fp32"), (310, 100003, 5, 0, "bf16"),
         (205, 200005, 0, 3, "fp16"), (2500, 3001, 0, 1, "bf16"), (2440, 4096, 0, 0, "fp16"), (2440, 1500, 1, 0, "fp32"),
         (1300, 9000, 0, 0, "bf16"), (2433, 6000, 0, 5, "fp16")]


@pytest.mark.parametrize("shape", LARGE, ids=lambda s: "x".join(map(str, s)))
def test_large_batches(shape):
    T, V, pad, shift, dtype = shape
    g, x, y = make_logits(V, T, V, dtype, pad=pad, shift=shift, banned=0.05, masked=0.3)
    rng = np.random.default_rng(T)
    lp = O.tuning.token_logprobs(x, y, 0.9)
    yt = cuda(y, torch.int64)
    e = tol_lp(x, y, lp, 0.9) + U * np.abs(lp)
    check("logps", tuning().token_logprobs(g, yt, temperature=0.9).cpu().numpy(), lp, e)
    old = np.float32(lp - rng.choice([-0.7, -0.1, 0.05, 0.6], T))
    ref = np.float32(lp + 0.4 * rng.standard_normal(T))
    adv = np.float32(rng.standard_normal(T))
    want = O.tuning.policy_loss(x, y, old, ref, adv, kl_coef=0.2, temperature=0.9)
    hide = lambda v: cuda(np.where(y >= 0, v, np.float32(np.nan)))  # noqa: E731
    runs = [tuning().policy_loss(g, yt, hide(old), hide(ref), hide(adv), kl_coef=0.2, temperature=0.9)
            for _ in range(2)]
    r = runs[0]
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    check("logps", r.logps.cpu().numpy(), lp, e)
    w = O.tuning.policy_weights(y)
    rho = np.where(y >= 0, np.exp(lp - old), 0.0)
    erho = rho * (e + U * (np.abs(lp) + np.abs(old) + 8))
    gap = np.where(y >= 0, ref - lp, 0.0)
    egap = e + U * (np.abs(gap) + np.abs(lp))
    dcoef = w * (erho * np.abs(adv) + 4 * U * np.abs(rho * adv) + 0.2 * (np.exp(gap) * egap + 8 * U * np.exp(gap)))
    check("loss", r.loss.cpu().numpy(), want["loss"], dcoef.sum() + 4 * U * np.sum(w * (np.abs(rho * adv) + 1)))
    check_grad(r.grad, x, y, lp, want["coef"], dcoef, want["grad"], dtype, 0.9)


# many short pairs, some longer ones, empty ones, rows before the first and past the last
SHORT = [  # P, rows per pair, V, pad, shift, dtype
    (1230, 2, 2101, 0, 1, "bf16"), (310, 7, 2300, 0, 0, "fp32"), (160, 2, 30011, 0, 3, "fp16"),
    (80, 2, 60001, 7, 0, "bf16"), (40, 2, 139255, 0, 0, "bf16"), (310, 3, 5000, 4, 2, "fp32"), (45, 1, 100003, 0, 1, "fp32"),
    (610, 2, 25001, 0, 1, "bf16"), (305, 2, 60001, 7, 0, "fp16"), (610, 3, 12501, 0, 0, "fp32"), (152, 2, 139255, 0, 3, "bf16"),
]


@pytest.mark.parametrize("even", [True, False], ids=["even", "ragged"])
@pytest.mark.parametrize("shape", SHORT, ids=lambda s: "x".join(map(str, s)))
def test_short_pairs(shape, even):
    P, each, V, pad, shift, dtype = shape
    T = P * each
    rng = np.random.default_rng(P + V)
    if even:
        borders = np.minimum(np.arange(2 * P + 1) * each // 2 + (1 if each == 1 else 0), T)
    else:
        borders = np.sort(np.minimum(rng.integers(2, T, 2 * P + 1), T - 3))
        borders[9:14] = borders[14] if borders[14] < T - 40 else borders[9]   # empty pairs, then one of 29 rows
        borders[15:] = np.maximum(borders[15:], borders[14] + 29)
    for average, smoothing, temperature, masked in ((False, 0.0, 1.0, 0.0), (True, 0.15, 1.4, 0.4)):
        g, x, y = make_logits(T + V, T, V, dtype, pad=pad, shift=shift, masked=masked)
        lp = O.tuning.token_logprobs(x, y, temperature)
        ref = np.float32(lp + 0.4 * rng.standard_normal(T))
        beta = 0.3
        want = O.tuning.preference_loss(x, y, borders, ref, beta, smoothing, average, temperature)
        given = np.where(y >= 0, ref, np.float32(np.nan))
        runs = [tuning().preference_loss(g, cuda(y, torch.int64), cuda(borders, torch.int64), cuda(given), beta=beta,
                                         label_smoothing=smoothing, average=average, temperature=temperature)
                for _ in range(2)]
        r = runs[0]
        for a, b in zip(*runs):
            assert torch.equal(a, b)
        e = tol_lp(x, y, lp, temperature) + U * np.abs(lp)
        check("logps", r.logps.cpu().numpy(), want["logps"], e)
        K = 2 * P
        n = [max(1, int((y[borders[k]:borders[k + 1]] >= 0).sum())) if average else 1 for k in range(K)]
        er = np.array([e[borders[k]:borders[k + 1]].sum() / n[k] for k in range(K)])
        check("ratios", r.ratios.cpu().numpy(), want["ratios"], er + 2 * U * np.abs(want["ratios"]) + 1e-12)
        eh = beta * (er[0::2] + er[1::2])
        check("margins", r.margins.cpu().numpy(), want["margins"], eh + 2 * U * np.abs(want["margins"]) + 1e-12)
        check("loss", r.loss.cpu().numpy(), want["loss"], eh.mean() + 2 * U * abs(want["loss"]))
        dcoef = np.zeros(T)
        for k in range(K):
            dcoef[borders[k]:borders[k + 1]] = beta / P * eh[k // 2] / 4 / n[k]
        check_grad(r.grad, x, y, lp, want["coef"], dcoef, want["grad"], dtype, temperature)


def test_all_rows_left_out():
    g, _, _ = make_logits(3, 20, 3000, "bf16")
    g.fill_(float("nan"))
    y = torch.full((20,), -1, device="cuda", dtype=torch.int64)
    nan = torch.full((20,), float("nan"), device="cuda")
    r = tuning().preference_loss(g, y, cuda([0, 10, 20], torch.int64), nan, average=True)
    assert abs(float(r.loss) - np.log(2.0)) < 1e-6 and not r.grad.any() and not r.logps.any()
    for off in (None, cuda([0, 10, 20], torch.int64)):
        p = tuning().policy_loss(g, y, nan, nan, nan, offsets=off, kl_coef=0.1)
        assert float(p.loss) == 0.0 and float(p.kl) == 0.0 and not p.grad.any()


@pytest.mark.parametrize("V", [90, 2600])
def test_gradients_by_differences(V):
    """The directional derivative of the oracle's loss against the kernel's gradient (fp32 logits).  The gradient's
    entries are within 1e-5 of |g_t|; a direction of unit entries adds at most 1e-5 sum |g| sqrt(V) of that, and the
    central difference (h = 1e-5) about 1e-9."""
    T = 30
    g, x, y = make_logits(V, T, V, "fp32", masked=0.2)
    x[y < 0] = 0.0
    rng = np.random.default_rng(0)
    lp = O.tuning.token_logprobs(x, y)
    ref = np.float32(lp + 0.4 * rng.standard_normal(T))
    old = np.float32(lp - rng.choice([-0.7, -0.1, 0.05, 0.6], T))
    adv = np.float32(rng.standard_normal(T))
    d = rng.choice([-1.0, 1.0], x.shape)
    borders = [0, 8, 15, 22, 30]
    h = 1e-5
    loss = lambda z: O.tuning.preference_loss(z, y, borders, ref)["loss"]  # noqa: E731
    r = tuning().preference_loss(g, cuda(y, torch.int64), cuda(borders, torch.int64), cuda(ref))
    c = O.tuning.preference_loss(x, y, borders, ref)["coef"]
    got = float((r.grad.double().cpu().numpy() * d).sum())
    assert abs(got - (loss(x + h * d) - loss(x - h * d)) / (2 * h)) < 1e-5 * np.abs(c).sum() * np.sqrt(V) + 1e-8
    loss = lambda z: O.tuning.policy_loss(z, y, old, ref, adv, kl_coef=0.1)["loss"]  # noqa: E731
    r = tuning().policy_loss(g, cuda(y, torch.int64), cuda(old), cuda(ref), cuda(adv), kl_coef=0.1)
    c = O.tuning.policy_loss(x, y, old, ref, adv, kl_coef=0.1)["coef"]
    got = float((r.grad.double().cpu().numpy() * d).sum())
    assert abs(got - (loss(x + h * d) - loss(x - h * d)) / (2 * h)) < 1e-5 * np.abs(c).sum() * np.sqrt(V) + 1e-8


def test_row_offsets_past_32_bits():
    """Three rows whose elements start more than 2^31 apart, and a broadcast row."""
    V, ld = 3001, (1 << 31) + 24
    store = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(store, (3, V), (ld, 1))
    g, _, y = make_logits(2, 3, V, "bf16")
    x.copy_(g)
    yt, z = cuda(y, torch.int64), cuda(np.zeros(3))
    one = g[:1].expand(3, V)
    for given in (x, one):
        v = given.double().cpu().numpy()
        lp = O.tuning.token_logprobs(v, y)
        e = tol_lp(v, y, lp, 1.0) + U * np.abs(lp)
        off = [0, 1, 3]
        want = O.tuning.preference_loss(v, y, off, np.zeros(3), 0.1)
        r = tuning().preference_loss(given, yt, cuda(off, torch.int64), z, beta=0.1)
        check("logps", r.logps.cpu().numpy(), lp, e)
        check_grad(r.grad, v, y, lp, want["coef"], np.full(3, 0.1 * 0.1 * e.sum()), want["grad"], "bf16", 1.0)


def test_another_stream():
    s = torch.cuda.Stream()
    g, x, y = make_logits(8, 64, 9001, "bf16")
    z = cuda(np.zeros(64))
    yt = cuda(y, torch.int64)
    want = tuning().policy_loss(g, yt, z - 2, z - 2, z + 1, kl_coef=0.1)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        h = torch.zeros_like(g)
        for _ in range(20):
            h.add_(1)
        h.copy_(g)
        got = tuning().policy_loss(h, yt, z - 2, z - 2, z + 1, kl_coef=0.1)
        grads = [got.grad.clone()]
        norm = tuning().clip_grad_norm(grads, 1e-3)
    s.synchronize()
    assert torch.equal(got.grad, want.grad) and torch.equal(got.loss, want.loss)
    assert abs(float(norm) - float(want.grad.double().norm())) < 1e-5 * float(norm)


# ---------------------------------------------------------------------------------------------- the gradients' norm

def make_grads(seed, sizes, kinds, scale=1.0):
    rng = np.random.default_rng(seed)
    out = []
    for k, n in enumerate(sizes):
        store = torch.zeros(n + 9, dtype=DTYPES[kinds[k % len(kinds)]], device="cuda")
        v = store[k % 3:k % 3 + n]          # every alignment of an element
        v.copy_(torch.from_numpy((scale * rng.standard_normal(n)).astype(np.float32)))
        out.append(v)
    return out


# squares: 2 u each, at most 40 additions per thread and chunk in fp32, then fp64: relative error of the norm below
# 64 u; a scaled element has that, the scale's rounding, its own and half a unit of its type
NORM_TOL = 64 * U


@pytest.mark.parametrize("kinds", [("fp32",), ("bf16",), ("fp16",), ("fp32", "bf16", "fp16")], ids="-".join)
@pytest.mark.parametrize("sizes", [[1], [0, 3], [5, 0, 17, 8192, 8193, 16385, 100003], [3_000_001], [7] * 40,
                                   list(range(1, 700))], ids=lambda s: "%d_tensors_%d" % (len(s), sum(s)))
@pytest.mark.parametrize("max_norm", [0.5, 1e6])
def test_clip_grad_norm(sizes, kinds, max_norm):
    grads = make_grads(len(sizes), sizes, kinds)
    old = [g.double().cpu().numpy() for g in grads]
    norm, want = O.tuning.clip_grad_norm(old, max_norm)
    out = [torch.full_like(g, 7.0) for g in grads]
    got = tuning().clip_grad_norm(grads, max_norm, out=out)
    assert abs(float(got) - norm) <= NORM_TOL * norm
    in_place = [g.clone() for g in grads]
    tuning().clip_grad_norm(in_place, max_norm)
    for k, (g, o, i, w) in enumerate(zip(grads, out, in_place, want)):
        kind = kinds[k % len(kinds)]
        assert np.array_equal(g.double().cpu().numpy(), old[k])       # untouched
        assert torch.equal(o, i)
        tol = (NORM_TOL + 4 * U + HALF[kind][0]) * np.abs(w) + HALF[kind][1]
        check("out", o.double().cpu().numpy(), w, tol if norm > max_norm else 0.0)


@pytest.mark.parametrize("scale", [1e-42, 1e-30, 1e-20, 1e18, 1e25, 3e37])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_norms_over_the_whole_range(scale, kind):
    grads = make_grads(4, [1000, 77], [kind], scale) + make_grads(5, [3001], [kind], scale * 1e-3)
    old = [g.double().cpu().numpy() for g in grads]
    norm, want = O.tuning.clip_grad_norm(old, 1.0)
    got = tuning().clip_grad_norm(grads, 1.0)
    # values below fp32's smallest normal keep their size, and the norm its own spacing
    assert abs(float(got) - norm) <= NORM_TOL * norm + 2.0 ** -149 if norm < 3.4e38 else float(got) == np.inf
    for g, w in zip(grads, want):
        check("out", g.double().cpu().numpy(), w, (NORM_TOL + 4 * U + HALF[kind][0]) * np.abs(w) + 2.0 ** -126)


def test_mixed_magnitudes():
    x = torch.randn(5000, device="cuda")
    x[::3] *= 1e-25
    x[1::3] *= 1e22
    norm = float(tuning().clip_grad_norm([x.clone()], 1.0))
    assert abs(norm - float(x.double().norm())) <= NORM_TOL * norm


def test_norms_that_are_no_numbers():
    x = torch.ones(3000, device="cuda")
    x[17] = float("nan")
    y = torch.ones(9, device="cuda", dtype=torch.bfloat16)
    assert torch.isnan(tuning().clip_grad_norm([x, y], 1.0)) and torch.isnan(x).all() and torch.isnan(y).all()
    x = torch.ones(3000, device="cuda")
    x[17] = float("-inf")
    assert tuning().clip_grad_norm([x], 1.0) == float("inf")
    assert torch.isnan(x[17]) and not x[:17].any() and not x[18:].any()
    z = [torch.zeros(100, device="cuda")]
    assert tuning().clip_grad_norm(z, 1.0) == 0.0 and not z[0].any()


def test_clip_permuted_gradients():
    x = torch.randn(40, 33, device="cuda")
    want = x / x.norm()
    g = x.clone().t()
    tuning().clip_grad_norm([g], 1.0)
    assert torch.allclose(g.t(), want, rtol=1e-5)


# --------------------------------------------------------------------------------------------------------- refusals

def refused(f, *args, status=N.NMD_ERR_INVALID, **kw):
    with pytest.raises(N.NmdError) as e:
        f(*args, **kw)
    assert e.value.status == status


def test_refusals():
    t = tuning()
    x = torch.zeros(4, 10, device="cuda")
    y = torch.zeros(4, device="cuda", dtype=torch.int64)
    v = torch.zeros(4, device="cuda")
    off = cuda([0, 2, 4], torch.int64)
    for bad in (x.double(), x.cpu(), x[0], x.t(), x[:, ::2], x[:, :0], None):
        refused(t.token_logprobs, bad, y)
    for bad in (y.int(), y[:3], y.cpu(), y[None], None):
        refused(t.token_logprobs, x, bad)
    for temperature in (0.0, -1.0, float("nan"), float("inf"), 1e-300):
        refused(t.token_logprobs, x, y, temperature=temperature)
    for bad in (off[:2], off[:1], cuda([0, 1, 2, 4], torch.int64), off.int(), off[None], off.cpu()):
        refused(t.preference_loss, x, y, bad, v)
    for bad in (v[:3], v.double(), v.cpu(), None):
        refused(t.preference_loss, x, y, off, bad)
    refused(t.preference_loss, x, y, off, v, beta=float("nan"))
    for smoothing in (-0.1, 1.0, float("nan")):
        refused(t.preference_loss, x, y, off, v, label_smoothing=smoothing)
    refused(t.policy_loss, x, y, v, None, v, kl_coef=0.1)
    refused(t.policy_loss, x, y, None, v, v)
    refused(t.policy_loss, x, y, v, v, v[:2])
    refused(t.policy_loss, x, y, v, v, v, offsets=off[:1])
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-1.0), dict(clip_high=float("inf")),
               dict(kl_coef=-0.1), dict(kl_coef=float("nan"))):
        refused(t.policy_loss, x, y, v, v, v, **kw)
    A, B = torch.zeros(4, 8, device="cuda"), torch.zeros(9, 8, device="cuda")
    for a, b in ((A, B[:, :7]), (A, B.bfloat16()), (A, B.cpu()), (A.double(), B.double()), (A[0], B), (A, B[:0]),
                 (A[:, :0], B[:, :0]), (torch.zeros(4, 257, device="cuda"), torch.zeros(9, 257, device="cuda"))):
        refused(t.factor_logprobs, a, b, y)
    refused(t.factor_logprobs, A, B, y[:3])
    refused(t.factor_logprobs, A, B, y, temperature=0.0)
    for max_norm in (0.0, -1.0, float("nan"), float("inf")):
        refused(t.clip_grad_norm, [x.clone()], max_norm)
    refused(t.clip_grad_norm, [], 1.0)
    for bad in (x.double(), x.cpu(), x[:, :5], x[:1].expand(4, 10)):
        refused(t.clip_grad_norm, [v, bad], 1.0)
    for out in ([x, x], [v], [x.t()], [x.bfloat16()], [x.cpu()]):
        refused(t.clip_grad_norm, [x], 1.0, out=out)


def test_refusals_of_the_library():
    """The C entries check what the Python layer never passes."""
    L = N.lib()
    x = torch.zeros(4, 16, device="cuda")
    y = torch.zeros(4, device="cuda", dtype=torch.int64)
    o = torch.zeros(64, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    call = lambda **k: L.nmd_token_logprobs(*[{**dict(a=x.data_ptr(), b=0, c=4, d=16, e=16, f=y.data_ptr(), g=1.0,  # noqa: E731
                                                      h=o.data_ptr(), i=None), **k}[n] for n in "abcdefghi"])
    assert call() == N.NMD_OK
    for k in (dict(a=None), dict(b=3), dict(b=-1), dict(c=-1), dict(c=(1 << 27) + 1), dict(d=0), dict(d=1 << 31),
              dict(e=-1), dict(f=None), dict(h=None), dict(a=x.data_ptr() + 2)):
        assert call(**k) == N.NMD_ERR_INVALID, k
    off = cuda([0, 2, 4], torch.int64)
    pol = lambda **k: L.nmd_policy_loss(*[{**dict(  # noqa: E731
        a=x.data_ptr(), b=0, c=4, d=16, e=16, f=y.data_ptr(), g=o.data_ptr(), h=o.data_ptr(), i=o.data_ptr(),
        j=off.data_ptr(), k=2, l=0.2, m=0.2, n=0.0, o=1.0, p=o.data_ptr(), q=o[8:].data_ptr(), r=None, s=0,
        t=ws.data_ptr(), u=1 << 20, v=None), **k}[n] for n in "abcdefghijklmnopqrstuv"])
    assert pol() == N.NMD_OK
    assert pol(u=16) == N.NMD_ERR_WORKSPACE and pol(t=None) == N.NMD_ERR_WORKSPACE
    assert pol(t=ws.data_ptr() + 16) == N.NMD_ERR_WORKSPACE
    assert pol(r=x.data_ptr(), s=16) == N.NMD_ERR_INVALID            # the gradient over the logits
    assert pol(r=ws[4096:].data_ptr(), s=15) == N.NMD_ERR_INVALID    # rows of the gradient overlap
    assert pol(k=0) == N.NMD_ERR_INVALID
    torch.cuda.synchronize()
