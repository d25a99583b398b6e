"""Newton-Schulz orthogonalisation and the Muon step against the fp64 oracle (oracle/tuning.py).

Tolerance, in the Frobenius norm.  Each step forms A = X X^T, B = b A + c A^2 and X' = (a I + B) X.  With X, A and a I
+ B held to 22 bits (2^-23 each way) and each sum of products taken in fp32 with at most n roundings in a row, an entry
of a product is off by g sum |x| |y|, g = 2^-21 + n 2^-23 (the tensor cores' additions round towards zero, up to a unit),
so with |.| the Frobenius and |.|_2 the spectral norm
    e_A  = g |X|^2,   e_B = |b| e_A + |c| (2 |A|_2 e_A + g |A|^2) + 2^-22 |a I + B|,
    e_X' = e_B |X|_2 + g |a I + B| |X| + 2^-22 |X'|.
What is off after step i goes through the remaining steps: an odd polynomial f of the singular values changes by at most
max |(f(s) - f(t)) / (s - t)| over pairs s, t of +- the singular values (0 among them for what is not square).  The
last rounding adds half a unit of the type.  The norm's own roundings scale X by 1 + 2^-22 at most, like an error of X0.
"""
import numpy as np
import pytest

import oracle as O
from gpu_common import require_gpu
from paper_2608_21607_gb300 import nmd as N

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
MUON = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module", autouse=True)
def gpu():
    return require_gpu()


def tuning():
    from paper_2608_21607_gb300 import tuning as t
    return t


def roundings(*sums):
    """Additions in a row of the longest of these sums: chunks of at most 256 products are summed 16 at a time, three
    products each, then added up."""
    return max(48 + n / 128 for n in sums)


def tolerance(G, steps, coefficients, dtype, eps=1e-7):
    a, b, c = coefficients
    s = np.linalg.svd(G, compute_uv=False) / (np.linalg.norm(G) + eps)
    if min(G.shape) != max(G.shape):
        s = np.append(s, 0.0)
    g = 2.0 ** -21 + roundings(min(G.shape), max(G.shape)) * 2.0 ** -23
    r = min(G.shape)
    f = lambda t: a * t + b * t ** 3 + c * t ** 5  # noqa: E731
    errors, at = [2.0 ** -22 * np.linalg.norm(s)], [s]
    for _ in range(steps):
        X, X2, A = np.linalg.norm(s), s.max(), np.linalg.norm(s ** 2)
        aB = np.linalg.norm(np.append(a + b * s ** 2 + c * s ** 4, a * np.ones(max(0, r - len(s)))))
        e_A = g * X ** 2
        e_B = abs(b) * e_A + abs(c) * (2 * X2 ** 2 * e_A + g * A ** 2) + 2.0 ** -22 * aB
        s = f(s)
        errors.append(e_B * X2 + g * aB * X + 2.0 ** -22 * np.linalg.norm(s))
        at.append(s)
    total = 0.0
    for i, (e, v) in enumerate(zip(errors, at)):
        if len(v) > 400:
            v = np.quantile(v, np.linspace(0, 1, 400))
        both = np.concatenate([v, -v])
        out = both
        slope = np.ones(len(both))
        for _ in range(i, steps):
            slope = slope * (a + 3 * b * out ** 2 + 5 * c * out ** 4)
            out = f(out)
        d = both[:, None] - both[None, :]
        with np.errstate(divide="ignore", invalid="ignore"):
            q = np.where(np.abs(d) > 1e-9, np.abs(out[:, None] - out[None, :]) / np.abs(d), 0.0)
        total += e * max(q.max(), np.abs(slope).max())
    return total + HALF[dtype] * np.linalg.norm(at[-1]) + (2.0 ** -25 * np.sqrt(G.size) if dtype == "fp16" else 0.0)


def gradient(rows, cols, seed=0, strong=4, noise=0.2, size=1e-3):
    rng = np.random.default_rng(seed)
    k = max(1, min(strong, rows, cols))
    x = rng.standard_normal((rows, k)) @ rng.standard_normal((k, cols)) / np.sqrt(k)
    return size * (x + noise * rng.standard_normal((rows, cols)))


def place(x, dtype, layout="rows"):
    """`x` on the GPU with its rows adjacent, its columns adjacent, or every second element of padded rows."""
    t = torch.from_numpy(np.asarray(x)).to("cuda").to(DTYPES[dtype])
    if layout == "rows":
        return t
    if layout == "columns":
        return t.t().contiguous().t()
    if layout == "padded":
        big = torch.full((t.shape[0], t.shape[1] + 3), float("nan"), device="cuda", dtype=t.dtype)
        big[:, :t.shape[1]] = t
        return big[:, :t.shape[1]]
    if layout == "shifted":
        big = torch.full((t.numel() + 1,), float("nan"), device="cuda", dtype=t.dtype)
        big[1:] = t.reshape(-1)
        return big[1:].view(t.shape)
    big = torch.full((t.shape[0], 2 * t.shape[1] + 1), float("nan"), device="cuda", dtype=t.dtype)
    big[:, 1::2] = t
    return big[:, 1::2]


def check(G, steps=5, coefficients=MUON, dtype=None, **kw):
    dtype = dtype or {v: k for k, v in DTYPES.items()}[G.dtype]
    got = tuning().orthogonalize(G, steps=steps, coefficients=coefficients, **kw)
    assert got.shape == G.shape and got.dtype == G.dtype
    x = G.double().cpu().numpy()
    want = O.tuning.orthogonalize(x, steps, coefficients)
    err = np.linalg.norm(got.double().cpu().numpy() - want)
    tol = tolerance(x, steps, coefficients, dtype)
    assert err <= tol, (err, tol, np.linalg.norm(want))
    return got, err, tol


SIZES = [(1, 1), (1, 7), (9, 1), (2, 2), (5, 3), (3, 17), (16, 16), (31, 33), (64, 64), (65, 64), (64, 200), (127, 128),
         (128, 128), (129, 127), (200, 31), (255, 256), (257, 256), (300, 511), (1000, 8), (8, 2000), (5000, 64), (33, 4099),
         (2000, 130), (513, 700)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_orthogonalize(dtype, rows, cols):
    check(place(gradient(rows, cols), dtype))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["rows", "columns", "padded", "shifted", "apart"])
@pytest.mark.parametrize("rows,cols", [(1, 5), (40, 40), (72, 301), (301, 72), (500, 9), (260, 270)])
def test_orthogonalize_layouts(dtype, layout, rows, cols):
    G = place(gradient(rows, cols, 1), dtype, layout)
    plain, _, _ = check(G.contiguous())
    got, _, _ = check(G)
    if layout in ("padded", "shifted"):
        assert torch.equal(got, plain)
    for out_layout in ("rows", "columns", "apart"):
        out = place(np.zeros((rows, cols)), dtype, out_layout)
        assert tuning().orthogonalize(G, out=out) is out
        assert torch.equal(out, got)
    assert tuning().orthogonalize(G, out=G) is G
    assert torch.equal(G, got)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
@pytest.mark.parametrize("rows,cols", [(50, 50), (300, 40), (70, 1000)])
def test_orthogonalize_steps(steps, rows, cols):
    check(place(gradient(rows, cols, 2), "fp32"), steps)


def test_orthogonalize_many_steps():
    """Sixteen steps of a map that converges (a, b, c = 15/8, -5/4, 3/8) reach the orthogonal factor itself."""
    for rows, cols in ((60, 60), (33, 400), (700, 90)):
        G = place(gradient(rows, cols, 3, strong=40, noise=1.0), "fp32")
        got, _, _ = check(G, 16, (1.875, -1.25, 0.375))
        U, s, Vt = np.linalg.svd(G.double().cpu().numpy(), full_matrices=False)
        if s[-1] / np.linalg.norm(s) * 1.875 ** 14 > 10:
            assert np.linalg.norm(got.double().cpu().numpy() - U @ Vt) < 1e-4 * np.sqrt(min(rows, cols))


@pytest.mark.parametrize("rows,cols", [(24, 24), (100, 30), (30, 500), (300, 300)])
def test_orthogonalize_low_rank(rows, cols):
    """Fewer directions than columns, equal columns, columns and rows of zeros."""
    for noise in (0.0, 1e-4):
        x = gradient(rows, cols, 4, strong=3, noise=noise)
        x[:, 3] = x[:, 5]
        x[:, 7] = 0.0
        x[2] = 0.0
        check(place(x, "fp32"))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols", [(40, 40), (20, 3000), (300, 290)])
def test_orthogonalize_zero_and_sizes(dtype, rows, cols):
    t = tuning()
    zero = torch.zeros(rows, cols, device="cuda", dtype=DTYPES[dtype])
    assert torch.equal(t.orthogonalize(zero), zero)
    assert torch.equal(t.orthogonalize(zero, eps=1e-300), zero)
    g = gradient(rows, cols, 5, size=1.0)
    for size in ((1e-30, 1e-5, 1e15, 1e36) if dtype != "fp16" else (1e-3, 1e3)):
        check(place(size * g, dtype))
    check(place(g, dtype))


def test_orthogonalize_nothing():
    for shape in ((0, 5), (5, 0), (0, 0)):
        x = torch.zeros(shape, device="cuda")
        assert tuning().orthogonalize(x).shape == shape


@pytest.mark.parametrize("rows,cols", [(10, 10), (60, 5000), (400, 300)])
def test_orthogonalize_not_finite(rows, cols):
    """A NaN or an infinity shows everywhere."""
    for bad in (float("nan"), float("inf")):
        for dtype in DTYPES.values():
            x = torch.randn(rows, cols, device="cuda").to(dtype)
            x[rows // 2, cols - 1] = bad
            assert not tuning().orthogonalize(x).isfinite().any()


def test_orthogonalize_past_the_range():
    """Coefficients that take singular values out of range give no finite result instead of a wrong one."""
    x = torch.randn(50, 60, device="cuda")
    got = tuning().orthogonalize(x, steps=16, coefficients=(30.0, 40.0, 50.0))
    assert not got.isfinite().all()


@pytest.mark.parametrize("rows,cols,dtype", [(20000, 32, "fp32"), (64, 30000, "bf16"), (1100, 1000, "fp32"), (900, 4100, "bf16"),
                                             (30001, 256, "fp16"), (2049, 1025, "fp32")])
def test_orthogonalize_larger(rows, cols, dtype):
    check(place(gradient(rows, cols, 6), dtype))


def test_orthogonalize_against_differences():
    """The map's change along a direction is that of the oracle (a central difference in fp64)."""
    G, D = gradient(40, 90, 7, strong=40, noise=1.0, size=1.0), gradient(40, 90, 8, size=1.0)
    h = 2.0 ** -9
    t = tuning().orthogonalize
    got = (t(place(G + h * D, "fp32")).double() - t(place(G - h * D, "fp32")).double()).cpu().numpy() / (2 * h)
    want = (O.tuning.orthogonalize(G + h * D) - O.tuning.orthogonalize(G - h * D)) / (2 * h)
    # inputs rounded to fp32 go through the same map: their own share is an error of X0 of 2^-24
    tol = (tolerance(G + h * D, 5, MUON, "fp32") + tolerance(G - h * D, 5, MUON, "fp32")) / (2 * h) * 1.1
    assert np.linalg.norm(got - want) <= tol


def round_to(dtype):
    return lambda m: torch.from_numpy(m).to(torch.float32).to(DTYPES[dtype]).double().numpy()


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("types", [("fp32", "fp32", "fp32"), ("bf16", "bf16", "fp32"), ("fp16", "fp32", "fp16"),
                                   ("fp32", "bf16", "bf16")])
@pytest.mark.parametrize("rows,cols,layouts", [
    (1, 1, ("rows", "rows", "rows")), (64, 64, ("rows", "rows", "rows")), (20, 333, ("rows", "columns", "padded")),
    (333, 20, ("columns", "rows", "apart")), (270, 300, ("rows", "rows", "columns")), (4000, 32, ("rows", "rows", "rows"))])
def test_muon_step(nesterov, types, rows, cols, layouts):
    x = [gradient(rows, cols, 10, size=1.0), gradient(rows, cols, 11), gradient(rows, cols, 12)]
    W, G, M = (place(v, d, l) for v, d, l in zip(x, types, layouts))
    w, g, m = (v.double().cpu().numpy() for v in (W, G, M))
    kw = dict(lr=0.05, beta=0.9, nesterov=nesterov, weight_decay=0.3)
    tuning().muon_step(W, G, M, **kw)
    # the momentum is rounded once (its own type) after fp32 products: the oracle's from the same start
    exact = 0.9 * m + 0.1 * g
    got_m = M.double().cpu().numpy()
    assert np.all(np.abs(got_m - exact) <= (HALF[types[2]] + 3 * 2.0 ** -24) * (np.abs(0.9 * m) + np.abs(0.1 * g)) + 2.0 ** -25)
    want, _ = O.tuning.muon_step(w, g, m, round_momentum=lambda _: got_m, **kw)
    U = 0.9 * got_m + 0.1 * g if nesterov else got_m
    scale = max(1.0, rows / cols) ** 0.5
    tol = 0.05 * scale * 1.01 * tolerance(U, 5, MUON, "fp32") + (HALF[types[0]] + 3 * 2.0 ** -24) * (np.linalg.norm(want) + 0.05 * scale * 1.3 * min(rows, cols) ** 0.5)
    assert np.linalg.norm(W.double().cpu().numpy() - want) <= tol
    assert torch.equal(G.double().cpu(), torch.from_numpy(g))


def test_muon_step_defaults_and_scale():
    for scale in (None, 0.2):
        W, G, M = (place(gradient(90, 40, k), "fp32") for k in range(3))
        want, m = O.tuning.muon_step(*(v.double().cpu().numpy() for v in (W, G, M)), lr=0.1, scale=scale)
        tuning().muon_step(W, G, M, lr=0.1, scale=scale)
        assert np.linalg.norm(W.double().cpu().numpy() - want) <= 1e-4 * np.linalg.norm(want)
        np.testing.assert_allclose(M.double().cpu().numpy(), m, rtol=1e-6, atol=1e-10)
    # lr = 0: the weights stay, the momentum does not
    W0 = W.clone()
    tuning().muon_step(W, G, M, lr=0.0, weight_decay=0.5)
    assert torch.equal(W, W0)


def test_equal_bits_streams_and_replay():
    t = tuning()
    for rows, cols in ((64, 64), (5000, 40), (300, 700)):
        G = place(gradient(rows, cols, 20), "fp32")
        W, M = torch.zeros_like(G), torch.zeros_like(G)
        first = t.orthogonalize(G)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            assert torch.equal(t.orthogonalize(G), first)
            side.synchronize()
            graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = t.orthogonalize(G)
            with torch.cuda.graph(other, stream=side, pool=graph.pool()):
                t.muon_step(W, G, M, lr=1.0, nesterov=False, beta=0.0, scale=1.0)
        side.synchronize()
        for _ in range(3):
            graph.replay()
            other.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(M, G)
        assert torch.allclose(W, -3 * first, rtol=1e-5, atol=1e-6)


def test_versions():
    W, G, M = (place(gradient(20, 10, k), "fp32") for k in range(3))
    for written in (W, M):
        leaf = torch.ones_like(W, requires_grad=True)
        loss = (leaf * written).sum()
        tuning().muon_step(W, G, M, lr=0.1)
        with pytest.raises(RuntimeError):
            loss.backward()
    with torch.inference_mode():
        tuning().orthogonalize(torch.randn(5, 6, device="cuda"))
    parameter = torch.nn.Parameter(torch.randn(30, 20, device="cuda"))
    tuning().muon_step(parameter, G[:, :1].expand(20, 20)[:1].expand(30, 20), torch.zeros(30, 20, device="cuda"), lr=0.1)
    assert parameter.isfinite().all() and parameter.requires_grad


def refused(f, *args, **kw):
    with pytest.raises(N.NmdError) as e:
        f(*args, **kw)
    assert e.value.status == N.NMD_ERR_INVALID


def test_refusals():
    t = tuning()
    x = torch.ones(6, 4, device="cuda")
    for bad in (x.cpu(), x.double(), x[0], x.int(), None, torch.zeros(16385, 1, device="cuda").expand(16385, 16385)):
        refused(t.orthogonalize, bad)
    for kw in (dict(steps=0), dict(steps=17), dict(coefficients=(1.0, 2.0)), dict(coefficients=(float("nan"), 0.0, 0.0)),
               dict(eps=0.0), dict(eps=float("nan")), dict(out=x[:5]), dict(out=x.bfloat16()), dict(out=x.cpu()),
               dict(out=x[:1].expand(6, 4))):
        refused(t.orthogonalize, x, **kw)
    flat = torch.ones(60, device="cuda")
    refused(t.orthogonalize, flat[:24].view(6, 4), out=flat[20:44].view(6, 4))
    refused(t.orthogonalize, flat[:16].view(4, 4), out=flat[:16].view(4, 4).t())
    W, G, M = x.clone(), x.clone(), x.clone()
    for bad in (x.cpu(), x.double(), x[:5], None, x.t()):
        refused(t.muon_step, bad, G, M, lr=0.1)
        refused(t.muon_step, W, bad, M, lr=0.1)
        refused(t.muon_step, W, G, bad, lr=0.1)
    for args in ((W, W, M), (W, G, W), (W, G, G), (W, G, x[:1].expand(6, 4)), (x[:1].expand(6, 4), G, M)):
        refused(t.muon_step, *args, lr=0.1)
    for kw in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=0.1, beta=1.0), dict(lr=0.1, beta=-0.5),
               dict(lr=0.1, weight_decay=-1.0), dict(lr=0.1, scale=float("inf")), dict(lr=0.1, steps=0), dict(lr=0.1, eps=0.0)):
        refused(t.muon_step, W, G, M, **kw)
    assert torch.equal(W, x) and torch.equal(M, x) and (flat == 1).all()


@pytest.mark.parametrize("rows,cols,dtype", [(100000, 64, "fp32"), (64, 130000, "fp32"), (117000, 33, "bf16"), (155648, 17, "fp32"),
                                             (155649, 17, "fp32"), (40, 97281, "fp16"), (58369, 50, "fp32")])
def test_orthogonalize_tall(rows, cols, dtype):
    """Long sides at which the tiles of a CTA no longer fit shared memory, or no longer fit on chip."""
    check(place(gradient(rows, cols, 9), dtype))


def test_several_streams_at_once():
    """Steps that each want more than half of the SMs at a time, on three streams."""
    t = tuning()
    Gs = [place(gradient(rows, cols, k), "fp32") for k, (rows, cols) in enumerate(((20000, 64), (30000, 33), (64, 25000)))]
    want = [t.orthogonalize(G) for G in Gs]
    streams = [torch.cuda.Stream() for _ in Gs]
    torch.cuda.synchronize()
    got = [[], [], []]
    for _ in range(10):
        for k, (G, s) in enumerate(zip(Gs, streams)):
            with torch.cuda.stream(s):
                got[k].append(t.orthogonalize(G))
    torch.cuda.synchronize()
    for k in range(3):
        assert all(torch.equal(x, want[k]) for x in got[k])


@pytest.mark.parametrize("rows,cols,dtype", [(70, 240001, "fp32"), (129, 131000, "bf16"), (515, 33001, "fp16"), (2000, 8400, "fp32")])
@pytest.mark.parametrize("layout", ["rows", "columns"])
def test_orthogonalize_wide(rows, cols, dtype, layout):
    """Long sides split over many CTAs, by rows and by columns in memory; a step is its update."""
    G = place(gradient(rows, cols, 13), dtype, layout)
    check(G)
    W, M = torch.zeros_like(G), torch.zeros_like(G)
    tuning().muon_step(W, G, M, lr=1.0, beta=0.0, nesterov=False, scale=1.0)
    assert torch.equal(W, -tuning().orthogonalize(G))


@pytest.mark.parametrize("rows,cols,dtype", [(1400, 3000, "bf16"), (2433, 2500, "fp16"), (1290, 20001, "bf16"), (1281, 2300, "fp32")])
@pytest.mark.parametrize("layout", ["rows", "columns"])
def test_orthogonalize_large(rows, cols, dtype, layout):
    """Tiles of 256 columns: the update's of 16-bit results, and at (2433, 2500) the symmetric products' too."""
    G = place(gradient(rows, cols, 17), dtype, layout)
    check(G)
    W, M = torch.zeros_like(G), torch.zeros_like(G)
    tuning().muon_step(W, G, M, lr=1.0, beta=0.0, nesterov=False, scale=1.0)
    assert torch.equal(W, -tuning().orthogonalize(G))
