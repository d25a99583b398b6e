"""The distance of Newton-Schulz results from the fp64 oracle, on every way through the kernels, held to a small
multiple of what fp32 products are off by (newton_schulz.py has the arithmetic): a piece or a product that is lost
shows a hundred times over."""
import numpy as np
import pytest

import newton_schulz as ns
from gpu_common import require_gpu

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF16, FP16 = torch.bfloat16, torch.float16
SPACING = {BF16: 2.0 ** -7, FP16: 2.0 ** -10}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    return require_gpu()


def tuning():
    from paper_2608_21607_gb300 import tuning as t
    return t


def place(x, dtype=torch.float32, layout="rows"):
    t = torch.from_numpy(np.asarray(x)).to("cuda").to(dtype)
    return t if layout == "rows" else t.t().contiguous().t()


def seen(x):
    return x.double().cpu().numpy()


# Short sides up to 64, on chip: one CTA, up to eight that add up all sums themselves, up to 32, more, tiles in TMEM.
# Others as products: sums whole (of up to 20 blocks of 64, or of many tiles), in more than 16 parts, in fewer; tiles
# of 64 and of 128 columns; a short side too long for the chip.
STRIP = [(5, 3), (16, 16), (64, 64), (100, 40), (1000, 60), (3000, 24), (20000, 64), (20001, 33), (120000, 64)]
PRODUCTS = [(65, 66), (300, 511), (1100, 1000), (4000, 100), (24001, 66), (2000, 600), (3001, 300), (2000, 1700), (2300, 1281),
            (160001, 17)]


@pytest.mark.parametrize("layout", ["rows", "columns"])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("long,short", STRIP + PRODUCTS)
def test_fp32_results(long, short, turned, layout):
    G = place(ns.gradient(*((short, long) if turned else (long, short)), seed=long), layout=layout)
    got = tuning().orthogonalize(G)
    want, off = ns.expected(seen(G))
    err = np.linalg.norm(seen(got) - want)
    print("%d x %d %s: %.2e of the norm, allowed %.2e" % (*G.shape, layout, err / np.linalg.norm(want), off / np.linalg.norm(want)))
    assert err <= off


@pytest.mark.parametrize("rows,cols,kw", [(64, 64, dict(noise=0.02)), (3000, 48, dict(noise=1e-3)), (300, 300, dict(noise=0.02)),
                                          (100, 4000, dict(noise=1e-3)), (600, 900, dict(strong=40, noise=1.0))])
@pytest.mark.parametrize("steps", [1, 2, 3, 5, 7])
def test_fp32_results_of_other_gradients(rows, cols, kw, steps):
    G = place(ns.gradient(rows, cols, 3, **kw))
    want, off = ns.expected(seen(G), steps)
    assert np.linalg.norm(seen(tuning().orthogonalize(G, steps=steps)) - want) <= off


def test_sixteen_steps_of_a_map_that_converges():
    for rows, cols in ((60, 60), (33, 400), (700, 90)):
        G = place(ns.gradient(rows, cols, 4, strong=40, noise=1.0))
        k = (1.875, -1.25, 0.375)
        want, off = ns.expected(seen(G), 16, k)
        assert np.linalg.norm(seen(tuning().orthogonalize(G, steps=16, coefficients=k)) - want) <= off


@pytest.mark.parametrize("rows,cols", [(40, 40), (20, 3000), (300, 290), (900, 100)])
@pytest.mark.parametrize("below", [0, 1, 4, 7, 7.9, 8.1, 12, 30, 60, 95])
def test_updates_smaller_than_eps(rows, cols, below):
    """|X| of 2^-below to start with.  Its elements are held to 2^-37 where |X| is 2^-8 or more, which beside their root
    mean square (2^-8 / 300) is 2^-21, and half of that on average: within what the bound has for the pieces."""
    g = ns.gradient(rows, cols, 6)
    eps = 1.0
    G = place(g / np.linalg.norm(g) * 2.0 ** -below)
    want, off = ns.expected(seen(G), eps=eps)
    assert np.linalg.norm(want) > 0.0
    assert np.linalg.norm(seen(tuning().orthogonalize(G, eps=eps)) - want) <= off


# tiles of 64, 128 and 256 columns, sums of 256 on the tensor cores, the strip kernel
SIXTEEN = [(64, 64), (5000, 64), (300, 511), (4000, 100), (20001, 256), (2000, 600), (3000, 1400), (2500, 2433)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("long,short", SIXTEEN)
def test_16_bit_results(long, short, turned, dtype):
    G = place(ns.gradient(*((short, long) if turned else (long, short)), seed=short), dtype)
    got = tuning().orthogonalize(G)
    want, off = ns.expected(seen(G), sixteen=True)
    right = seen(torch.from_numpy(want).to(dtype))
    err, allowed = np.linalg.norm(seen(got) - right), ns.rounded_apart(off, want, SPACING[dtype])
    size = np.linalg.norm(want)
    print("%d x %d %s: %.2e from the rounded definition, allowed %.2e" % (*G.shape, dtype, err / size, allowed / size))
    assert err <= allowed


@pytest.mark.parametrize("rows,cols", [(64, 64), (33, 20000), (1000, 60), (300, 511), (4000, 100), (2047, 1001)])
@pytest.mark.parametrize("weight,grad", [("rows", "rows"), ("rows", "columns"), ("columns", "rows")])
def test_fp32_steps_of_16_bit_gradients(rows, cols, weight, grad):
    """Weights of 0 show the update itself; the gradient in the weights' memory order and in the other."""
    G = place(ns.gradient(rows, cols, 5), BF16, grad)
    W, M = place(np.zeros((rows, cols)), layout=weight), place(np.zeros((rows, cols)), layout=weight)
    tuning().muon_step(W, G, M, lr=1.0, beta=0.0, nesterov=False, scale=-1.0)
    assert torch.equal(M, G.float())
    want, off = ns.expected(seen(G))
    assert np.linalg.norm(seen(W) - want) <= off
