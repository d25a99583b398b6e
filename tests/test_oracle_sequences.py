"""The oracle's beam search, reordering and orthogonalisation against brute force, and the refusals of the library's
entries (they come before anything touches a GPU)."""
import ctypes as C
import itertools

import numpy as np
import pytest

import oracle as O
from paper_2608_21607_gb300 import build as B
from paper_2608_21607_gb300 import nmd as N

T = O.tuning


def test_beam_search_finds_the_best_chain():
    """As wide as the number of prefixes, it is an exhaustive search over the chains of a table."""
    rng = np.random.default_rng(0)
    V, steps = 4, 3
    table = rng.standard_normal((V, V))
    lp = table - np.log(np.exp(table).sum(1, keepdims=True))
    best = sorted(itertools.product(range(V), repeat=steps),
                  key=lambda c: -sum(lp[a, b] for a, b in zip((0,) + c, c)))
    last, scores, paths = np.array([0]), np.zeros((1, 1)), [()]
    for _ in range(steps):
        scores, parents, tokens, _ = T.beam_select(table[last], scores, min(64, V * len(paths)))
        paths = [paths[p] + (int(v),) for p, v in zip(parents[0], tokens[0])]
        last = tokens[0]
    assert paths == best


def test_beam_select_order_and_what_is_left_out():
    x = np.zeros((3, 4))
    x[1, 2] = -np.inf
    s, p, t, f = T.beam_select(x, [[0.0, 0.0, -np.inf]], 9, end=3)
    np.testing.assert_allclose(s[0, :3], -np.log(3.0))
    assert t[0].tolist() == [0, 1, 3, 0, 1, 2, 3, -1, -1] and p[0].tolist() == [1, 1, 1, 0, 0, 0, 0, 0, 0]
    assert f[0].tolist() == [False, False, True, False, False, False, True, False, False]
    x[0, 0] = np.nan
    s, p, t, f = T.beam_select(x, [[0.0, -5.0, -1.0]], 3, finished=[[False, True, True]], end=1)
    assert t[0].tolist() == [1, 1, -1] and p[0].tolist() == [2, 1, 0] and f[0].tolist() == [True, True, False]
    assert s[0, :2].tolist() == [-1.0, -5.0]


def test_beam_reorder():
    x = np.arange(24).reshape(2, 6, 2)
    parents = np.array([[2, 2, 0], [1, -1, 3]])
    y = T.beam_reorder(x, parents, dim=1)
    assert np.array_equal(y, x[:, [2, 2, 0, 4, 4, 5]])


@pytest.mark.parametrize("shape", [(5, 5), (9, 4), (3, 11), (1, 6), (7, 1)])
def test_orthogonalize_is_the_matrix_iteration(shape):
    rng = np.random.default_rng(1)
    G = rng.standard_normal(shape)
    a, b, c = 3.4445, -4.7750, 2.0315
    X = G / (np.linalg.norm(G) + 1e-7)
    for _ in range(5):
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
    np.testing.assert_allclose(T.orthogonalize(G), X, atol=1e-12)
    s = np.linalg.svd(T.orthogonalize(G), compute_uv=False)
    assert s.min() > 0.2 and s.max() < 1.3
    assert np.array_equal(T.orthogonalize(0 * G), 0 * G)


def test_muon_step():
    rng = np.random.default_rng(2)
    W, G, M = rng.standard_normal((3, 8, 2))
    W1, M1 = T.muon_step(W, G, M, lr=0.1, beta=0.9, nesterov=False, weight_decay=0.5)
    np.testing.assert_allclose(M1, 0.9 * M + 0.1 * G)
    np.testing.assert_allclose(W1, 0.95 * W - 0.1 * 2.0 * T.orthogonalize(M1))
    W2, _ = T.muon_step(W, G, M, lr=0.1, beta=0.9, scale=1.0)
    np.testing.assert_allclose(W2, W - 0.1 * T.orthogonalize(0.9 * M1 + 0.1 * G))


# ------------------------------------------------------------------------------------------- refusals of the library

@pytest.fixture(scope="module")
def L():
    B.build()
    return N.lib()


P = 1 << 20   # an address that nothing reads: the calls end before


def select(L, **kw):
    a = dict(logits=P, dtype=0, B=2, K=3, V=10, ld=10, scores=P, finished=None, end=-1, width=3, temperature=1.0,
             out=P, parents=P, tokens=P, done=None)
    a.update(kw)
    return L.nmd_beam_select(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(logits=P + 2), dict(dtype=3), dict(dtype=-1), dict(B=-1), dict(B=1 << 21), dict(K=0),
    dict(K=65), dict(V=0), dict(V=1 << 31), dict(ld=-1), dict(scores=None), dict(finished=P), dict(end=10),
    dict(end=-2), dict(width=0), dict(width=129), dict(temperature=0.0), dict(temperature=float("nan")),
    dict(temperature=float("inf")), dict(out=None), dict(parents=None), dict(tokens=None)])
def test_beam_select_refuses(L, bad):
    assert select(L, **bad) == N.NMD_ERR_INVALID


def test_beam_select_of_no_groups(L):
    assert select(L, B=0, logits=None) == N.NMD_OK


def reorder(L, states, B=2, K=3, width=3, parents=8 * P):
    table = (N.nmd_beam_state * len(states))(*[N.nmd_beam_state(*s) for s in states])
    return L.nmd_beam_reorder(len(states), C.addressof(table), B, K, width, parents, None)


@pytest.mark.parametrize("states,kw", [
    ([(None, P, 1, 0, 0, 8, 8, 8)], {}), ([(P, None, 1, 0, 0, 8, 8, 8)], {}),
    ([(P, P, 1, 0, 0, 8, 8, 9)], {}),                       # rows over one another
    ([(P, P, 2, 40, 40, 8, 8, 8)], {}),                     # the second outer index within the first
    ([(P, P, 2, 8, 8, 8, 8, 8)], {}), ([(P, P, -1, 0, 0, 8, 8, 8)], {}), ([(P, P, 1, 0, 0, -8, -8, 8)], {}),
    ([(P, P, 1, 0, 0, 8, 8, -8)], {}), ([(P, P, 1, 0, 0, 8, 16, 8)], {}),
    ([(P, P, 1, 0, 0, 8, 8, 8)], dict(width=4)),            # in place, of another width
    ([(P, P + 40, 1, 0, 0, 8, 8, 8)], {}),                  # what is written starts in what is read
    ([(P, P - 40, 1, 0, 0, 8, 8, 8)], {}),
    ([(P, P + 100, 1, 0, 0, 8, 8, 8), (P + 60, P + 130, 1, 0, 0, 8, 8, 8)], {}),
    ([(P, P + 200, 1, 0, 0, 8, 8, 8), (P + 220, P + 220, 1, 0, 0, 8, 8, 8)], {}),
    ([(P, P + 200, 1, 0, 0, 8, 8, 8), (P + 8, P + 8, 1, 0, 0, 8, 8, 8)], {}),
    ([(P, P, 1, 0, 0, 8, 8, 8)], dict(parents=P + 40)), ([(2 * P, P, 1, 0, 0, 8, 8, 8)], dict(parents=P - 40)),
    ([(P, P, 1, 0, 0, 8, 8, 8)], dict(parents=None)), ([(P, P, 1, 0, 0, 8, 8, 8)], dict(B=-1)),
    ([(P, P, 1, 0, 0, 8, 8, 8)], dict(K=65, width=65)), ([(P, P, 1, 0, 0, 8, 8, 8)], dict(K=0, width=0)),
    ([(P, P, 1 << 45, 1 << 45, 1 << 45, 8, 8, 8)], {})])
def test_beam_reorder_refuses(L, states, kw):
    assert reorder(L, states, **kw) == N.NMD_ERR_INVALID


def test_beam_reorder_of_nothing(L):
    assert reorder(L, []) == N.NMD_OK
    assert reorder(L, [(None, None, 1, 0, 0, 8, 8, 0), (None, None, 0, 0, 0, 8, 8, 8)]) == N.NMD_OK
    assert reorder(L, [(None, None, 1, 0, 0, 8, 8, 8)], B=0) == N.NMD_OK
    assert L.nmd_beam_reorder(1, None, 2, 3, 3, 8 * P, None) == N.NMD_ERR_INVALID
    assert L.nmd_beam_reorder(-1, None, 2, 3, 3, P, None) == N.NMD_ERR_INVALID


def ortho(L, **kw):
    a = dict(update=P, dtype=0, rows=6, cols=4, rs=4, cs=1, steps=5, k=(3.4, -4.8, 2.0), eps=1e-7, out=2 * P, ors=4,
             ocs=1, ws=4 * P, nbytes=1 << 24)
    a.update(kw)
    if a["k"] is not None:
        a["k"] = (C.c_double * 3)(*a["k"])
    return L.nmd_orthogonalize(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(update=None), dict(update=P + 1), dict(dtype=3), dict(rows=-1), dict(rows=1 << 31), dict(rows=20000, cols=20000),
    dict(rs=-1), dict(cs=-1), dict(steps=0), dict(steps=17), dict(k=None), dict(k=(float("nan"), 0, 0)), dict(eps=0.0),
    dict(eps=float("nan")), dict(out=None), dict(ors=3), dict(ocs=0), dict(out=P + 4), dict(out=P, ors=5),
    dict(out=P + 92)])
def test_orthogonalize_refuses(L, bad):
    assert ortho(L, **bad) == N.NMD_ERR_INVALID


def test_orthogonalize_workspace(L):
    for bad in (dict(ws=None), dict(ws=4 * P + 16), dict(nbytes=100)):
        assert ortho(L, **bad) == N.NMD_ERR_WORKSPACE
    assert ortho(L, rows=0) == N.NMD_OK and ortho(L, cols=0, update=None, out=None) == N.NMD_OK
    n = C.c_size_t(0)
    for rows, cols in ((-1, 3), (3, 1 << 31), (16385, 16385)):
        assert L.nmd_orthogonalize_workspace_bytes(rows, cols, C.byref(n)) == N.NMD_ERR_INVALID
    assert L.nmd_orthogonalize_workspace_bytes(3, 3, None) == N.NMD_ERR_INVALID


def muon(L, w=(P, 0, 4, 1), g=(2 * P, 0, 4, 1), m=(3 * P, 0, 4, 1), **kw):
    a = dict(rows=6, cols=4, lr=0.1, beta=0.9, nesterov=1, decay=0.0, scale=1.0, steps=5, k=(3.4, -4.8, 2.0), eps=1e-7,
             ws=4 * P, nbytes=1 << 24)
    a.update(kw)
    a["k"] = (C.c_double * 3)(*a["k"])
    keep = [v and N.nmd_matrix(*v) for v in (w, g, m)]
    at = [None if x is None else C.addressof(x) for x in keep]
    return L.nmd_muon_step(*at, *a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(w=None), dict(g=None), dict(m=None), dict(w=(None, 0, 4, 1)), dict(g=(2 * P, 3, 4, 1)), dict(m=(3 * P, 0, 0, 1)),
    dict(w=(P, 0, 3, 1)), dict(w=(2 * P, 0, 4, 1)), dict(m=(2 * P + 4, 0, 4, 1)), dict(w=(3 * P + 92, 0, 4, 1)),
    dict(lr=float("nan")), dict(lr=-1.0), dict(beta=1.0), dict(beta=-0.1), dict(decay=-1.0), dict(scale=float("inf")),
    dict(eps=-1.0), dict(steps=0), dict(rows=-1)])
def test_muon_step_refuses(L, bad):
    assert muon(L, **bad) == N.NMD_ERR_INVALID


def test_muon_step_workspace(L):
    assert muon(L, ws=None) == N.NMD_ERR_WORKSPACE and muon(L, nbytes=64) == N.NMD_ERR_WORKSPACE
    assert muon(L, rows=0) == N.NMD_OK
