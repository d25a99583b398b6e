"""The bound of the precision tests, on the CPU: steps on two fp16 pieces keep it, and steps that lose a piece do not."""
import numpy as np
import pytest

import newton_schulz as ns


@pytest.mark.parametrize("rows,cols,kw", [
    (16, 16, {}), (64, 64, {}), (90, 700, {}), (300, 511, {}), (511, 300, {}), (1000, 60, {}), (100, 4000, {}),
    (300, 40, dict(strong=40, noise=1.0)), (300, 300, dict(noise=0.02)), (100, 4000, dict(noise=1e-3))])
def test_lost_pieces_are_seen(rows, cols, kw):
    G = ns.gradient(rows, cols, 1, **kw).astype(np.float32).astype(np.float64)
    want, off = ns.expected(G)
    assert np.linalg.norm(ns.steps_on_pieces(G) - want) <= off
    for lost in (dict(cross=False), dict(count=1)):
        assert np.linalg.norm(ns.steps_on_pieces(G, **lost) - want) > 5 * off


@pytest.mark.parametrize("rows,cols", [(64, 64), (300, 511), (100, 4000)])
def test_lost_pieces_are_seen_in_16_bits(rows, cols):
    G = ns.gradient(rows, cols, 2).astype(np.float32).astype(np.float64)
    want, off = ns.expected(G, sixteen=True)
    right = want.astype(np.float16).astype(np.float64)
    allowed = ns.rounded_apart(off, want, 2.0 ** -10)
    assert np.linalg.norm(ns.steps_on_pieces(G).astype(np.float16) - right) <= allowed
    for lost in (dict(cross=False), dict(count=1)):
        assert np.linalg.norm(ns.steps_on_pieces(G, **lost).astype(np.float16) - right) > 2 * allowed
