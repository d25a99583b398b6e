"""Beam search's selection and the reordering of states against the fp64 oracle (oracle/tuning.py).

A selected score is the beam's score plus a log-probability, which is off by at most TOL = u (128 + 4 R + 4 |lp|), u =
2^-24 and R the spread of the row's finite z = x / temperature (each term of the sum carries the roundings of its
exponent, 3 u R, and of the exponential, 4 u; order and merges of the sum add at most 104 u), and is rounded once to
fp32.  Beams and columns have to be the oracle's wherever its neighbouring values lie further apart than twice that;
where they do not, the value of what was taken has to be within it.  Rows that are copies of one another are equal in
every bit, so ties of whole rows count.
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


@pytest.fixture(scope="module", autouse=True)
def gpu():
    return require_gpu()


def tuning():
    from paper_2608_21607_gb300 import tuning as t
    return t


def cuda(v, dtype=None):
    return torch.as_tensor(np.asarray(v)).to("cuda", dtype)


def make(seed, B, K, V, dtype, *, pad=0, shift=0, scale=2.5, unused=0.0, finished=0.0, banned=0.0):
    """(logits on the GPU, scores, finished or None): logits of stride V + pad, `shift` elements into the storage; rows
    that are not read hold NaN."""
    rng = np.random.default_rng(seed)
    x = (scale * rng.standard_normal((B * K, V))).astype(np.float32)
    if banned:
        x[:, rng.permutation(V)[:int(banned * V)]] = -np.inf
    scores = np.sort(-10.0 + 3.0 * rng.standard_normal((B, K)), axis=1)[:, ::-1].astype(np.float32)
    scores[rng.random((B, K)) < unused] = -np.inf
    done = rng.random((B, K)) < finished if finished else None
    off = ~np.isfinite(scores) if done is None else done | ~np.isfinite(scores)
    x[off.reshape(-1)] = np.nan
    flat = torch.full((B * K * (V + pad) + shift,), float("nan"), device="cuda", dtype=DTYPES[dtype])
    rows = flat[shift:].view(B * K, V + pad)[:, :V]
    rows.copy_(torch.from_numpy(x))
    return rows, scores, done


def check(rows, scores, done, width, end=None, temperature=1.0, got=None):
    if got is None:
        got = tuning().beam_select(rows, cuda(scores), width=width, finished=None if done is None else cuda(done), end=end,
                                   temperature=temperature)
    x = rows.double().cpu().numpy()
    B, K = scores.shape
    V = x.shape[1]
    # one more than asked for: the last one may have a neighbour
    best, parents, tokens, fin = O.tuning.beam_select(x, scores, min(width + 1, K * V + 1), done, end, temperature)
    spread = 0.0
    live = [z[np.isfinite(z)] / temperature for z in x]
    for z in live:
        if len(z):
            spread = max(spread, z.max() - z.min())
    alike = np.unique(np.concatenate([np.nan_to_num(x, nan=7e77), scores.reshape(-1, 1)], 1), axis=0, return_inverse=True)[1]
    alike = alike.reshape(B, K)
    s, p, t = (v.cpu().numpy() for v in (got.scores, got.parents, got.tokens))
    assert s.shape == p.shape == t.shape == (B, width) and got.scores.dtype == torch.float32
    for b in range(B):
        for i in range(width):
            want = best[b, i] if i < best.shape[1] else -np.inf
            if want == -np.inf:
                assert s[b, i] == -np.inf and p[b, i] == 0 and t[b, i] == -1
                continue
            tol = U * (128 + 4 * spread + 4 * abs(want)) + U * abs(want)
            assert abs(s[b, i] - want) <= tol, (b, i, s[b, i], want, tol)
            with np.errstate(invalid="ignore"):
                clear = np.abs(best[b] - want) > 2 * tol
            clear |= (best[b] == want) & (alike[b, parents[b]] == alike[b, parents[b, i]])
            if clear.all():
                assert (p[b, i], t[b, i]) == (parents[b, i], tokens[b, i]), (b, i, want)
        pairs = [(p[b, i], t[b, i]) for i in range(width) if t[b, i] >= 0]
        assert len(set(pairs)) == len(pairs)
    if end is None:
        assert got.finished is None
    else:
        assert np.array_equal(got.finished.cpu().numpy(), (t == end))
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,K,V,width", [
    (1, 1, 1, 1), (1, 1, 2, 2), (3, 2, 7, 5), (2, 5, 3, 20), (4, 3, 1, 7), (5, 4, 255, 4), (2, 8, 1000, 16),
    (3, 64, 33, 128), (1, 64, 700, 64), (7, 1, 4097, 3), (2, 3, 20011, 6), (1, 4, 139255, 4), (1, 1, 70001, 128),
    (40, 5, 513, 5), (1, 32, 9001, 64), (6, 14, 312, 14), (2, 3, 1024, 48), (2, 3, 1025, 48), (3, 33, 34, 66), (2, 22, 461, 44),
    (1, 16, 1142, 16), (2, 64, 1000, 128), (1, 64, 1024, 40), (1, 8, 64, 128)])
def test_select(dtype, B, K, V, width):
    check(*make(B * 7 + K, B, K, V, dtype), width)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 3), (8, 5), (13, 8)])
def test_select_strides(dtype, pad, shift):
    rows, scores, done = make(1, 6, 4, 1003, dtype, pad=pad, shift=shift, unused=0.3, finished=0.3)
    check(rows, scores, done, 6, end=1002, temperature=0.7)


@pytest.mark.parametrize("V", [5, 300, 30001])
def test_select_unused_finished_banned(V):
    rows, scores, done = make(2, 20, 6, V, "bf16", unused=0.4, finished=0.4, banned=0.3)
    scores[0] = -np.inf        # a group without a beam
    done[1] = True             # a group that is done
    scores[1] = np.arange(6) - 9.0
    done[2], scores[2, 1:] = False, -np.inf      # the first step: one beam
    scores[2, 0] = 0.0
    rows[12:13] = torch.randn(1, V, device="cuda", dtype=torch.bfloat16)
    check(rows, scores, done, 12, end=min(3, V - 1))
    check(rows, scores, done, 3, end=0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [64, 5000, 140000])
def test_select_ties(dtype, V):
    """Equal logits, equal rows: the lowest beam, then the lowest column."""
    rows = torch.zeros(6, V, device="cuda", dtype=DTYPES[dtype])
    scores = np.zeros((2, 3), np.float32)
    got = check(rows, scores, None, 9)
    assert got.parents.cpu().tolist() == [[0] * 9] * 2 and got.tokens.cpu().tolist() == [list(range(9))] * 2
    for v in (V - 1, V // 2, 17):
        rows[:, v] = 3.0
    got = check(rows, scores, None, 10)
    first = sorted([17, V // 2, V - 1])
    assert got.parents.cpu().tolist() == [[0] * 3 + [1] * 3 + [2] * 3 + [0]] * 2
    assert got.tokens.cpu().tolist() == [first * 3 + [0]] * 2
    rows[:, 1::2] *= -1.0      # zeros of either sign are equal
    got = check(rows * 0, scores, None, 4)
    assert got.tokens.cpu().tolist() == [[0, 1, 2, 3]] * 2


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [40, 9000])
def test_select_rising_and_falling_rows(dtype, V):
    """Every column better than all before it, and the other way around."""
    ramp = torch.linspace(-8, 8, V, device="cuda").to(DTYPES[dtype])
    rows = torch.stack([ramp, ramp.flip(0), ramp, -ramp.abs()]).contiguous()
    check(rows, np.array([[-1.0, -1.25], [-3.0, -2.0]], np.float32), None, 40)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V,shift", [(1100, 0), (9001, 3), (50000, 1), (139255, 0)])
@pytest.mark.parametrize("width", [1, 4, 32, 33, 128])
def test_select_equal_and_flat_rows(dtype, V, shift, width):
    """Rows of one value, of three, and of nearly one: nothing but the columns tells many offers apart."""
    g = torch.Generator(device="cuda").manual_seed(V + width)
    store = torch.zeros(4 * V + shift, device="cuda", dtype=DTYPES[dtype])
    rows = store[shift:].view(4, V)
    rows[1] = torch.randint(0, 3, (V,), device="cuda", generator=g).to(rows.dtype) / 2
    rows[2] = torch.randint(0, 2, (V,), device="cuda", generator=g).to(rows.dtype)
    rows[2, V // 2:] = 1.0 + 1 / 128
    rows[3] = (1 + 1e-3 * torch.randn(V, device="cuda", generator=g)).to(rows.dtype)
    got = tuning().beam_select(rows, torch.zeros(4, 1, device="cuda"), width=width)
    assert (got.parents == 0).all()
    for i in range(4):   # in each row the order of the logits, of equal ones that of the columns
        want = torch.sort(rows[i].float(), descending=True, stable=True).indices[:width]
        assert torch.equal(got.tokens[i], want)
    check(rows, np.array([[-1.0, -1.25], [-3.0, -2.0]], np.float32), None, width)


def test_select_masked_values():
    """Rows masked with the type's lowest value, +inf and NaN, banned altogether, and tiny temperatures."""
    for dtype in DTYPES:
        low = torch.finfo(DTYPES[dtype]).min
        rows = torch.randn(8, 999, device="cuda").to(DTYPES[dtype])
        rows[0, 10:] = low
        rows[1] = low
        rows[2] = float("-inf")
        rows[3, 7] = float("inf")
        rows[4, 998] = float("nan")
        rows[5, :998] = float("-inf")
        rows[6, 500] = -low
        scores = np.zeros((1, 8), np.float32)
        got = check(rows, scores, None, 40)
        assert not set(got.parents[0, got.tokens[0] >= 0].tolist()) & {2, 3, 4}
        for temperature in (1e-3, 50.0):
            check(rows[[0, 5, 7]], np.zeros((1, 3), np.float32), None, 12, temperature=temperature)
        nothing = tuning().beam_select(rows[2:5], cuda(np.zeros((3, 1), np.float32)))
        assert torch.isneginf(nothing.scores).all() and (nothing.tokens == -1).all() and (nothing.parents == 0).all()


def test_select_nan_scores_offer_nothing():
    rows = torch.randn(4, 50, device="cuda")
    got = check(rows, np.array([[np.nan, np.inf, -np.inf, -1.0]], np.float32), None, 60)
    assert set(got.parents[0, :50].tolist()) == {3}


def test_select_large_offsets():
    """Rows past 2^31 elements from the first."""
    V, ld = 100, 1 << 29
    flat = torch.zeros(5 * ld + V, device="cuda", dtype=torch.float16)
    rows = torch.as_strided(flat, (6, V), (ld, 1))
    rows.copy_(torch.randn(6, V, device="cuda"))
    check(rows, np.zeros((2, 3), np.float32), None, 5)


def test_select_equal_calls_give_equal_bits_and_replay():
    rows, scores, done = make(5, 9, 6, 30011, "bf16", finished=0.2)
    s, d = cuda(scores), cuda(done)
    t = tuning()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = t.beam_select(rows, s, finished=d, end=5)
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            out = t.beam_select(rows, s, finished=d, end=5)
    side.synchronize()
    s.add_(0.5)
    graph.replay()
    want = t.beam_select(rows, s, finished=d, end=5)
    torch.cuda.synchronize()
    for a, b in zip(out, want):
        assert torch.equal(a, b)
    assert torch.equal(first.tokens, check(rows, scores, done, 6, end=5).tokens)
    s.sub_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, first):
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------------------------------------- reorder

ANY = [torch.int64, torch.int32, torch.float32, torch.bfloat16, torch.float16, torch.uint8, torch.bool, torch.float64]


def values(shape, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randint(0, 200, shape, device="cuda", generator=g)
    return (x % 2 == 0) if dtype == torch.bool else x.to(dtype)


def moved(x, parents, dim=0, out=None):
    y = O.tuning.beam_reorder(x.double().cpu().numpy(), parents, dim, None if out is None else out.double().cpu().numpy())
    return torch.from_numpy(np.ascontiguousarray(y)).to("cuda")


@pytest.mark.parametrize("dtype", ANY, ids=[str(d).split(".")[1] for d in ANY])
@pytest.mark.parametrize("B,K,inner", [(1, 1, 1), (1, 4, 7), (3, 2, 64), (2, 5, 1001), (5, 64, 33), (1, 33, 5000), (2, 8, 40000)])
def test_reorder_in_place(dtype, B, K, inner):
    rng = np.random.default_rng(K)
    parents = rng.integers(0, K, (B, K))
    x = values((B * K, inner), dtype)
    want = moved(x, parents)
    assert tuning().beam_reorder(x, cuda(parents)) is x
    assert torch.equal(x.double(), want)
    tuning().beam_reorder(x, cuda(np.tile(np.arange(K), (B, 1))))
    assert torch.equal(x.double(), want)


@pytest.mark.parametrize("dtype", [torch.int64, torch.bfloat16, torch.uint8])
@pytest.mark.parametrize("K,w", [(4, 4), (3, 7), (64, 128), (5, 1), (1, 9)])
def test_reorder_into_another(dtype, K, w):
    rng = np.random.default_rng(w)
    parents = rng.integers(0, K, (3, w))
    parents[0, 0], parents[2, w - 1] = -1, K       # these stay as they are
    x, y = values((2, 3 * K, 5, 31), dtype), values((2, 3 * w, 5, 31), dtype, 1)
    want = moved(x, parents, 1, y)
    before = x.clone()
    assert tuning().beam_reorder(x, cuda(parents), dim=1, out=y) is y
    assert torch.equal(y.double(), want) and torch.equal(x, before)


@pytest.mark.parametrize("shift", [0, 1, 3])
def test_reorder_several_views(shift):
    """Used parts of longer rows, layers before the rows, rows before the layers, states between each other's bytes;
    what lies around them stays."""
    rng = np.random.default_rng(3)
    B, K = 4, 6
    parents = rng.integers(0, K, (B, K))
    history = values((B * K, 50 + shift), torch.int64)
    cache = values((3, B * K, 2, 10 + shift, 8), torch.bfloat16)
    both = values((B * K, 2, 101), torch.float16)
    layers = values((B * K, 3, 33), torch.float32)
    flat = values((B * K * 77 + 5,), torch.uint8)
    whole = [history, cache, both, layers, flat]
    before = [v.clone() for v in whole]
    states = [history[:, shift:41 + shift], cache[:, :, :, :9], both[:, 0], both[:, 1], layers.transpose(0, 1)[1:],
              flat[shift:shift + B * K * 77].view(B * K, 77)]
    dims = [0, 1, 0, 0, 1, 0]
    t = tuning()
    want = [moved(x, parents, d) if x.dim() != 5 else None for x, d in zip(states, dims)]
    p = cuda(parents)
    t.beam_reorder([s for s, d in zip(states, dims) if d == 0], p)
    t.beam_reorder([s for s, d in zip(states, dims) if d == 1][1:], p, dim=1)
    for x, w in zip(states, want):
        if w is not None:
            assert torch.equal(x.double(), w)
    # whole rows with elements that are not adjacent are refused, each element for itself is not
    with pytest.raises(N.NmdError):
        t.beam_reorder(states[1], p, dim=1)
    assert torch.equal(cache, before[1])
    t.beam_reorder(cache, p, dim=1)
    assert torch.equal(cache.double(), moved(before[1], parents, 1))
    h = before[0].clone()
    h[:, shift:41 + shift] = want[0].long()
    assert torch.equal(history, h)
    l = before[3].clone()
    l.transpose(0, 1)[1:] = want[4].float()
    assert torch.equal(layers, l)
    assert torch.equal(flat[:shift], before[4][:shift]) and torch.equal(flat[shift + B * K * 77:], before[4][shift + B * K * 77:])


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("inner", [1, 2, 3, 127, 8191, 8193, 20001])
@pytest.mark.parametrize("K", [2, 7, 64])
def test_reorder_rows_of_any_phase(shift, inner, K):
    """16-bit rows that start at every multiple of two bytes; what lies around them stays."""
    rng = np.random.default_rng(inner)
    parents = rng.integers(0, K, (3, K))
    flat = values((3 * K * (inner + 1) + 9,), torch.bfloat16, inner)
    rows = flat[shift:shift + 3 * K * (inner + 1)].view(3 * K, inner + 1)[:, :inner]
    want, before = moved(rows, parents), flat.clone()
    tuning().beam_reorder(rows, cuda(parents))
    assert torch.equal(rows.double(), want)
    before[shift:shift + 3 * K * (inner + 1)].view(3 * K, inner + 1)[:, :inner] = want.to(torch.bfloat16)
    assert torch.equal(flat, before)
    other = torch.zeros(3 * K, inner, device="cuda", dtype=torch.bfloat16)
    tuning().beam_reorder(rows, cuda(parents), out=other)
    assert torch.equal(other.double(), moved(rows, parents))


def test_reorder_the_same_state_twice():
    parents = cuda([[1, 2, 0, 0]])
    x = torch.arange(4, device="cuda")[:, None].repeat(1, 999)
    tuning().beam_reorder([x, x], parents)
    assert x[:, 0].tolist() == [2, 0, 1, 1] and x[:, 998].tolist() == [2, 0, 1, 1]


def test_reorder_many_and_empty_states():
    rng = np.random.default_rng(4)
    parents = rng.integers(0, 3, (2, 3))
    xs = [values((6, n), d, n) for n, d in zip(list(range(0, 70)) + [20000, 0], ANY * 9)]
    want = [moved(x, parents) for x in xs]
    assert tuning().beam_reorder(xs, cuda(parents)) is xs
    for x, w in zip(xs, want):
        assert torch.equal(x.double(), w)
    tuning().beam_reorder([], cuda(parents))
    none = torch.zeros(0, 5, device="cuda")
    tuning().beam_reorder(none, torch.zeros(0, 3, device="cuda", dtype=torch.int64))


def test_reorder_large_offsets():
    """Rows past 2^31 and 2^32 bytes from the first."""
    x = torch.zeros(4, (1 << 30) + 9, device="cuda", dtype=torch.uint8)
    for k in range(4):
        x[k, -3:] = k + 1
        x[k, :2] = 10 * (k + 1)
    tuning().beam_reorder(x, cuda([[3, 3, 0, 1]]))
    assert x[:, -1].tolist() == [4, 4, 1, 2] and x[:, 0].tolist() == [40, 40, 10, 20]


def test_reorder_raises_versions_and_replays():
    x = torch.arange(12.0, device="cuda").view(4, 3)
    parents = cuda([[0, 0, 1, 2]])
    leaf = torch.ones(4, 3, device="cuda", requires_grad=True)
    loss = (leaf * x).sum()
    tuning().beam_reorder(x, parents)
    with pytest.raises(RuntimeError):
        loss.backward()
    graph = torch.cuda.CUDAGraph()
    y = torch.arange(4, device="cuda")[:, None].repeat(1, 5)
    with torch.cuda.graph(graph):
        tuning().beam_reorder(y, parents)
    assert y[:, 0].tolist() == [0, 1, 2, 3]
    graph.replay()
    assert y[:, 0].tolist() == [0, 0, 1, 2]
    parents.copy_(cuda([[3, 1, 1, 0]]))
    graph.replay()
    torch.cuda.synchronize()
    assert y[:, 4].tolist() == [2, 0, 0, 0]


# --------------------------------------------------------------------------------------------------------- refusals

def refused(f, *args, **kw):
    with pytest.raises(N.NmdError) as e:
        f(*args, **kw)
    assert e.value.status == N.NMD_ERR_INVALID


def test_refusals():
    t = tuning()
    x, s = torch.zeros(6, 10, device="cuda"), torch.zeros(2, 3, device="cuda")
    f = torch.zeros(2, 3, device="cuda", dtype=torch.bool)
    for bad in (x.cpu(), x.double(), x[0], x[:, ::2], x[:, :0], None):
        refused(t.beam_select, bad, s)
    for bad in (s[:1], s.double(), s.cpu(), s.view(-1), s.view(2, 3, 1), None, torch.zeros(6, 0, device="cuda")):
        refused(t.beam_select, x, bad)
    for kw in (dict(width=0), dict(width=129), dict(finished=f), dict(finished=f.int(), end=1), dict(finished=f[:1], end=1),
               dict(finished=f.cpu(), end=1), dict(end=10), dict(end=-1), dict(temperature=0.0),
               dict(temperature=float("nan"))):
        refused(t.beam_select, x, s, **kw)
    refused(t.beam_select, torch.zeros(65, 10, device="cuda"), torch.zeros(1, 65, device="cuda"))
    p = torch.zeros(2, 3, device="cuda", dtype=torch.int64)
    for bad in (p.int(), p.cpu(), p[0], None, p[:, :2], torch.zeros(4, 3, device="cuda", dtype=torch.int64)):
        refused(t.beam_reorder, x, bad)
    for bad in (x.cpu(), x[:4], x[:, ::2], x[:1].expand(6, 10), x.t(), None, [x, None]):
        refused(t.beam_reorder, bad, p)
    refused(t.beam_reorder, x, p, dim=2)
    refused(t.beam_reorder, x, p, dim=-1)
    for out in (x[:4], x.double(), x.cpu(), x[:, :9], [x, x], x.view(6, 10, 1), torch.zeros(66, device="cuda").as_strided((6, 10), (0, 1))):
        refused(t.beam_reorder, x, p, out=out)
    flat = torch.zeros(200, device="cuda")
    a, b = flat[:60].view(6, 10), flat[50:110].view(6, 10)
    refused(t.beam_reorder, a, p, out=b)
    refused(t.beam_reorder, [a, flat[120:180].view(6, 10)], p, out=[flat[60:120].view(6, 10), flat[100:160].view(6, 10)])
    assert not x.any() and not flat.any()
