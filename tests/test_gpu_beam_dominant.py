"""Rows in which a column or a few hold nearly all of the probability, and what is selected beside them lies up to the
end of fp32's exponents below (86 to 88 in the logits' units over the temperature is 2^-124 to 2^-127).

Within a row the order of the offers is that of the logits, of equal ones that of the columns, so the columns are
compared exactly.  Scores: the tolerance of test_gpu_beam.py, u (128 + 4 R + 4 |lp|) and one rounding, R <= 210.
"""
import numpy as np
import pytest

import oracle as O
from gpu_common import require_gpu

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = 2.0 ** -24
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    return require_gpu()


def check(rows, width, temperature):
    """One beam a group: every row by itself."""
    from paper_2608_21607_gb300 import tuning as t

    got = t.beam_select(rows, torch.zeros(len(rows), 1, device="cuda"), width=width, temperature=temperature)
    want = torch.sort(rows.float(), dim=1, descending=True, stable=True).indices[:, :width]
    wrong = (got.tokens != want).any(1).nonzero().view(-1).tolist()
    assert not wrong, (wrong, got.tokens[wrong[0]].tolist(), want[wrong[0]].tolist())
    assert (got.parents == 0).all()
    # one row's scores, by the oracle
    best, _, tokens, _ = O.tuning.beam_select(rows[:1].double().cpu().numpy(), [[0.0]], width, temperature=temperature)
    assert np.array_equal(got.tokens[:1].cpu().numpy(), tokens)
    assert np.all(np.abs(got.scores[:1].cpu().numpy() - best) <= U * (128 + 4 * 210 + 5 * np.abs(best)))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("temperature", [1.0, 0.05, 4.0])
@pytest.mark.parametrize("width", [1, 2, 8, 33])
@pytest.mark.parametrize("V", [20000, 139255])
def test_one_column_dominates(dtype, temperature, width, V):
    """The largest column, lower ones of other threads in the first round of loads, and a better one in the next round,
    at each place of a vector of the largest column's own thread."""
    per = 16 // DTYPES[dtype].itemsize            # elements of a vector
    gaps = np.arange(83.0, 90.0, 0.25)
    stride = (V + per - 1) // per * per           # rows from 16-byte boundaries
    rows = torch.full((len(gaps) * per, stride), -200.0 * temperature, device="cuda", dtype=DTYPES[dtype])[:, :V]
    first = 1024 * per                            # columns of a round of 256 threads with four vectors
    rows[:, 0] = 0.0
    for i, gap in enumerate(gaps):
        for place in range(per):
            rows[i * per + place, 80 * per:80 * per + 37 * width:37] = -(gap + 0.75) * temperature
            rows[i * per + place, first + place] = -gap * temperature
    check(rows, width, temperature)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("temperature", [1.0, 0.05])
@pytest.mark.parametrize("width", [48, 128])
@pytest.mark.parametrize("odd", [0, 1])
def test_a_few_columns_dominate(dtype, temperature, width, odd):
    """Dominating columns in forty threads, every second column spread over the end of the exponents, the others below."""
    V = 60011
    g = torch.Generator(device="cuda").manual_seed(width)
    rows = ((-85.0 - 4.0 * torch.rand((6, V), device="cuda", generator=g)) * temperature).to(DTYPES[dtype])
    rows[:, 1 - odd::2] = -200.0 * temperature
    for r in range(6):
        at = torch.randint(0, 2000, (40,), device="cuda", generator=g)
        rows[r, at] = (torch.rand(40, device="cuda", generator=g) * temperature).to(rows.dtype)
    check(rows, width, temperature)
