"""Views that torch negates or conjugates only when they are read: their memory holds other values than they show, so
operators that read memory refuse them, and rows are copied only between views of one kind."""
import pytest

from gpu_common import require_gpu
from paper_2608_21607_gb300 import nmd as N

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    return require_gpu()


def refused(f, *args, **kw):
    with pytest.raises(N.NmdError) as e:
        f(*args, **kw)
    assert e.value.status == N.NMD_ERR_INVALID


def test_updates_that_are_negated_when_read():
    from paper_2608_21607_gb300 import tuning as t

    z = torch.randn(6, 4, device="cuda", dtype=torch.complex64)
    update = z.conj().imag
    assert update.is_neg()
    x = torch.randn(6, 4, device="cuda")
    refused(t.orthogonalize, update)
    refused(t.orthogonalize, x, out=update)
    for at in range(3):
        matrices = [torch.randn(6, 4, device="cuda") for _ in range(3)]
        matrices[at] = update
        refused(t.muon_step, *matrices, lr=0.1)
    # what it shows, laid out
    assert torch.equal(t.orthogonalize(update.resolve_neg()), -t.orthogonalize(z.imag))


def test_states_of_two_kinds():
    from paper_2608_21607_gb300 import tuning as t

    parents = torch.tensor([[1, 0, 0]], device="cuda")
    z = torch.randn(3, 5, device="cuda", dtype=torch.complex64)
    refused(t.beam_reorder, z.conj(), parents, out=torch.empty_like(z))
    refused(t.beam_reorder, z, parents, out=torch.empty_like(z).conj())
    refused(t.beam_reorder, z.conj().imag[:, :1], parents, out=torch.empty(3, 1, device="cuda"))
    want = z.conj()[[1, 0, 0]]
    out = torch.empty_like(z).conj()
    t.beam_reorder(z.conj(), parents, out=out)
    assert torch.equal(out, want)
    t.beam_reorder(z.conj(), parents)                     # in place: rows change places, whatever they show
    assert torch.equal(z.conj().resolve_conj(), want.resolve_conj())
