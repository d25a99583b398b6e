"""A cooperative launch that is refused (a context with a part of the SMs) leaves no step half taken: the products that
need no co-residency take the strip kernel's place.  The refusal is made on the host: the library is linked once more
with a launch call in between that answers "too large" to cooperative launches and passes everything else on.

Tolerance: both ways are within 2^-17 of the result's norm on these well-conditioned updates (fp32 steps come out about
1e-6 off, and the pieces' 22 bits and the sums' roundings towards zero are within eight of theirs).
"""
import ctypes as C
import glob
import os
import subprocess

import numpy as np
import pytest

import oracle as O
from gpu_common import require_gpu
from paper_2608_21607_gb300 import build as B
from paper_2608_21607_gb300 import nmd as N

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BETWEEN = r"""
#include <cuda_runtime.h>
static int refused = 0;
extern "C" int launches_refused() { return refused; }
extern "C" cudaError_t __real_cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void** args);
extern "C" cudaError_t __wrap_cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void** args) {
  for (unsigned i = 0; i < c->numAttrs; ++i)
    if (c->attrs[i].id == cudaLaunchAttributeCooperative && c->attrs[i].val.cooperative) {
      ++refused;
      return cudaErrorCooperativeLaunchTooLarge;
    }
  return __real_cudaLaunchKernelExC(c, f, args);
}
"""


@pytest.fixture(scope="module")
def refusing(tmp_path_factory):
    """The library whose cooperative launches are refused."""
    require_gpu()
    d = str(tmp_path_factory.mktemp("refusing"))
    src, so = os.path.join(d, "between.cpp"), os.path.join(d, "librefusing.so")
    with open(src, "w") as f:
        f.write(BETWEEN)
    subprocess.run([B.nvcc(), "-shared", "-o", so, src] + sorted(glob.glob(os.path.join(B.BUILD, "*.o"))) + B.ARCH
                   + ["-Xcompiler", "-fPIC", "-Xlinker", "--wrap=cudaLaunchKernelExC"], check=True, capture_output=True)
    return C.CDLL(so)


@pytest.mark.parametrize("rows,cols,layout", [(200, 64, "rows"), (1000, 40, "columns"), (64, 5000, "rows"),
                                              (20000, 33, "rows"), (17, 30001, "columns"), (64, 64, "rows")])
@pytest.mark.parametrize("types", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32)])
def test_step_without_cooperative_launches(refusing, monkeypatch, rows, cols, layout, types):
    from paper_2608_21607_gb300 import tuning as t

    rng = np.random.default_rng(rows)
    W, G, M = (torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).cuda() for _ in range(3))
    G = G.to(types[0])
    if layout == "columns":
        W, M = W.t().contiguous().t(), M.t().contiguous().t()
    w, g, m = (v.double().cpu().numpy() for v in (W, G, M))
    for name in ("nmd_muon_step", "nmd_orthogonalize"):
        f = getattr(refusing, name)
        f.argtypes, f.restype = getattr(N.lib(), name).argtypes, C.c_int
        monkeypatch.setitem(t._calls, name, f)
    before = refusing.launches_refused()
    t.muon_step(W, G, M, lr=1.0, beta=0.5, scale=1.0)
    assert refusing.launches_refused() == before + (max(rows, cols) > 128)
    got = M.double().cpu().numpy()
    np.testing.assert_allclose(got, 0.5 * m + 0.5 * g, rtol=1e-6, atol=1e-6)
    want, _ = O.tuning.muon_step(w, g, m, lr=1.0, beta=0.5, scale=1.0, round_momentum=lambda _: got)
    moved = np.linalg.norm(want - w)
    assert np.linalg.norm(W.double().cpu().numpy() - want) <= 2.0 ** -17 * moved + 2.0 ** -24 * np.linalg.norm(want)
    # the result by itself, of the update's type
    got = t.orthogonalize(G).double().cpu().numpy()
    want = O.tuning.orthogonalize(g)
    half = 2.0 ** -24 if types[0] == torch.float32 else 2.0 ** -8
    assert np.linalg.norm(got - want) <= (2.0 ** -17 + half) * np.linalg.norm(want)
