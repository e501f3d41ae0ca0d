"""The bounded waits of the orthogonalised updates, made to run out on purpose without
faulting anything.

In libdora_timeout_test.so these waits give up after 5 ms.  For matrices of many tiles the
first pair of CTAs never copies the operands of its first product (nor expects their bytes);
for small ones the first CTA never says that its first product is done.  The kernels must
end by themselves and report DORA_ERR_TIMEOUT; the context and the list must stay usable."""
import ctypes

import pytest
import torch

import __graft_entry__ as G
import paper_2609_34325_gb300 as P
from helpers import dev
from paper_2609_34325_gb300 import build as B

pytestmark = pytest.mark.gpu
DORA_ERR_TIMEOUT = 4               # include/dora.h: a bounded pipeline wait ran out
SMALL = [(64, 787), (100, 37), (128, 128), (9, 1500)]
LARGE = [(640, 700), (300, 1000), (1536, 384), (257, 511)] * 3


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _timeout(monkeypatch, name, *args, **kw):
    """An entry point through the test library."""
    lib = ctypes.CDLL(B.TIMEOUT_TEST_LIB_PATH)
    fn = getattr(lib, name)
    fn.restype, fn.argtypes = P._SIGS[name]
    status = torch.zeros(1, dtype=torch.int32, device=dev())
    with monkeypatch.context() as m:
        m.setattr(P, "load_library", lambda: lib)
        getattr(P, name)(*args, status=status, **kw)
    torch.cuda.synchronize()       # the launches ended: every wait was bounded
    return int(status.item())


def _matrices(shapes, seed):
    g = torch.Generator(device=dev()).manual_seed(seed)
    return [torch.randn(s, generator=g, device=dev()) for s in shapes]


def test_a_product_that_is_not_done_leaves_its_matrix(monkeypatch):
    grads = _matrices(SMALL, 1)
    outs = [torch.zeros_like(x, dtype=torch.bfloat16) for x in grads]
    lst = P.MatrixList(grads, outs=outs)
    P.dora_orthogonalize(lst)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    for _ in range(2):
        for o in outs:
            o.fill_(7.0)
        assert _timeout(monkeypatch, "dora_orthogonalize", lst) == DORA_ERR_TIMEOUT
        assert bool((outs[0] == 7.0).all())
        assert all(torch.equal(o, w) for o, w in zip(outs[1:], want[1:]))
    P.dora_orthogonalize(lst)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_operands_that_never_come(monkeypatch):
    grads = _matrices(LARGE, 2)
    outs = [torch.zeros_like(x, dtype=torch.bfloat16) for x in grads]
    lst = P.MatrixList(grads, outs=outs)
    P.dora_orthogonalize(lst)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    for _ in range(2):                     # twice: the kernel left nothing behind
        for o in outs:
            o.fill_(7.0)
        assert _timeout(monkeypatch, "dora_orthogonalize", lst) == DORA_ERR_TIMEOUT
        assert any(bool((o == 7.0).all()) for o in outs)
        P.dora_orthogonalize(lst)
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_weights_of_a_step_that_was_given_up(monkeypatch):
    grads = _matrices(SMALL, 3)
    params, momentum = _matrices(SMALL, 4), [torch.zeros_like(x) for x in grads]
    lst = P.MatrixList(grads, params=params, momentum=momentum)
    before = [p.clone() for p in params]
    assert _timeout(monkeypatch, "dora_muon_step", lst, 0.1) == DORA_ERR_TIMEOUT
    assert torch.equal(params[0], before[0]) and bool(momentum[0].any())
    assert all(not torch.equal(p, b) for p, b in zip(params[1:], before[1:]))
