"""The bounded waits of the policy loss's ring, made to run out on purpose without
faulting anything.

In libdora_timeout_test.so these waits give up after 5 ms, and the first CTA never
copies its second row (nor expects its bytes), so that its sum and gradient warps
wait for a stage that stays empty, and with them the other CTAs of its cluster.  The
kernel must end by itself, report DORA_ERR_TIMEOUT and leave the rows of that CTA or
cluster NaN and all others right; the context must stay usable."""
import ctypes

import pytest
import torch

import __graft_entry__ as G
import paper_2609_34325_gb300 as P
from helpers import dev
from paper_2609_34325_gb300 import build as B

pytestmark = pytest.mark.gpu
DORA_ERR_TIMEOUT = 4               # include/dora.h: a bounded pipeline wait ran out


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _timeout_loss(monkeypatch, *args, **kw):
    """dora_policy_loss through the test library."""
    lib = ctypes.CDLL(B.TIMEOUT_TEST_LIB_PATH)
    lib.dora_policy_loss.restype, lib.dora_policy_loss.argtypes = P._SIGS["dora_policy_loss"]
    with monkeypatch.context() as m:
        m.setattr(P, "load_library", lambda: lib)
        P.dora_policy_loss(*args, **kw)


# one CTA a row, and clusters of two, four and eight; several rows each
@pytest.mark.parametrize("rows,classes", [(700, 20000), (300, 50000), (200, 100000), (80, 200000)])
def test_a_wait_that_runs_out_leaves_its_rows_nan_and_the_others_right(rows, classes, monkeypatch):
    g = torch.Generator(device=dev()).manual_seed(rows)
    z = torch.randn(rows, classes, generator=g, device=dev()).to(torch.bfloat16)
    act = torch.randint(0, classes, (rows,), generator=g, device=dev()).int()
    old = torch.full((rows,), -10.0, device=dev())
    adv = torch.randn(rows, generator=g, device=dev())

    def buffers():
        return {"logp": torch.full((rows,), 7.0, device=dev()),
                "entropy": torch.full((rows,), 7.0, device=dev()),
                "row_loss": torch.full((rows,), 7.0, device=dev()),
                "totals": torch.full((6,), 7.0, device=dev()), "grad": torch.full_like(z, 7.0)}

    def call(run, out, status):
        run(z, act, old, adv, out["logp"], P.alloc_policy_workspace(dev()), grad=out["grad"],
            entropy_coef=0.01, entropy=out["entropy"], row_loss=out["row_loss"],
            totals=out["totals"], status=status)
        torch.cuda.synchronize()           # the launch ended: every wait was bounded

    want = buffers()
    call(P.dora_policy_loss, want, None)
    for _ in range(2):                     # twice: the kernel left nothing behind
        out = buffers()
        status = torch.zeros(1, dtype=torch.int32, device=dev())
        call(lambda *a, **kw: _timeout_loss(monkeypatch, *a, **kw), out, status)
        assert int(status.item()) == DORA_ERR_TIMEOUT
        lost = torch.isnan(out["logp"])
        assert 1 < int(lost.sum()) < rows // 2 and bool(lost[0])
        for n in ("logp", "entropy", "row_loss", "grad"):
            assert bool(torch.isnan(out[n][lost]).all()), n
            assert torch.equal(out[n][~lost], want[n][~lost]), n
        assert bool(torch.isnan(out["totals"]).all())
        # what follows in an update sees it without a status word
        norm = torch.zeros(2, device=dev())
        P.dora_grad_norm(P.ParamList([out["grad"]]), 1.0, norm)
        assert not bool(torch.isfinite(norm[0]))
    again = buffers()
    call(P.dora_policy_loss, again, None)
    for n in want:
        assert torch.equal(again[n], want[n]), n
