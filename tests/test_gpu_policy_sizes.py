"""Sizes past the 32 bits of the policy losses' entry points are refused, not cut
down to what fits."""
import pytest
import torch

import __graft_entry__ as G
import paper_2609_34325_gb300 as P
from helpers import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def test_policy_loss_of_more_classes_than_32_bits_hold():
    one, action = torch.zeros(1, device=dev()), torch.zeros(1, dtype=torch.int32, device=dev())
    z = torch.empty(1, 2 ** 32 + 5, dtype=torch.bfloat16, device=dev())
    z[:, :16] = 0.0
    logp = torch.full((1,), 7.0, device=dev())
    with pytest.raises(ValueError):
        P.dora_policy_loss(z, action, one, one, logp)
    with pytest.raises(ValueError):
        P.dora_policy_loss(z.view(-1, 1), action, one, one, logp)
    torch.cuda.synchronize()
    assert float(logp) == 7.0
    P.dora_policy_loss(z, action, one, one, logp, classes=4)       # of which four count
    assert abs(float(logp) + 1.3862944) < 1e-6


def test_sequence_loss_of_more_scores_than_32_bits_hold():
    scores = torch.empty(2 ** 32 + 8, device=dev())
    cu = torch.tensor([0, 5], dtype=torch.int32, device=dev())
    k = torch.ones(1, dtype=torch.int32, device=dev())
    one, logp = torch.zeros(1, device=dev()), torch.full((1,), 7.0, device=dev())
    with pytest.raises(ValueError):
        P.dora_pl_policy_loss(scores, cu, k, torch.zeros(1, 1, dtype=torch.int32, device=dev()),
                              one, one, logp)
    torch.cuda.synchronize()
    assert float(logp) == 7.0
