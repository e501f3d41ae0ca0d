"""Memory that the policy update's entry points allocate themselves belongs to the
stream that they write and use it on."""
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


def _stream_of(t):
    """The stream whose memory the allocator took a tensor from."""
    at = t.data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= at < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


def test_lists_and_states_are_memory_of_their_stream():
    g = [torch.randn(n, device=dev()) for n in (1000, 5)]
    m = [torch.zeros_like(t) for t in g]
    v = [torch.zeros_like(t) for t in g]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lst = P.ParamList(g, params=[t.clone() for t in g], exp_avg=m, exp_avg_sq=v, stream=side)
    state = P.alloc_adam_state(dev(), stream=side)
    assert side.cuda_stream != torch.cuda.current_stream().cuda_stream
    assert _stream_of(lst.data) == side.cuda_stream == _stream_of(state)
    torch.cuda.synchronize()
    P.dora_adam_step(lst, state, 1e-3, stream=side)
    side.synchronize()
    assert int(state[:8].view(torch.int64).item()) == 1
    assert bool(torch.allclose(m[0], 0.1 * g[0], rtol=1e-6, atol=0))
    for t in (P.ParamList(g).data, P.alloc_adam_state(dev())):
        assert _stream_of(t) == torch.cuda.current_stream().cuda_stream
