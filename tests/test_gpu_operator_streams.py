"""The operators on the runtime's own stream handles: the null stream by both of its names and the calling thread's stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2111_01264_amd as P


class Handle:
    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.mark.parametrize("handle", [0, 1, 2], ids=["null", "hipStreamLegacy", "hipStreamPerThread"])
def test_the_runtime_s_own_handles(handle):
    g = torch.Generator(device="cuda")
    g.manual_seed(handle)
    x, w = torch.randn(5, 300, generator=g, device="cuda"), torch.randn(40, 300, generator=g, device="cuda")
    u = torch.rand(5, generator=g, device="cuda")

    def run(stream):
        q, s, v, t = (torch.zeros(5, 304, dtype=torch.int8, device="cuda"), torch.zeros(5, device="cuda"), torch.zeros(40, 304, dtype=torch.int8, device="cuda"), torch.zeros(40, device="cuda"))
        y, index, logp = torch.zeros(5, 40, device="cuda"), torch.full((5,), -7, dtype=torch.int32, device="cuda"), torch.zeros(5, device="cuda")
        torch.cuda.synchronize()
        P.q8_quantize_rows(x, P.DQN_TYPE_FP32, 300, 5, 300, q, 304, s, None, 0, stream)
        P.q8_quantize_rows(w, P.DQN_TYPE_FP32, 300, 40, 300, v, 304, t, None, 0, stream)
        P.q8_linear(q, 304, s, v, 304, t, None, 0, 5, 40, 300, y, P.DQN_TYPE_FP32, 40, stream)
        P.policy_sample(y, P.DQN_TYPE_FP32, 40, 5, 40, None, None, None, None, u, index, logp, None, 0, stream)
        torch.cuda.synchronize()
        return y, index, logp

    got, want = run(Handle(handle)), run(torch.cuda.Stream())
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.all(got[1] >= 0)
