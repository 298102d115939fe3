"""The operators at the most rows and columns that they accept, thin where the other side would not fit: every row is answered, and nothing behind the last."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2111_01264_amd as P
from tests.test_gpu_q8_linear import run


@pytest.mark.parametrize("M,N,K", [(P.Q8_LINEAR_MAX_ROWS, 3, 17), (3, P.Q8_LINEAR_MAX_ROWS, 17), (17, P.Q8_LINEAR_MAX_ROWS, 48), (P.Q8_LINEAR_MAX_ROWS, 130, 16), (1, 1, P.Q8_LINEAR_MAX_K)])
def test_products(M, N, K):
    run(M, N, K, "bf16", relu=True)
    run(M, N, K, "fp32", pad=((-K) % 16, (-K) % 16, 1))


@pytest.mark.parametrize("cols", [1, 5, 70])
def test_rows_to_levels(cols):
    rows = P.Q8_QUANTIZE_MAX_ROWS
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    x = torch.randint(-127, 128, (rows, cols), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    x[:, 0] = 127   # a row's largest: its levels are its values
    q, scale = torch.zeros(rows + 1, cols, dtype=torch.int8, device="cuda"), torch.zeros(rows + 1, device="cuda")
    f = x.half()
    torch.cuda.synchronize()
    P.q8_quantize_rows(f, P.DQN_TYPE_FP16, cols, rows, cols, q, cols, scale, None, 0, None)
    torch.cuda.synchronize()
    assert torch.equal(q[:rows], x) and torch.all(scale[:rows] == 1.0) and torch.all(q[rows] == 0) and scale[rows].item() == 0.0


@pytest.mark.parametrize("n", [1, 3, 64, 70])
def test_draws(n):
    rows = P.POLICY_SAMPLE_MAX_ROWS
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    x = torch.zeros(rows, n, device="cuda").bfloat16()
    at = torch.randint(n, (rows,), generator=g, device="cuda")
    x.scatter_(1, at[:, None], 1.0)
    u = torch.rand(rows, generator=g, device="cuda")
    index, logp = torch.full((rows + 1,), -7, dtype=torch.int32, device="cuda"), torch.full((rows + 1,), 9.0, device="cuda")
    k, m = torch.ones(rows, dtype=torch.int32, device="cuda"), torch.ones(rows, device="cuda")
    assert P.policy_sample_workspace(rows, n) == 0
    for filters in (dict(top_k=k, min_p=None), dict(top_k=None, min_p=m)):   # each leaves the largest score alone
        index[:rows] = -5
        torch.cuda.synchronize()
        P.policy_sample(x, P.DQN_TYPE_BF16, n, rows, n, None, filters["top_k"], None, filters["min_p"], u, index, logp, None, 0, None)
        torch.cuda.synchronize()
        assert torch.equal(index[:rows].long(), at) and torch.all(logp[:rows] == 0) and index[rows].item() == -7 and logp[rows].item() == 9.0
