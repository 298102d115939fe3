"""policy_sample: scores of +infinity share the whole mass, also where top-k keeps more entries than there are of them, at every length at which another kernel does the row."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_policy_sample import INF, TYPES, Call, gen


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [50, 700, 3000, 20001, 60000])
def test_fewer_infinities_than_top_k_keeps(kind, n):
    g = gen(n)
    x = torch.randn(5, n, generator=g, device="cuda")
    x[0, 1] = INF
    x[1, 1] = INF; x[1, n - 1] = INF
    x[2, ::2] = INF
    x[3] = -INF; x[3, n // 3] = INF
    x[4] = INF
    x = x.to(TYPES[kind][0])
    for k in (0, 1, 2, 5, 40, 193, 500, n - 1):
        for f in (dict(), dict(p=[1.0] * 5), dict(p=[0.7] * 5), dict(m=[0.5] * 5), dict(t=[2.0] * 5)):
            c = Call(x, n, torch.rand(5, generator=g, device="cuda"), k=[k] * 5, **f)
            assert c.run() <= 5
            got = c.index[:5].long()
            assert torch.all(got >= 0) and torch.all(x.gather(1, got[:, None]) == INF)
