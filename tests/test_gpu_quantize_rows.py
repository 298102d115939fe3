"""q8_quantize_rows against the oracle in 64 bits, through the C boundary: the levels are equal, the scales off by one rounding,
the values by theirs."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2111_01264_amd as P
from oracle import actor

TYPES = {"fp32": (torch.float32, P.DQN_TYPE_FP32), "bf16": (torch.bfloat16, P.DQN_TYPE_BF16), "fp16": (torch.float16, P.DQN_TYPE_FP16)}


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def check(x, ldx, rows, cols, code, q, scale, values):
    want_q, want_s = actor.quantize_rows(f64(x)[:rows, :cols])
    if q is not None:
        assert np.array_equal(q.cpu().numpy()[:, :cols], want_q)
    s = scale.cpu().numpy().astype(np.float64)
    ok = np.isfinite(want_s)
    assert np.array_equal(np.isnan(s), ~ok)
    # one rounding to fp32: half a step, or half the smallest subnormal
    assert np.all(np.abs(s - want_s)[ok] <= np.maximum(want_s[ok] * 2.0 ** -24, 2.0 ** -150))
    if values is not None:
        v, want = f64(values)[:, :cols], want_q * want_s[:, None]
        eps = torch.finfo(values.dtype).eps / 2
        tiny = torch.finfo(values.dtype).tiny * eps   # half a step of the subnormals
        # the scale's rounding, the product's and the result's
        bound = np.abs(want) * (2 * 2.0 ** -24 + eps) * (1 + 2.0 ** -20) + tiny + 127 * 2.0 ** -149
        assert np.all(np.abs(v - want)[ok] <= bound[ok]) and np.all(np.isnan(v[~ok]))


def run(x, ldx, rows, cols, code, want_q=True, want_values=True, stream=None, guard=3):
    dt = x.dtype
    q = torch.full((rows + 1, cols + guard), 77, dtype=torch.int8, device="cuda") if want_q else None
    v = torch.full((rows + 1, cols + guard), 5.0, dtype=dt, device="cuda") if want_values else None
    scale = torch.full((rows + 1,), -1.0, device="cuda")
    torch.cuda.synchronize()
    P.q8_quantize_rows(x, code, ldx, rows, cols, q, cols + guard, scale, v, cols + guard, stream)
    torch.cuda.synchronize()
    # what lies behind the last column and the last row stays as it was
    for t, mark in ((q, 77), (v, 5.0)):
        if t is not None:
            assert torch.all(t[rows] == mark) and torch.all(t[:rows, cols:] == mark)
    assert scale[rows].item() == -1.0
    check(x, ldx, rows, cols, code, None if q is None else q[:rows], scale[:rows], None if v is None else v[:rows])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (2, 15), (5, 16), (4, 17), (2, 63), (2, 511), (2, 512), (3, 1000), (2, 2048), (7, 2049), (33, 3136), (2, 4095), (3, 4096), (2, 4097),
                                       (3, 8192), (2, 8209), (2, 16384), (2, 16401), (1, 33001), (1, 65536), (2, 70003), (600, 40)])
def test_sizes(kind, rows, cols):
    dt, code = TYPES[kind]
    g = torch.Generator(device="cuda")
    g.manual_seed(rows * 100003 + cols)
    x = (torch.randn(rows, cols + 2, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(dt)
    run(x, cols + 2, rows, cols, code)
    if cols in (17, 3136, 4097):
        run(x, cols + 2, rows, cols, code, want_q=False)
        run(x, cols + 2, rows, cols, code, want_values=False)
        dense = x[:, :cols].contiguous()
        run(dense, cols, rows, cols, code, guard=0)


@pytest.mark.parametrize("kind", list(TYPES))
def test_borders_between_levels(kind):
    """Largest magnitudes and values whose quotients lie half way between two levels, or as near to that as the type allows."""
    dt, code = TYPES[kind]
    rows = []
    for top in (127.0, 254.0, 381.0, 63.5, 100.0, 1.0, 3.0, 129.0):
        r = [top] + [sign * (k + 0.5) * top / 127.0 for k in range(0, 126) for sign in (1, -1)]
        r = torch.tensor(r, dtype=torch.float64).to(dt)
        up, down = (torch.nextafter(r.float(), torch.full((), s * 1e9)).to(dt) for s in (1, -1))
        for t in (r, up, down):
            t[0] = top
            rows.append(torch.clamp(t.float(), -top, top).to(dt))
    x = torch.stack(rows).cuda()
    run(x, x.shape[1], x.shape[0], x.shape[1], code)


@pytest.mark.parametrize("kind", list(TYPES))
def test_rows_of_zeros_of_the_type_s_ends_and_not_finite(kind):
    dt, code = TYPES[kind]
    fin = torch.finfo(dt)
    for cols in (5, 300, 5000):
        x = torch.zeros(9, cols, dtype=torch.float32)
        x[1, cols // 2] = -0.0
        x[2] = torch.linspace(-1, 1, cols) * fin.max
        x[3] = torch.linspace(-1, 1, cols) * (fin.tiny * 4)
        x[4, 3] = fin.tiny * fin.eps       # the smallest subnormal alone
        x[5, cols - 1] = float("nan")
        x[6, 0] = float("inf")
        x[7, 1] = float("-inf")
        x[8] = 1.0
        x = x.to(dt).cuda()
        run(x, cols, 9, cols, code)


def test_empty_rows_and_unaligned_views():
    scale = torch.full((4,), -1.0, device="cuda")
    P.q8_quantize_rows(None, P.DQN_TYPE_FP32, 0, 3, 0, None, 0, scale, None, 0, None)
    torch.cuda.synchronize()
    assert scale.tolist() == [0.0, 0.0, 0.0, -1.0]
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    for kind, (dt, code) in TYPES.items():
        big = torch.randn(6, 700, generator=g, device="cuda").to(dt)
        for off in (1, 2, 3, 5, 8):
            x = big[1:5, off:off + 601]
            run(x, 700, 4, 601, code)


def test_another_stream_and_a_replayed_graph():
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    stream = torch.cuda.Stream()
    x = torch.randn(40, 3136, generator=g, device="cuda").bfloat16()
    run(x, 3136, 40, 3136, P.DQN_TYPE_BF16, stream=stream)
    q, scale = torch.zeros(40, 3136, dtype=torch.int8, device="cuda"), torch.zeros(40, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        P.q8_quantize_rows(x, P.DQN_TYPE_BF16, 3136, 40, 3136, q, 3136, scale, None, 0, stream)
    for _ in range(3):
        x.copy_(torch.randn(40, 3136, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(x, 3136, 40, 3136, P.DQN_TYPE_BF16, q, scale, None)
