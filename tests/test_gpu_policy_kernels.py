"""policy_sample kernel by kernel: rows of more than 256 vectors by workgroups of 256 and 1024 threads, and rows shared out among workgroups.  Every test asserts which kernels its
sizes reach, so that a moved line cannot empty it.  Bounds are those of test_gpu_policy_sample."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2111_01264_amd as P
from tests.gpu_kernels import kernels_of
from tests.test_gpu_policy_sample import INF, NAN, TYPES, Call, gen

N = 60000   # shared out, at up to 64 rows


def shared_out(call):
    assert P.policy_sample_workspace(call.rows, call.n) > 0
    names = kernels_of(call.enqueue)
    assert len(names) == (4 if call.k is not None or call.p is not None else 3) and all("policy_split_kernel" in s for s in names), names
    return call


def one_workgroup(call, threads):
    assert P.policy_sample_workspace(call.rows, call.n) == 0
    names = kernels_of(call.enqueue)
    assert len(names) == 1 and "policy_row_kernel" in names[0] and "Li%dE" % threads in names[0], names
    return call


@pytest.mark.parametrize("kind", list(TYPES))
def test_masks_infinities_and_nan(kind):
    dt, _ = TYPES[kind]
    low = torch.finfo(dt).min
    g = gen(N)
    x = torch.randn(12, N, generator=g, device="cuda")
    x[0] = -INF                                     # nothing left
    x[1] = -INF; x[1, N - 1] = -3.0                 # one left, the last
    x[2, : N - 2] = low                             # masked with the type's lowest value
    x[3] = low                                      # all of it: a row of equals
    x[4, N // 2] = NAN                              # in one part only
    x[5, 1] = INF; x[5, N - 1] = INF                # share the mass, in the first and the last part
    x[6, N - 1] = NAN; x[6, 0] = INF
    x[7, 0] = torch.finfo(dt).max; x[7, 1] = low
    x[8, : N - 1] = -INF; x[8, 0] = NAN
    x[9, 5000:] = -INF                              # whole parts without a score
    x[10, : N - 300] = -INF
    x[11] = INF
    x = x.to(dt)
    for t in (1.0, 0.0, 1e-30, 1e30):
        for k, p in ((0, 1.0), (3, 1.0), (500, 1.0), (0, 0.9), (2, 0.5), (40000, 0.8)):
            c = shared_out(Call(x, N, torch.rand(12, generator=g, device="cuda"), [t] * 12, [k] * 12, [p] * 12))
            c.run()
            assert c.index[[0, 4, 6, 8]].tolist() == [-1] * 4 and torch.isnan(c.logp[[0, 4, 6, 8]]).all()


def test_equal_scores_go_by_index():
    """Weights of exactly 1: kept sets and borders are whole numbers, with no rounding anywhere."""
    x = torch.zeros(6, N, device="cuda")
    x[:, 1::2] = -0.0   # the same score
    x[3, ::3] = -INF
    x[4] = torch.finfo(torch.float32).min
    x[5] = INF
    live = np.flatnonzero(np.arange(N) % 3)
    for k in (0, 2, 192, N // 2, N - 1):
        for p in (1.0, 0.5, 0.25):
            for u in (0.0, 0.25, 0.5, 1 - 2.0 ** -24):
                c = shared_out(Call(x, N, [u] * 6, k=[k] * 6, p=[p] * 6))
                c.enqueue()
                torch.cuda.synchronize()
                got = c.index[:6].tolist()
                size = k if k else N
                kept = size if p == 1.0 else int(np.ceil(p * size))
                for r in (0, 1, 2, 4, 5):
                    assert got[r] == int(np.floor(u * kept)), (r, k, p, u)
                size = min(k, len(live)) if k else len(live)
                kept = size if p == 1.0 else int(np.ceil(p * size))
                assert got[3] == live[int(np.floor(u * kept))], (k, p, u)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("step", [1.0, 1 / 16, 1 / 512])
def test_equals_at_the_border_lie_in_many_parts(kind, step):
    """Scores of few values: a filter's border falls among equals from all parts, which the lists hold (a fine step) or do not (a coarse one)."""
    g = gen(int(1 / step))
    x = (torch.round(2 * torch.randn(8, N, generator=g, device="cuda") / step) * step).to(TYPES[kind][0])
    for seed in range(2):
        c = shared_out(Call(x, N, torch.rand(8, generator=g, device="cuda"), k=[50, 192, 193, 5000, 0, 0, 700, 20000], p=[1.0, 0.7, 1.0, 1.0, 0.3, 0.95, 0.5, 0.9]))
        c.run()


def test_refused_settings_and_the_ends_of_u():
    g = gen(1)
    x = torch.randn(9, N, generator=g, device="cuda")
    c = shared_out(Call(x, N, [0.5] * 9, t=[-1.0, NAN, INF, 1.0, 1.0, 1.0, -0.0, 1.0, 1.0], p=[1.0, 1.0, 1.0, NAN, 1.0, 1.0, 1.0, -0.5, 2.0], m=[0.0, 0.0, 0.0, 0.0, NAN, 0.0, 0.0, 0.0, -1.0]))
    c.u[5] = NAN
    c.run()
    assert c.index[:6].tolist() == [-1] * 6 and (c.index[6:9] >= 0).all()
    for u in (-3.0, 0.0, 1.0 - 2.0 ** -24, 1.0, 1e30, INF, -INF):
        shared_out(Call(x, N, [u] * 9, k=[0, 7, 0, 1, N, -5, 2, N + 9, 3])).run()
        shared_out(Call(x, N, [u] * 9, p=[0.1, 0.5, 0.9, 0.99, 0.999, 1.0, 0.3, 0.0, 1e-30])).run()
        shared_out(Call(x, N, [u] * 9, m=[0.0, 0.5, 1.0, 2.0, 0.1, 0.01, 1e-30, INF, -INF])).run()


@pytest.mark.parametrize("kind", list(TYPES))
def test_pitches_and_alignments(kind):
    g = gen(2)
    n, ld = 50001, 50006
    big = (2 * torch.randn(6, ld, generator=g, device="cuda")).to(TYPES[kind][0])
    for off in (0, 1, 2, 3, 5):
        shared_out(Call(big[:, off:off + n], n, torch.rand(6, generator=g, device="cuda"), k=[0, 0, 20, 0, 900, 4000], p=[1.0, 0.9, 1.0, 0.5, 1.0, 0.7])).run()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,n,threads", [(5, 700, 256), (5, 8191, 256), (5, 16384, 256), (5, 16385, 1024), (140, 20001, 1024), (257, 16385, 256)])
def test_one_workgroup_per_row(kind, rows, n, threads):
    """What the rows above go through where they are not shared out: masks, infinities, equals and alignment under every filter."""
    dt, _ = TYPES[kind]
    g = gen(rows + n)
    big = (2 * torch.randn(rows, n + 5, generator=g, device="cuda")).to(dt)
    big[0] = -INF
    big[1, ::3] = INF
    big[2] = torch.round(big[2])
    big[3, 7:] = torch.finfo(dt).min
    big[4, n // 3] = NAN
    rep = lambda v: [v[r % len(v)] for r in range(rows)]  # noqa: E731
    for off in (0, 3):
        x, u = big[:, off:off + n], torch.rand(rows, generator=g, device="cuda")
        for f in (dict(), dict(k=rep([5, 192, 193, 600])), dict(p=rep([0.9, 0.5, 0.99])), dict(k=rep([300, 50, 0, 1000]), p=rep([0.5, 0.95, 0.8]), m=rep([0.0, 0.02]))):
            one_workgroup(Call(x, n, u, t=rep([1.0, 0.5, 1.0, 2.0, 1.0, 0.0, 20.0]), **f), threads).run()


def test_replayed_graphs_and_streams_with_a_workspace_each():
    """The graphs of all calls in flight together, each on a stream of its own, several times; the workspaces are never cleared in between."""
    g = gen(7)

    def make(rows, n, dt, **f):
        return Call((3 * torch.randn(rows, n, generator=g, device="cuda")).to(dt), n, torch.rand(rows, generator=g, device="cuda"), **{k: [v] * rows for k, v in f.items()})
    f32, bf16 = torch.float32, torch.bfloat16
    calls = [shared_out(make(2, N, f32, k=50, p=0.9)), shared_out(make(2, N, f32, p=0.9)), shared_out(make(3, N, f32)), shared_out(make(2, N, bf16, k=5000, p=0.5)),
             shared_out(make(1, 131072, bf16, k=40, p=0.95)), one_workgroup(make(140, 20000, bf16, p=0.9), 1024), one_workgroup(make(20, 40000, f32, k=300), 1024), one_workgroup(make(260, 30000, bf16, p=0.9), 256),
             one_workgroup(make(30, 3000, f32, k=1000, p=0.9), 256), make(30, 18, f32, p=0.9)]
    streams, graphs = [torch.cuda.Stream() for _ in calls], []
    for c, s in zip(calls, streams):
        c.enqueue(s)
    for c, s in zip(calls, streams):
        c.check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.enqueue(s)
        graphs.append(graph)
    for _ in range(3):
        for c in calls:
            c.x.copy_(3 * torch.randn(c.rows, c.n, generator=g, device="cuda"))
            c.u.copy_(torch.rand(c.rows, generator=g, device="cuda"))
            c.index[:c.rows] = -3
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        for c in calls:
            c.check()
